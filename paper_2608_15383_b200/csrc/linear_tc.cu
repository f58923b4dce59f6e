// exmoe_linear on tcgen05: D = W X^T with the weights' rows as the MMA's M and the tokens as its N, so that a warp's lanes hold consecutive
// outputs of one token: they are read and written in runs of 32 whatever the rows' distances and alignment are.
//
// Two forms.  `linear_split_kernel`: a tile of 128 rows by up to 64 tokens per cluster of CL CTAs, which split K and add their parts through
// the cluster's shared memory in a fixed order.  `linear_pair_kernel`: persistent pairs of CTAs (cta_group::2), 256 rows by up to 256 tokens.
// Both: TMA into a ring of 64-wide stages with the 128-byte swizzle, one warp issuing the MMAs, two accumulators in turn.  An MMA truncates what it adds
// (a few units of 2^-24 of all that its chain has summed): over a whole K of thousands that would show in a binary32 result.  So chains of kChain stages (32 MMAs)
// start from zero, and warps take them out of tensor memory and add them to binary32 sums in registers; only the pairs' BF16 results come from chains of up to 1024 MMAs.
//
// With a second matrix a tile's 128 rows are 64 of W and the same 64 of U: a row's two factors are 64 lanes of tensor memory apart and meet in shared memory.
#include <algorithm>
#include <mutex>

#include "common.cuh"
#include "frag.cuh"
#include "linear.cuh"
#include "mbar.cuh"
#include "tc.cuh"

namespace exmoe {

namespace {

constexpr int kSms = 148;
constexpr int kChain = 8;                                                  // stages
constexpr int kABytes = BM * 128;                                          // weights of a stage: 128 rows of 64 elements
__device__ int g_linear_status;                                            // sticky: EXMOE_ERR_TIMEOUT

__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr));
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const float* v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};"
                 ::"r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])),
                 "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7])), "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, int rank) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
    return at;
}
__device__ __forceinline__ void in_flight_end(uint32_t bar, uint32_t parity, long long budget) {
    const long long t0 = clock64();
    while (!mbar_try_at(bar, parity) && clock64() - t0 < budget) {}
}
// Takes up to 64 columns of a chain's accumulator (this warp's lanes) into acc: in pieces of 8, `cols` of them in use.
__device__ __forceinline__ void drain(uint32_t at, int cols, bool first, float (&acc)[64]) {
#pragma unroll
    for (int c = 0; c < 64; c += 16) {
        if (c < cols) {
            uint32_t r[8], s[8];
            tmem_ld8(at + c, r);
            if (c + 8 < cols) tmem_ld8(at + c + 8, s);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[c + i] = first ? __uint_as_float(r[i]) : acc[c + i] + __uint_as_float(r[i]);
            if (c + 8 < cols) {
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[c + 8 + i] = first ? __uint_as_float(s[i]) : acc[c + 8 + i] + __uint_as_float(s[i]);
            }
        }
    }
}

// ---- clusters that split K -------------------------------------------------------------------------------------------
// 128 rows by up to 64 tokens; a CTA takes a CL-th of K.  Two CTAs fit an SM, so that one loads while another finishes, and so that the next call's can
// be set up while this one's are at work.  The weights are requested into L2 before the wait for the kernel in front (which may still be writing them: L2 has
// what it writes), and read behind it.  Bound by latencies one after the other (wait, first stage, exchange) and by the 57 bytes a clock that an SM takes in: replayed,
// 45 tokens 5632 -> 2048 10.1 us (23 MB: 2.3 TB/s), two matrices 2048 -> 5632 13 us (46 MB: 3.5 TB/s).
constexpr int kSplitThreads = 256, kSplitTokens = 64, kSplitDrain = 4, kSplitStages = 11;
constexpr int kSplitRoom = 104 * 1024, kSplitRoomWide = 208 * 1024;        // of the ring: of two CTAs per SM, of one
struct SplitShared {                                                       // in front of the ring, which then holds the CTA's part of the tile: float [BN][BM]
    uint64_t full[kSplitStages], empty[kSplitStages], acc_full[2], acc_empty[2], drained;
    uint32_t tmem;
    int abort_flag;
};
static_assert(kSplitTokens * BM * 4 <= kSplitRoom && sizeof(SplitShared) <= 1024, "room");

__device__ __forceinline__ void mma_one(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void prefetch_2d(const CUtensorMap* map, int x, int y) {
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y) : "memory");
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory"); }

// The CTA's share of the tile's tokens, summed over the cluster's CL <= PEERS CTAs in order and finished: a thread has one output of every (256 / kRows)-th
// token, as many at a time as it has of a usual share, so that all parts are on their way together; their residuals are requested before the parts are there.
template <typename O, bool GATED, int PEERS>
struct Finish {
    static constexpr int kRows = GATED ? BM / 2 : BM, kEvery = kSplitThreads / kRows, kBatch = (PEERS == 2 ? 16 : PEERS == 4 ? 12 : 8) / (GATED ? 2 : 1);
    const LinearArgs& a;
    int nn, row, c0, c_end, CL;
    long long t0;
    O res[kBatch];
    __device__ __forceinline__ Finish(const LinearArgs& args, int n0, long long tile_t0, int rank, int cluster, int BN, int tid) : a(args), CL(cluster), t0(tile_t0) {
        const int share = (BN + CL - 1) / CL;
        row = tid % kRows;
        nn = n0 + row;
        c0 = rank * share + tid / kRows;
        c_end = (int)min((long long)min(BN, (rank + 1) * share), a.T - t0);
        if (nn >= a.N) c_end = 0;
        load(c0);
    }
    __device__ __forceinline__ void load(int from) {
        if (!a.residual) return;
        const O* p = static_cast<const O*>(a.residual) + (t0 + from) * a.ld_res + nn;
#pragma unroll
        for (int i = 0; i < kBatch; ++i, p += kEvery * a.ld_res)
            if (from + i * kEvery < c_end) res[i] = *p;
    }
    __device__ __forceinline__ void operator()(uint32_t part) {
        if (c0 >= c_end) return;
        const float bias = a.bias ? a.bias[nn] : 0.f, bias_up = GATED && a.bias_up ? a.bias_up[nn] : 0.f;
        for (int c = c0; c < c_end; c += kBatch * kEvery) {
            float g[PEERS][kBatch], u[PEERS][kBatch];
#pragma unroll
            for (int p = 0; p < PEERS; ++p)
                if (p < CL) {
                    const uint32_t from = at_rank(part, p) + 4 * row;
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) {                     // (again the last one behind the end)
                        const uint32_t at = from + 4 * BM * min(c + i * kEvery, c_end - 1);
                        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(g[p][i]) : "r"(at) : "memory");
                        if (GATED) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(u[p][i]) : "r"(at + 4 * kRows) : "memory");
                    }
                }
#pragma unroll
            for (int p = 1; p < PEERS; ++p)
                if (p < CL)
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) {
                        g[0][i] += g[p][i];
                        if (GATED) u[0][i] += u[p][i];
                    }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) g[0][i] += bias;
            activate_all(g[0], a.act);
            if (GATED)
#pragma unroll
                for (int i = 0; i < kBatch; ++i) g[0][i] *= u[0][i] + bias_up;
            if (a.residual)
#pragma unroll
                for (int i = 0; i < kBatch; ++i) g[0][i] += (float)res[i];
            O* out = static_cast<O*>(a.out) + (t0 + c) * a.ld_out + nn;
#pragma unroll
            for (int i = 0; i < kBatch; ++i, out += kEvery * a.ld_out)
                if (c + i * kEvery < c_end) store_out(out, g[0][i]);
            load(c + kBatch * kEvery);
        }
    }
};

// STUCK (exmoe_debug_linear_timeout): the second stage's barrier asks for an arrival that nobody makes.
template <typename O, bool GATED, int PEERS, bool STUCK>
__global__ void __launch_bounds__(kSplitThreads, 2)
linear_split_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_u, const __grid_constant__ CUtensorMap map_x,
                    const __grid_constant__ LinearArgs a, int BN, int CL, int row_tiles, int stages) {
    extern __shared__ unsigned char raw[];
    SplitShared& sm = *reinterpret_cast<SplitShared*>(raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u));
    unsigned char* ring = reinterpret_cast<unsigned char*>(&sm) + 1024;
    constexpr int kRows = GATED ? BM / 2 : BM;                             // outputs of a tile
    constexpr long long budget = STUCK ? kWaitBudgetTest : kWaitBudget;
    const int tid = threadIdx.x, lane = tid & 31, warp = warp_uniform(tid >> 5);
    const int rank = (int)blockIdx.x % CL, tile = (int)blockIdx.x / CL;
    const int n0 = tile % row_tiles * kRows, t0 = tile / row_tiles * BN, stage_bytes = kABytes + BN * 128;
    const int blocks = (a.K + 63) / 64, kb0 = (int)((long long)blocks * rank / CL), n = (int)((long long)blocks * (rank + 1) / CL) - kb0;
    volatile int* abort_flag = &sm.abort_flag;
    if (warp == 0 && lane < 3) prefetch_map(lane == 0 ? &map_w : lane == 1 ? &map_x : &map_u);
    if (warp == 1) {
        for (int i = lane; i < n; i += 32) {
            prefetch_2d(&map_w, (kb0 + i) * 64, n0);
            if (GATED) prefetch_2d(&map_u, (kb0 + i) * 64, n0);
        }
    }
    if (tid == 0) {
        for (int s = 0; s < stages; ++s) {
            mbar_init(&sm.full[s], STUCK && s == 1 ? 2 : 1);
            mbar_init(&sm.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sm.acc_full[b], 1);
            mbar_init(&sm.acc_empty[b], kSplitDrain);
        }
        mbar_init(&sm.drained, 1);
        sm.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem)), "r"(2 * kSplitTokens));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem;
    grid_dependency_wait();
    grid_launch_dependents();
    const uint32_t full = smem_u32(sm.full), empty = smem_u32(sm.empty), acc_full = smem_u32(sm.acc_full), acc_empty = smem_u32(sm.acc_empty), ring_at = smem_u32(ring);
    bool ok = true;
    float acc[64];
    if (warp == 0) {
        int i = 0, s = 0, turn = 0;
        for (; i < n; ++i) {
            if (turn > 0) ok = mbar_wait_warp(empty + 8 * s, (turn - 1) & 1, abort_flag, &g_linear_status, budget);
            if (!ok) break;
            if (elect_one()) {
                const uint32_t at = ring_at + s * stage_bytes;
                const int k = (kb0 + i) * 64;
                mbar_expect_tx(&sm.full[s], (uint32_t)stage_bytes);
                tma_load_2d(at, &map_w, k, n0, &sm.full[s]);
                if (GATED) tma_load_2d(at + kABytes / 2, &map_u, k, n0, &sm.full[s]);
                tma_load_2d(at + kABytes, &map_x, k, t0, &sm.full[s]);
            }
            __syncwarp();
            if (++s == stages) {
                s = 0;
                ++turn;
            }
        }
        if (!ok)                                                           // the copies in flight end before their memory is used again
            for (int j = 0; j < stages; ++j)
                if (turn > 0 || j < s) in_flight_end(full + 8 * j, (j < s ? turn : turn - 1) & 1, budget);
    } else if (warp == 1) {
        const uint32_t idesc = make_idesc(BN);
        const uint64_t da0 = make_desc_b(ring_at), db0 = make_desc_b(ring_at + kABytes);
        int s = 0;
        uint32_t turn = 0;
        for (int i = 0; i < n; ++i) {
            const int c = i / kChain, buf = c & 1;
            if (i % kChain == 0 && c >= 2) ok = mbar_wait_warp(acc_empty + 8 * buf, (c / 2 - 1) & 1, abort_flag, &g_linear_status, budget);
            if (ok) ok = mbar_wait_warp(full + 8 * s, turn, abort_flag, &g_linear_status, budget);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t off = (uint64_t)(s * stage_bytes >> 4);
#pragma unroll
                for (int j = 0; j < 4; ++j)                                // K = 16: 32 bytes on
                    mma_one(tmem + buf * kSplitTokens, da0 + off + 2 * j, db0 + off + 2 * j, idesc, j > 0 || i % kChain > 0);
                tc_commit_at(empty + 8 * s);
                if (i % kChain == kChain - 1 || i == n - 1) tc_commit_at(acc_full + 8 * buf);
            }
            __syncwarp();
            if (++s == stages) {
                s = 0;
                turn ^= 1;
            }
        }
        if (!ok) {                                                         // given up: the MMAs in flight end before their operands' memory is used again
            if (elect_one()) tc_commit_at(smem_u32(&sm.drained));
            __syncwarp();
            in_flight_end(smem_u32(&sm.drained), 0, budget);
        }
    } else if (warp >= 4) {
        const int chains = (n + kChain - 1) / kChain;
        for (int c = 0; c < chains; ++c) {
            const int buf = c & 1;
            ok = mbar_wait_warp(acc_full + 8 * buf, (c >> 1) & 1, abort_flag, &g_linear_status, budget);
            if (!ok) break;
            tc_fence_after();
            drain(tmem + ((uint32_t)(32 * (warp & 3)) << 16) + buf * kSplitTokens, BN, c == 0, acc);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(acc_empty + 8 * buf);
        }
    }
    Finish<O, GATED, PEERS> finish(a, n0, t0, rank, CL, BN, tid);
    __syncthreads();                                                       // the ring has been read (or is given up), the accumulators too
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * kSplitTokens));
    if (warp >= 4) {
        float* part = reinterpret_cast<float*>(ring) + 32 * (warp & 3) + lane;
#pragma unroll
        for (int i = 0; i < 64; ++i)
            if (i < BN) part[i * BM] = acc[i];
    }
    if (CL > 1) {
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }
    finish(ring_at);
    if (CL > 1) {
        cluster_arrive();                                                  // nobody reads this CTA's shared memory any more
        cluster_wait();
    }
}

template <typename O, bool GATED, int PEERS, bool STUCK = false>
int launch_split(const LinearArgs& a, int BN, int CL, bool wide, cudaStream_t st) {
    constexpr int kRows = GATED ? BM / 2 : BM;
    alignas(64) CUtensorMap mw, mu, mx;
    if (encode_map(&mw, a.w, a.N, a.K, a.ld_w, kRows) || encode_map(&mu, GATED ? a.w_up : a.w, a.N, a.K, GATED ? a.ld_up : a.ld_w, kRows) ||
        encode_map(&mx, a.x, a.T, a.K, a.ld_x, BN))
        return EXMOE_ERR_CUDA;
    static SmemOnce once;
    const auto kern = linear_split_kernel<O, GATED, PEERS, STUCK>;
    static_assert(2 * (kSplitRoom + 2048 + 1024) <= 228 * 1024 && kSplitRoomWide + 2048 <= 227 * 1024, "shared memory of two CTAs, of one");
    if (!allow_smem(kern, kSplitRoomWide + 2048, once)) return EXMOE_ERR_CUDA;
    const int row_tiles = (a.N + kRows - 1) / kRows;
    const long long ctas = (long long)row_tiles * ((a.T + BN - 1) / BN) * CL;
    if (ctas > INT32_MAX) return EXMOE_ERR_SHAPE;
    const int room = wide ? kSplitRoomWide : kSplitRoom, stages = std::min(kSplitStages, room / (kABytes + BN * 128));
    cudaLaunchConfig_t lc{};
    lc.gridDim = dim3((unsigned)ctas);
    lc.blockDim = dim3(kSplitThreads);
    lc.dynamicSmemBytes = (size_t)room + 2048;
    lc.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)CL;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = CL > 1 ? 2 : 1;
#ifdef EXMOE_DISABLE_PDL
    lc.attrs = attr + 1;
    --lc.numAttrs;
#endif
    if (cudaLaunchKernelEx(&lc, kern, mw, mu, mx, a, BN, CL, row_tiles, stages) != cudaSuccess) {
        cudaGetLastError();
        return EXMOE_ERR_CUDA;
    }
    count_launch();
    return EXMOE_OK;
}

// ---- pairs of CTAs ---------------------------------------------------------------------------------------------------
// 256 rows (128 in each CTA; 64 of W and 64 of U) by BN tokens (half of their operand in each CTA).  Both CTAs load; the first one's barriers count the bytes of both, its
// second warp issues the pair's MMAs, whose commits arrive in both.  16 warps of each CTA drain its half of the accumulators and finish the tile
// while the next one's chains run.  Bound by the tensor pipe: 4096 tokens 2048 -> 5632 with two matrices 125 us (92 % of its cycles, 1513 TFLOP/s); 8192 tokens 2048 -> 2048
// with residuals 52 us (78 %: the four rounds' last tiles are finished in the open).
constexpr int kPairThreads = 32 * 20, kPairTokens = 256, kDrainWarps = 16;
constexpr int kPairStage = kABytes + kPairTokens / 2 * 128;
template <bool GATED>
struct __align__(1024) PairShared {
    static constexpr int kStages = GATED ? 5 : 6;
    unsigned char ring[kStages][kPairStage];
    float meet[GATED ? kDrainWarps : 1][GATED ? 4 : 1][8][32];             // the factors that a warp's partner needs
    uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], drained;
    uint32_t tmem;
    int abort_flag;
};

__device__ __forceinline__ void mma_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void commit_pair(uint32_t bar) {                // arrives at this barrier in both CTAs
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((unsigned short)3) : "memory");
}
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {    // `bar` may be the other CTA's
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");     // (released to the cluster it would wait for the stores before it)
}
__device__ __forceinline__ void two_warps_sync(int barrier) {
    __syncwarp();
    asm volatile("barrier.cta.sync.aligned %0, 64;" ::"r"(barrier) : "memory");
}

// Eight tokens of a warp's 32 outputs: read, finished, written.  Addresses are a base that all lanes share and 32 bits of a lane's own: steps from token
// to token are then uniform instructions, and a call without residuals or with whole runs has none of their predicates (21 instructions per element
// otherwise, and a product of K = 512 takes twice as long as its MMAs).
template <typename O>
struct Outputs {
    const char* res;                                                       // of the first token's first output; null without one
    char* out;
    long long res_step, out_step;                                          // bytes from token to token
    int left, act;                                                         // tokens that exist
    uint32_t lane_at;                                                      // bytes
    bool in;                                                               // this lane's output exists
    __device__ __forceinline__ void load(int c, O (&r)[8]) const {
        if (!res || !in) return;
        const char* p = res + c * res_step;
        if (c + 8 <= left) {
#pragma unroll
            for (int i = 0; i < 8; ++i, p += res_step) r[i] = *reinterpret_cast<const O*>(p + lane_at);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i, p += res_step)
                if (c + i < left) r[i] = *reinterpret_cast<const O*>(p + lane_at);
        }
    }
    __device__ __forceinline__ void store(int c, float (&v)[8], const O (&r)[8]) const {
        if (!in) return;
        if (res) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += (float)r[i];
        }
        char* p = out + c * out_step;
        if (c + 8 <= left) {
#pragma unroll
            for (int i = 0; i < 8; ++i, p += out_step) store_out(reinterpret_cast<O*>(p + lane_at), v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i, p += out_step)
                if (c + i < left) store_out(reinterpret_cast<O*>(p + lane_at), v[i]);
        }
    }
};
// The pairs work side by side on tiles of kGroup rows of tiles and as many columns as it takes: what they read at a time is then few weights and few
// tokens (8192 tokens, 8192 -> 8192 outputs: 700 us instead of 805 along whole columns; 4 and 16 rows of tiles are no faster).
constexpr int kGroup = 8;
struct TileAt { int row, token; };
__device__ __forceinline__ TileAt tile_at(int tile, int row_tiles, int token_tiles) {
    const int group = tile / (kGroup * token_tiles), in_group = tile - group * kGroup * token_tiles, rows = min(kGroup, row_tiles - group * kGroup);
    return {group * kGroup + in_group % rows, in_group / rows};
}

// CHAIN: stages of a chain of MMAs; 0: all of K is one.
template <typename O, bool GATED, int CHAIN, bool STUCK>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
linear_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_u, const __grid_constant__ CUtensorMap map_x,
                   const __grid_constant__ LinearArgs a, int BN, int row_tiles, int token_tiles) {
    using S = PairShared<GATED>;
    extern __shared__ unsigned char raw[];
    S& sm = *reinterpret_cast<S*>(raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u));
    constexpr int kRows = GATED ? BM / 2 : BM;                             // outputs of a CTA's half of a tile
    constexpr long long budget = STUCK ? kWaitBudgetTest : kWaitBudget;
    const int tid = threadIdx.x, lane = tid & 31, warp = warp_uniform(tid >> 5);
    const int rank = (int)blockIdx.x & 1, pair = (int)blockIdx.x >> 1, pairs = (int)gridDim.x >> 1, tiles = row_tiles * token_tiles;
    volatile int* abort_flag = &sm.abort_flag;
    if (tid == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(&sm.full[s], STUCK && s == 1 ? 2 : 1);
            mbar_init(&sm.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sm.acc_full[b], 1);
            mbar_init(&sm.acc_empty[b], 2 * kDrainWarps);
        }
        mbar_init(&sm.drained, 1);
        sm.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0 && lane < 3) prefetch_map(lane == 0 ? &map_w : lane == 1 ? &map_x : &map_u);
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem)), "r"(2 * kPairTokens));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::);
    }
    tc_fence_before();
    cluster_arrive();
    cluster_wait();
    tc_fence_after();
    const uint32_t tmem = sm.tmem;
    grid_dependency_wait();
    grid_launch_dependents();
    constexpr bool kChained = CHAIN > 0;
    const int blocks = (a.K + 63) / 64, per_chain = kChained ? CHAIN : blocks, chains = (blocks + per_chain - 1) / per_chain;
    const uint32_t full = smem_u32(sm.full), empty = smem_u32(sm.empty), acc_full = smem_u32(sm.acc_full), acc_empty = smem_u32(sm.acc_empty);
    const uint32_t ring = smem_u32(sm.ring[0]);
    bool ok = true;
    if (warp == 0) {
        const uint32_t first_full = at_rank(full, 0);
        int s = 0, turn = 0;                                               // stage, turns of the ring
        for (int tile = pair; tile < tiles && ok; tile += pairs) {
            const TileAt at_tile = tile_at(tile, row_tiles, token_tiles);
            const int n0 = (at_tile.row * 2 + rank) * kRows, t0 = at_tile.token * BN + rank * (BN / 2);
            for (int i = 0; i < blocks; ++i) {
                if (turn > 0) ok = mbar_wait_warp(empty + 8 * s, (turn - 1) & 1, abort_flag, &g_linear_status, budget);
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t at = ring + s * kPairStage, bar = first_full + 8 * s;
                    if (rank == 0) mbar_expect_tx(&sm.full[s], 2 * (uint32_t)(kABytes + BN / 2 * 128));
                    tma_load_pair(at, &map_w, i * 64, n0, bar);
                    if (GATED) tma_load_pair(at + kABytes / 2, &map_u, i * 64, n0, bar);
                    tma_load_pair(at + kABytes, &map_x, i * 64, t0, bar);
                }
                __syncwarp();
                if (++s == S::kStages) {
                    s = 0;
                    ++turn;
                }
            }
        }
        if (!ok && rank == 0)                                              // the copies in flight end (the other CTA's are counted here too)
            for (int j = 0; j < S::kStages; ++j)
                if (turn > 0 || j < s) in_flight_end(full + 8 * j, (j < s ? turn : turn - 1) & 1, budget);
    } else if (warp == 1 && rank == 0) {
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(2 * BM >> 4) << 24);
        const uint64_t da0 = make_desc_b(ring), db0 = make_desc_b(ring + kABytes);
        int s = 0, chain = 0, in_chain = 0;
        uint32_t turn = 0;
        for (int tile = pair; tile < tiles && ok; tile += pairs) {
            for (int i = 0; i < blocks; ++i) {
                const int buf = chain & 1;
                if (in_chain == 0 && chain >= 2) ok = mbar_wait_warp(acc_empty + 8 * buf, (chain / 2 - 1) & 1, abort_flag, &g_linear_status, budget);
                if (ok) ok = mbar_wait_warp(full + 8 * s, turn, abort_flag, &g_linear_status, budget);
                if (!ok) break;
                tc_fence_after();
                const bool ends = in_chain == per_chain - 1 || i == blocks - 1;
                if (elect_one()) {
                    const uint64_t off = (uint64_t)(s * kPairStage >> 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j)                            // K = 16: 32 bytes on
                        mma_pair(tmem + buf * kPairTokens, da0 + off + 2 * j, db0 + off + 2 * j, idesc, j > 0 || in_chain > 0);
                    commit_pair(empty + 8 * s);
                    if (ends) commit_pair(acc_full + 8 * buf);
                }
                __syncwarp();
                in_chain = ends ? 0 : in_chain + 1;
                chain += ends;
                if (++s == S::kStages) {
                    s = 0;
                    turn ^= 1;
                }
            }
        }
        if (!ok) {                                                         // the MMAs in flight end
            if (elect_one()) asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(&sm.drained)) : "memory");
            __syncwarp();
            in_flight_end(smem_u32(&sm.drained), 0, budget);
        }
    } else if (warp >= 4) {
        const int d = warp - 4, quarter = warp & 3, group = d >> 2, cw = BN / 4;   // a quarter of the columns, on the warp's 32 lanes
        const bool is_up = GATED && quarter >= 2;
        const uint32_t my_empty = at_rank(acc_empty, 0);
        // A tile's residuals are requested into L2 while its sums are made, unless they are BF16 and a pair's other tiles hide them in a long K (us with / without: 8192 tokens
        // 64 -> 2048 21.6 / 24.9, 1024 -> 2048 32.4 / 33.3, 2048 -> 2048 53.1 / 52.1, FP32 73.3 / 76.2; one round of tiles, 2048 tokens 2048 -> 2048 18.5 / 18.9).
        const bool into_l2 = kChained || tiles <= pairs || blocks <= 16;
        const uint32_t lanes = tmem + ((uint32_t)(32 * quarter) << 16) + group * cw;
        int chain = 0;
        for (int tile = pair; tile < tiles; tile += pairs) {               // (a warp that has given up stores nothing, but keeps its appointments)
            const TileAt at_tile = tile_at(tile, row_tiles, token_tiles);
            const int n0 = (at_tile.row * 2 + rank) * kRows + 32 * (GATED ? quarter & 1 : quarter), nn = n0 + lane;
            const long long t0 = (long long)at_tile.token * BN + group * cw;
            const float* b = is_up ? a.bias_up : a.bias;
            const float bias = b && nn < a.N ? b[nn] : 0.f;
            Outputs<O> to{a.residual ? static_cast<const char*>(a.residual) + (t0 * a.ld_res + n0) * (int)sizeof(O) : nullptr,
                          static_cast<char*>(a.out) + (t0 * a.ld_out + n0) * (int)sizeof(O), a.ld_res * (int)sizeof(O), a.ld_out * (int)sizeof(O),
                          (int)max(0ll, min((long long)cw, a.T - t0)), a.act, lane * (uint32_t)sizeof(O), nn < a.N};
            // The runs of eight tokens that this warp finishes: with a second factor lanes of W the even ones, lanes of U the odd ones.  Residuals are
            // requested two of them ahead, the first ones before the tile's sums are there.
            constexpr int kStep = GATED ? 16 : 8;
            const int c_first = GATED && is_up ? 8 : 0;
            if (into_l2 && to.res && n0 < a.N)
                for (int i = lane; i < min(cw, to.left); i += 32) asm volatile("prefetch.global.L2 [%0];" ::"l"(to.res + i * to.res_step));
            O res[2][8];
            if (c_first < cw) to.load(c_first, res[0]);
            if (c_first + kStep < cw) to.load(c_first + kStep, res[1]);
            int buf = chain & 1;
            if (kChained && chains > 1) {
                // the chains' sums go back to where the last one was
                float acc[64];
                for (int c = 0; c < chains && ok; ++c, ++chain) {
                    buf = chain & 1;
                    ok = mbar_wait_warp(acc_full + 8 * buf, (chain >> 1) & 1, abort_flag, &g_linear_status, budget);
                    if (!ok) break;
                    tc_fence_after();
                    drain(lanes + buf * kPairTokens, cw, c == 0, acc);
                    if (c == chains - 1) break;
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_cluster(my_empty + 8 * buf);
                }
                if (ok) {
#pragma unroll
                    for (int c = 0; c < 64; c += 8)
                        if (c < cw) tmem_st8(lanes + buf * kPairTokens + c, acc + c);
                    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                }
                ++chain;
            } else {
                if (ok) ok = mbar_wait_warp(acc_full + 8 * buf, (chain >> 1) & 1, abort_flag, &g_linear_status, budget);
                tc_fence_after();
                ++chain;
            }
            if (!ok) to.in = false;
            const auto sums = [&](int c, float (&v)[8]) {                  // eight columns from c on, bias included
                uint32_t r[8];
                tmem_ld8(lanes + buf * kPairTokens + c, r);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]) + bias;
            };
            const int partner = d ^ 2, barrier = 1 + (d & 1) + 2 * group;
            if constexpr (GATED) {
#pragma unroll 1
                for (int c = 8 - c_first; c < cw; c += 16) {
                    float v[8];
                    sums(c, v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sm.meet[d][c >> 4][i][lane] = v[i];
                }
                two_warps_sync(barrier);
            }
            const auto finish = [&](int c, O (&r)[8]) {
                float v[8];
                sums(c, v);
                if constexpr (GATED) {
                    float other[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float o = sm.meet[partner][c >> 4][i][lane];
                        other[i] = is_up ? v[i] : o;
                        v[i] = is_up ? o : v[i];
                    }
                    activate_all(v, a.act);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] *= other[i];
                } else {
                    activate_all(v, a.act);
                }
                to.store(c, v, r);
                if (c + 2 * kStep < cw) to.load(c + 2 * kStep, r);
            };
#pragma unroll 1
            for (int c = c_first; c < cw; c += 2 * kStep) {
                finish(c, res[0]);
                if (c + kStep < cw) finish(c + kStep, res[1]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_cluster(my_empty + 8 * buf);
            if constexpr (GATED) two_warps_sync(barrier);
        }
    }
    tc_fence_before();
    cluster_arrive();                                                      // neither CTA's memory nor barriers are in use any more
    cluster_wait();
    tc_fence_after();
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * kPairTokens));
}

// Chains in front of a BF16 result are as long as K up to kLongChain stages, 1024 MMAs, and stay in tensor memory until they are finished.  Each truncates by
// 1e-7 of what it has summed (measured: 1e-4 over 1024 of them where all products have one sign, a fortieth of a BF16 half step; 6e-3, more than a whole one, over 65536).
constexpr int kLongChain = 256;
template <typename O, bool GATED, int CHAIN, bool STUCK>
int launch_pair(const LinearArgs& a, int BN, cudaStream_t st) {
    using S = PairShared<GATED>;
    constexpr int kRows = GATED ? BM / 2 : BM;
    alignas(64) CUtensorMap mw, mu, mx;
    if (encode_map(&mw, a.w, a.N, a.K, a.ld_w, kRows) || encode_map(&mu, GATED ? a.w_up : a.w, a.N, a.K, GATED ? a.ld_up : a.ld_w, kRows) ||
        encode_map(&mx, a.x, a.T, a.K, a.ld_x, BN / 2))
        return EXMOE_ERR_CUDA;
    static SmemOnce once;
    const auto kern = linear_pair_kernel<O, GATED, CHAIN, STUCK>;
    constexpr int smem = (int)sizeof(S) + 1024;
    static_assert(smem <= 227 * 1024, "shared memory");
    if (!allow_smem(kern, smem, once)) return EXMOE_ERR_CUDA;
    const int row_tiles = (a.N + 2 * kRows - 1) / (2 * kRows);
    const long long tiles = (long long)row_tiles * ((a.T + BN - 1) / BN);
    if (tiles > INT32_MAX) return EXMOE_ERR_SHAPE;
    cudaLaunchConfig_t lc{};
    lc.gridDim = dim3(2 * (unsigned)std::min<long long>(tiles, kSms / 2));
    lc.blockDim = dim3(kPairThreads);
    lc.dynamicSmemBytes = smem;
    lc.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
#ifdef EXMOE_DISABLE_PDL
    lc.numAttrs = 0;
#endif
    if (cudaLaunchKernelEx(&lc, kern, mw, mu, mx, a, BN, row_tiles, (a.T + BN - 1) / BN) != cudaSuccess) {
        cudaGetLastError();
        return EXMOE_ERR_CUDA;
    }
    count_launch();
    return EXMOE_OK;
}

// How many clusters of one to eight CTAs the device holds at once, with one CTA per SM and with two.  (GPCs differ in their SMs, devices in their GPCs:
// 15 clusters of eight CTAs, 22 of six, 33 of four, 74 of two where these figures were taken.)
constexpr int kMostCluster = 8;
struct Clusters { int wide[kMostCluster + 1], narrow[kMostCluster + 1]; };
const Clusters* clusters_held() {
    static Clusters held[64];
    static std::once_flag once[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
    std::call_once(once[dev], [dev] {
        const auto kern = linear_split_kernel<float, false, 8, false>;
        cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSplitRoomWide + 2048);
        for (int c = 1; c <= kMostCluster; ++c)
            for (int wide = 0; wide < 2; ++wide) {
                cudaLaunchConfig_t lc{};
                lc.gridDim = dim3((unsigned)c);
                lc.blockDim = dim3(kSplitThreads);
                lc.dynamicSmemBytes = (wide ? kSplitRoomWide : kSplitRoom) + 2048;
                cudaLaunchAttribute attr[1];
                attr[0].id = cudaLaunchAttributeClusterDimension;
                attr[0].val.clusterDim.x = (unsigned)c;
                attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
                lc.attrs = attr;
                lc.numAttrs = 1;
                int n = 0;
                if (cudaOccupancyMaxActiveClusters(&n, kern, &lc) != cudaSuccess) {
                    cudaGetLastError();
                    n = 0;
                }
                (wide ? held[dev].wide : held[dev].narrow)[c] = n;
            }
    });
    return &held[dev];
}

// Which form, and its tile, by what they take in clocks of an SM (1.9 GHz): from the times below, each model within 15 % of them or so.
//   pair    a stage what shared memory takes for four k-steps' operands, 4 (64 + BN / 4), a tile 1500 besides, a call 6000
//   split   a stage its bytes at 57 a clock (what an SM takes in), twice where SMs are shared; a call 8000, 250 for every part of the exchange and 1500 for
//           clusters of more than four CTAs, which start late once they are many
//   both    weights from HBM at 3400 bytes a clock, and 10000 (7000) besides
// us, replayed from a graph, weights from HBM, split in clusters of 2 / 3 / 4 / 6 and pair: 64 tokens of 2048 -> 2048 9.2 / 7.1 / 6.7 / 7.1 and 9.6; 45 of 5632 -> 2048
// 14.3 / 11.1 / 10.4 / 10.1 and 20.3; 45 of 2048 -> 5632 with two matrices 13.5 / 11.7 / 16 / 18 and 13.2; 512 of 2048 -> 2048 12 (split at best) and 9.5.
template <typename O, bool GATED, bool STUCK = false>
int launch_tc(const LinearArgs& a, cudaStream_t st) {
    const int row_tiles = (a.N + (GATED ? 63 : 127)) / (GATED ? 64 : 128), blocks = (a.K + 63) / 64;
    const long long pair_rows = (row_tiles + 1) / 2;
    int pair_BN = 256;
    long long pair_cost = INT64_MAX;
    for (int BN = 256; BN >= 64; BN -= 32) {
        const long long rounds = (pair_rows * ((a.T + BN - 1) / BN) + kSms / 2 - 1) / (kSms / 2), cost = rounds * (blocks * (long long)(256 + BN) + 1500) + 6000;
        if (cost < pair_cost) {
            pair_cost = cost;
            pair_BN = BN;
        }
    }
    const long long from_hbm = (GATED ? 4ll : 2ll) * a.N * a.K / 3400;
    pair_cost = std::max(pair_cost, from_hbm + 10000);
    const int BN = a.T >= 64 ? 64 : (a.T + 15) / 16 * 16, stage = kABytes + BN * 128;
    const long long tiles = (long long)row_tiles * ((a.T + BN - 1) / BN);
    const Clusters* held = clusters_held();
    int CL = 1;
    bool wide = false;
    long long split_cost = INT64_MAX;
    for (int c = 1; held && c <= std::min(kMostCluster, std::max(1, blocks / 2)); ++c) {
        if (held->narrow[c] <= 0) continue;
        const int n = (blocks + c - 1) / c;
        const bool alone = tiles <= held->wide[c];
        const long long turns = alone ? 1 : 2 * ((tiles + held->narrow[c] - 1) / held->narrow[c]), cost = turns * n * (stage / 57) + 8000 + 250 * c + (c > 4 && tiles * c > 64 ? 1500 : 0);
        if (cost < split_cost) {
            split_cost = cost;
            CL = c;
            wide = alone && (long long)n * stage > 280 * 1024;              // (8 stages of 24 KB: 8.2 us wide, 6.7 with room for the next call's CTAs; 16: 10.5, 11.6)
        }
    }
    if (pair_cost < std::max(split_cost, from_hbm + 7000)) {
        if constexpr (sizeof(O) == 4) return launch_pair<O, GATED, kChain, STUCK>(a, pair_BN, st);
        else return blocks <= kLongChain ? launch_pair<O, GATED, 0, STUCK>(a, pair_BN, st) : launch_pair<O, GATED, kLongChain, STUCK>(a, pair_BN, st);
    }
    if constexpr (STUCK) return launch_split<O, GATED, 8, true>(a, BN, CL, wide, st);
    if (CL <= 2) return launch_split<O, GATED, 2>(a, BN, CL, wide, st);
    return CL <= 4 ? launch_split<O, GATED, 4>(a, BN, CL, wide, st) : launch_split<O, GATED, 8>(a, BN, CL, wide, st);
}

}  // namespace

int launch_linear_tc(const LinearArgs& a, int type, cudaStream_t st) {
    if (type == EXMOE_F32) return a.w_up ? launch_tc<float, true>(a, st) : launch_tc<float, false>(a, st);
    return a.w_up ? launch_tc<__nv_bfloat16, true>(a, st) : launch_tc<__nv_bfloat16, false>(a, st);
}

int launch_linear_tc_stuck(const LinearArgs& a, cudaStream_t st) { return launch_tc<__nv_bfloat16, false, true>(a, st); }

extern "C" int exmoe_linear_status(void) {
    int v = 0;
    const int zero = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&v, g_linear_status, sizeof v) != cudaSuccess ||
        (v && cudaMemcpyToSymbol(g_linear_status, &zero, sizeof zero) != cudaSuccess))
        return EXMOE_ERR_CUDA;
    return v;
}

}  // namespace exmoe
