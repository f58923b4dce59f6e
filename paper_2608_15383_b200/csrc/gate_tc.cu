// The gate on many tokens: the logits as a GEMM on tcgen05, then the choice, in one kernel.
//
// A cluster of CL CTAs (as many, up to eight, as 148 SMs have room for) takes 128 tokens, the MMA's M; each multiplies a CL-th of K by
// all experts, its N = MT x 128.  Tokens and weights come by TMA into a ring of kStages 64-wide stages.
//   Rounding, as measured (no document states it; the bound below takes more than was seen).  An MMA truncates: every product to 2^-25 of the binade of the largest one (or of the accumulator), its result to 24 bits; at
// most 17 / 4 + 1 = 5.25 units of 2^-23 of the magnitudes summed so far.  In one chain over K, each MMA would lose that much of all that
// the ones before have summed, H / 16 times.  So only kChain stages (8 MMAs) make a chain that starts from zero; sixteen warps take its
// accumulator out of tensor memory, which has two of them, and add it to binary32 sums in registers behind the next chain's MMAs.
// What is left is bounded in the units that decide (`cost` below): the products of an MMA count once for it and each that follows in its
// chain, and once for every addition behind that, and with weighted norms, summed by the same warps from the stages' tiles, Cauchy's
// inequality gives dz = 2^-24 sqrt(sum c |x|^2) sqrt(sum c |w|^2).  With chains of one stage the main loop took 50 thousand cycles instead of 40
// (gate below; twice as many drains), and the bounds of longer ones mark more.
//   Choice.  The partial logits go to shared memory; the CTA that owns a token (128 / CL each) adds the CL parts, and a warp chooses
// (gate.cuh).  Where a decision rests on less than the bound, the token waits; behind the others, all sixteen warps compute the logits that
// matter in binary64, a warp per logit, and its choice goes on.
//   What bounds it, at 8192 tokens of d_model 4096, 256 experts, 8 of 4 of 8 groups by the two largest, sigmoid with a balance bias (64
// clusters of two): 58.8 us replayed from a graph, of 91 thousand cycles per CTA (106 in the last) 38 in the main loop, 31 in its 64 tokens' exchange and
// choices, 17 in the near-ties (3 tokens, 8 logits), the rest in barriers.  The main loop runs at the rate of shared memory (a stage's 48 KB come in by TMA and
// go out to the MMAs and to the norms: 1,150 cycles at 128 bytes each; the tensor pipe is busy for 17 % of the kernel), the choices at that of
// instructions, the near-ties at the latency of code that few tokens run.  The bytes alone would take 10.8 us.  With eight CTAs per cluster (up to 2048 tokens) the
// exchange takes 9 of 40 thousand cycles.
#include <algorithm>

#include "gate.cuh"
#include "mbar.cuh"
#include "tc.cuh"

namespace exmoe {

namespace {

constexpr int kTokens = 128, kStages = 4, kChain = 2, kDrainWarps = 16, kThreads = 32 * (4 + kDrainWarps), kPad = 4;
constexpr int kRowBytes = 128;                                             // 64 elements
__device__ int g_gate_status;                                              // sticky: EXMOE_ERR_TIMEOUT

__device__ __forceinline__ void mma_f16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr));
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
__device__ __forceinline__ float ld_rank(uint32_t addr, int rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at_rank(addr, rank)) : "memory");
    return v;
}
// The parts of a token's logits, added to z [32 PER], and of its size: from this CTA's on, four CTAs' in flight.  A lane's pieces of 16
// bytes (8: PER = 2) are as far apart as a warp reads at once.
template <int PER>
__device__ __forceinline__ void load_logits(uint32_t part, uint32_t size_at, int rank, int CL, int lane, float* z, float& size) {
    constexpr int W = PER == 2 ? 2 : 4, N = PER / W;
    float v[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) v[j] = 0.f;
    for (int i0 = 0; i0 < CL; i0 += 4) {
        float from[4][PER], s[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i0 + i < CL) {
                const uint32_t at = at_rank(part, (rank + i0 + i) & (CL - 1)) + 4 * W * lane;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if constexpr (W == 2)
                        asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];" : "=f"(from[i][0]), "=f"(from[i][1]) : "r"(at) : "memory");
                    else
                        asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];"
                                     : "=f"(from[i][4 * j]), "=f"(from[i][4 * j + 1]), "=f"(from[i][4 * j + 2]), "=f"(from[i][4 * j + 3]) : "r"(at + 512 * j) : "memory");
                }
                s[i] = ld_rank(size_at, (rank + i0 + i) & (CL - 1));
            }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i0 + i < CL) {
#pragma unroll
                for (int j = 0; j < PER; ++j) v[j] += from[i][j];
                size += s[i];
            }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if constexpr (W == 2)
            *reinterpret_cast<float2*>(z + 2 * lane) = make_float2(v[0], v[1]);
        else
            *reinterpret_cast<float4*>(z + 4 * lane + 128 * j) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
    }
    __syncwarp();
}
__device__ __forceinline__ void add_pair(float& a, float& b, uint32_t x, uint32_t y) {      // two binary32 additions in one instruction
    asm("{\n\t.reg .b64 s, t;\n\tmov.b64 s, {%0, %1};\n\tmov.b64 t, {%2, %3};\n\tadd.rn.f32x2 s, s, t;\n\tmov.b64 {%0, %1}, s;\n\t}" : "+f"(a), "+f"(b) : "r"(x), "r"(y));
}
// sum of squares of 16 bytes of BF16, in pairs of BF16 sums: short by less than 4 2^-9 of itself
__device__ __forceinline__ void square(__nv_bfloat162& sum, const uint4& v) {
    const uint32_t r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = *reinterpret_cast<const __nv_bfloat162*>(&r[i]);
        sum = __hfma2(p, p, sum);
    }
}

__device__ __forceinline__ void in_flight_end(uint32_t bar, uint32_t parity, long long budget) {
    const long long t0 = clock64();
    while (!mbar_try_at(bar, parity) && clock64() - t0 < budget) {}
}

// the choosing warps' barrier
__device__ __forceinline__ void choosers_sync() {
    __syncwarp();
    asm volatile("barrier.cta.sync.aligned 1, %0;" ::"n"(32 * kDrainWarps) : "memory");
}
__device__ __forceinline__ bool choosers_or(bool v) {
    uint32_t r;
    __syncwarp();
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred.aligned q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)v), "n"(32 * kDrainWarps) : "memory");
    return r != 0;
}

template <int PER>
struct Warp {                                                              // a choosing warp's share of shared memory
    ChoiceRoom<PER> room;
    double z64[32 * PER];                                                  // logits computed again
};
constexpr int kTodoUsed = 10;
__device__ __forceinline__ int todo_at(int i) { return i < 8 ? i : kTodoKept + i - 8; }
constexpr int kParts = 2 * kDrainWarps;
constexpr int kItems = 512;                                               // two tokens with all of their logits
// A token that waits for logits to be computed again; its logits are back in its row of `part`, which no other CTA reads.
struct Waiting {
    int token, first;                                                      // in the tile; first item | how many << 16, -1: there was no room for them
    float dz;
    uint32_t todo[kTodoUsed];                                              // the words of 256 experts, kTodoKept, kTodoStage
    Picks picks;
};
template <int MT, int PER>
struct __align__(1024) Shared {
    static constexpr int kStage = (MT * 128 + kTokens) * kRowBytes;
    union {
        unsigned char ring[kStages][kStage];                               // weights, then tokens; rows of 128 bytes, swizzled
        struct {
            float part[kTokens][MT * 128 + kPad];                          // this CTA's part of the logits, read by the cluster; rows four banks apart
            Warp<PER> warp[kDrainWarps];
        } s;
    };
    float size[kTokens], balance[32 * PER];
    float w2_max[kDrainWarps];
    int n_waiting, n_items, wide;
    Waiting waiting[kTokens];
    double item_z[kItems];                                                 // logits to compute again
    unsigned short item_expert[kItems], item_waiting[kItems];
    uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], drained;
    uint32_t tmem;
    int abort_flag;
};

// STUCK (exmoe_debug_gate_timeout): the second stage's barrier asks for an arrival that nobody makes.
template <int MT, int PER, bool STUCK>
__global__ void __launch_bounds__(kThreads, 1)
gate_tc_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const __nv_bfloat16* hidden,
               const __nv_bfloat16* __restrict__ w_router, const float* __restrict__ bias, const float* addend, int T, int H,
               const __grid_constant__ GateArgs g, int CL, int32_t* ids, float* weights) {
    using S = Shared<MT, PER>;
    constexpr long long budget = STUCK ? kWaitBudgetTest : kWaitBudget;
    constexpr int COLS = MT * 128 / 4;                      // accumulator columns of a drain warp: a quarter of them, on its 32 lanes
    extern __shared__ unsigned char raw[];
    S& sm = *reinterpret_cast<S*>(raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u));
    const int tid = threadIdx.x, lane = tid & 31, warp = warp_uniform(tid >> 5);
    const int rank = (int)blockIdx.x % CL, t0 = (int)blockIdx.x / CL * kTokens;
    volatile int* abort_flag = &sm.abort_flag;
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm.full[s], STUCK && s == 1 ? 2 : 1);
            mbar_init(&sm.empty[s], 1 + kDrainWarps);                      // the MMAs and the warps that add up the squares
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sm.acc_full[b], 1);
            mbar_init(&sm.acc_empty[b], kDrainWarps);
        }
        mbar_init(&sm.drained, 1);
        sm.abort_flag = 0;
        sm.n_waiting = sm.n_items = sm.wide = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem)), "r"(2 * MT * kTokens));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm.tmem;
    grid_dependency_wait();
    grid_launch_dependents();
    const int blocks = (H + 63) / 64, kb0 = blocks * rank / CL, n = blocks * (rank + 1) / CL - kb0;
    const uint32_t full = smem_u32(sm.full), empty = smem_u32(sm.empty), acc_full = smem_u32(sm.acc_full), acc_empty = smem_u32(sm.acc_empty);
    float acc[COLS], x2 = 0.f;
#pragma unroll
    for (int i = 0; i < COLS; ++i) acc[i] = 0.f;
    const int d = warp - 4, quarter = warp & 3;                            // drain warps: d of kDrainWarps
    const int col0 = (d >> 2) * COLS;                                      // token 32 quarter + lane, experts col0 ..
    bool ok = true;
    if (warp == 0) {
        // The ring unrolled, so that the MMAs' operands are constants away from two descriptors, and the next stage's barrier looked at
        // before this stage's MMAs: what stands between two MMAs is time that the tensor pipe may run dry.
        constexpr uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(MT * 128 >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);   // N: experts
        static_assert(kStages % (2 * kChain) == 0, "a turn of the ring leaves off where it began");
        constexpr int kTurns = kStages / (2 * kChain);                     // of the two accumulators in a turn of the ring
        const uint64_t dw0 = make_desc_b(smem_u32(sm.ring[0])), dx0 = make_desc_b(smem_u32(sm.ring[0]) + MT * 128 * kRowBytes);
        uint32_t turn = 0;                                                 // parity of the ring's turn
        bool ready = false;
        for (int i0 = 0; i0 < n && ok; i0 += kStages, turn ^= 1) {
#pragma unroll
            for (int s = 0; s < kStages; ++s) {
                if (i0 + s >= n) break;
                const int buf = s / kChain & 1, use = s / (2 * kChain), next = (s + 1) % kStages;
                if (s % kChain == 0 && (i0 > 0 || use > 0)) {              // the accumulator's use number i0 / kStages * kTurns + use
                    ok = mbar_wait_warp(acc_empty + 8 * buf, (kTurns % 2 ? turn + use + 1 : use + 1) & 1, abort_flag, &g_gate_status, budget);
                    if (!ok) break;
                }
                if (!ready) {
                    ok = mbar_wait_warp(full + 8 * s, turn, abort_flag, &g_gate_status, budget);
                    if (!ok) break;
                }
                tc_fence_after();
                const bool seen = i0 + s + 1 < n && mbar_look_at(full + 8 * next, next ? turn : turn ^ 1);
                if (elect_one()) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)                            // K = 16: 32 bytes on
                        mma_f16(tmem + buf * MT * 128, dx0 + (uint64_t)(s * S::kStage + 32 * j >> 4), dw0 + (uint64_t)(s * S::kStage + 32 * j >> 4), idesc,
                                j > 0 || s % kChain > 0);
                    tc_commit_at(empty + 8 * s);
                    if (s % kChain == kChain - 1 || i0 + s == n - 1) tc_commit_at(acc_full + 8 * buf);
                }
                __syncwarp();
                ready = __all_sync(0xffffffffu, seen);
            }
        }
        if (!ok) {                                                         // given up: the MMAs in flight end before their operands' memory is used again
            if (elect_one()) tc_commit_at(smem_u32(&sm.drained));
            __syncwarp();
            in_flight_end(smem_u32(&sm.drained), 0, budget);
        }
    } else if (warp == 1) {
        int i = 0;
        for (; i < n; ++i) {
            const int s = i % kStages;
            if (i >= kStages) ok = mbar_wait_warp(empty + 8 * s, (i / kStages - 1) & 1, abort_flag, &g_gate_status, budget);
            if (!ok) break;
            if (elect_one()) {
                mbar_expect_tx(&sm.full[s], S::kStage);
                tma_load_2d(smem_u32(sm.ring[s]), &map_w, (kb0 + i) * 64, 0, &sm.full[s]);
                tma_load_2d(smem_u32(sm.ring[s]) + MT * 128 * kRowBytes, &map_x, (kb0 + i) * 64, t0, &sm.full[s]);
            }
            __syncwarp();
        }
        for (int j = max(0, i - kStages); j < i; ++j) in_flight_end(full + 8 * (j % kStages), (j / kStages) & 1, budget);   // and so do the copies
    } else if (warp < 4) {
        for (int e = tid - 64; e < 32 * PER; e += 64) sm.balance[e] = g.balance && e < g.E ? g.balance[e] : 0.f;
    } else {
        // a quarter of a token's row, and a half (MT = 2) or a quarter of an expert's
        constexpr int WQ = MT == 2 ? 4 : 2;                                // 16-byte pieces
        const int u = tid - 128, xr = u >> 2, wr = MT == 2 ? u >> 1 : u >> 2;
        float w2 = 0.f;
        for (int i = 0; i < n; ++i) {
            const int s = i % kStages, c = i / kChain, buf = c & 1;
            ok = mbar_wait_warp(full + 8 * s, (i / kStages) & 1, abort_flag, &g_gate_status, budget);
            if (!ok) break;
            const __nv_bfloat162 zero(__float2bfloat16(0.f), __float2bfloat16(0.f));
            __nv_bfloat162 a[2] = {zero, zero}, b[WQ];
            const unsigned char *wt = sm.ring[s] + wr * kRowBytes, *xt = sm.ring[s] + (MT * 128 + xr) * kRowBytes;
            uint4 xv[2], wv[WQ];
#pragma unroll
            for (int j = 0; j < 2; ++j) xv[j] = *reinterpret_cast<const uint4*>(xt + ((((u & 3) * 2 + j) ^ (xr & 7)) << 4));
#pragma unroll
            for (int j = 0; j < WQ; ++j) wv[j] = *reinterpret_cast<const uint4*>(wt + ((((MT == 2 ? u & 1 : u & 3) * WQ + j) ^ (wr & 7)) << 4));
#pragma unroll
            for (int j = 0; j < 2; ++j) square(a[j], xv[j]);
#pragma unroll
            for (int j = 0; j < WQ; ++j) {
                b[j] = zero;
                square(b[j], wv[j]);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive_at(empty + 8 * s);
            // What is lost for the products of one MMA: 2 x 5.25 units of 2^-24 in it and in each that follows in its chain, an addition for each
            // chain from its own on, one per CTA; with S_j the products of MMA j and loss = sum c_j S_j <= sqrt(sum c_j |x_j|^2) sqrt(sum c_j |w_j|^2).
            auto cost = [&](int step) {
                return 10.5f * (float)(4 * kChain - 4 * (i % kChain) - step) + (float)((n - 1) / kChain - c + 1 + CL);
            };
            x2 = fmaf(cost(u & 3), __low2float(a[0]) + __high2float(a[0]) + (__low2float(a[1]) + __high2float(a[1])), x2);
#pragma unroll
            for (int j = 0; j < WQ; j += 2)
                w2 = fmaf(cost((MT == 2 ? 2 * (u & 1) : u & 3) + j / 2), __low2float(b[j]) + __high2float(b[j]) + (__low2float(b[j + 1]) + __high2float(b[j + 1])), w2);
            if (i % kChain < kChain - 1 && i < n - 1) continue;
            ok = mbar_wait_warp(acc_full + 8 * buf, (c >> 1) & 1, abort_flag, &g_gate_status, budget);
            if (!ok) break;
            tc_fence_after();
            const uint32_t at = tmem + ((uint32_t)(32 * quarter) << 16) + buf * MT * 128 + col0;
#pragma unroll
            for (int k = 0; k < COLS; k += 16) {
                uint32_t r[16];
                tmem_ld16(at + k, r);
                tc_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; j += 2) add_pair(acc[k + j], acc[k + j + 1], r[j], r[j + 1]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(acc_empty + 8 * buf);
        }
        x2 += __shfl_xor_sync(0xffffffffu, x2, 1);
        x2 += __shfl_xor_sync(0xffffffffu, x2, 2);
        w2 += __shfl_xor_sync(0xffffffffu, w2, 1);
        if (MT == 1) w2 += __shfl_xor_sync(0xffffffffu, w2, 2);
        if (!ok) w2 = INFINITY;                                            // nothing is known of the logits: all will be computed again
        w2 = warp_max(w2);                                                 // rows behind the last expert are zeros
        if (lane == 0) sm.w2_max[d] = w2;
    }
    __syncthreads();                                                       // the ring has been read, the accumulators too
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * MT * kTokens));
    if (warp >= 4) {
#pragma unroll
        for (int i = 0; i < COLS; i += 4)
            *reinterpret_cast<float4*>(&sm.s.part[32 * quarter + lane][col0 + i]) = make_float4(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
        float w2 = 0.f;
#pragma unroll
        for (int i = 0; i < kDrainWarps; ++i) w2 = fmaxf(w2, sm.w2_max[i]);
        const int c0 = 8 * kb0, chunks = min(8 * n, H / 8 - c0);           // this part of K
        if (w2 == 0.f) {                                                   // the same for all warps
            bool any = false;
            for (int e = d; e < g.E && !any; e += kDrainWarps) any = any_number(reinterpret_cast<const uint4*>(w_router + (size_t)e * H) + c0, chunks, lane, 32);
            w2 = choosers_or(any) ? kLeastSquare : 0.f;
        }
        const int u = tid - 128;                                           // the bound for this part, with the largest |w| of all experts
        for (unsigned rows = __ballot_sync(0xffffffffu, x2 == 0.f) & 0x11111111u; rows; rows &= rows - 1) {
            const int from = __ffs(rows) - 1;
            const long long t = t0 + ((u & ~31) + from >> 2);
            if (t < T && any_number(reinterpret_cast<const uint4*>(hidden + t * H) + c0, chunks, lane, 32) && lane == from) x2 = kLeastSquare;
        }
        if ((u & 3) == 0) sm.size[u >> 2] = w2 < INFINITY ? sqrtf(least_of(x2)) * sqrtf(least_of(w2)) : INFINITY;
    }
    cluster_arrive();
    cluster_wait();
    if (warp >= 4) {
        Warp<PER>& my = sm.s.warp[d];
        ChoiceRoom<PER>& room = my.room;
        const float* balance = g.balance ? sm.balance : nullptr;
        const float added = bias || addend ? kAddedRel : 0.f;
        const int owned = kTokens / CL, chunks = H / 8;
        // Round 0: the CTA's tokens.  The rounds behind it: those that wait, done by the warps together: first the logits, then the choices.
        for (int round = 0, n_tok = owned, log_p = 0;; ++round) {
            if (round > 0) {
                for (int f = d; f < n_tok; f += kDrainWarps) {
                    Waiting& w = sm.waiting[f];
                    const Marked marked(w.todo, w.token >= 0 ? (g.E + 31) / 32 : 0, lane);   // a word per lane
                    const int total = marked.count();
                    int first = 0;
                    if (lane == 0 && total) first = atomicAdd(&sm.n_items, total);
                    first = __shfl_sync(0xffffffffu, first, 0);
                    if (lane == 0) w.first = first + total <= kItems ? first | total << 16 : -1;
                    int at = first + marked.up_to - __popc(marked.word);
                    for (unsigned r = marked.word; r; r &= r - 1, ++at)
                        if (at < kItems) {
                            sm.item_expert[at] = (unsigned short)(32 * lane + __ffs(r) - 1);
                            sm.item_waiting[at] = (unsigned short)f;
                        }
                }
                choosers_sync();
                const int n_items = min(sm.n_items, kItems);
                log_p = log_parts(n_items, kParts);
                // once more with logit_wide where one of the sums needs it (from then on in every round)
                for (bool wide = false;; wide = true) {
                    for (int u = d; u < n_items << log_p; u += kDrainWarps) {
                        const int j = u >> log_p, part = u & ((1 << log_p) - 1), e = sm.item_expert[j];
                        const long long t = t0 + sm.waiting[sm.item_waiting[j]].token;
                        const float b = bias && part == 0 ? bias[e] : 0.f, add = addend && part == 0 ? addend[(size_t)t * g.E + e] : 0.f;
                        const uint4 *x = reinterpret_cast<const uint4*>(hidden + t * H), *w = reinterpret_cast<const uint4*>(w_router + (size_t)e * H);
                        const int from = chunks * part >> log_p, to = chunks * (part + 1) >> log_p;
                        double z = wide ? logit_wide(x, w, from, to, lane) : logit_f64<false>(x, w, from, to, lane);
                        if (lane == 0 && !wide && needs_wide(z)) sm.wide = 1;
                        z += (double)b;
                        z += (double)add;
                        if (lane == 0) sm.item_z[u] = z;
                    }
                    choosers_sync();
                    if (wide || !sm.wide) break;
                }
                if (tid == 128) sm.n_items = 0;
            }
            bool open = false;
            for (int f = d; f < n_tok; f += kDrainWarps) {
                int tok = rank * owned + f, mode = GATE_NEW;
                float dz = 0.f;
                if (round == 0) {
                    if (t0 + tok >= T) break;
                    float size = 0.f;
                    load_logits<PER>(smem_u32(&sm.s.part[tok][0]), smem_u32(&sm.size[tok]), rank, CL, lane, room.z, size);
                    dz = 1.02f * 0x1p-24f * size + (addend && (bias || size > 0.f) ? 16.f * 0x1p-24f : 0.f);       // the norms are short by less than 2 %
                    if (bias || addend || g.E < 32 * PER) {
                        bool cancelled = false;
#pragma unroll
                        for (int j = 0; j < PER; ++j) {
                            const int e = lane + 32 * j;
                            float v = -INFINITY;
                            if (e < g.E) {
                                v = room.z[e];
                                if (bias) v += bias[e];
                                if (addend) {
                                    const float before = fabsf(v);
                                    v += addend[(size_t)(t0 + tok) * g.E + e];
                                    cancelled |= before > 2.f * fabsf(v) + 16.f;
                                }
                            }
                            room.z[e] = v;
                        }
                        if (__any_sync(0xffffffffu, cancelled)) dz = INFINITY;
                        __syncwarp();
                    }
                }
                Waiting& w = sm.waiting[f];
                if (round > 0) {
                    tok = w.token;
                    dz = w.dz;
                    if (tok < 0) continue;
                    if (w.first < 0) {                                     // no room for its logits: in the next round
                        open = true;
                        continue;
                    }
#pragma unroll
                    for (int j = 0; j < PER; ++j) room.z[lane + 32 * j] = sm.s.part[tok][lane + 32 * j];
                    if (lane < kTodoUsed) room.todo[todo_at(lane)] = w.todo[lane];
                    room.picks.at[lane] = w.picks.at[lane];
                    if (lane == 0) {
                        room.picks.n = w.picks.n;
                        room.picks.mx = w.picks.mx;
                        room.picks.sum = w.picks.sum;
                    }
                    __syncwarp();
                    const int first = w.first & 0xffff, count = w.first >> 16;
                    for (int j = first + lane; j < first + count; j += 32) {
                        double z = sm.item_z[j << log_p];
                        for (int p = 1; p < 1 << log_p; ++p) z += sm.item_z[(j << log_p) + p];
                        my.z64[sm.item_expert[j]] = z;
                    }
                    __syncwarp();
                }
                const float rel = dz > 0.f ? added : 0.f;
                int32_t* ids_t = ids + (size_t)(t0 + tok) * g.k;
                float* weights_t = weights + (size_t)(t0 + tok) * g.k;
                if (round > 0) mode = go_on<PER>(g, room, balance, my.z64, dz, rel, lane, ids_t, weights_t);
                const bool again = mode == GATE_WAITS || (mode != GATE_DONE && choose_fast<PER>(g, room, balance, dz, rel, lane, mode, ids_t, weights_t));
                if (again) {                                               // it waits; its logits go back to its row
                    int at = f;
                    if (round == 0) {
                        if (lane == 0) at = atomicAdd(&sm.n_waiting, 1);
                        at = __shfl_sync(0xffffffffu, at, 0);
                    }
                    if (lane < kTodoUsed) sm.waiting[at].todo[lane] = room.todo[todo_at(lane)];
                    sm.waiting[at].picks.at[lane] = room.picks.at[lane];
                    if (lane == 0) {
                        sm.waiting[at].picks.n = room.picks.n;
                        sm.waiting[at].picks.mx = room.picks.mx;
                        sm.waiting[at].picks.sum = room.picks.sum;
                        sm.waiting[at].token = tok;
                        sm.waiting[at].dz = dz;
                    }
#pragma unroll
                    for (int j = 0; j < PER; ++j) sm.s.part[tok][lane + 32 * j] = room.z[lane + 32 * j];
                    open = true;
                } else if (round > 0 && lane == 0) {
                    w.token = -1;
                }
                __syncwarp();
            }
            if (round == 0) cluster_arrive();                              // this warp has read the others' shared memory
            if (!choosers_or(open)) break;
            n_tok = sm.n_waiting;
        }
    } else {
        cluster_arrive();
    }
    cluster_wait();                                                        // nobody reads this CTA's shared memory any more
}

template <int MT, int PER, bool STUCK = false>
int launch_tc(const __nv_bfloat16* x, const __nv_bfloat16* w, const float* bias, const float* addend, int T, int H, const GateArgs& g, int32_t* ids,
              float* weights, cudaStream_t st) {
    using S = Shared<MT, PER>;
    static_assert(sizeof(S) + 1024 <= 227 * 1024, "shared memory");
    static SmemOnce once;
    alignas(64) CUtensorMap map_w, map_x;
    if (encode_map(&map_w, w, g.E, H, MT * 128) || encode_map(&map_x, x, T, H, kTokens)) return EXMOE_ERR_CUDA;
    const int tiles = (T + kTokens - 1) / kTokens;
    int CL = 8;
    while (CL > 1 && tiles * CL > kSms) CL /= 2;
    return launch(gate_tc_kernel<MT, PER, STUCK>, (unsigned)(tiles * CL), kThreads, CL, sizeof(S) + 1024, once, st, map_w, map_x, x, w, bias, addend, T, H, g, CL, ids, weights);
}

}  // namespace

int launch_gate_tc_stuck(const __nv_bfloat16* x, const __nv_bfloat16* w, int T, int H, const GateArgs& g, int32_t* ids, float* weights, cudaStream_t st) {
    return launch_tc<1, 2, true>(x, w, nullptr, nullptr, T, H, g, ids, weights, st);
}

int launch_gate_tc(const __nv_bfloat16* x, const __nv_bfloat16* w, const float* bias, const float* addend, int T, int H, const GateArgs& g, int32_t* ids,
                   float* weights, cudaStream_t st) {
    if (g.E <= 64) return launch_tc<1, 2>(x, w, bias, addend, T, H, g, ids, weights, st);
    if (g.E <= 128) return launch_tc<1, 4>(x, w, bias, addend, T, H, g, ids, weights, st);
    return launch_tc<2, 8>(x, w, bias, addend, T, H, g, ids, weights, st);
}

extern "C" int exmoe_gate_status(void) {
    int v = 0;
    const int zero = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&v, g_gate_status, sizeof v) != cudaSuccess ||
        (v && cudaMemcpyToSymbol(g_gate_status, &zero, sizeof zero) != cudaSuccess))
        return EXMOE_ERR_CUDA;
    return v;
}

}  // namespace exmoe
