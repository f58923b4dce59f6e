// Low-rank adapters of many requests beside a shared projection: out_t = base_t + scale_a * B_a (A_a x_t), a the adapter of
// token t.  exmoe_lora_plan groups the tokens by adapter once per step, exmoe_lora runs one projection's adapters over the groups.
// With ranks of 8 to 128 this is no work for the tensor pipe: what bounds it is memory at many tokens (x and base read, out written: 15.9 us
// for 8192 rows of 2048 columns) and the chain of latencies at few.
#include <algorithm>

#include "common.cuh"
#include "frag.cuh"
#include "mbar.cuh"

namespace exmoe {

namespace {

constexpr int kMaxAdapters = 1024, kMaxRank = 128, kMaxTokens = 1 << 29, kMaxDim = 1 << 30;   // rows and columns, rounded up, fit 32 bits
constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32;
constexpr int kSms = 148;
constexpr int kLoraThreads = 256, kLoraWarps = kLoraThreads / 32;

// A plan: header, tiles, then the tokens grouped by adapter (ascending, those without one last; inside a group ascending tokens).
// A tile is a run of at most tile_rows(T) rows of one group: few enough that clusters fill the chip, and more where there are tokens enough, since
// every tile reads its adapter.  8192 tokens of 12 requests, 2048 x 2048, rank 16, rows per tile / CTAs per tile, us: 64 / 1 43.0, 64 / 2 33.8,
// 64 / 4 38.9, 32 / 1 34.8, 32 / 2 38.9 (with about 10 of launch).
__host__ __device__ constexpr int tile_rows(int T) { return T >= 1184 ? 64 : T >= 592 ? 32 : 16; }
constexpr int kPlanMagic = 0x4c6f5241;
enum { LP_MAGIC = 0, LP_TOKENS = 1, LP_ADAPTERS = 2, LP_TILES = 3, LP_STATUS = 4, LP_WORDS = 16 };
struct LoraTile { int adapter, row0, nrows, pad; };                        // adapter -1: none
__host__ __device__ inline int plan_tiles(int T, int n) {                  // most tiles of a plan
    const int groups = T < n + 1 ? T : n + 1;
    return T / tile_rows(T) + groups;
}

// A counting sort by one CTA.  A warp takes a run of tokens in steps of 32 and counts its tokens of each group; a thread per group adds up the warps'
// counts; a scan over the groups gives their first rows and tiles; then every warp places its tokens behind those of the warps before it.
// Which lanes of a step have the same group comes from a ballot for each bit of its number (`match` takes 10 cycles for each value that
// differs) unless all have.  us, replayed from a graph, 16 adapters and long requests / 256 adapters, each token another: 64 tokens 2.6 / 2.9, 1024
// 3.2 / 4.4, 8192 5.8 / 17.0 (`match`: 26); 1000 adapters, 64 tokens 3.5 (a warp per group over the warps' counts: 16.9).  Bound by the steps'
// instructions, 50 in each of the two passes where requests are long; once per step of all layers.
__global__ void __launch_bounds__(kPlanThreads)
lora_plan_kernel(const int32_t* ids, int T, int n, int32_t* plan) {
    extern __shared__ int32_t sm[];
    int32_t* hist = sm;                                                    // [warp][n + 1]: this warp's tokens of a group, then those of the warps before it
    int32_t* count = hist + kPlanWarps * (n + 1);                          // [n + 1]
    int32_t* first = count + n + 1;                                        // [n + 1] first row of a group
    int32_t* tile0 = first + n + 1;                                        // [n + 1] its first tile
    __shared__ int bad, rows_of[kPlanWarps], tiles_of[kPlanWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, most = tile_rows(T);
    const unsigned lt = (1u << lane) - 1u;
    LoraTile* tiles = reinterpret_cast<LoraTile*>(plan + LP_WORDS);
    int32_t* perm = plan + LP_WORDS + 4 * plan_tiles(T, n);
    const int per = ((T + kPlanWarps - 1) / kPlanWarps + 31) & ~31, warps = per ? (T + per - 1) / per : 0;   // tokens of a warp, warps that have some
    for (int i = tid; i < warps * (n + 1); i += kPlanThreads) hist[i] = 0;
    if (tid == 0) bad = 0;
    grid_dependency_wait();
    grid_launch_dependents();
    __syncthreads();
    const int t_begin = min(T, warp * per), t_end = min(T, t_begin + per), bits = 32 - __clz(n);
    int32_t* mine = hist + warp * (n + 1);
    constexpr int KEPT = 8;                                                // steps whose ids, then groups, are in registers: 8192 tokens
    int kept[KEPT];
    unsigned same[KEPT];                                                   // lanes of the same group
#pragma unroll
    for (int i = 0; i < KEPT; ++i) kept[i] = t_begin + 32 * i + lane < t_end ? ids[t_begin + 32 * i + lane] : -1;
    auto look_at = [&](int id, bool in, int& group, unsigned& same) {
        if (id < -1 || id >= n) bad = 1;
        group = id >= 0 && id < n ? id : n;
        same = 0xffffffffu;
        const int of_first = __shfl_sync(0xffffffffu, group, 0);
        if (__all_sync(0xffffffffu, in && group == of_first)) return;      // mostly, where requests are long
        const unsigned valid = __ballot_sync(0xffffffffu, in);
        unsigned other = 0u;
#pragma unroll 4
        for (int b = 0; b < bits; ++b) {
            const unsigned m = __ballot_sync(0xffffffffu, group >> b & 1);
            other |= m ^ (unsigned)-(group >> b & 1);
        }
        same = valid & ~other;
    };
    auto count_step = [&](int group, unsigned same, bool in) {
        if (in && !(same & lt)) mine[group] += __popc(same);
        __syncwarp();
    };
    auto place_step = [&](int group, unsigned same, int t0, bool in) {
        if (in) perm[first[group] + mine[group] + __popc(same & lt)] = t0 + lane;
        __syncwarp();
        count_step(group, same, in);
    };
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
        const int t0 = t_begin + 32 * i;
        if (t0 >= t_end) break;
        look_at(kept[i], t0 + lane < t_end, kept[i], same[i]);
        count_step(kept[i], same[i], t0 + lane < t_end);
    }
    for (int t0 = t_begin + 32 * KEPT; t0 < t_end; t0 += 32) {
        int group;
        unsigned like;
        look_at(t0 + lane < t_end ? ids[t0 + lane] : -1, t0 + lane < t_end, group, like);
        count_step(group, like, t0 + lane < t_end);
    }
    __syncthreads();
    int rows = 0;                                                          // of group tid
    for (int b = tid; b <= n; b += kPlanThreads) {
        int sum = 0;
        for (int w0 = 0; w0 < warps; w0 += 8) {
            int c[8];
#pragma unroll
            for (int w = 0; w < 8; ++w) c[w] = w0 + w < warps ? hist[(w0 + w) * (n + 1) + b] : 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                if (w0 + w < warps) hist[(w0 + w) * (n + 1) + b] = sum;
                sum += c[w];
            }
        }
        count[b] = sum;
        if (b < n) rows = b == tid ? sum : rows;
    }
    static_assert(kMaxAdapters <= kPlanThreads && kPlanWarps == 32, "a thread per adapter, a lane per warp");
    int ir = rows, it = (rows + most - 1) / most;
    const int nt_mine = it;
    auto scan = [&](int& r, int& t) {                                      // sums up to this lane's
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, r, d), p = __shfl_up_sync(0xffffffffu, t, d);
            if (lane >= d) {
                r += o;
                t += p;
            }
        }
    };
    scan(ir, it);
    if (lane == 31) {
        rows_of[warp] = ir;
        tiles_of[warp] = it;
    }
    __syncthreads();
    int wr = rows_of[lane], wt = tiles_of[lane];
    scan(wr, wt);
    const int rows_all = __shfl_sync(0xffffffffu, wr, 31), tiles_all = __shfl_sync(0xffffffffu, wt, 31);
    const int r0 = __shfl_sync(0xffffffffu, wr, (warp + 31) & 31), q0 = __shfl_sync(0xffffffffu, wt, (warp + 31) & 31);
    if (tid < n) {
        first[tid] = (warp ? r0 : 0) + ir - rows;
        tile0[tid] = (warp ? q0 : 0) + it - nt_mine;
    }
    if (tid == 0) {                                                        // the tokens without an adapter come last
        first[n] = rows_all;
        tile0[n] = tiles_all;
    }
    const int nt = tiles_all + (T - rows_all + most - 1) / most;
    if (tid == 0) {
        plan[LP_MAGIC] = kPlanMagic;
        plan[LP_TOKENS] = T;
        plan[LP_ADAPTERS] = n;
        plan[LP_TILES] = nt;
        plan[LP_STATUS] = bad ? EXMOE_ERR_BAD_ADAPTER_ID : EXMOE_OK;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
        const int t0 = t_begin + 32 * i;
        if (t0 >= t_end) break;
        place_step(kept[i], same[i], t0, t0 + lane < t_end);
    }
    for (int t0 = t_begin + 32 * KEPT; t0 < t_end; t0 += 32) {
        int group;
        unsigned like;
        look_at(t0 + lane < t_end ? ids[t0 + lane] : -1, t0 + lane < t_end, group, like);
        place_step(group, like, t0, t0 + lane < t_end);
    }
    for (int i = tid; i < nt; i += kPlanThreads) {
        int b = 0, above = n + 1;                                          // the last group whose first tile is not behind this one: the others have none
        while (above - b > 1) {
            const int m = (b + above) / 2;
            if (tile0[m] <= i)
                b = m;
            else
                above = m;
        }
        const int row = (i - tile0[b]) * most;
        tiles[i] = LoraTile{b < n ? b : -1, first[b] + row, min(most, count[b] - row), 0};
    }
}

struct LoraArgs {
    int32_t* plan;
    const __nv_bfloat16 *x, *a, *b;
    const float* scale;
    const void* base;
    void* out;
    long long ld_x, ld_base, ld_out;
    int T, n, K, N, r;
};
// whether the plan is one for this call; a wrong one is reported and nothing else is done
__device__ __forceinline__ bool plan_fits(const LoraArgs& p, const int4& head) {
    static_assert(LP_MAGIC == 0 && LP_TOKENS == 1 && LP_ADAPTERS == 2 && LP_TILES == 3, "the header's first words");
    if (head.x == kPlanMagic && head.y == p.T && head.z == p.n) return true;
    if (blockIdx.x == 0 && threadIdx.x == 0) p.plan[LP_STATUS] = EXMOE_ERR_STATE;
    return false;
}

__device__ __forceinline__ void cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void st_cluster(uint32_t addr, const float4& v, uint32_t bar, int rank) {      // and counts its bytes on that CTA's barrier
    uint32_t at, b;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(b) : "r"(bar), "r"(rank));
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1,%2,%3,%4}, [%5];"
                 ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(b) : "memory");
}

// Eight consecutive columns of a row of base or out.  `vec`: they are 16-byte aligned; `n`: how many of them there are.
template <typename O> struct Cols;
template <> struct Cols<__nv_bfloat16> {
    uint4 w = make_uint4(0, 0, 0, 0);
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int n, bool vec) {
        w = make_uint4(0, 0, 0, 0);
        if (vec && n >= 8) {
            asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "l"(p) : "memory");
            return;
        }
        uint32_t h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = i < n ? (uint32_t)reinterpret_cast<const unsigned short*>(p)[i] : 0u;
        w = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
    }
    __device__ __forceinline__ float get(int i) const {
        const uint32_t r = i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w;
        return __uint_as_float(i & 1 ? r & 0xffff0000u : r << 16);
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            r[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        w = make_uint4(r[0], r[1], r[2], r[3]);
    }
    __device__ __forceinline__ void store(__nv_bfloat16* p, int n, bool vec) const {
        if (vec && n >= 8) {
            *reinterpret_cast<uint4*>(p) = w;
            return;
        }
        const uint32_t r[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) reinterpret_cast<unsigned short*>(p)[i] = (unsigned short)(r[i >> 1] >> (16 * (i & 1)));
    }
};
template <> struct Cols<float> {
    float w[8] = {};
    __device__ __forceinline__ void load(const float* p, int n, bool vec) {
        if (vec && n >= 8) {
            asm volatile("ld.global.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(w[0]), "=f"(w[1]), "=f"(w[2]), "=f"(w[3]) : "l"(p) : "memory");
            asm volatile("ld.global.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(w[4]), "=f"(w[5]), "=f"(w[6]), "=f"(w[7]) : "l"(p + 4) : "memory");
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = i < n ? p[i] : 0.f;
    }
    __device__ __forceinline__ float get(int i) const { return w[i]; }
    __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = v[i];
    }
    __device__ __forceinline__ void store(float* p, int n, bool vec) const {
        if (vec && n >= 8) {
            *reinterpret_cast<float4*>(p) = make_float4(w[0], w[1], w[2], w[3]);
            *reinterpret_cast<float4*>(p + 4) = make_float4(w[4], w[5], w[6], w[7]);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = w[i];
    }
};

// A cluster of CTAs per tile of up to 16 MB rows of one adapter.
//   shrink  v = A x: every CTA takes a part of K.  Operands go from global memory into the fragments of m16n8k16 MMAs in 16-byte
//           loads: a lane's eight consecutive k serve two MMAs of both operands, K being permuted alike on both sides.  A warp takes 16
//           ranks, all rows and every WK-th step of 32.
//   join    partial v of the warps, then of the CTAs (through the cluster's shared memory), added in a fixed order in binary32
//   expand  out = base + scale B v: every CTA takes a part of N; v as a sum of two BF16 numbers (three for binary32 outputs: 8 more
//           bits each), so that B's products lose nothing that the output holds.  A lane's columns of the four MMAs of 32 columns
//           are made consecutive by permuting the rows of B: 16-byte accesses to base and out.
// RP: rank, rounded up (zeros).
// Replayed from a graph with warm weights, 2048 x 2048: 1 token of rank 16 3.7 us, 64 tokens of 64 requests over 32 adapters 5.1, 8192 tokens of 12
// requests 23.7 (101 MB moved or 4.2 TB/s; a plain copy of as many bytes 15.9); 777 tokens 1408 x 2048 of rank 64 9.8.  A tile of 8192 tokens (weights cold)
// spends 2,500 of 44,000 cycles on its rows' numbers, 15,000 on shrink, 3,000 on the join and 22,000 on expand, waiting for loads in flight at 22 %
// occupancy (registers); neither prefetches into L2 nor loads a step ahead in registers (fewer CTAs per SM) gained.
template <typename O, int RP, int MB>
struct LoraSmem {
    static constexpr int TM = 16 * MB, WN = RP / 16, WK = kLoraWarps / WN, PS = RP + 8, VS = RP + 8, SPLIT = sizeof(O) == 4 ? 3 : 2;
    alignas(16) float sum[TM][RP];                                                     // this CTA's part of v, read by the cluster
    union {
        float part[WK][TM][PS];                                            // the warps' parts
        __nv_bfloat16 v[SPLIT][TM][VS];                                    // v as BF16 numbers, largest first
    };
    long long token[TM];
    uint64_t arrived[2];
    int abort_flag;
};
// The CTAs send each other their parts of v (st.async, counted by the receiver's barrier) instead of fetching them: a way across the cluster instead
// of a barrier and two ways (one row of rank 16: 1200 cycles of the call's 5600; fetched, 2800 of 7100).  Up to kOneHop numbers for a CTA every CTA sends all of its part
// to all; beyond, each adds up a CL-th of v and sends the sums (32 rows of rank 64, CL = 8: 64 KB for a CTA otherwise).  What a CTA
// receives is behind LoraSmem: [rank][TM][RP], or [rank][CL-th] and v.
constexpr int kOneHop = 4096;
// STUCK (exmoe_debug_lora_timeout): the barrier of a cluster's first CTA asks for an arrival that nobody makes.
template <typename O, int RP, int MB, bool STUCK>
__global__ void __launch_bounds__(kLoraThreads, RP <= 64 ? 2 : 1)
lora_kernel(LoraArgs p, int log_cl, bool one_hop) {
    using S = LoraSmem<O, RP, MB>;
    constexpr int TM = S::TM, WN = S::WN, WK = S::WK, U = MB == 1 ? 4 : MB == 2 ? 2 : 1;
    extern __shared__ __align__(16) unsigned char smem[];
    S& sm = *reinterpret_cast<S*>(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, q = lane >> 2, c = lane & 3;
    const int CL = 1 << log_cl, rank = (int)blockIdx.x & (CL - 1);
    grid_dependency_wait();
    grid_launch_dependents();
    const int at = (int)blockIdx.x >> log_cl;
    const int4 head = load_behind_wait_cg(reinterpret_cast<const int4*>(p.plan));
    const int4 entry = load_behind_wait_cg(reinterpret_cast<const int4*>(p.plan + LP_WORDS) + at);      // inside the plan, whatever it holds
    if (!plan_fits(p, head) || at >= head.w) return;                       // the same for a whole cluster
    const LoraTile tile{entry.x, entry.y, entry.z, entry.w};
    const int32_t* perm = p.plan + LP_WORDS + 4 * plan_tiles(p.T, p.n);
    const int nrows = tile.nrows, nmb = (nrows + 15) / 16;
    float* received = reinterpret_cast<float*>(smem + sizeof(S));
    const int used = 16 * nmb * RP;                                        // numbers of v
    if (CL > 1) {
        if (tid == 0 && tile.adapter >= 0) {
            sm.abort_flag = 0;
            mbar_init(&sm.arrived[0], STUCK && rank == 0 ? 2 : 1);
            mbar_init(&sm.arrived[1], 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            mbar_expect_tx(&sm.arrived[0], (one_hop ? CL : 1) * used * 4);
            mbar_expect_tx(&sm.arrived[1], used * 4);
        }
        __syncthreads();
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // this CTA can be sent to
    }
    if (tid < TM) sm.token[tid] = perm[tile.row0 + min(tid, nrows - 1)];   // rows behind the last repeat it; they are not stored
    __syncthreads();
    const int n_blocks = (p.N + 31) / 32;
    const bool vec = !((reinterpret_cast<uintptr_t>(p.out) | reinterpret_cast<uintptr_t>(p.base) | (p.ld_out | p.ld_base) * sizeof(O)) & 15);
    const O* base = static_cast<const O*>(p.base);
    O* out = static_cast<O*>(p.out);
    Cols<O> y[MB][2];
    auto load_base = [&](int nb) {
        const int col = 32 * nb + 8 * c;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (base && mb < nmb) y[mb][h].load(base + sm.token[16 * mb + 8 * h + q] * p.ld_base + col, p.N - col, vec);
    };
    if (tile.adapter < 0) {
        if (base != out)
            for (int nb = rank * kLoraWarps + warp; nb < n_blocks; nb += CL * kLoraWarps) {
                load_base(nb);
                const int col = 32 * nb + 8 * c;
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (16 * mb + 8 * h + q < nrows) y[mb][h].store(out + sm.token[16 * mb + 8 * h + q] * p.ld_out + col, p.N - col, vec);
            }
        return;
    }
    {   // shrink
        const int wn = warp % WN, wk = warp / WN;
        const int steps = (p.K + 31) / 32, s_end = steps * (rank + 1) >> log_cl;
        const uint4 *xrow[MB][2], *arow[2];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int h = 0; h < 2; ++h) xrow[mb][h] = reinterpret_cast<const uint4*>(p.x + sm.token[16 * mb + 8 * h + q] * p.ld_x) + c;
        bool has[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int row = 16 * wn + 8 * j + q;
            has[j] = row < p.r;
            arow[j] = reinterpret_cast<const uint4*>(p.a + ((size_t)tile.adapter * p.r + (has[j] ? row : 0)) * p.K) + c;
        }
        float acc[MB][2][4];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[mb][j][i] = 0.f;
        for (int s0 = (steps * rank >> log_cl) + wk; s0 < s_end; s0 += U * WK) {
            uint4 xv[U][MB][2], av[U][2];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int s = s0 + u * WK;
                const bool in = s < s_end && 32 * s + 8 * c < p.K;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    av[u][j] = make_uint4(0, 0, 0, 0);
                    if (in && has[j]) av[u][j] = arow[j][4 * s];
                }
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        xv[u][mb][h] = make_uint4(0, 0, 0, 0);
                        if (in && mb < nmb) xv[u][mb][h] = xrow[mb][h][4 * s];
                    }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
                    if (mb < nmb) {
                        const uint4 &lo = xv[u][mb][0], &hi = xv[u][mb][1];
#pragma unroll
                        for (int j = 0; j < 2; ++j) mma_m16n8k16(acc[mb][j], lo.x, hi.x, lo.y, hi.y, av[u][j].x, av[u][j].y);
#pragma unroll
                        for (int j = 0; j < 2; ++j) mma_m16n8k16(acc[mb][j], lo.z, hi.z, lo.w, hi.w, av[u][j].z, av[u][j].w);
                    }
        }
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *reinterpret_cast<float2*>(&sm.part[wk][16 * mb + 8 * h + q][16 * wn + 8 * j + 2 * c]) = make_float2(acc[mb][j][2 * h], acc[mb][j][2 * h + 1]);
    }
    __syncthreads();
    for (int i = 4 * tid; i < used; i += 4 * kLoraThreads) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WK; ++w) {
            const float4 o = *reinterpret_cast<const float4*>(&sm.part[w][i / RP][i % RP]);
            v.x += o.x;
            v.y += o.y;
            v.z += o.z;
            v.w += o.w;
        }
        *reinterpret_cast<float4*>(&sm.sum[0][0] + i) = v;
    }
    const int slice = used >> log_cl;                                           // two hops: what a CTA adds up
    if (CL > 1) {
        cluster_wait();
        for (int i = 4 * tid; i < used; i += 4 * kLoraThreads) {           // its own again
            const float4 v = *reinterpret_cast<const float4*>(&sm.sum[0][0] + i);
            if (one_hop) {
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < CL) st_cluster(smem_u32(received + rank * TM * RP + i), v, smem_u32(&sm.arrived[0]), (rank + r) & (CL - 1));
            } else {
                const int to = i / slice;
                st_cluster(smem_u32(received + (rank - to) * slice + i), v, smem_u32(&sm.arrived[0]), to);
            }
        }
    } else {
        __syncthreads();
    }
    // in flight meanwhile: what the first columns need
    const float scale = p.scale[tile.adapter];
    constexpr int KB = RP / 16;
    uint2 bf[4][KB];
    auto load_b = [&](int nb) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int col = 32 * nb + 8 * (q >> 1) + 2 * j + (q & 1);
            const __nv_bfloat16* row = p.b + ((size_t)tile.adapter * p.N + min(col, p.N - 1)) * p.r + 4 * c;
#pragma unroll
            for (int k = 0; k < KB; ++k) {
                bf[j][k] = make_uint2(0, 0);
                if (col < p.N && 16 * k + 4 * c < p.r) bf[j][k] = *reinterpret_cast<const uint2*>(row + 16 * k);
            }
        }
    };
    int nb = rank * kLoraWarps + warp;
    if (nb < n_blocks) {
        load_b(nb);
        load_base(nb);
    }
    // A peer that does not send (none does that) would leave this call's rows unwritten and the plan's status at EXMOE_ERR_TIMEOUT.
    auto joined = [&](int hop) {
        if (__syncthreads_and(mbar_wait(&sm.arrived[hop], 0, &sm.abort_flag, p.plan + LP_STATUS, STUCK ? kWaitBudgetTest : kWaitBudget))) return true;
        cluster_arrive();                                                  // nor may this CTA end while it can be sent to
        cluster_wait();
        return false;
    };
    auto add_parts = [&](const float* at, int stride) {                    // by rank; all in flight at once
        float4 from[8], v;
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < CL) from[r] = *reinterpret_cast<const float4*>(at + r * stride);
        v = from[0];
#pragma unroll
        for (int r = 1; r < 8; ++r)
            if (r < CL) {
                v.x += from[r].x;
                v.y += from[r].y;
                v.z += from[r].z;
                v.w += from[r].w;
            }
        return v;
    };
    if (CL > 1) {
        if (!joined(0)) return;
        if (!one_hop) {
            for (int i = 4 * tid; i < slice; i += 4 * kLoraThreads) {
                const float4 v = add_parts(received + i, slice);
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < CL) st_cluster(smem_u32(received + TM * RP + rank * slice + i), v, smem_u32(&sm.arrived[1]), (rank + r) & (CL - 1));
            }
            if (!joined(1)) return;
        }
    }
    for (int i = 4 * tid; i < used; i += 4 * kLoraThreads) {
        float4 all;
        if (CL == 1)
            all = *reinterpret_cast<const float4*>(&sm.sum[0][0] + i);
        else if (one_hop)
            all = add_parts(received + i, TM * RP);
        else
            all = *reinterpret_cast<const float4*>(received + TM * RP + i);
        float v[4] = {all.x, all.y, all.z, all.w};
        if (i % RP >= p.r) v[0] = v[1] = v[2] = v[3] = 0.f;                // behind the rank: an infinity in x made 0 x infinity of the zeros there
#pragma unroll
        for (int n = 0; n < S::SPLIT; ++n) {
            __nv_bfloat16 h[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                h[j] = __float2bfloat16(v[j]);
                const float f = __bfloat162float(h[j]);
                v[j] = fabsf(f) < INFINITY ? v[j] - f : 0.f;               // an infinity or NaN is all in the first
            }
            *reinterpret_cast<uint2*>(&sm.v[n][i / RP][i % RP]) = *reinterpret_cast<const uint2*>(h);
        }
    }
    __syncthreads();
    while (nb < n_blocks) {
        const int col = 32 * nb + 8 * c;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
            if (mb < nmb) {
                float d[4][4] = {};
#pragma unroll
                for (int k = 0; k < KB; ++k)
#pragma unroll
                    for (int n = S::SPLIT - 1; n >= 0; --n) {
                        const uint2 lo = *reinterpret_cast<const uint2*>(&sm.v[n][16 * mb + q][16 * k + 4 * c]);
                        const uint2 hi = *reinterpret_cast<const uint2*>(&sm.v[n][16 * mb + 8 + q][16 * k + 4 * c]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) mma_m16n8k16(d[j], lo.x, hi.x, lo.y, hi.y, bf[j][k].x, bf[j][k].y);
                    }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float o[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[i] = fmaf(scale, d[i >> 1][2 * h + (i & 1)], base ? y[mb][h].get(i) : 0.f);
                    y[mb][h].set(o);
                    if (16 * mb + 8 * h + q < nrows) y[mb][h].store(out + sm.token[16 * mb + 8 * h + q] * p.ld_out + col, p.N - col, vec);
                }
            }
        nb += CL * kLoraWarps;
        if (nb < n_blocks) {
            load_b(nb);
            load_base(nb);
        }
    }
}

template <typename O, int RP, int MB, bool STUCK = false>
int launch_lora(const LoraArgs& p, int tiles, int CL, cudaStream_t st) {
    using S = LoraSmem<O, RP, MB>;
    static SmemOnce once;
    const auto kern = lora_kernel<O, RP, MB, STUCK>;
    const bool one_hop = CL * S::TM * RP <= kOneHop;
    constexpr int most = (int)sizeof(S) + std::max(kOneHop, 2 * S::TM * RP) * 4;
    static_assert(sizeof(S) % 16 == 0 && most <= (RP <= 64 ? 112 : 224) * 1024, "shared memory, of a second CTA too");
    if (!allow_smem(kern, most, once)) return EXMOE_ERR_CUDA;
    const size_t smem = sizeof(S) + (CL == 1 ? 0 : one_hop ? CL : 2) * S::TM * RP * 4;
    cudaLaunchConfig_t lc{};
    lc.gridDim = dim3((unsigned)(tiles * CL));
    lc.blockDim = dim3(kLoraThreads);
    lc.dynamicSmemBytes = smem;
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
    if (cudaLaunchKernelEx(&lc, kern, p, CL == 8 ? 3 : CL == 4 ? 2 : CL == 2 ? 1 : 0, one_hop) != cudaSuccess) {
        cudaGetLastError();
        return EXMOE_ERR_CUDA;
    }
    count_launch();
    return EXMOE_OK;
}
template <typename O, int RP>
int launch_lora_rows(const LoraArgs& p, int tiles, int CL, cudaStream_t st) {
    switch (tile_rows(p.T)) {
        case 16: return launch_lora<O, RP, 1>(p, tiles, CL, st);
        case 32: return launch_lora<O, RP, 2>(p, tiles, CL, st);
        default: return launch_lora<O, RP, 4>(p, tiles, CL, st);
    }
}
template <typename O>
int launch_lora_rank(const LoraArgs& p, int tiles, int CL, cudaStream_t st) {
    if (p.r <= 16) return launch_lora_rows<O, 16>(p, tiles, CL, st);
    if (p.r <= 32) return launch_lora_rows<O, 32>(p, tiles, CL, st);
    if (p.r <= 64) return launch_lora_rows<O, 64>(p, tiles, CL, st);
    return launch_lora_rows<O, 128>(p, tiles, CL, st);
}

int check_plan(int T, int n) {
    if (T < 0 || T > kMaxTokens) return EXMOE_ERR_ARG;
    return n < 1 || n > kMaxAdapters ? EXMOE_ERR_SHAPE : EXMOE_OK;
}

// [rows, cols] elements of `es` bytes, rows `ld` elements apart: do two such ranges share a byte?  Column ranges of the same wider rows do not.
struct Range { uintptr_t at; long long rows, pitch, width; };
bool overlap(const Range& a, const Range& b) {
    if (!a.at || !b.at || a.rows <= 0 || b.rows <= 0) return false;
    const uintptr_t a_end = a.at + (a.rows - 1) * a.pitch + a.width, b_end = b.at + (b.rows - 1) * b.pitch + b.width;
    if (a_end <= b.at || b_end <= a.at) return false;
    if (a.pitch != b.pitch || a.rows == 1 || b.rows == 1) return true;
    const long long d = (long long)((b.at > a.at ? b.at - a.at : a.at - b.at) % (uintptr_t)a.pitch);   // column distance
    const Range &lo = b.at > a.at ? a : b, &hi = b.at > a.at ? b : a;
    return !(d >= lo.width && d + hi.width <= a.pitch);
}

}  // namespace

extern "C" int exmoe_lora_plan_bytes(int T, int num_adapters, size_t* bytes) {
    const int rc = check_plan(T, num_adapters);
    if (rc) return rc;
    if (!bytes) return EXMOE_ERR_ARG;
    *bytes = 4 * (LP_WORDS + 4 * (size_t)plan_tiles(T, num_adapters) + (size_t)T);
    return EXMOE_OK;
}

extern "C" int exmoe_lora_plan(const int32_t* adapter_ids, int T, int num_adapters, void* plan, void* stream) {
    const int rc = check_plan(T, num_adapters);
    if (rc) return rc;
    if ((!adapter_ids && T) || !plan || !aligned(4, adapter_ids) || !aligned(16, plan)) return EXMOE_ERR_ARG;
    const size_t smem = 4 * (size_t)(kPlanWarps + 3) * (num_adapters + 1);
    static SmemOnce once;
    if (!allow_smem(lora_plan_kernel, 4 * (kPlanWarps + 3) * (kMaxAdapters + 1), once)) return EXMOE_ERR_CUDA;
    cudaLaunchConfig_t lc{};
    lc.gridDim = dim3(1);
    lc.blockDim = dim3(kPlanThreads);
    lc.dynamicSmemBytes = smem;
    lc.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
#ifdef EXMOE_DISABLE_PDL
    lc.numAttrs = 0;
#endif
    if (cudaLaunchKernelEx(&lc, lora_plan_kernel, adapter_ids, T, num_adapters, (int32_t*)plan) != cudaSuccess) {
        cudaGetLastError();
        return EXMOE_ERR_CUDA;
    }
    count_launch();
    return EXMOE_OK;
}

extern "C" int exmoe_lora_plan_status(const void* plan) {
    if (!plan) return EXMOE_ERR_ARG;
    int32_t head[LP_WORDS];
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(head, plan, sizeof head, cudaMemcpyDeviceToHost) != cudaSuccess) return EXMOE_ERR_CUDA;
    return head[LP_MAGIC] == kPlanMagic ? head[LP_STATUS] : EXMOE_ERR_STATE;
}

static int lora_call(const exmoe_lora_shape* shape, void* plan, const void* x, int64_t ld_x, const void* a, const void* b, const float* scale, int T,
                     const void* base, int64_t ld_base, void* out, int64_t ld_out, int type, bool stuck, void* stream) {
    if (!shape || T < 0 || T > kMaxTokens || (type != EXMOE_F32 && type != EXMOE_BF16)) return EXMOE_ERR_ARG;
    const int n = shape->num_adapters, K = shape->d_in, N = shape->d_out, r = shape->rank;
    if (n < 1 || n > kMaxAdapters || K <= 0 || K % 8 || N <= 0 || r <= 0 || r % 8 || r > kMaxRank || K > kMaxDim || N > kMaxDim) return EXMOE_ERR_SHAPE;
    if (T == 0) return EXMOE_OK;
    if (!plan || !x || !a || !b || !scale || !out) return EXMOE_ERR_ARG;
    if (ld_x < K || ld_x % 8 || ld_out < N || (base && ld_base < N)) return EXMOE_ERR_ARG;
    const long long es = type == EXMOE_F32 ? 4 : 2;
    if (!aligned(16, plan, x, a, b) || !aligned(4, scale) || !aligned(es, base, out)) return EXMOE_ERR_ARG;
    auto range = [](const void* p, long long rows, long long ld, long long width, long long es) {
        return Range{reinterpret_cast<uintptr_t>(p), rows, ld * es, width * es};
    };
    size_t plan_size = 0;
    exmoe_lora_plan_bytes(T, n, &plan_size);
    const Range o = range(out, T, ld_out, N, es), bs = range(base, T, ld_base, N, es);
    if ((!(base == out && (ld_base == ld_out || T == 1)) && overlap(o, bs)) || overlap(o, range(x, T, ld_x, K, 2)) || overlap(o, range(a, 1, 0, (long long)n * r * K, 2)) ||
        overlap(o, range(b, 1, 0, (long long)n * r * N, 2)) || overlap(o, range(scale, 1, 0, n, 4)) || overlap(o, range(plan, 1, 0, (long long)plan_size, 1)))
        return EXMOE_ERR_ARG;
    const LoraArgs args{(int32_t*)plan, (const __nv_bfloat16*)x, (const __nv_bfloat16*)a, (const __nv_bfloat16*)b, scale, base, out,
                        ld_x, ld_base, ld_out, T, n, K, N, r};
    // As many CTAs per tile (a power of two up to eight) as the chip has room for if every adapter is in use.
    const int tiles = plan_tiles(T, n);
    int CL = 8;
    while (CL > 1 && (long long)tiles * CL > 2 * kSms) CL /= 2;
    if (stuck) {
        if (type != EXMOE_BF16 || tile_rows(T) != 16 || r > 64 || CL == 1) return EXMOE_ERR_SHAPE;
        return r <= 16 ? launch_lora<__nv_bfloat16, 16, 1, true>(args, tiles, CL, (cudaStream_t)stream)
                       : launch_lora<__nv_bfloat16, 64, 1, true>(args, tiles, CL, (cudaStream_t)stream);
    }
    return type == EXMOE_F32 ? launch_lora_rank<float>(args, tiles, CL, (cudaStream_t)stream) : launch_lora_rank<__nv_bfloat16>(args, tiles, CL, (cudaStream_t)stream);
}

extern "C" int exmoe_lora(const exmoe_lora_shape* shape, void* plan, const void* x, int64_t ld_x, const void* a, const void* b,
                          const float* scale, int T, const void* base, int64_t ld_base, void* out, int64_t ld_out, int type,
                          void* stream) {
    return lora_call(shape, plan, x, ld_x, a, b, scale, T, base, ld_base, out, ld_out, type, false, stream);
}

extern "C" int exmoe_debug_lora_timeout(const exmoe_lora_shape* shape, void* plan, const void* x, const void* a, const void* b, const float* scale, int T, void* out,
                                       void* stream) {
    if (!shape || T == 0) return EXMOE_ERR_ARG;
    return lora_call(shape, plan, x, shape->d_in, a, b, scale, T, nullptr, 0, out, shape->d_out, EXMOE_BF16, true, stream);
}

}  // namespace exmoe
