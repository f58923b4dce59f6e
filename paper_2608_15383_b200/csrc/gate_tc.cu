// The gate on many tokens: the logits as a GEMM on tcgen05, then the choice, in one kernel.
//
// A cluster of CL CTAs takes 128 tokens; each multiplies a CL-th of K: weights of all experts (up to MT x 128 rows, the MMA's M) and
// tokens (N = 128) come by TMA into a ring of 64-wide stages, and a stage's four MMAs of K = 16 start from zero.  An MMA truncates:
// every product to 2^-25 of the largest one's (and the accumulator's) binade, the result to 24 bits; four of them one after
// another lose at most 4 (17 / 4 + 1) units of 2^-23 of S = sum |x_i w_i|, while the 64 MMAs of 1024 elements, each truncating what the
// ones before have summed, would lose as many times more.  So sixteen warps take every stage's accumulator out of tensor memory, which
// has two of them, and add it to binary32 sums in registers, behind the MMAs of the next stage; they also add up |x|^2 and |w|^2
// from the stages' tiles.  The partial logits go to shared memory, the CTA that owns a token adds the CL parts, and a warp makes its
// choice (gate.cuh), with the logits that decide computed again in binary64 where they are closer than the bound.
#include <algorithm>

#include "gate.cuh"
#include "mbar.cuh"
#include "tc.cuh"

namespace exmoe {

namespace {

constexpr int kTokens = 128, kStages = 4, kDrainWarps = 16, kThreads = 32 * (4 + kDrainWarps);
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
template <int PER>
__device__ __forceinline__ void add_run(uint32_t addr, int rank, float (&v)[PER]) {
    const uint32_t at = at_rank(addr, rank);
    if constexpr (PER == 2) {
        float a, b;
        asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];" : "=f"(a), "=f"(b) : "r"(at) : "memory");
        v[0] += a;
        v[1] += b;
    } else {
#pragma unroll
        for (int i = 0; i < PER; i += 4) {
            float a, b, c, d;
            asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(a), "=f"(b), "=f"(c), "=f"(d) : "r"(at + 4 * i) : "memory");
            v[i] += a;
            v[i + 1] += b;
            v[i + 2] += c;
            v[i + 3] += d;
        }
    }
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

template <int MT, int PER>
struct Warp {                                                              // a choosing warp's share of shared memory
    ChoiceRoom<PER> room;
    double z64[32 * PER];
};
template <int MT, int PER>
struct __align__(1024) Shared {
    static constexpr int kStage = (MT * 128 + kTokens) * kRowBytes;
    union {
        unsigned char ring[kStages][kStage];                               // weights, then tokens; rows of 128 bytes, swizzled
        struct {
            float part[kTokens][MT * 128];                                 // this CTA's part of the logits, read by the cluster
            Warp<MT, PER> warp[kDrainWarps];
        } s;
    };
    float x2[kTokens], w2[MT * 128], balance[32 * PER];
    float w2_max[kDrainWarps];
    int items, item[kDrainWarps * 32 * PER];                               // logits to compute again: warp << 16 | expert
    uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2];
    uint32_t tmem;
    int abort_flag;
};

template <int MT, int PER>
__global__ void __launch_bounds__(kThreads, 1)
gate_tc_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const __nv_bfloat16* hidden,
               const __nv_bfloat16* __restrict__ w_router, const float* __restrict__ bias, const float* addend, int T, int H,
               const __grid_constant__ GateArgs g, int CL, int32_t* ids, float* weights) {
    using S = Shared<MT, PER>;
    constexpr int EP = MT * 128, COLS = MT * kTokens / 4;                  // accumulator columns of a drain warp: a quarter of them, on its 32 lanes
    extern __shared__ unsigned char raw[];
    S& sm = *reinterpret_cast<S*>(raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u));
    const int tid = threadIdx.x, lane = tid & 31, warp = warp_uniform(tid >> 5);
    const int rank = (int)blockIdx.x % CL, t0 = (int)blockIdx.x / CL * kTokens;
    volatile int* abort_flag = &sm.abort_flag;
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm.full[s], 1);
            mbar_init(&sm.empty[s], 1 + kDrainWarps);                      // the MMAs and the warps that add up the squares
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sm.acc_full[b], 1);
            mbar_init(&sm.acc_empty[b], kDrainWarps);
        }
        sm.abort_flag = 0;
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
    float acc[COLS];
#pragma unroll
    for (int i = 0; i < COLS; ++i) acc[i] = 0.f;
    const int d = warp - 4, quarter = warp & 3;                            // drain warps: d of kDrainWarps
    const int mt = MT == 2 ? d >> 3 : 0, col0 = (d >> 2) * COLS % kTokens; // experts mt * 128 + 32 quarter + lane, tokens col0 ..
    bool ok = true;
    if (warp == 0) {
        const uint32_t idesc = make_idesc(kTokens);
        for (int i = 0; i < n; ++i) {
            const int s = i % kStages, buf = i & 1;
            if (i >= 2) ok = mbar_wait_warp(acc_empty + 8 * buf, ((i >> 1) - 1) & 1, abort_flag, &g_gate_status);
            if (ok) ok = mbar_wait_warp(full + 8 * s, (i / kStages) & 1, abort_flag, &g_gate_status);
            if (!ok) break;
            tc_fence_after();
            const uint64_t dw = make_desc_b(smem_u32(sm.ring[s])), dx = make_desc_b(smem_u32(sm.ring[s]) + MT * 128 * kRowBytes);
            if (elect_one()) {
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j)                            // K = 16: 32 bytes on
                        mma_f16(tmem + (buf * MT + m) * kTokens, dw + (uint64_t)(m * 128 * kRowBytes + 32 * j >> 4), dx + (uint64_t)(32 * j >> 4), idesc, j > 0);
                tc_commit_at(empty + 8 * s);
                tc_commit_at(acc_full + 8 * buf);
            }
            __syncwarp();
        }
    } else if (warp == 1) {
        for (int i = 0; i < n; ++i) {
            const int s = i % kStages;
            if (i >= kStages) ok = mbar_wait_warp(empty + 8 * s, (i / kStages - 1) & 1, abort_flag, &g_gate_status);
            if (!ok) break;
            if (elect_one()) {
                mbar_expect_tx(&sm.full[s], S::kStage);
                tma_load_2d(smem_u32(sm.ring[s]), &map_w, (kb0 + i) * 64, 0, &sm.full[s]);
                tma_load_2d(smem_u32(sm.ring[s]) + MT * 128 * kRowBytes, &map_x, (kb0 + i) * 64, t0, &sm.full[s]);
            }
            __syncwarp();
        }
    } else if (warp < 4) {
        for (int e = tid - 64; e < 32 * PER; e += 64) sm.balance[e] = g.balance && e < g.E ? g.balance[e] : 0.f;
    } else {
        // a quarter of a token's row, and a half (MT = 2) or a quarter of an expert's
        constexpr int WQ = MT == 2 ? 4 : 2;                                // 16-byte pieces
        const int u = tid - 128, xr = u >> 2, wr = MT == 2 ? u >> 1 : u >> 2;
        float x2 = 0.f, w2 = 0.f;
        for (int i = 0; i < n; ++i) {
            const int s = i % kStages, buf = i & 1;
            ok = mbar_wait_warp(full + 8 * s, (i / kStages) & 1, abort_flag, &g_gate_status);
            if (!ok) break;
            const __nv_bfloat162 zero(__float2bfloat16(0.f), __float2bfloat16(0.f));
            __nv_bfloat162 a = zero, b = zero;
            const unsigned char *wt = sm.ring[s] + wr * kRowBytes, *xt = sm.ring[s] + (MT * 128 + xr) * kRowBytes;
#pragma unroll
            for (int j = 0; j < 2; ++j) square(a, *reinterpret_cast<const uint4*>(xt + ((((u & 3) * 2 + j) ^ (xr & 7)) << 4)));
#pragma unroll
            for (int j = 0; j < WQ; ++j) square(b, *reinterpret_cast<const uint4*>(wt + ((((MT == 2 ? u & 1 : u & 3) * WQ + j) ^ (wr & 7)) << 4)));
            __syncwarp();
            if (lane == 0) mbar_arrive_at(empty + 8 * s);
            x2 += __low2float(a) + __high2float(a);
            w2 += __low2float(b) + __high2float(b);
            ok = mbar_wait_warp(acc_full + 8 * buf, (i >> 1) & 1, abort_flag, &g_gate_status);
            if (!ok) break;
            tc_fence_after();
            const uint32_t at = tmem + ((uint32_t)(32 * quarter) << 16) + (buf * MT + mt) * kTokens + col0;
#pragma unroll
            for (int c = 0; c < COLS; c += 16) {
                uint32_t r[16];
                tmem_ld16(at + c, r);
                tc_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[c + j] += __uint_as_float(r[j]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(acc_empty + 8 * buf);
        }
        x2 += __shfl_xor_sync(0xffffffffu, x2, 1);
        x2 += __shfl_xor_sync(0xffffffffu, x2, 2);
        w2 += __shfl_xor_sync(0xffffffffu, w2, 1);
        if (MT == 1) w2 += __shfl_xor_sync(0xffffffffu, w2, 2);
        if ((u & 3) == 0) sm.x2[xr] = x2;
        if (MT == 2 ? (u & 1) == 0 : (u & 3) == 0) sm.w2[wr] = w2;
    }
    __syncthreads();                                                       // the ring has been read, the accumulators too
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * MT * kTokens));
    if (warp >= 4)
#pragma unroll
        for (int i = 0; i < COLS; ++i) sm.s.part[col0 + i][mt * 128 + 32 * quarter + lane] = acc[i];
    cluster_arrive();
    cluster_wait();
    if (warp >= 4) {
        float w2 = 0.f;
        for (int e = tid - 128; e < EP; e += 32 * kDrainWarps) {
            float v = 0.f;
            for (int r = 0; r < CL; ++r) v += ld_rank(smem_u32(&sm.w2[e]), r);
            w2 = v;                                                        // rows behind the last expert are zeros
        }
        w2 = warp_max(w2);
        if (lane == 0) sm.w2_max[d] = w2;
    }
    bool all_ok = true;                                                    // of the whole cluster: a part of the logits is missing otherwise
    for (int r = 0; r < CL; ++r) {
        int f;
        asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(f) : "r"(at_rank(smem_u32(&sm.abort_flag), r)) : "memory");
        all_ok &= f == 0;
    }
    __syncthreads();
    if (warp >= 4 && all_ok) {
        Warp<MT, PER>& my = sm.s.warp[d];
        ChoiceRoom<PER>& room = my.room;
        float w2 = 0.f;
#pragma unroll
        for (int i = 0; i < kDrainWarps; ++i) w2 = fmaxf(w2, sm.w2_max[i]);
        const float* balance = g.balance ? sm.balance : nullptr;
        const int owned = kTokens / CL, chunks = H / 8;
        for (int i = d; i - d < owned; i += kDrainWarps) {                 // the warps together, so that they share what is computed again
            const int tok = rank * owned + i;
            const long long t = t0 + tok;
            const bool live = i < owned && t < T;
            if (tid == 128) sm.items = 0;
            float dz = 0.f;
            if (live) {
                float v[PER], x2 = 0.f;
#pragma unroll
                for (int j = 0; j < PER; ++j) v[j] = 0.f;
                for (int r = 0; r < CL; ++r) {
                    add_run<PER>(smem_u32(&sm.s.part[tok][PER * lane]), r, v);
                    x2 += ld_rank(smem_u32(&sm.x2[tok]), r);
                }
                bool cancelled = false;
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    const int e = PER * lane + j;
                    if (e < g.E) {
                        if (bias) v[j] += bias[e];
                        if (addend) {
                            const float before = fabsf(v[j]);
                            v[j] += addend[t * g.E + e];
                            cancelled |= before > 2.f * fabsf(v[j]) + 16.f;
                        }
                    } else {
                        v[j] = -INFINITY;
                    }
                }
                store_run<PER>(room.z + PER * lane, v);
                __syncwarp();
                // the tensor cores' 2 x 21, an addition per stage, one per CTA; the norms are short by less than 2 %
                dz = 1.02f * (float)(42 + (blocks + CL - 1) / CL + CL) * 0x1p-24f * sqrtf(x2) * sqrtf(w2) + (addend ? 16.f * 0x1p-24f : 0.f);
                if (__any_sync(0xffffffffu, cancelled)) dz = INFINITY;
            }
            int32_t* ids_t = ids + t * g.k;
            float* weights_t = weights + t * g.k;
            bool open = live;                                              // not chosen yet
            for (bool decided = false;; decided = true) {
                open = open && choose_fast<PER>(g, room, balance, dz, bias || addend ? kAddedRel : 0.f, lane, decided, ids_t, weights_t);
                if (!choosers_or(open)) break;
                if (open) {
                    unsigned es = 32 * lane < g.E ? room.todo[lane] : 0u;  // a word per lane
                    int at = 0;
                    if (es) at = atomicAdd(&sm.items, __popc(es));
                    for (; es; es &= es - 1) sm.item[at++] = d << 16 | (32 * lane + __ffs(es) - 1);
                }
                choosers_sync();
                for (int j = d; j < sm.items; j += kDrainWarps) {
                    const int who = sm.item[j] >> 16, e = sm.item[j] & 0xffff;
                    const long long u = t - d + who;                       // that warp's token
                    const double z = logit_f64(reinterpret_cast<const uint4*>(hidden + u * H), reinterpret_cast<const uint4*>(w_router + (size_t)e * H), chunks, lane);
                    if (lane == 0) sm.s.warp[who].z64[e] = z + (bias ? (double)bias[e] : 0.0) + (addend ? (double)addend[u * g.E + e] : 0.0);
                }
                choosers_sync();
                if (tid == 128) sm.items = 0;
                if (!open) continue;
                const uint32_t stage = room.todo[kTodoStage];
                if (stage == GATE_GROUPS) {
                    choose_groups<PER>(g, room, my.z64, my.z64, lane);
                    continue;
                }
                if (stage == GATE_EXPERTS)
                    choose_again<PER>(g, room, my.z64, lane, ids_t, weights_t);
                else
                    choose_exact(g, my.z64, reinterpret_cast<unsigned long long*>(room.z), lane, ids_t, weights_t);       // z and c
                open = false;
            }
            __syncwarp();
        }
    }
    cluster_arrive();                                                      // nobody reads this CTA's shared memory any more
    cluster_wait();
}

template <int MT, int PER>
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
    return launch(gate_tc_kernel<MT, PER>, (unsigned)(tiles * CL), kThreads, CL, sizeof(S) + 1024, once, st, map_w, map_x, x, w, bias, addend, T, H, g, CL, ids, weights);
}

}  // namespace

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
