// The gate of a sparse block (exmoe_gate): scores, balance bias, groups, top-k, weights; from hidden states or from logits.
#include <cooperative_groups.h>

#include <algorithm>

#include "frag.cuh"
#include "gate.cuh"

namespace exmoe {

namespace {

namespace cg = cooperative_groups;

constexpr int kMaxTokens = 1 << 29;                                        // grids and row counts fit 32 bits
constexpr int kGateThreads = 256, kGateWarps = kGateThreads / 32;

// What the other forms do not take (more than 512 experts or 32 choices, rows too long for their shared memory): one CTA per token,
// everything in binary64, whose additions bound it (products of BF16 values are exact in binary32).  64 experts of 2048, one token: 18.4 us
// a call, 6.0 in the first version of the form for few tokens below.
__global__ void __launch_bounds__(kGateThreads)
gate_token_kernel(const __nv_bfloat16* hidden, const __nv_bfloat16* __restrict__ w_router, const float* __restrict__ bias,
                  const float* addend, int H, const __grid_constant__ GateArgs g, int32_t* ids, float* weights) {
    extern __shared__ __align__(16) unsigned char smem[];
    double* z = reinterpret_cast<double*>(smem);
    unsigned long long* key = reinterpret_cast<unsigned long long*>(z + g.E);
    uint4* xs = reinterpret_cast<uint4*>(smem + (((size_t)g.E * 16 + 15) & ~size_t(15)));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, chunks = H / 8;
    const size_t t = blockIdx.x;
    grid_dependency_wait();
    const uint4* xrow = reinterpret_cast<const uint4*>(hidden + t * H);
    for (int i = tid; i < chunks; i += kGateThreads) xs[i] = xrow[i];
    __syncthreads();
    for (int e = warp; e < g.E; e += kGateWarps) {
        const double s = logit_f64<true>(xs, reinterpret_cast<const uint4*>(w_router + (size_t)e * H), 0, chunks, lane);
        if (lane == 0) z[e] = s + (bias ? (double)bias[e] : 0.0) + (addend ? (double)addend[t * g.E + e] : 0.0);
    }
    __syncthreads();
    if (warp == 0) choose_exact(g, z, key, lane, ids + t * g.k, weights + t * g.k);
}

// One warp per token: the latency of a row's loads, then the choice's instructions.  16 tokens of 64 experts 2.4 us (replayed from a graph), 8191 BF16
// rows of 256 experts, 8 of 3 of 8 groups, 8.8 us (818 instructions a token, 6 us of issue), of which the bytes would take 0.7; 16-byte loads instead of 2-byte ones
// changed nothing.  Longer-lived warps that take several tokens each lost (a choice's
// latency is then in the open).  PER: experts per lane of choose_fast, 0: all in binary64.  Shared memory, per warp: logits_room(), and the balance
// bias where choose_fast reads it.
template <int PER>
__host__ __device__ constexpr size_t logits_room(int E) {
    if constexpr (PER > 0)
        return sizeof(ChoiceRoom<PER>) + 8 * 32 * PER;
    else
        return 16 * (size_t)E;
}
template <typename Z, int PER>
__global__ void __launch_bounds__(kGateThreads, PER <= 8 ? 4 : 2)
gate_logits_kernel(const Z* logits, long long ld, int T, const __grid_constant__ GateArgs g, int32_t* ids, float* weights) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    unsigned char* mine = smem + warp * logits_room<PER>(g.E);
    const size_t t = (size_t)blockIdx.x * warps + warp;
    grid_dependency_wait();
    grid_launch_dependents();
    const Z* row = logits + (long long)t * ld;
    double *z64, *key;
    if constexpr (PER > 0) {
        float* balance = nullptr;
        if (g.balance) {
            balance = reinterpret_cast<float*>(smem + warps * logits_room<PER>(g.E));
            for (int e = threadIdx.x; e < 32 * PER; e += blockDim.x) balance[e] = e < g.E ? g.balance[e] : 0.f;
            __syncthreads();
        }
        if (t >= (size_t)T) return;
        ChoiceRoom<PER>& room = *reinterpret_cast<ChoiceRoom<PER>*>(mine);
        float v[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) v[i] = lane + 32 * i < g.E ? (float)row[lane + 32 * i] : -INFINITY;
#pragma unroll
        for (int i = 0; i < PER; ++i) room.z[lane + 32 * i] = v[i];
        __syncwarp();
        z64 = reinterpret_cast<double*>(mine + sizeof(ChoiceRoom<PER>));
        key = reinterpret_cast<double*>(room.z);                           // z and c
        bool all = false;                                                  // everything in binary64 after all
        for (int mode = GATE_NEW; choose_fast<PER>(g, room, balance, 0.f, 0.f, lane, mode, ids + t * g.k, weights + t * g.k); mode = GATE_DECIDED) {
            const uint32_t stage = room.todo[kTodoStage];
            if (stage == GATE_GROUPS) {
                choose_groups<PER>(g, room, nullptr, z64, lane);
                continue;
            }
            if (stage == GATE_EXPERTS && finish_choice<PER>(g, room, balance, nullptr, 0.f, 0.f, lane, ids + t * g.k, weights + t * g.k)) return;
            all = true;
            break;
        }
        if (!all) return;
        __syncwarp();
    } else {
        if (t >= (size_t)T) return;
        z64 = reinterpret_cast<double*>(mine);
        key = z64 + g.E;
    }
    for (int e = lane; e < g.E; e += 32) z64[e] = (double)(float)row[e];
    __syncwarp();
    choose_exact(g, z64, reinterpret_cast<unsigned long long*>(key), lane, ids + t * g.k, weights + t * g.k);
}


// ---- few tokens: a cluster of eight CTAs shares the experts of TB tokens -----------------------------------------------
// As many warps as a 64-expert router has rows, so that a row's 4 KB are in flight at once.  Logits in binary32: chains of four products, two
// to a chunk, a lane's H / 256 chunks one after another, a tree over the lanes.  Each addition is off by 2^-24 of what is summed, so
// the products of chunk j count 4 + 1 + (chunks - j) + 5 times: sum c_j S_j <= sqrt(sum c_j |x_j|^2) sqrt(sum c_j |w_j|^2) such units.  Bias and
// addend are off by 2^-24 of the sum before and of the logit (where the
// former is larger than twice the latter + 16, all logits are computed again).  They travel through the cluster's shared
// memory to the CTA that owns the token (i % 8), whose first warp chooses; where that rests on less than the bound, its warps
// compute the logits that matter once more in binary64.  What bounds it is the chain of latencies: weights from memory, sums, the
// exchange in the cluster, the choice.  64 experts of 2048, replayed from a graph: one token 4.9 us, 37 tokens 6.2, or 9.0 with a near-tie.
template <int PER>
struct __align__(16) FewRoom {
    ChoiceRoom<PER> room;
    float balance[32 * PER];
    double z64[32 * PER];
};
// Four tokens per cluster from here on: 16 tokens one / four 5.9 / 6.4, 32 tokens 8.6 / 7.2 us (64 experts of 2048); 16.1 / 19.2 and 23.5 / 19.2 (256 of 4096).
constexpr int kFewCluster = 8, kFewFour = 24;
template <int TB, int PER>
__global__ void __launch_bounds__(kGateThreads, 2)                         // else the compiler may take 80 registers, and fewer loads are in flight: 37 tokens 6.1 -> 7.4 us
gate_few_kernel(const __nv_bfloat16* hidden, const __nv_bfloat16* __restrict__ w_router, const float* __restrict__ bias, const float* addend, int T, int H,
                const __grid_constant__ GateArgs g, int32_t* ids, float* weights) {
    static_assert(TB <= kFewCluster, "a CTA owns at most one token");
    extern __shared__ __align__(16) unsigned char smem[];
    FewRoom<PER>& sm = *reinterpret_cast<FewRoom<PER>*>(smem);
    ChoiceRoom<PER>& room = sm.room;
    float* z = room.z;
    uint4* xs = reinterpret_cast<uint4*>(smem + sizeof(FewRoom<PER>));     // [TB][H / 8]
    __shared__ float w2_of[kFewCluster * kGateWarps], x2_of[kGateWarps];
    __shared__ int cancelled;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, chunks = H / 8;
    const int rank = blockIdx.x % kFewCluster, t0 = (blockIdx.x / kFewCluster) * TB, n_tok = min(TB, T - t0);
    grid_dependency_wait();
    grid_launch_dependents();
    constexpr int JB = 8;                                                  // chunks of an expert in flight
    const int gw = rank * kGateWarps + warp;
    uint4 raw[JB];
    auto fetch = [&](int e, int j0) {
#pragma unroll
        for (int j = 0; j < JB; ++j) {
            const int i = lane + 32 * (j0 + j);
            raw[j] = make_uint4(0, 0, 0, 0);
            if (i < chunks && e < g.E) raw[j] = reinterpret_cast<const uint4*>(w_router + (size_t)e * H)[i];
        }
    };
    fetch(gw, 0);                                                          // in flight while the hidden rows are staged
    const uint4* xrow = reinterpret_cast<const uint4*>(hidden + (size_t)t0 * H);
    for (int i = tid; i < n_tok * chunks; i += kGateThreads) xs[i] = xrow[i];
    for (int i = n_tok * chunks + tid; i < TB * chunks; i += kGateThreads) xs[i] = make_uint4(0, 0, 0, 0);
    cg::cluster_group cluster = cg::this_cluster();
    if (tid == 0) cancelled = 0;
    for (int e = tid; e < 32 * PER; e += kGateThreads) {
        if (e >= g.E) z[e] = -INFINITY;
        if (g.balance) sm.balance[e] = e < g.E ? g.balance[e] : 0.f;
    }
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // every CTA runs: its memory may be written
    const int nj = (chunks + 31) / 32;
    auto cost = [&](int j) { return (float)(10 + nj - j); };
    {
        float x2 = 0.f;                                                    // sum c |x|^2 of the token that this CTA owns
        if (rank < n_tok)
            for (int i = tid; i < chunks; i += kGateThreads) x2 = fmaf(cost(i >> 5), square8(xs[(size_t)rank * chunks + i]), x2);
        x2 = warp_sum_f32(x2);
        if (lane == 0) x2_of[warp] = x2;
    }
    bool joined = false;
    float w2_top = 0.f;
    for (int e = gw; e < g.E; e += kFewCluster * kGateWarps) {
        float acc[TB], w2 = 0.f;
#pragma unroll
        for (int t = 0; t < TB; ++t) acc[t] = 0.f;
        for (int j0 = 0; j0 < nj; j0 += JB) {
            if (j0 > 0 || e != gw) fetch(e, j0);
#pragma unroll
            for (int j = 0; j < JB; ++j) {
                if (j0 + j >= nj) break;
                const int i = lane + 32 * (j0 + j);
                float w[8];
                unpack8(raw[j], w);
                w2 = fmaf(cost(j0 + j), dot8(w, w), w2);
#pragma unroll
                for (int t = 0; t < TB; ++t) {
                    float x[8];
                    unpack8(i < chunks ? xs[t * chunks + i] : make_uint4(0, 0, 0, 0), x);
                    acc[t] += dot8(w, x);
                }
            }
        }
        if (!joined) {                                                     // before the first store into another CTA's memory
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            joined = true;
        }
        w2_top = fmaxf(w2_top, warp_sum_f32(w2));
        const float b = bias ? bias[e] : 0.f;
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            float sum = warp_sum_f32(acc[t]);
            if (lane == 0 && t < n_tok) {
                sum += b;
                if (addend) {
                    const float before = fabsf(sum);
                    sum += addend[(size_t)(t0 + t) * g.E + e];
                    if (before > 2.f * fabsf(sum) + 16.f) *cluster.map_shared_rank(&cancelled, t) = 1;
                }
                cluster.map_shared_rank(z, t)[e] = sum;
            }
        }
    }
    if (!joined) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (lane < kFewCluster) cluster.map_shared_rank(w2_of, lane)[gw] = w2_top;
    cluster.sync();
    if (rank >= n_tok) return;
    const size_t t = t0 + rank;
    float dz = 0.f;
    if (warp == 0) {
        float w2 = 0.f, x2 = 0.f;
#pragma unroll
        for (int i = 0; i < kFewCluster * kGateWarps; i += 32) w2 = fmaxf(w2, w2_of[i + lane]);
        w2 = warp_max(w2);
#pragma unroll
        for (int i = 0; i < kGateWarps; ++i) x2 += x2_of[i];
        if (x2 == 0.f && any_number(xs + (size_t)rank * chunks, chunks, lane, 32)) x2 = kLeastSquare;
        // the norms come out of binary32 sums, short by less than 1 %
        dz = x2 == 0.f && !(bias && addend) ? 0.f : 1.01f * 0x1p-24f * sqrtf(least_of(x2)) * sqrtf(fmaxf(w2, kLeastSquare)) + (addend ? 16.f * 0x1p-24f : 0.f);
        if (cancelled) dz = INFINITY;
    }
    const float* balance = g.balance ? sm.balance : nullptr;
    const float rel = (bias || addend) && dz > 0.f ? kAddedRel : 0.f;
    int32_t* ids_t = ids + t * g.k;
    float* weights_t = weights + t * g.k;
    for (int mode = GATE_NEW;;) {
        const bool open = warp == 0 && (mode == GATE_WAITS || (mode != GATE_DONE && choose_fast<PER>(g, room, balance, dz, rel, lane, mode, ids_t, weights_t)));
        if (!__syncthreads_or(open)) return;
        int item = 0;
        for (int b = 0; 32 * b < g.E; ++b)
            for (unsigned es = room.todo[b]; es; es &= es - 1, ++item) {
                if (item % kGateWarps != warp) continue;
                const int e = 32 * b + __ffs(es) - 1;
                const double v = logit_f64<true>(xs + (size_t)rank * chunks, reinterpret_cast<const uint4*>(w_router + (size_t)e * H), 0, chunks, lane);
                if (lane == 0) sm.z64[e] = v + (bias ? (double)bias[e] : 0.0) + (addend ? (double)addend[t * g.E + e] : 0.0);
            }
        __syncthreads();
        if (warp == 0) mode = go_on<PER>(g, room, balance, sm.z64, dz, rel, lane, ids_t, weights_t);
    }
}

int check_gate(const exmoe_shape* shape, const exmoe_gate* gate, int T, GateArgs* a) {
    if (!shape || !gate || T < 0 || T > kMaxTokens) return EXMOE_ERR_ARG;
    if ((gate->score != EXMOE_SCORE_SOFTMAX && gate->score != EXMOE_SCORE_SIGMOID) ||
        (gate->group_score != EXMOE_GROUP_MAX && gate->group_score != EXMOE_GROUP_TOP2) || (gate->renormalise != 0 && gate->renormalise != 1))
        return EXMOE_ERR_ARG;
    if (shape->num_experts <= 0 || shape->num_experts > 4096 || shape->top_k <= 0) return EXMOE_ERR_SHAPE;
    if (gate->num_groups < 1 || gate->num_groups > 32 || shape->num_experts % gate->num_groups || gate->top_groups < 1 ||
        gate->top_groups > gate->num_groups)
        return EXMOE_ERR_SHAPE;
    const int size = shape->num_experts / gate->num_groups;
    if (shape->top_k > gate->top_groups * size) return EXMOE_ERR_SHAPE;
    int log_lanes = 5;
    while (gate->num_groups << log_lanes > 32) --log_lanes;
    *a = GateArgs{shape->num_experts, shape->top_k, gate->num_groups, size, gate->top_groups, gate->score == EXMOE_SCORE_SIGMOID,
                  gate->group_score == EXMOE_GROUP_TOP2, gate->renormalise != 0, gate->weight_scale, nullptr, 1 << log_lanes, log_lanes, (size + (1 << log_lanes) - 1) >> log_lanes, -1, 1.f / (float)size};
    if (shape->num_experts <= kFastExperts) {                              // choose_fast's run of a lane
        const int run = shape->num_experts <= 64 ? 2 : shape->num_experts <= 128 ? 4 : shape->num_experts <= 256 ? 8 : 16;
        for (int l = 0; l <= 5; ++l)
            if (run << l == size) a->log_run = l;
    }
    return EXMOE_OK;
}

// From how many tokens on the tensor cores (at most 256 experts) are faster than four tokens per cluster, by the size of the router's matrix.
// us, four / tensor cores, means of four batches: 16 experts of d_model 512: 256 tokens 10.2 / 10.9, 384: 13.9 / 10.9.   64 of 2048: 128 9.1 / 12.0,
// 192: 13.7 / 12.8.   128 of 2048: 128 14.8 / 17.1, 192: 20.0 / 18.1.   256 of 1024: 128 14.9 / 16.9, 192: 20.9 / 16.9.   64 of 4096: 128 14.0 / 14.7,
// 192: 18.2 / 14.7.   256 of 4096: 48 19.5 / 21.4, 64: 26.7 / 24.5.
constexpr int kManyExperts = 256;
constexpr int many_tokens(int E, int H) {
    const long long n = (long long)E * H;
    return n <= 1 << 14 ? 288 : n <= 3 << 16 ? 176 : n <= 1 << 19 ? 150 : 56;
}

// A call's kernels by the number of experts: what choose_fast holds per lane.
template <int TB, int PER>
int launch_few(const __nv_bfloat16* x, const __nv_bfloat16* w, const float* bias, const float* addend, int T, int H, const GateArgs& g, int32_t* ids,
               float* wts, cudaStream_t st) {
    static SmemOnce once;
    const size_t smem = sizeof(FewRoom<PER>) + (size_t)TB * H * 2;
    return launch(gate_few_kernel<TB, PER>, (unsigned)((T + TB - 1) / TB * kFewCluster), kGateThreads, kFewCluster, smem, once, st, x, w, bias, addend, T, H, g, ids, wts);
}
template <int TB>
int launch_few(const __nv_bfloat16* x, const __nv_bfloat16* w, const float* bias, const float* addend, int T, int H, const GateArgs& g, int32_t* ids,
               float* wts, cudaStream_t st) {
    if (g.E <= 64) return launch_few<TB, 2>(x, w, bias, addend, T, H, g, ids, wts, st);
    if (g.E <= 128) return launch_few<TB, 4>(x, w, bias, addend, T, H, g, ids, wts, st);
    if (g.E <= 256) return launch_few<TB, 8>(x, w, bias, addend, T, H, g, ids, wts, st);
    return launch_few<TB, 16>(x, w, bias, addend, T, H, g, ids, wts, st);
}
template <typename Z, int PER>
int launch_logits(const Z* z, long long ld, int T, const GateArgs& g, int32_t* ids, float* wts, cudaStream_t st) {
    static SmemOnce once;
    const size_t bias = PER && g.balance ? 128 * PER : 0, room = logits_room<PER>(g.E);
    const int warps = std::max(1, std::min(kGateWarps, (int)((kGateSmemMax - bias) / room)));
    return launch(gate_logits_kernel<Z, PER>, (unsigned)(((long long)T + warps - 1) / warps), 32 * warps, 1, warps * room + bias, once, st, z, ld, T, g, ids, wts);
}
template <typename Z>
int launch_logits(const Z* z, long long ld, int T, const GateArgs& g, int32_t* ids, float* wts, cudaStream_t st) {
    if (g.E > kFastExperts || g.k > kFastChoices) return launch_logits<Z, 0>(z, ld, T, g, ids, wts, st);
    if (g.E <= 64) return launch_logits<Z, 2>(z, ld, T, g, ids, wts, st);
    if (g.E <= 128) return launch_logits<Z, 4>(z, ld, T, g, ids, wts, st);
    if (g.E <= 256) return launch_logits<Z, 8>(z, ld, T, g, ids, wts, st);
    return launch_logits<Z, 16>(z, ld, T, g, ids, wts, st);
}

}  // namespace

extern "C" int exmoe_route_gated(const exmoe_shape* shape, const exmoe_gate* gate, const void* hidden_bf16, const void* router_bf16,
                                 const float* bias, const float* addend, const float* balance, int T, int32_t* topk_ids,
                                 float* topk_weights, void* stream) {
    GateArgs g;
    const int rc = check_gate(shape, gate, T, &g);
    if (rc) return rc;
    const int H = shape->d_model;
    if (H <= 0 || H % 8 || 2 * (size_t)H + 16 * (size_t)g.E > (size_t)kGateSmemMax) return EXMOE_ERR_SHAPE;
    if (T == 0) return EXMOE_OK;
    if (!hidden_bf16 || !router_bf16 || !topk_ids || !topk_weights) return EXMOE_ERR_ARG;
    if (!aligned(16, hidden_bf16, router_bf16) || !aligned(4, bias, addend, balance, topk_ids, topk_weights)) return EXMOE_ERR_ARG;
    g.balance = balance;
    const __nv_bfloat16 *x = (const __nv_bfloat16*)hidden_bf16, *w = (const __nv_bfloat16*)router_bf16;
    cudaStream_t st = (cudaStream_t)stream;
    if (g.E <= kManyExperts && g.k <= kFastChoices && T >= many_tokens(g.E, H) && H >= 64) return launch_gate_tc(x, w, bias, addend, T, H, g, topk_ids, topk_weights, st);
    if (g.E <= kFastExperts && g.k <= kFastChoices && sizeof(FewRoom<16>) + 8 * (size_t)H <= (size_t)kGateSmemMax)
        return T < kFewFour ? launch_few<1>(x, w, bias, addend, T, H, g, topk_ids, topk_weights, st) : launch_few<4>(x, w, bias, addend, T, H, g, topk_ids, topk_weights, st);
    static SmemOnce once;
    return launch(gate_token_kernel, (unsigned)T, kGateThreads, 1, 2 * (size_t)H + 16 * (size_t)g.E, once, st, x, w, bias, addend, H, g, topk_ids, topk_weights);
}

extern "C" int exmoe_debug_gate_timeout(const exmoe_shape* shape, const exmoe_gate* gate, const void* hidden_bf16, const void* router_bf16, int T, int32_t* topk_ids,
                                       float* topk_weights, void* stream) {
    GateArgs g;
    const int rc = check_gate(shape, gate, T, &g);
    if (rc) return rc;
    const int H = shape->d_model;
    if (g.E > 64 || g.k > kFastChoices || H % 8 || H < 1024 || 2 * (size_t)H + 16 * (size_t)g.E > (size_t)kGateSmemMax) return EXMOE_ERR_SHAPE;
    if (T == 0 || !hidden_bf16 || !router_bf16 || !topk_ids || !topk_weights) return EXMOE_ERR_ARG;
    if (!aligned(16, hidden_bf16, router_bf16) || !aligned(4, topk_ids, topk_weights)) return EXMOE_ERR_ARG;
    return launch_gate_tc_stuck((const __nv_bfloat16*)hidden_bf16, (const __nv_bfloat16*)router_bf16, T, H, g, topk_ids, topk_weights, (cudaStream_t)stream);
}

extern "C" int exmoe_gate_logits(const exmoe_shape* shape, const exmoe_gate* gate, const void* logits, int type, int64_t row_stride,
                                 const float* balance, int T, int32_t* topk_ids, float* topk_weights, void* stream) {
    GateArgs g;
    const int rc = check_gate(shape, gate, T, &g);
    if (rc) return rc;
    if ((type != EXMOE_F32 && type != EXMOE_BF16) || row_stride < 0 || (T > 1 && row_stride < g.E)) return EXMOE_ERR_ARG;
    if (T == 0) return EXMOE_OK;
    if (!logits || !topk_ids || !topk_weights) return EXMOE_ERR_ARG;
    if (!aligned(type == EXMOE_F32 ? 4 : 2, logits) || !aligned(4, balance, topk_ids, topk_weights)) return EXMOE_ERR_ARG;
    g.balance = balance;
    cudaStream_t st = (cudaStream_t)stream;
    return type == EXMOE_F32 ? launch_logits((const float*)logits, row_stride, T, g, topk_ids, topk_weights, st)
                             : launch_logits((const __nv_bfloat16*)logits, row_stride, T, g, topk_ids, topk_weights, st);
}

}  // namespace exmoe
