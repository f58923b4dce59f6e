// Products with an epilogue (exmoe_linear): out = residual + act(x W^T + bias), or residual + act(x W^T + bias) * (x U^T + bias_up).
#include <algorithm>

#include "common.cuh"
#include "frag.cuh"
#include "linear.cuh"

namespace exmoe {

namespace {

constexpr int kMaxTokens = 1 << 29, kMaxDim = 1 << 30, kSms = 148;
__host__ __device__ constexpr int few_chain(int warps) { return 32 * 16 * warps; }        // the K that chains of 32 MMAs of a CTA's warps make

// Few tokens.  A CTA takes 16 rows of W (8 of W and 8 of U: the two factors meet in one lane) and 8 NT tokens; its warps split K.
// Weights are the MMA's rows: a lane's 16 bytes of a row are k = 8 c .. 8 c + 7 of every 32, the k that two MMAs take from it, and the
// tokens are read in the same order.
// A CTA goes through groups of rows; a warp has its next weights and tokens on their way while the group's parts are added up.
// WARPS: 8, two CTAs per SM, or, where the SMs have a group each at most, 16 that share it (us, replayed from a graph, 8 / 16 warps: 2048 -> 2048 outputs 3.5 / 3.2,
// 5632 -> 2048 7.4 / 6.2, 16 tokens 9.6 / 8.2; 2048 -> 5632 6.2 / 7.5, gated 8.7 / 10.2, 8192 -> 8192 22.4 / 25.8).  Either way an SM has 128 KB
// (NT = 2: 64) of weights on their way.  Bound by HBM and by 2 us of launch and latency: one token, two matrices 2048 -> 5632, 46 MB in 8.7 us (5.3 TB/s); 5632 -> 2048, 23 MB in
// 6.2 us (3.7 TB/s).
// LONG: chains of 32 MMAs, added in binary32 in shared memory.  The instructions truncate what they add (3.5e-4 over 8192 of them where all products have
// one sign).  (In a form of its own: the loop around it takes calls with one chain 0.3 us; FP32 8192 -> 8192 outputs 23.5 -> 23.9 us with 1 token, 24.5 -> 25.2 with 8.)
template <typename O, int NT, bool GATED, int WARPS, bool LONG>
__global__ void __launch_bounds__(32 * WARPS, 16 / WARPS)
linear_few_kernel(const __grid_constant__ LinearArgs a, int rows, int groups) {
    constexpr int kFewThreads = 32 * WARPS, kFewWarps = WARPS, kAhead = (NT == 1 ? 64 : 32) / WARPS;
    constexpr int kChain = few_chain(WARPS) / (32 * WARPS * kAhead);              // batches of a chain
    __shared__ float part[2][kFewWarps][NT][16][9];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    {   // into L2, before the wait (the kernel in front may be writing them: L2 has what it writes)
        const long long n0 = (long long)blockIdx.x * rows;
        const int n_rows = (int)min((long long)rows, a.N - n0);
        if (tid < (GATED ? 2 : 1) * n_rows) {
            const __nv_bfloat16* row = tid < n_rows ? a.w + (n0 + tid) * a.ld_w : a.w_up + (n0 + tid - n_rows) * a.ld_up;
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(row), "r"(2 * min(a.K, 1 << 19)) : "memory");
        }
    }
    grid_dependency_wait();
    grid_launch_dependents();
    const uint4 zero = make_uint4(0, 0, 0, 0);
    const int blocks = (a.K + 31) / 32, batches = max(1, (blocks + kFewWarps * kAhead - 1) / (kFewWarps * kAhead));
    uint4 va[kAhead], vb[kAhead], vx[kAhead][NT];
    const auto load = [&](int group, int batch) {
        const long long n0 = (long long)group * rows;
        const int n_rows = (int)min((long long)rows, a.N - n0);
        const bool row_a = g < n_rows, row_b = GATED ? row_a : 8 + g < n_rows;
        const __nv_bfloat16* wa = a.w + (n0 + g) * a.ld_w + 8 * c;
        const __nv_bfloat16* wb = GATED ? a.w_up + (n0 + g) * a.ld_up + 8 * c : a.w + (n0 + 8 + g) * a.ld_w + 8 * c;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int k = (warp + (batch * kAhead + u) * kFewWarps) * 32;
            const bool in = k + 8 * c < a.K;
            va[u] = in && row_a ? *reinterpret_cast<const uint4*>(wa + k) : zero;
            vb[u] = in && row_b ? *reinterpret_cast<const uint4*>(wb + k) : zero;
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const int t = 8 * i + g;
                vx[u][i] = in && t < a.T ? *reinterpret_cast<const uint4*>(a.x + t * a.ld_x + 8 * c + k) : zero;
            }
        }
    };
    int group = blockIdx.x;
    if (group < groups) load(group, 0);
    for (int turn = 0; group < groups; turn ^= 1) {
        const int next = group + (int)gridDim.x;
        int first = 0;
        do {
            float acc[NT][4];
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = 0.f;
            for (int batch = first; batch < (LONG ? min(batches, first + kChain) : batches); ++batch) {
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        mma_m16n8k16(acc[i], va[u].x, vb[u].x, va[u].y, vb[u].y, vx[u][i].x, vx[u][i].y);
                        mma_m16n8k16(acc[i], va[u].z, vb[u].z, va[u].w, vb[u].w, vx[u][i].z, vx[u][i].w);
                    }
                if (batch + 1 < batches) load(group, batch + 1);
                else if (next < groups) load(next, 0);
            }
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float& p = part[turn][warp][i][g + 8 * (j >> 1)][2 * c + (j & 1)];
                    p = LONG && first ? p + acc[i][j] : acc[i][j];
                }
            first += kChain;
        } while (LONG && first < batches);
        __syncthreads();                                                   // (a warp writes these parts again behind the next one: all have read them by then)
        const long long n0 = (long long)group * rows;
        const int n_rows = (int)min((long long)rows, a.N - n0);
        for (int i = tid; i < NT * 8 * n_rows; i += kFewThreads) {
            const int r = i % n_rows, tt = i / n_rows, nt = tt >> 3, col = tt & 7;
            const long long n = n0 + r;
            if (tt >= a.T) continue;
            float v = 0.f, u = 0.f;
#pragma unroll
            for (int w = 0; w < kFewWarps; ++w) {
                v += part[turn][w][nt][r][col];
                if (GATED) u += part[turn][w][nt][8 + r][col];
            }
            v = activate(v + (a.bias ? a.bias[n] : 0.f), a.act);
            if (GATED) v *= u + (a.bias_up ? a.bias_up[n] : 0.f);
            if (a.residual) v += load_out<O>(a.residual, tt * a.ld_res + n);
            store_out(static_cast<O*>(a.out) + tt * a.ld_out + n, v);
        }
        group = next;
    }
}

template <typename O, int NT, bool GATED, int WARPS, bool LONG>
int launch_few(const LinearArgs& a, cudaStream_t st) {
    // as many rows, up to 16 (8 of each matrix), as spread evenly over the CTAs that the chip holds
    constexpr int most = GATED ? 8 : 16;
    constexpr long long ctas = kSms * (16 / WARPS);
    const long long turns = (a.N + most * ctas - 1) / (most * ctas), rows = (a.N + ctas * turns - 1) / (ctas * turns);
    cudaLaunchConfig_t lc{};
    const long long groups = (a.N + rows - 1) / rows;
    lc.gridDim = dim3((unsigned)std::min(groups, ctas));
    lc.blockDim = dim3(32 * WARPS);
    lc.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
#ifdef EXMOE_DISABLE_PDL
    lc.numAttrs = 0;
#endif
    if (cudaLaunchKernelEx(&lc, linear_few_kernel<O, NT, GATED, WARPS, LONG>, a, (int)rows, (int)groups) != cudaSuccess) {
        cudaGetLastError();
        return EXMOE_ERR_CUDA;
    }
    count_launch();
    return EXMOE_OK;
}
constexpr int kFewTokens = 16;                                             // (two MMAs of 8: 16 tokens 2048 -> 2048 4.1 us; on tcgen05 17 take 5.6)
template <typename O, bool GATED, int WARPS>
int launch_few_tokens(const LinearArgs& a, cudaStream_t st) {
    constexpr int kMostShort = few_chain(WARPS) * (sizeof(O) == 4 ? 1 : 32);    // (in front of a BF16 result 1024 MMAs: 1e-4, a fortieth of half a step)
    if (a.K <= kMostShort) return a.T <= 8 ? launch_few<O, 1, GATED, WARPS, false>(a, st) : launch_few<O, 2, GATED, WARPS, false>(a, st);
    return a.T <= 8 ? launch_few<O, 1, GATED, WARPS, true>(a, st) : launch_few<O, 2, GATED, WARPS, true>(a, st);
}
template <typename O, bool GATED>
int launch_few_tokens(const LinearArgs& a, cudaStream_t st) {
    return a.N <= kSms * (GATED ? 8 : 16) ? launch_few_tokens<O, GATED, 16>(a, st) : launch_few_tokens<O, GATED, 8>(a, st);
}

}  // namespace

static int linear_call(const exmoe_linear_shape* shape, const void* x, int64_t ld_x, const void* w, int64_t ld_w, const float* bias, const void* w_up,
                       int64_t ld_w_up, const float* bias_up, int T, const void* residual, int64_t ld_residual, void* out, int64_t ld_out, int type, bool stuck,
                       void* stream) {
    if (!shape || T < 0 || T > kMaxTokens || (type != EXMOE_F32 && type != EXMOE_BF16)) return EXMOE_ERR_ARG;
    const int K = shape->d_in, N = shape->d_out;
    if (shape->activation < EXMOE_ACT_NONE || shape->activation > EXMOE_ACT_SILU) return EXMOE_ERR_ARG;
    if (K <= 0 || K % 8 || N <= 0 || K > kMaxDim || N > kMaxDim) return EXMOE_ERR_SHAPE;
    if (T == 0) return EXMOE_OK;
    if (!x || !w || !out || (bias_up && !w_up)) return EXMOE_ERR_ARG;
    if (ld_x < K || ld_x % 8 || ld_w < K || ld_w % 8 || (w_up && (ld_w_up < K || ld_w_up % 8)) || ld_out < N || (residual && ld_residual < N)) return EXMOE_ERR_ARG;
    const long long es = type == EXMOE_F32 ? 4 : 2;
    if (!aligned(16, x, w, w_up) || !aligned(4, bias, bias_up) || !aligned(es, residual, out)) return EXMOE_ERR_ARG;
    const Range o = range_of(out, T, ld_out, N, es);
    if ((!(residual == out && (ld_residual == ld_out || T == 1)) && overlap(o, range_of(residual, T, ld_residual, N, es))) || overlap(o, range_of(x, T, ld_x, K, 2)) ||
        overlap(o, range_of(w, N, ld_w, K, 2)) || overlap(o, range_of(w_up, N, ld_w_up, K, 2)) || overlap(o, range_of(bias, 1, 0, N, 4)) ||
        overlap(o, range_of(bias_up, 1, 0, N, 4)))
        return EXMOE_ERR_ARG;
    const LinearArgs a{(const __nv_bfloat16*)x, (const __nv_bfloat16*)w, (const __nv_bfloat16*)w_up, bias, bias_up, residual, out, ld_x, ld_w, ld_w_up,
                       ld_residual, ld_out, T, K, N, shape->activation};
    cudaStream_t st = (cudaStream_t)stream;
    if (stuck) return T > kFewTokens && K >= 1024 ? launch_linear_tc_stuck(a, st) : EXMOE_ERR_SHAPE;
    if (T > kFewTokens) return launch_linear_tc(a, type, st);
    if (type == EXMOE_F32) return w_up ? launch_few_tokens<float, true>(a, st) : launch_few_tokens<float, false>(a, st);
    return w_up ? launch_few_tokens<__nv_bfloat16, true>(a, st) : launch_few_tokens<__nv_bfloat16, false>(a, st);
}

extern "C" int exmoe_linear(const exmoe_linear_shape* shape, const void* x, int64_t ld_x, const void* w, int64_t ld_w, const float* bias, const void* w_up,
                            int64_t ld_w_up, const float* bias_up, int T, const void* residual, int64_t ld_residual, void* out, int64_t ld_out, int type,
                            void* stream) {
    return linear_call(shape, x, ld_x, w, ld_w, bias, w_up, ld_w_up, bias_up, T, residual, ld_residual, out, ld_out, type, false, stream);
}

extern "C" int exmoe_debug_linear_timeout(const exmoe_linear_shape* shape, const void* x, const void* w, int T, void* out, void* stream) {
    if (!shape || T == 0) return EXMOE_ERR_ARG;
    return linear_call(shape, x, shape->d_in, w, shape->d_in, nullptr, nullptr, 0, nullptr, T, nullptr, 0, out, shape->d_out, EXMOE_BF16, true, stream);
}

}  // namespace exmoe
