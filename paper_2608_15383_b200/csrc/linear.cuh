// What the kernels of exmoe_linear share: arguments, activations, access to results.
#pragma once
#include "common.cuh"

namespace exmoe {

struct LinearArgs {
    const __nv_bfloat16 *x, *w, *w_up;   // w_up: null without a second factor
    const float *bias, *bias_up;         // or null
    const void* residual;                // or null
    void* out;
    long long ld_x, ld_w, ld_up, ld_res, ld_out;
    int T, K, N, act;
};

__device__ __forceinline__ float activate(float v, int act) {
    switch (act) {
        case EXMOE_ACT_RELU: return v < 0.f ? 0.f : v;                     // a NaN stays one
        case EXMOE_ACT_GELU: {
            // v Phi(v) = max(v, 0) - |v| Phi(-|v|), and Phi(-x) by Abramowitz and Stegun's 7.1.26: (a1 t + ... + a5 t^5) exp(-x^2 / 2) / 2 with
            // t = 1 / (1 + p x / sqrt 2), off by 7.5e-8 at most, and with binary32's roundings by
            // 2.9e-7 (measured; near 0, where Phi is a half).  (normcdff: 130 instructions instead of 15, more than a large product has time for.)
            const float x = fabsf(v), t = __fdividef(1.f, fmaf(0.3275911f * 0.70710678f, x, 1.f));
            const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
            return (v > 0.f ? v : 0.f) - fminf(x, 100.f) * (0.5f * poly * __expf(-0.5f * v * v));
        }
        case EXMOE_ACT_GELU_TANH: {                                        // (1 + tanh y) / 2 = 1 / (1 + exp(-2 y))
            const float y = 0.7978845608028654f * fmaf(0.044715f * v * v, v, v);
            return __fdividef(v, 1.f + __expf(-2.f * y));
        }
        case EXMOE_ACT_SILU: return __fdividef(v, 1.f + __expf(-v));
        default: return v;
    }
}
// (One branch for all: the code of the others is not fetched.)
template <int N>
__device__ __forceinline__ void activate_all(float (&v)[N], int act) {
    switch (act) {
        case EXMOE_ACT_RELU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = activate(v[i], EXMOE_ACT_RELU);
            break;
        case EXMOE_ACT_GELU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = activate(v[i], EXMOE_ACT_GELU);
            break;
        case EXMOE_ACT_GELU_TANH:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = activate(v[i], EXMOE_ACT_GELU_TANH);
            break;
        case EXMOE_ACT_SILU:
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = activate(v[i], EXMOE_ACT_SILU);
            break;
    }
}

template <typename O> __device__ __forceinline__ float load_out(const void* p, long long at);
template <> __device__ __forceinline__ float load_out<float>(const void* p, long long at) { return static_cast<const float*>(p)[at]; }
template <> __device__ __forceinline__ float load_out<__nv_bfloat16>(const void* p, long long at) { return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]); }
__device__ __forceinline__ void store_out(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_out(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

// More than a few tokens, on tensor cores (linear_tc.cu).
int launch_linear_tc(const LinearArgs& a, int type, cudaStream_t st);
int launch_linear_tc_stuck(const LinearArgs& a, cudaStream_t st);

}  // namespace exmoe
