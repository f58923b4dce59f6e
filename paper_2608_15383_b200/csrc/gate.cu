// The gate of a sparse block (exmoe_gate): scores, balance bias, groups, top-k, weights; from hidden states or from logits.
#include <algorithm>

#include "gate.cuh"

namespace exmoe {

namespace {

constexpr int kGateThreads = 256, kGateWarps = kGateThreads / 32;
constexpr int kGateSmemMax = 200 * 1024;

// One CTA per token, everything in binary64: products of BF16 values are exact in binary32.
__global__ void __launch_bounds__(kGateThreads)
gate_token_kernel(const __nv_bfloat16* hidden, const __nv_bfloat16* __restrict__ w_router, const float* __restrict__ bias,
                  const float* addend, int H, GateArgs g, int32_t* ids, float* weights) {
    extern __shared__ __align__(16) unsigned char smem[];
    double* z = reinterpret_cast<double*>(smem);
    unsigned long long* key = reinterpret_cast<unsigned long long*>(z + g.E);
    uint4* xs = reinterpret_cast<uint4*>(smem + (((size_t)g.E * 16 + 15) & ~size_t(15)));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, chunks = H / 8;
    const size_t t = blockIdx.x;
    const uint4* xrow = reinterpret_cast<const uint4*>(hidden + t * H);
    for (int i = tid; i < chunks; i += kGateThreads) xs[i] = xrow[i];
    __syncthreads();
    for (int e = warp; e < g.E; e += kGateWarps) {
        const uint4* wrow = reinterpret_cast<const uint4*>(w_router + (size_t)e * H);
        double s = 0.0;
        for (int i = lane; i < chunks; i += 32) {
            const uint4 wv = wrow[i], xv = xs[i];
            const uint32_t wr[4] = {wv.x, wv.y, wv.z, wv.w}, xr[4] = {xv.x, xv.y, xv.z, xv.w};
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                s += (double)(__uint_as_float(wr[n] << 16) * __uint_as_float(xr[n] << 16));
                s += (double)(__uint_as_float(wr[n] & 0xffff0000u) * __uint_as_float(xr[n] & 0xffff0000u));
            }
        }
        s = warp_sum_f64(s);
        if (lane == 0) z[e] = s + (bias ? (double)bias[e] : 0.0) + (addend ? (double)addend[t * g.E + e] : 0.0);
    }
    __syncthreads();
    if (warp == 0) choose_exact(g, z, key, lane, ids + t * g.k, weights + t * g.k);
}

// One warp per token.
template <typename Z>
__global__ void __launch_bounds__(kGateThreads)
gate_logits_kernel(const Z* logits, long long ld, int T, GateArgs g, int32_t* ids, float* weights) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double* z = reinterpret_cast<double*>(smem) + (size_t)warp * 2 * g.E;
    unsigned long long* key = reinterpret_cast<unsigned long long*>(z + g.E);
    const size_t t = (size_t)blockIdx.x * (blockDim.x >> 5) + warp;
    if (t >= (size_t)T) return;
    for (int e = lane; e < g.E; e += 32) z[e] = (double)(float)logits[(long long)t * ld + e];
    __syncwarp();
    choose_exact(g, z, key, lane, ids + t * g.k, weights + t * g.k);
}

int check_gate(const exmoe_shape* shape, const exmoe_gate* gate, int T, GateArgs* a) {
    if (!shape || !gate || T < 0) return EXMOE_ERR_ARG;
    if ((gate->score != EXMOE_SCORE_SOFTMAX && gate->score != EXMOE_SCORE_SIGMOID) ||
        (gate->group_score != EXMOE_GROUP_MAX && gate->group_score != EXMOE_GROUP_TOP2) || (gate->renormalise != 0 && gate->renormalise != 1))
        return EXMOE_ERR_ARG;
    if (shape->num_experts <= 0 || shape->num_experts > 4096 || shape->top_k <= 0) return EXMOE_ERR_SHAPE;
    if (gate->num_groups < 1 || gate->num_groups > 32 || shape->num_experts % gate->num_groups || gate->top_groups < 1 ||
        gate->top_groups > gate->num_groups)
        return EXMOE_ERR_SHAPE;
    const int size = shape->num_experts / gate->num_groups;
    if (shape->top_k > gate->top_groups * size) return EXMOE_ERR_SHAPE;
    *a = GateArgs{shape->num_experts, shape->top_k, gate->num_groups, size, gate->top_groups, gate->score == EXMOE_SCORE_SIGMOID,
                  gate->group_score == EXMOE_GROUP_TOP2, gate->renormalise != 0, gate->weight_scale, nullptr};
    return EXMOE_OK;
}
int launched() {
    if (cudaGetLastError() != cudaSuccess) return EXMOE_ERR_CUDA;
    count_launch();
    return EXMOE_OK;
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
    if ((reinterpret_cast<uintptr_t>(hidden_bf16) | reinterpret_cast<uintptr_t>(router_bf16)) & 15) return EXMOE_ERR_ARG;
    g.balance = balance;
    static SmemOnce once;
    if (!allow_smem(gate_token_kernel, kGateSmemMax, once)) return EXMOE_ERR_CUDA;
    gate_token_kernel<<<T, kGateThreads, 2 * (size_t)H + 16 * (size_t)g.E, (cudaStream_t)stream>>>(
        (const __nv_bfloat16*)hidden_bf16, (const __nv_bfloat16*)router_bf16, bias, addend, H, g, topk_ids, topk_weights);
    return launched();
}

extern "C" int exmoe_gate_logits(const exmoe_shape* shape, const exmoe_gate* gate, const void* logits, int type, int64_t row_stride,
                                 const float* balance, int T, int32_t* topk_ids, float* topk_weights, void* stream) {
    GateArgs g;
    const int rc = check_gate(shape, gate, T, &g);
    if (rc) return rc;
    if ((type != EXMOE_F32 && type != EXMOE_BF16) || row_stride < 0 || (T > 1 && row_stride < g.E)) return EXMOE_ERR_ARG;
    if (T == 0) return EXMOE_OK;
    if (!logits || !topk_ids || !topk_weights) return EXMOE_ERR_ARG;
    g.balance = balance;
    const int warps = std::max(1, std::min(kGateWarps, (int)(kGateSmemMax / (16 * (size_t)g.E))));
    const size_t smem = (size_t)warps * 16 * g.E;
    const unsigned ctas = (unsigned)(((long long)T + warps - 1) / warps);
    static SmemOnce once[2];
    if (type == EXMOE_F32) {
        if (!allow_smem(gate_logits_kernel<float>, kGateSmemMax, once[0])) return EXMOE_ERR_CUDA;
        gate_logits_kernel<float><<<ctas, 32 * warps, smem, (cudaStream_t)stream>>>((const float*)logits, row_stride, T, g, topk_ids, topk_weights);
    } else {
        if (!allow_smem(gate_logits_kernel<__nv_bfloat16>, kGateSmemMax, once[1])) return EXMOE_ERR_CUDA;
        gate_logits_kernel<__nv_bfloat16><<<ctas, 32 * warps, smem, (cudaStream_t)stream>>>((const __nv_bfloat16*)logits, row_stride, T, g, topk_ids, topk_weights);
    }
    return launched();
}

}  // namespace exmoe
