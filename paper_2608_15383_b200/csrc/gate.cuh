// The choice of a gate (exmoe_gate) from a token's logits, shared by the kernels that end in it.
#pragma once
#include "common.cuh"

namespace exmoe {

struct GateArgs {
    int E, k, G, size, top_groups;     // experts, choices, groups, experts per group, groups kept (G where there are no groups)
    bool sigmoid, top2, renorm;
    float scale;
    const float* balance;              // [E] or null
};

// Doubles as integers of the same order: 0 is left for an expert that cannot be chosen, 1 is a NaN, -infinity follows; zeros of both signs are equal.
__device__ __forceinline__ unsigned long long order_key(double v) {
    if (v != v) return 1ull;
    const unsigned long long b = (unsigned long long)__double_as_longlong(v + 0.0);
    return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ double warp_sum_f64(double s) {
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
    return s;
}

// The groups that keep their experts (a bit each), from lane g's value of group g.
template <typename T>
__device__ __forceinline__ unsigned kept_groups(T value, int G, int top_groups, int lane) {
    int before = 0;
    for (int g = 0; g < G; ++g) {
        const T v = __shfl_sync(0xffffffffu, value, g);
        before += v > value || (v == value && g < lane);
    }
    return __ballot_sync(0xffffffffu, lane < G && before < top_groups);
}

// The whole choice in binary64, by one warp.  z: the token's logits, key: room for as many integers (both in shared memory).
__device__ __noinline__ void choose_exact(const GateArgs& g, const double* z, unsigned long long* key, int lane, int32_t* ids, float* weights) {
    const double kMasked = -INFINITY;
    double* c = reinterpret_cast<double*>(key);
    const bool grouped = g.top_groups < g.G;
    double mx = kMasked, inv = 1.0;
    if (!g.sigmoid) {
        for (int e = lane; e < g.E; e += 32) mx = fmax(mx, z[e]);          // fmax leaves a NaN out
#pragma unroll
        for (int m = 16; m >= 1; m >>= 1) mx = fmax(mx, __shfl_xor_sync(0xffffffffu, mx, m));
        if (mx == kMasked) mx = 0.0;
        double sum = 0.0;
        for (int e = lane; e < g.E; e += 32) sum += exp(z[e] - mx);
        sum = warp_sum_f64(sum);
        inv = sum == 0.0 ? 0.0 : 1.0 / sum;
    }
    auto score = [&](double v) { return g.sigmoid ? 1.0 / (1.0 + exp(-v)) : exp(v - mx) * inv; };
    unsigned kept = 0xffffffffu;
    const bool by_score = g.balance || (grouped && g.top2);
    if (by_score)
        for (int e = lane; e < g.E; e += 32)
            c[e] = z[e] == kMasked ? kMasked : score(z[e]) + (g.balance ? (double)g.balance[e] : 0.0);
    __syncwarp();
    const double* by = g.balance ? c : z;                                  // what orders the experts
    if (grouped) {
        double value = kMasked;
        if (lane < g.G) {
            const double* v = (g.top2 ? c : by) + lane * g.size;
            double a = kMasked, b = kMasked;
            for (int i = 0; i < g.size; ++i) {
                if (v[i] > a) {
                    b = a;
                    a = v[i];
                } else if (v[i] > b) {
                    b = v[i];
                }
            }
            value = g.top2 && b > kMasked ? a + b : a;
        }
        kept = kept_groups(value, g.G, g.top_groups, lane);
        __syncwarp();
    }
    for (int e = lane; e < g.E; e += 32) key[e] = !grouped || (kept >> (e / g.size) & 1u) ? order_key(by[e]) : 0ull;
    double total = 0.0;
    for (int j = 0; j < g.k; ++j) {
        unsigned long long best = 0;
        int at = 0x7fffffff;
        for (int e = lane; e < g.E; e += 32)
            if (key[e] > best) {                                           // ascending e: the first maximum wins
                best = key[e];
                at = e;
            }
        const unsigned hi = __reduce_max_sync(0xffffffffu, (unsigned)(best >> 32));
        const unsigned lo = __reduce_max_sync(0xffffffffu, (unsigned)(best >> 32) == hi ? (unsigned)best : 0u);
        const bool mine = (unsigned)(best >> 32) == hi && (unsigned)best == lo;
        const int e = (int)__reduce_min_sync(0xffffffffu, mine ? (unsigned)at : 0x7fffffffu);
        total += score(z[e]);
        if (lane == 0) {
            ids[j] = e;
            key[e] = 0ull;
        }
        __syncwarp();
    }
    const double f = g.renorm ? (total == 0.0 ? 0.0 : 1.0 / total) : 1.0;
    for (int j = lane; j < g.k; j += 32) weights[j] = (float)(score(z[ids[j]]) * f * (double)g.scale);
}

}  // namespace exmoe
