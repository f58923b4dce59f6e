// What a gate is trained with: how often each expert was chosen, the balance loss, the z loss (exmoe_balance_loss), and the gradient of
// the mixture weights and of both losses on the logits (exmoe_gate_backward).
//
// Scores of a token.  Softmax: with m the largest logit, e_i = exp(z_i - m), q_i = e_i / sum e.  Sigmoid: s_i = 1 / (1 + exp(-z_i)),
// q_i = s_i / sum s.  Numerator and sum are both multiplied by exp(-c), c = min(m, 0), so that a row whose sigmoids all leave binary32's range
// keeps its q: with u = exp(-|z|), s_i exp(-c) = a / (1 + u), a = exp(z_i - c) where c < 0, else 1 or u by the sign of z_i.
// log sum exp z = m + log sum e.
//
// Every row is read once and stays in the registers of its team of lanes; column sums stay in registers too (a lane has the same experts in
// every row), and are joined in a fixed order: the results do not depend on the order in which blocks run.
#include <algorithm>

#include "common.cuh"
#include "frag.cuh"
#include "gate.cuh"

namespace exmoe {

namespace {

constexpr int kMaxTokens = 1 << 29, kMaxExperts = 4096;
constexpr int kSms = 148;
constexpr int kJoinThreads = 512, kJoinCtas = 8, kWindow = 512;
constexpr int kTurnsAlone = 8;                                             // rows in turn up to which one CTA is faster than tiles and a second step

template <typename Z> __device__ __forceinline__ float to_float(Z v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// A team of L lanes per row, each with V experts in runs of W: expert (j L + lane) W + i.  Up to 32 lanes they are (part of) a warp, beyond
// that the whole CTA.
constexpr int kMostSums = 5;
template <int L, int THREADS>
struct Team {
    static constexpr bool kCta = L > 32;
    static constexpr int kThreads = kCta ? L : THREADS, kWarps = kThreads / 32, kTeams = kThreads / L;
    int lane, index;                   // in the team; of the team in its CTA
    float* room;                       // [kMostSums kWarps], for teams of several warps
    __device__ Team(float* r) : lane((int)threadIdx.x % L), index((int)threadIdx.x / L), room(r) {}
    __device__ __forceinline__ void sync() const {
        if constexpr (kCta) __syncthreads();
        else __syncwarp();
    }
    // the largest / the sum over the team of each of N values, in one go
    template <int N>
    __device__ __forceinline__ void max(float (&v)[N]) const {
        if constexpr (L == 32) {
#pragma unroll
            for (int i = 0; i < N; ++i) asm("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(v[i]));
        } else {
            reduce(v, [](float a, float b) { return fmaxf(a, b); }, -INFINITY);
        }
    }
    template <int N>
    __device__ __forceinline__ void sum(float (&v)[N]) const { reduce(v, [](float a, float b) { return a + b; }, 0.f); }
    template <int N, typename F>
    __device__ __forceinline__ void reduce(float (&v)[N], F f, float none) const {
        static_assert(N <= kMostSums, "room");
#pragma unroll
        for (int m = (kCta ? 32 : L) / 2; m >= 1; m >>= 1)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = f(v[i], __shfl_xor_sync(0xffffffffu, v[i], m));
        if constexpr (kCta) {
            __syncthreads();
            if ((threadIdx.x & 31) == 0)
#pragma unroll
                for (int i = 0; i < N; ++i) room[i * kWarps + (threadIdx.x >> 5)] = v[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = none;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) v[i] = f(v[i], room[i * kWarps + w]);
            }
        }
    }
    __device__ __forceinline__ bool any(bool v) const {                    // of the team's warp, or of the CTA: enough to agree on a way
        if constexpr (kCta) return __syncthreads_or(v);
        else return __any_sync(0xffffffffu, v);
    }
};

// A row's logits; what v holds behind the last expert stays.
template <typename Z, int W, int L, int V>
__device__ __forceinline__ void load_row(const Z* row, int E, int lane, float (&v)[V]) {
#pragma unroll
    for (int j = 0; j < V / W; ++j) {
        const int e = (j * L + lane) * W;
        if constexpr (W == 1) {
            if (e < E) v[j] = to_float(row[e]);
        } else {                                                           // E is a multiple of W
            if (e < E) {
                if constexpr (sizeof(Z) == 4) {
                    const float4 r = *reinterpret_cast<const float4*>(row + e);
                    v[4 * j] = r.x, v[4 * j + 1] = r.y, v[4 * j + 2] = r.z, v[4 * j + 3] = r.w;
                } else {
                    const uint2 r = *reinterpret_cast<const uint2*>(row + e);
                    v[4 * j] = __uint_as_float(r.x << 16), v[4 * j + 1] = __uint_as_float(r.x & 0xffff0000u);
                    v[4 * j + 2] = __uint_as_float(r.y << 16), v[4 * j + 3] = __uint_as_float(r.y & 0xffff0000u);
                }
            }
        }
    }
}
template <typename Z, int W, int L, int V>
__device__ __forceinline__ void store_row(Z* row, int E, int lane, const float (&v)[V]) {
#pragma unroll
    for (int j = 0; j < V / W; ++j) {
        const int e = (j * L + lane) * W;
        if (e >= E) continue;
        if constexpr (W == 1) {
            if constexpr (sizeof(Z) == 4) row[e] = v[j];
            else row[e] = __float2bfloat16(v[j]);
        } else if constexpr (sizeof(Z) == 4) {
            *reinterpret_cast<float4*>(row + e) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        } else {
            const __nv_bfloat162 a = __floats2bfloat162_rn(v[4 * j], v[4 * j + 1]), b = __floats2bfloat162_rn(v[4 * j + 2], v[4 * j + 3]);
            *reinterpret_cast<uint2*>(row + e) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
        }
    }
}

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float exp2_of(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// exp(x) for x <= 0 by the hardware's 2^x: off by 2 units of 2^-23 and by the product's rounding, |x| 2^-24 (which with that of the difference that x is
// is what a score far below the largest is off by; the function with the exact argument takes three times the instructions, which
// would bound these kernels).  Results below 2^-126 are 0.
__device__ __forceinline__ float exp_below(float x) { return exp2_of(x * kLog2e); }
__device__ __forceinline__ float recip(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Pairs of binary32 numbers: two operations in one instruction.
struct Two { unsigned long long bits; };
__device__ __forceinline__ Two two(float a, float b) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.bits) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void split(Two v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v.bits)); }
__device__ __forceinline__ Two operator+(Two a, Two b) {
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}
__device__ __forceinline__ Two operator*(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}
__device__ __forceinline__ Two fma(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits), "l"(c.bits));
    return r;
}
__device__ __forceinline__ float both(Two v) {
    float a, b;
    split(v, a, b);
    return a + b;
}
// e = exp(v - top) and their sum, top the largest.  The difference comes first, exact next to top: what v log2(e) - top log2(e) in one step takes from the
// rounding of top log2(e) is a factor on all of a row's terms, 1 % at logits of 1e5, and outside of binary32 from 1.5e9 on.  Each term is exp_below's, bit
// by bit, so that a chosen expert's own is in proportion to the sum.
template <int V>
__device__ __forceinline__ float exps_below(const float (&v)[V], float top, float (&e)[V]) {
    const Two shift = two(-top, -top), scale = two(kLog2e, kLog2e);
    Two sum = two(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < V; j += 2) {
        float a, b;
        split((two(v[j], v[j + 1]) + shift) * scale, a, b);
        e[j] = exp2_of(a);
        e[j + 1] = exp2_of(b);
        sum = sum + two(e[j], e[j + 1]);
    }
    return both(sum);
}
// A sigmoid times exp(-c) (see the top; c <= 0), and 1 - sigmoid.
__device__ __forceinline__ float scaled_sigmoid(float z, float c, float& rest) {
    const float u = exp_below(-fabsf(z)), inv = recip(1.f + u), small = u * inv;
    rest = z < 0.f ? inv : small;                                          // (NaN: both are)
    return c < 0.f ? exp_below(z - c) * inv : z < 0.f ? small : inv;
}
// All of a row's: the sigmoids s, s (1 - s) = u / (1 + u)^2, and the sum of the former; both times exp(-c).
template <int V>
__device__ __forceinline__ float sigmoids(const float (&v)[V], float c, float (&s)[V], float (&slope)[V]) {
    if (c < 0.f) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float rest;
            s[j] = scaled_sigmoid(v[j], c, rest);
            slope[j] = s[j] * rest;
            sum += s[j];
        }
        return sum;
    }
    const Two one = two(1.f, 1.f);
    Two sum = two(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < V; j += 2) {
        const Two u = two(exp_below(-fabsf(v[j])), exp_below(-fabsf(v[j + 1])));
        float a, b, x, y;
        split(one + u, a, b);
        const Two inv = two(recip(a), recip(b)), small = u * inv;
        split(inv, a, b);
        split(small, x, y);
        s[j] = v[j] < 0.f ? x : a;
        s[j + 1] = v[j + 1] < 0.f ? y : b;
        split(small * inv, slope[j], slope[j + 1]);
        sum = sum + two(s[j], s[j + 1]);
    }
    return both(sum);
}
// The logarithm of a row's sum of exponentials; 0 for a row without any expert left.
__device__ __forceinline__ float log_sum(float base, float sum) { return sum == 0.f ? 0.f : base + __logf(sum); }
__device__ __forceinline__ float inverse(float sum) { return sum == 0.f ? 0.f : recip(sum); }

// The first sequence that ends at t or behind it, by a warp: offsets [S + 1] ascend.  Whatever they hold, the answer is in [0, S].
__device__ __forceinline__ int first_ending_at(const int32_t* offsets, int S, int t, int lane) {
    int lo = 0, hi = S;                                                    // the answer is in [lo, hi]
    while (hi > lo) {
        const int step = (hi - lo + 31) / 32, at = min(lo + step * lane, hi);
        const unsigned ends = __ballot_sync(0xffffffffu, at >= hi || offsets[at + 1] >= t);
        const int f = __ffs(ends) - 1;                                     // -1: none of the probes
        if (f < 0) {
            lo = min(lo + step * 31 + 1, hi);
        } else {
            hi = min(lo + step * f, hi);
            lo = f ? min(lo + step * (f - 1) + 1, hi) : hi;
        }
    }
    return lo;
}

struct BalanceArgs {
    const void* z;
    long long ld;
    const int32_t* ids;
    const uint8_t* mask;
    const int32_t* offsets;            // [S + 1] or null: one sequence of all tokens
    int S, T, E, k;
    bool sigmoid;
    int rows, tiles;                   // a tile: `rows` consecutive tokens
    float* losses;
    int32_t* counts;
    float* sums;
    int32_t* kept;
    // Scratch.  What a tile has of the sequence that goes on from the tile before it ([0]), and of the one that goes on behind it ([1])
    double *tile_loss, *tile_z;        // [tiles] losses of the sequences that lie in it; squares of its tokens' logarithms
    double* joined;                    // [2 kJoinCtas]
    float* part_sums;                  // [tiles][2][E]
    int32_t* part_counts;              // [tiles][2][E]
    int32_t* part_kept;                // [tiles][2]
    int32_t *tile_kept, *tile_some;    // [tiles] tokens that count; its sequences that have any
    int32_t* tile_open;                // [tiles][2] the sequence that begins in it and goes on behind it, or -1, and its last tile
};

__device__ __forceinline__ float loss_factor(int E, int k, int n) { return n ? (float)E / ((float)k * (float)n * (float)n) : 0.f; }

__device__ __forceinline__ void cluster_sync() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Sums of N values over the CTA, for thread 0, in a fixed order.
template <int N, int THREADS>
__device__ __forceinline__ void cta_sums(double (&v)[N]) {
    constexpr int WARPS = THREADS / 32;
    __shared__ double room[N][WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum_f64(v[i]);
    __syncthreads();
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) room[i][warp] = v[i];
    __syncthreads();
    if (warp == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = warp_sum_f64(lane < WARPS ? room[i][lane] : 0.0);
}

struct Open { int tile, last, s; };                                       // a sequence that goes on behind the tile it begins in, and its last tile
constexpr int kMostTiles = kSms;

// A lane's expert of tile t of a sequence; zeros behind its last.
__device__ __forceinline__ void load_part(const BalanceArgs& a, const Open& o, int chunk, int t, int lane, float& sum, int& count, int& n) {
    sum = 0.f;
    count = n = 0;
    if (t > o.last) return;
    const size_t at = 2 * (size_t)t + (t == o.tile), e = at * a.E + min(32 * chunk + lane, a.E - 1);
    sum = __ldcg(a.part_sums + e);
    count = __ldcg(a.part_counts + e);
    n = __ldcg(a.part_kept + at);
}

__device__ __forceinline__ bool ascends(const BalanceArgs& a, int first, int step) {
    bool ok = true;
    if (a.offsets)
        for (int s = first; s < a.S; s += step) {
            const int from = __ldcg(a.offsets + s), to = __ldcg(a.offsets + s + 1);
            ok = ok && from >= 0 && from <= to && to <= a.T;
        }
    return ok;
}
__device__ __forceinline__ void write_losses(const BalanceArgs& a, double balance, double some, double squares, double n, bool wrong) {
    a.losses[0] = wrong ? NAN : some > 0 ? (float)(balance / some) : 0.f;
    a.losses[1] = wrong ? NAN : n > 0 ? (float)(squares / n) : 0.f;
}

// Second step: the sequences that tiles share, and the losses.  A cluster, whose CTAs have a part each: a warp per 32 experts of a sequence, or several where there are few
// of these.  Bound by the latencies of what depends on one another: the wait, the list, the parts, the exchange.  About 4 us of a replayed call.
__global__ void __launch_bounds__(kJoinThreads)
balance_join_kernel(const __grid_constant__ BalanceArgs a) {
    constexpr int WARPS = kJoinThreads / 32;
    __shared__ float red_sum[WARPS][32];
    __shared__ int32_t red_count[WARPS][32], red_kept[WARPS], before[(kMostTiles + 31) / 32];
    __shared__ Open open[kMostTiles];                                      // in the order of their tiles
    const int cta = (int)blockIdx.x, ctas = (int)gridDim.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    grid_dependency_wait();
    grid_launch_dependents();
    const int chunks = (a.E + 31) / 32;
    // what the tiles have found of the losses, on its way while the rest is added up: by the first CTA
    double tile_loss = 0.0, tile_z = 0.0, tile_kept = 0.0, tile_some = 0.0;
    if (cta == 0 && tid < a.tiles) {
        tile_loss = __ldcg(a.tile_loss + tid);
        tile_z = __ldcg(a.tile_z + tid);
        tile_kept = (double)__ldcg(a.tile_kept + tid);
        tile_some = (double)__ldcg(a.tile_some + tid);
    }
    int n_open;
    if (!a.offsets) {
        n_open = a.tiles > 1;
    } else {
        static_assert(kMostTiles <= kJoinThreads, "a tile per thread");
        const int s = tid < a.tiles ? __ldcg(a.tile_open + 2 * tid) : -1, last = tid < a.tiles ? __ldcg(a.tile_open + 2 * tid + 1) : 0;
        const unsigned mine = __ballot_sync(0xffffffffu, s >= 0);
        if (lane == 0 && warp < (kMostTiles + 31) / 32) before[warp] = __popc(mine);
        __syncthreads();
        int at = __popc(mine & ((1u << lane) - 1u));
        n_open = 0;
#pragma unroll
        for (int w = 0; w < (kMostTiles + 31) / 32; ++w) {
            if (w < warp) at += before[w];
            n_open += before[w];
        }
        if (s >= 0) open[at] = Open{tid, last, s};
        __syncthreads();
    }
    double loss = 0.0, some = 0.0;
    const auto finish = [&](int s, int c, float sum, int count, int n) {   // by one warp
        const int e = 32 * c + lane;
        if (e < a.E) {
            a.sums[(size_t)s * a.E + e] = sum;
            a.counts[(size_t)s * a.E + e] = count;
            loss += (double)((float)count * loss_factor(a.E, a.k, n)) * (double)sum;
        }
        if (c == 0 && lane == 0) {
            a.kept[s] = n;
            some += n > 0;
        }
    };
    // An item: 32 experts of a sequence.  As many warps share its tiles (a power of two, inside a CTA) as there are for each.
    const int items = n_open * chunks, all = ctas * WARPS;
    int share = 1;
    while (share < WARPS && 2 * share * items <= all) share *= 2;
    const int group = (cta * WARPS + warp) / share, in_group = warp & (share - 1), groups = all / share;
    for (int i0 = 0; i0 < items; i0 += groups) {
        const int i = i0 + group, at = i < items ? i / chunks : 0, c = i - at * chunks;
        Open o{0, -1, 0};
        if (i < items) o = a.offsets ? open[at] : Open{0, a.tiles - 1, 0};
        constexpr int kFlight = 12;
        float sum = 0.f;
        int count = 0, n = 0;
        for (int t0 = o.tile + in_group; t0 <= o.last; t0 += kFlight * share) {
            float f[kFlight];
            int m[kFlight], l[kFlight];
#pragma unroll
            for (int u = 0; u < kFlight; ++u) load_part(a, o, c, t0 + u * share, lane, f[u], m[u], l[u]);
#pragma unroll
            for (int u = 0; u < kFlight; ++u) {
                sum += f[u];
                count += m[u];
                n += l[u];
            }
        }
        if (share > 1) {
            red_sum[warp][lane] = sum;
            red_count[warp][lane] = count;
            if (lane == 0) red_kept[warp] = n;
            __syncthreads();
            if (in_group == 0)
                for (int w = 1; w < share; ++w) {
                    sum += red_sum[warp + w][lane];
                    count += red_count[warp + w][lane];
                    n += red_kept[warp + w];
                }
            __syncthreads();
        }
        if (i < items && in_group == 0) finish(o.s, c, sum, count, n);
    }
    const bool bad = __syncthreads_or(!ascends(a, cta * kJoinThreads + tid, ctas * kJoinThreads));
    double v[4] = {loss + tile_loss, some + tile_some, tile_z, tile_kept};
    cta_sums<4, kJoinThreads>(v);
    if (bad) v[1] = -1e300;
    if (cta && tid == 0) {
        __stcg(a.joined + cta, v[0]);
        __stcg(a.joined + kJoinCtas + cta, v[1]);
    }
    if (ctas > 1) cluster_sync();
    if (cta || warp) return;
    if (lane) v[0] = v[1] = 0.0;
    if (lane > 0 && lane < ctas) {
        v[0] = __ldcg(a.joined + lane);
        v[1] = __ldcg(a.joined + kJoinCtas + lane);
    }
    v[0] = warp_sum_f64(v[0]);
    v[1] = warp_sum_f64(v[1]);
    if (lane == 0) write_losses(a, v[0], v[1], v[2], v[3], v[1] < 0.0);
}

template <int L, int V, int THREADS>
constexpr size_t balance_smem() {
    using TM = Team<L, THREADS>;
    return (size_t)(TM::kCta ? 1 : TM::kWarps) * L * V * 4 + (size_t)L * V * 4;
}

// First step: a CTA per tile, so that an SM has one start and one end; the offsets of a few hundred sequences are read at once.  ONLY: there is one tile, and no second step.
// 131072 x 64 binary32 in one sequence: 12 of the call's 16.5 us replayed, of which 4 are start and end and the rest reads 38 MB at 4.7 TB/s; issue slots 55 % busy.
// Rows in registers ahead, four rows per team and requests into L2 measure the same.  What a CTA does for a sequence takes 2 us however short it is.
template <typename Z, int W, int L, int V, int THREADS, bool ONLY>
__global__ void __launch_bounds__(Team<L, THREADS>::kThreads)
balance_kernel(const __grid_constant__ BalanceArgs a) {
    using TM = Team<L, THREADS>;
    extern __shared__ __align__(16) unsigned char smem[];
    float* red = reinterpret_cast<float*>(smem);                           // [warp][L V] column sums
    int32_t* hist = reinterpret_cast<int32_t*>(red + (TM::kCta ? 1 : TM::kWarps) * L * V);   // [L V]
    __shared__ float room[kMostSums * TM::kWarps];
    __shared__ int32_t window[kWindow + 1];
    __shared__ int n_kept;
    constexpr int U = V <= 8 && !TM::kCta ? 2 : 1;
    const TM team(room);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, E = a.E, k = a.k;
    const int t0 = (int)min((long long)a.T, (long long)blockIdx.x * a.rows), t1 = (int)min((long long)a.T, (long long)t0 + a.rows);
    const bool last = (int)blockIdx.x == a.tiles - 1;
    for (int e = tid; e < L * V; e += TM::kThreads) hist[e] = 0;
    if (tid == 0) n_kept = 0;
    __syncthreads();                                                       // warps of one sequence meet nowhere else before they count
    grid_dependency_wait();
    grid_launch_dependents();
    const Z* z = static_cast<const Z*>(a.z);
    double loss = 0.0, squares = 0.0;
    int some = 0, total = 0, open = -1, open_last = 0;                                    // of the tile (the same in all threads)
    int s = 0, in_window = kWindow;
    if (a.offsets) {
        if (a.S <= kWindow) {                                              // all of them at once
            __shared__ int first_seq;
            if (tid == 0) first_seq = a.S;
            for (int i = tid; i <= a.S; i += TM::kThreads) window[i] = __ldcg(a.offsets + i);
            __syncthreads();
            for (int i = tid; i < a.S; i += TM::kThreads)
                if (window[i + 1] >= t0 && (i == 0 || window[i] < t0)) atomicMin(&first_seq, i);
            __syncthreads();
            s = in_window = first_seq;
        } else {
            s = first_ending_at(a.offsets, a.S, t0, lane);
        }
    }
    for (; s < a.S; ++s, ++in_window) {
        int from = 0, to = a.T;
        if (a.offsets) {
            if (in_window == kWindow) {                                    // (never where all are there: S is at most that)
                __syncthreads();
                for (int i = tid; i <= kWindow; i += TM::kThreads) window[i] = s + i <= a.S ? __ldcg(a.offsets + s + i) : 0;
                in_window = 0;
                __syncthreads();
            }
            from = window[in_window];
            to = window[in_window + 1];
            if (from < 0 || from > to || to > a.T) break;                  // found by the second step too
        }
        if (from >= t1 && !(last && from == a.T)) break;
        const int lo = max(from, t0), hi = min(to, t1);
        if (lo >= hi && from < t0) continue;                               // ends where the tile begins
        float acc[V], sq = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.f;
        int mine = 0;
        // A team takes U rows at a time: their loads are on their way together, and one's sums over the team while another's are.
        const int rows = hi - lo, row0 = TM::kCta ? 0 : warp * (32 / L), own = TM::kCta ? 0 : lane / L;
        const Z* z_row = z + ((long long)lo + row0 + own) * a.ld;
        const int32_t* id_row = a.ids + ((long long)lo + row0 + own) * k + team.lane;
        const long long z_step = TM::kTeams * a.ld, id_step = (long long)TM::kTeams * k;
        for (int r = row0; r < rows; r += U * TM::kTeams) {
            float v[U][V], mx[U], sums[2 * U];
            bool on[U];
            int id[U];
#pragma unroll
            for (int u = 0; u < U; ++u, z_row += z_step, id_row += id_step) {
                const int at = r + u * TM::kTeams + own;
                on[u] = at < rows;
                id[u] = -1;
#pragma unroll
                for (int j = 0; j < V; ++j) v[u][j] = -INFINITY;
                if (on[u]) {                                               // (a masked row too: what it holds goes nowhere)
                    load_row<Z, W, L, V>(z_row, E, team.lane, v[u]);
                    if (team.lane < k) id[u] = *id_row;
                    if (a.mask) on[u] = a.mask[lo + at];
                    if (k > L && on[u])
                        for (int j = L; team.lane + j < k; j += L) {
                            const int more = id_row[j];
                            if ((unsigned)more < (unsigned)E) atomicAdd(hist + more, 1);
                        }
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                mx[u] = v[u][0];
#pragma unroll
                for (int j = 1; j < V; ++j) mx[u] = fmaxf(mx[u], v[u][j]);
            }
            team.max(mx);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (on[u] && (unsigned)id[u] < (unsigned)E) atomicAdd(hist + id[u], 1);
                mine += on[u] && team.lane == 0;
                mx[u] = mx[u] == -INFINITY ? 0.f : mx[u];
                float e[V];
                sums[u] = exps_below(v[u], mx[u], e);
                if (a.sigmoid) {
                    float slope[V];
                    sums[U + u] = sigmoids(v[u], fminf(mx[u], 0.f), e, slope);
                }
#pragma unroll
                for (int j = 0; j < V; ++j) v[u][j] = e[j];
            }
            if (a.sigmoid) {
                team.sum(sums);
            } else {
                float one[U];
#pragma unroll
                for (int u = 0; u < U; ++u) one[u] = sums[u];
                team.sum(one);
#pragma unroll
                for (int u = 0; u < U; ++u) sums[u] = sums[U + u] = one[u];
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (on[u]) {
                    const float lse = log_sum(mx[u], sums[u]), inv = inverse(sums[U + u]);
                    const Two scale = two(inv, inv);
#pragma unroll
                    for (int j = 0; j < V; j += 2) split(fma(two(v[u][j], v[u][j + 1]), scale, two(acc[j], acc[j + 1])), acc[j], acc[j + 1]);
                    if (team.lane == 0) sq = fmaf(lse, lse, sq);
                }
        }
        squares += (double)sq;
        // the sequence's (part of the) sums: over the warp's teams, over the warps
        if constexpr (!TM::kCta) {
#pragma unroll
            for (int m = L; m < 32; m <<= 1)
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] += __shfl_xor_sync(0xffffffffu, acc[j], m);
#pragma unroll
            for (int m = 1; m < 32; m <<= 1) mine += __shfl_xor_sync(0xffffffffu, mine, m);
        }
        if (TM::kCta ? tid == 0 : lane == 0) atomicAdd(&n_kept, mine);
        if (lane < L)
#pragma unroll
            for (int j = 0; j < V / W; ++j)
#pragma unroll
                for (int i = 0; i < W; ++i) red[(TM::kCta ? 0 : warp * L * V) + (j * L + team.lane) * W + i] = acc[j * W + i];
        __syncthreads();
        const int n = n_kept;
        const bool whole = from >= t0 && to <= t1;
        const size_t at = whole ? (size_t)s : 2 * (size_t)blockIdx.x + (from >= t0);
        float* sums = (whole ? a.sums : a.part_sums) + at * E;
        int32_t* counts = (whole ? a.counts : a.part_counts) + at * E;
        const float factor = whole ? loss_factor(E, k, n) : 0.f;
        for (int e = tid; e < E; e += TM::kThreads) {
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < (TM::kCta ? 1 : TM::kWarps); ++w) sum += red[w * L * V + e];
            const int count = hist[e];
            sums[e] = sum;
            counts[e] = count;
            hist[e] = 0;
            if (whole) loss += (double)((float)count * factor) * (double)sum;
        }
        if (tid == 0) (whole ? a.kept : a.part_kept)[at] = n;
        total += n;
        if (whole) some += n > 0;
        else if (from >= t0) {
            open = s;
            open_last = (to - 1) / a.rows;
        }
        __syncthreads();
        if (tid == 0) n_kept = 0;
        __syncthreads();
    }
    double v2[2] = {loss, squares};
    cta_sums<2, TM::kThreads>(v2);
    if constexpr (ONLY) {
        const bool bad = __syncthreads_or(!ascends(a, tid, TM::kThreads));
        if (tid == 0) write_losses(a, v2[0], some, v2[1], total, bad);
    } else if (tid == 0) {
        a.tile_loss[blockIdx.x] = v2[0];
        a.tile_z[blockIdx.x] = v2[1];
        a.tile_kept[blockIdx.x] = total;
        a.tile_some[blockIdx.x] = some;
        a.tile_open[2 * blockIdx.x] = open;
        a.tile_open[2 * blockIdx.x + 1] = open_last;
    }
}

constexpr int kBackThreads = 256, kBackPerSm = 768;                        // threads of a CTA, of an SM: 80 registers each (128 for V = 16)
template <int L, int V>
__host__ __device__ constexpr int back_ctas() {
    constexpr int threads = Team<L, kBackThreads>::kThreads, all = V <= 8 ? kBackPerSm : 512;
    return all > threads ? all / threads : 1;
}

struct BackwardArgs {
    const void* z;
    long long ld, ld_out;
    void* out;
    const int32_t* ids;
    const float *d_weights, *d_losses; // or null
    const int32_t *counts, *kept;
    const uint8_t* mask;
    const int32_t* offsets;
    int S, T, E, k, rows;              // rows: consecutive tokens of a warp (of a CTA, for teams of a CTA)
    bool sigmoid, renorm;
    float scale;
};

// dz of a row (see the top of the file for q; G_e = d_balance E c_e / (S' k T_s^2), what the balance loss changes by with a score):
//   softmax   q_e (G_e - sum q G)                            sigmoid   q_e (1 - s_e) (G_e - sum q G)
//   z loss    d_z 2 / N  lse  softmax(z)_e
//   weights w_j = scale s_j: softmax    p_e ([e chosen] d_e - sum p d),   sigmoid   s_e (1 - s_e) d_e      with d = scale dw
//   ... divided by their sum, r the shares: softmax    r_e (d_e - sum r d),   sigmoid   r_e (1 - s_e) (d_e - sum r d)
// The chosen ones' logits are read again and their shares taken from their own largest: they may all be lost beside the row's.  What goes to
// single experts passes through a row of shared memory that is zero between rows.
// Bound by instructions: 32768 x 256 (sigmoid, renormalised, both losses) 28.5 us replayed, 56 % of the issue slots, 551 instructions per row where 67 MB would take 10.6 us;
// 768 threads per SM have 80 registers each
// (the weights alone, when this was chosen: 22.2 us, with 1280 threads 30.9).
template <typename Z, int W, int L, int V>
__global__ void __launch_bounds__(Team<L, kBackThreads>::kThreads, back_ctas<L, V>())
gate_backward_kernel(const __grid_constant__ BackwardArgs a) {
    using TM = Team<L, kBackThreads>;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float room[kMostSums * TM::kWarps];
    __shared__ float loss_scale[2];
    const TM team(room);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, E = a.E, k = a.k;
    float* row_add = reinterpret_cast<float*>(smem) + team.index * L * V;
    for (int i = tid; i < TM::kTeams * L * V; i += TM::kThreads) reinterpret_cast<float*>(smem)[i] = 0.f;
    grid_dependency_wait();
    grid_launch_dependents();
    const long long unit = TM::kCta ? blockIdx.x : (long long)blockIdx.x * TM::kWarps + warp;
    const long long t_begin = unit * a.rows, t_end = min((long long)a.T, t_begin + a.rows);
    const bool losses = a.d_losses != nullptr, weights = a.d_weights != nullptr, one = k <= L;
    const Z* z = static_cast<const Z*>(a.z);
    constexpr int kStep = TM::kCta ? 1 : 32 / L;
    const int lane_row = TM::kCta ? 0 : lane / L;
    const Z* z_row = z + (t_begin + lane_row) * a.ld;
    Z* out_row = static_cast<Z*>(a.out) + (t_begin + lane_row) * a.ld_out;
    const int32_t* id_row = weights ? a.ids + (t_begin + lane_row) * k + team.lane : nullptr;
    const float* dw_row = weights ? a.d_weights + (t_begin + lane_row) * k + team.lane : nullptr;
    const long long z_step = kStep * a.ld, out_step = kStep * a.ld_out, id_step = (long long)kStep * k;
    const bool has_id = weights && team.lane < k;
    const int rows = t_end > t_begin ? (int)(t_end - t_begin) : 0;
    float v[V];
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = -INFINITY;
    // With a whole warp per row, its ids, weights' gradients and mask come a row ahead of it, and its logits into L1.  (With several rows per warp that
    // takes longer: 131072 x 64 31.9 us instead of 29.6.)  The first one is on its way before the sums over the sequences.
    constexpr bool kAhead = L >= 32;
    int next_id = -1;
    float next_d = 0.f;
    bool next_on = false;
    const auto request = [&](int r, const Z* row, const int32_t* ids, const float* dw) {
        next_on = r + lane_row < rows;
        next_id = -1;
        if (next_on) {
            if constexpr (kAhead)
#pragma unroll
            for (int j = 0; j < V / W; ++j)
                if ((j * L + team.lane) * W < E) asm volatile("prefetch.global.L1 [%0];" ::"l"(row + (j * L + team.lane) * W));
            if (has_id) {
                next_id = *ids;
                next_d = *dw;
            }
            if (a.mask) next_on = a.mask[t_begin + r + lane_row];
        }
    };
    if (kAhead && rows > 0) request(0, z_row, id_row, dw_row);
    if (a.d_losses) {                                                      // S' and N
        double all[2] = {0.0, 0.0};
        if (a.S == 1) {
            all[0] = (double)a.kept[0];
            all[1] = all[0] > 0;
        } else {
            for (int s = tid; s < a.S; s += TM::kThreads) {
                const int m = a.kept[s];
                all[0] += m;
                all[1] += m > 0;
            }
            cta_sums<2, TM::kThreads>(all);
        }
        if (tid == 0) {
            loss_scale[0] = all[1] > 0 ? a.d_losses[0] * (float)E / ((float)all[1] * (float)k) : 0.f;
            loss_scale[1] = all[0] > 0 ? 2.f * a.d_losses[1] / (float)all[0] : 0.f;
        }
    }
    __syncthreads();
    const float balance = losses ? loss_scale[0] : 0.f, z_scale = losses ? loss_scale[1] : 0.f;
    float g[V];                                                            // G of the sequence
#pragma unroll
    for (int j = 0; j < V; ++j) g[j] = 0.f;
    int s = -1, s_from = 0, s_to = 0;
    if (losses && t_begin < t_end) s = a.offsets ? first_ending_at(a.offsets, a.S, (int)t_begin + 1, lane) - 1 : -1;
    for (int r = 0; r < rows; r += kStep, z_row += z_step, out_row += out_step, id_row += id_step, dw_row += id_step) {
        if constexpr (!kAhead) request(r, z_row, id_row, dw_row);
        const bool in = r + lane_row < rows, on = next_on;
        const long long t = t_begin + r + lane_row;
        const int id0 = next_id;
        const float d0 = a.scale * next_d;
        if (in) load_row<Z, W, L, V>(z_row, E, team.lane, v);
        const bool first = on && (unsigned)id0 < (unsigned)E;
        const float zj0 = first ? to_float(z_row[id0]) : 0.f;              // of this lane's chosen expert
        if (kAhead && r + kStep < rows) request(r + kStep, z_row + z_step, id_row + id_step, dw_row + id_step);
        float share0 = 0.f, rest0 = 1.f;
        // f(expert, its logit, scale times its weight's gradient, place) of the team's lanes' chosen experts behind the first one of each
        const auto others = [&](auto f) {
            if (on)
                for (int j = L; team.lane + j < k; j += L) {
                    const int id = id_row[j];
                    if ((unsigned)id < (unsigned)E) f(id, to_float(z_row[id]), a.scale * dw_row[j], team.lane + j);
                }
        };
        bool counts = losses && on;
        if (counts && t >= s_to) {                                         // the next sequence that ends behind t
            do {
                ++s;
                s_from = a.offsets ? (s < a.S ? a.offsets[s] : INT32_MAX) : 0;
                s_to = a.offsets ? (s < a.S ? a.offsets[s + 1] : INT32_MAX) : a.T;
            } while (t >= s_to && s < a.S);
            const float n = s < a.S ? (float)a.kept[s] : 0.f, f = n > 0.f ? balance / (n * n) : 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int e = (j / W * L + team.lane) * W + j % W;
                g[j] = s < a.S && e < E ? f * (float)a.counts[(size_t)s * E + e] : 0.f;
            }
        }
        counts = counts && s < a.S && t >= s_from;
        float mx[2] = {v[0], -INFINITY};                                   // of the row, of the chosen
#pragma unroll
        for (int j = 1; j < V; ++j) mx[0] = fmaxf(mx[0], v[j]);
        if (weights && a.renorm) {
            if (first) mx[1] = zj0;
            if (!one) others([&](int, float zj, float, int) { mx[1] = fmaxf(mx[1], zj); });
            team.max(mx);
        } else {
            float m1[1] = {mx[0]};
            team.max(m1);
            mx[0] = m1[0];
        }
        const float top = mx[0] == -INFINITY ? 0.f : mx[0], most = mx[1] == -INFINITY ? 0.f : mx[1];
        const float c = fminf(top, 0.f), c_chosen = a.renorm ? fminf(most, 0.f) : 0.f;
        // scores: times exp(-c) / exp(-top), with 1 - s (sigmoid); sums: of the scores, of scores G, of exponentials (z loss), of the chosen ones' shares, of shares d
        float dz[V], sums[5] = {0.f, 0.f, 0.f, 0.f, 0.f};
        const bool with_z = z_scale != 0.f;
        if (a.sigmoid) {
            if (losses) {
                if (with_z) sums[2] = exps_below(v, top, dz);
                float sg[V];
                sums[0] = sigmoids(v, c, sg, dz);
                Two dot = two(0.f, 0.f);
#pragma unroll
                for (int j = 0; j < V; j += 2) dot = fma(two(sg[j], sg[j + 1]), two(g[j], g[j + 1]), dot);
                sums[1] = both(dot);
            }
        } else {
            sums[0] = exps_below(v, top, dz);
            Two dot = two(0.f, 0.f);
#pragma unroll
            for (int j = 0; j < V; j += 2) dot = fma(two(dz[j], dz[j + 1]), two(g[j], g[j + 1]), dot);
            sums[1] = both(dot);
        }
        const auto share_of = [&](float zj, float& rest) {
            rest = 1.f;
            return a.sigmoid ? scaled_sigmoid(zj, c_chosen, rest) : exp_below(zj - (a.renorm ? most : top));
        };
        if (weights) {
            if (first) {
                share0 = share_of(zj0, rest0);
                sums[3] = share0;
                sums[4] = share0 * d0;
                row_add[id0] = __int_as_float(team.lane + 1);
            }
            if (!one)
                others([&](int id, float zj, float d, int j) {
                    float rest;
                    const float share = share_of(zj, rest);
                    sums[3] += share;
                    sums[4] = fmaf(share, d, sums[4]);
                    row_add[id] = __int_as_float(j + 1);
                });
        }
        if (weights) {
            team.sum(sums);
        } else {
            float three[3] = {sums[0], sums[1], sums[2]};
            team.sum(three);
            sums[0] = three[0], sums[1] = three[1], sums[2] = three[2];
        }
        const float inv = inverse(sums[0]), mean = sums[1] * inv;
        if (weights) {
            // The chosen ones' part goes through row_add; where an expert is named twice, one after the other.
            team.sync();
            bool twice = first && __float_as_int(row_add[id0]) != team.lane + 1;
            if (!one) others([&](int id, float, float, int j) { twice |= __float_as_int(row_add[id]) != j + 1; });
            twice = team.any(twice);
            const float share_scale = a.renorm ? inverse(sums[3]) : a.sigmoid ? 1.f : inv, d_mean = a.renorm ? sums[4] * share_scale : 0.f;
            const auto part = [&](float zj, float d) {
                float rest;
                const float share = share_of(zj, rest);
                return share * share_scale * rest * (d - d_mean);
            };
            if (!twice) {
                if (first) row_add[id0] = share0 * share_scale * rest0 * (d0 - d_mean);
                if (!one) others([&](int id, float zj, float d, int) { row_add[id] = part(zj, d); });
            } else {
                if (first) row_add[id0] = 0.f;
                if (!one) others([&](int id, float, float, int) { row_add[id] = 0.f; });
                team.sync();
                if (on && team.lane == 0)
                    for (int j = 0; j < k; ++j) {
                        const int id = id_row[j];
                        if ((unsigned)id < (unsigned)E) row_add[id] += part(to_float(z_row[id]), a.scale * dw_row[j]);
                    }
            }
            team.sync();
        }
        if (a.sigmoid) {
            if (counts) {
                const Two scale = two(inv, inv), shift = two(-mean * inv, -mean * inv);
#pragma unroll
                for (int j = 0; j < V; j += 2) split(two(dz[j], dz[j + 1]) * fma(two(g[j], g[j + 1]), scale, shift), dz[j], dz[j + 1]);
                if (with_z) {
                    float e[V];
                    exps_below(v, top, e);
                    const float zl = z_scale * log_sum(top, sums[2]) * inverse(sums[2]);
                    const Two z2 = two(zl, zl);
#pragma unroll
                    for (int j = 0; j < V; j += 2) split(fma(two(e[j], e[j + 1]), z2, two(dz[j], dz[j + 1])), dz[j], dz[j + 1]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) dz[j] = 0.f;
            }
        } else if (on) {
            const float zl = (counts && with_z ? z_scale * log_sum(top, sums[0]) : 0.f) - (weights && !a.renorm ? sums[4] * inv : 0.f) - (counts ? mean : 0.f);
            const float on_g = counts ? inv : 0.f;
            const Two scale = two(on_g, on_g), shift = two(zl * inv, zl * inv);
#pragma unroll
            for (int j = 0; j < V; j += 2) split(two(dz[j], dz[j + 1]) * fma(two(g[j], g[j + 1]), scale, shift), dz[j], dz[j + 1]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) dz[j] = 0.f;
        }
        if (weights) {
#pragma unroll
            for (int j = 0; j < V / W; ++j) {
                const float* at = row_add + (j * L + team.lane) * W;
                if constexpr (W == 4) {
                    const float4 r = *reinterpret_cast<const float4*>(at);
                    dz[4 * j] += r.x, dz[4 * j + 1] += r.y, dz[4 * j + 2] += r.z, dz[4 * j + 3] += r.w;
                } else {
                    dz[j] += *at;
                }
            }
            team.sync();
            if (first) row_add[id0] = 0.f;
            if (!one) others([&](int id, float, float, int) { row_add[id] = 0.f; });
            team.sync();
        }
        if (in) store_row<Z, W, L, V>(out_row, E, team.lane, dz);
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------

struct Tiling { int rows, tiles; bool wide; };
// One CTA where it has few rows in turn, else one per SM: of 512 threads, which start and meet sooner, or, for sequences of many rows and where registers
// allow, of 1024 (us, 512 / 1024, replayed from a graph: 4096 x 64 7.4 / 8.8, 65536 x 128 in 2000 sequences 63 / 74, 131072 x 64 17.8 / 16.7).
Tiling tiling(int T, int E, int S) {
    const int at_once = E <= 64 ? 64 : E <= 128 ? 32 : E <= 1024 ? 16 : 1;     // rows that 512 threads have in hand
    if (T <= kTurnsAlone * at_once) return {std::max(1, T), 1, false};
    const int rows = std::max(at_once, (int)(((long long)T + kSms - 1) / kSms));
    return {rows, (int)(((long long)T + rows - 1) / rows), E <= 256 && rows >= 4 * at_once && T / S >= 4 * at_once};
}
size_t scratch_bytes(int E, const Tiling& t) {
    if (t.tiles == 1) return 0;
    return 8 * (2 * (size_t)t.tiles + 2 * kJoinCtas) + 4 * (4 * (size_t)t.tiles * E + 2 * (size_t)t.tiles + 4 * (size_t)t.tiles);
}

template <typename Z, int W, int L, int V>
int launch_balance(const BalanceArgs& a, bool wide, cudaStream_t st) {
    static SmemOnce once[3];
    constexpr int threads = Team<L, 512>::kThreads;
    constexpr size_t smem = balance_smem<L, V, 512>();
    if (a.tiles == 1) return launch(balance_kernel<Z, W, L, V, 512, true>, 1, threads, 1, smem, once[0], st, a);
    int rc;
    if constexpr (L * V <= 256) {
        if (wide) rc = launch(balance_kernel<Z, W, L, V, 1024, false>, (unsigned)a.tiles, 1024, 1, balance_smem<L, V, 1024>(), once[1], st, a);
        else rc = launch(balance_kernel<Z, W, L, V, 512, false>, (unsigned)a.tiles, threads, 1, smem, once[2], st, a);
    } else {
        rc = launch(balance_kernel<Z, W, L, V, 512, false>, (unsigned)a.tiles, threads, 1, smem, once[2], st, a);
    }
    if (rc) return rc;
    static SmemOnce join;
    const int ctas = a.offsets ? kJoinCtas : std::min(kJoinCtas, (a.E + 31) / 32);
    return launch(balance_join_kernel, (unsigned)ctas, kJoinThreads, ctas, 0, join, st, a);
}
template <typename Z, int W>
int launch_balance(const BalanceArgs& a, bool wide, cudaStream_t st) {
    if (a.E <= 64) return launch_balance<Z, W, 8, 8>(a, wide, st);
    if (a.E <= 128) return launch_balance<Z, W, 16, 8>(a, wide, st);
    if (a.E <= 256) return launch_balance<Z, W, 32, 8>(a, wide, st);
    if (a.E <= 512) return launch_balance<Z, W, 32, 16>(a, wide, st);
    if (a.E <= 1024) return launch_balance<Z, W, 32, 32>(a, wide, st);
    return launch_balance<Z, W, 512, 8>(a, wide, st);
}

template <typename Z, int W, int L, int V>
int launch_backward(BackwardArgs a, cudaStream_t st) {
    using TM = Team<L, kBackThreads>;
    static SmemOnce once;
    // rows per warp (CTA): as many as leave every SM its share of the CTAs that it holds at once
    constexpr int at_once = TM::kCta ? 1 : 32 / L, per_sm = back_ctas<L, V>();
    const long long units = (long long)kSms * per_sm * (TM::kCta ? 1 : TM::kWarps);
    const long long turns = ((long long)a.T + units * at_once - 1) / (units * at_once);
    a.rows = (int)std::min<long long>(turns * at_once, a.T);
    const long long per_cta = (long long)a.rows * (TM::kCta ? 1 : TM::kWarps);
    return launch(gate_backward_kernel<Z, W, L, V>, (unsigned)((a.T + per_cta - 1) / per_cta), TM::kThreads, 1, (size_t)TM::kTeams * L * V * 4, once, st, a);
}
template <typename Z, int W>
int launch_backward(const BackwardArgs& a, cudaStream_t st) {
    if (a.E <= 64) return launch_backward<Z, W, 8, 8>(a, st);
    if (a.E <= 128) return launch_backward<Z, W, 16, 8>(a, st);
    if (a.E <= 256) return launch_backward<Z, W, 32, 8>(a, st);
    if (a.E <= 512) return launch_backward<Z, W, 32, 16>(a, st);
    if (a.E <= 1024) return launch_backward<Z, W, 128, 8>(a, st);
    return launch_backward<Z, W, 512, 8>(a, st);
}

// Four logits per load where every row begins on a boundary of four and ends on one.
bool in_fours(const void* p, long long ld, int rows, int E, int es) { return E % 4 == 0 && (ld % 4 == 0 || rows <= 1) && aligned(4 * es, p); }

int check_loss(const exmoe_shape* shape, const exmoe_gate* gate, int type, int64_t row_stride, int T, int S, const int32_t* offsets, GateArgs* g) {
    const int rc = check_gate(shape, gate, T, g);
    if (rc) return rc;
    if ((type != EXMOE_F32 && type != EXMOE_BF16) || row_stride < 0 || (T > 1 && row_stride < g->E)) return EXMOE_ERR_ARG;
    if (S < 1 || S > kMaxTokens || (S > 1 && !offsets)) return EXMOE_ERR_ARG;
    return EXMOE_OK;
}

}  // namespace

extern "C" int exmoe_balance_scratch_bytes(const exmoe_shape* shape, int T, size_t* bytes) {
    if (!shape || !bytes || T < 0 || T > kMaxTokens) return EXMOE_ERR_ARG;
    if (shape->num_experts <= 0 || shape->num_experts > kMaxExperts) return EXMOE_ERR_SHAPE;
    *bytes = scratch_bytes(shape->num_experts, tiling(T, shape->num_experts, 1));   // (as many tiles whatever the sequences are)
    return EXMOE_OK;
}

extern "C" int exmoe_balance_loss(const exmoe_shape* shape, const exmoe_gate* gate, const void* logits, int type, int64_t row_stride, const int32_t* topk_ids,
                                  const uint8_t* mask, const int32_t* offsets, int num_sequences, int T, float* losses, int32_t* counts, float* score_sums,
                                  int32_t* kept, void* scratch, void* stream) {
    GateArgs g;
    const int rc = check_loss(shape, gate, type, row_stride, T, num_sequences, offsets, &g);
    if (rc) return rc;
    const Tiling t = tiling(T, g.E, num_sequences);
    if ((T && (!logits || !topk_ids)) || !losses || !counts || !score_sums || !kept || (!scratch && scratch_bytes(g.E, t))) return EXMOE_ERR_ARG;
    const int es = type == EXMOE_F32 ? 4 : 2;
    if (!aligned(es, logits) || !aligned(4, topk_ids, offsets, losses, counts, score_sums, kept) || !aligned(8, scratch)) return EXMOE_ERR_ARG;
    const long long SE = (long long)num_sequences * g.E;
    const Range ranges[] = {range_of(losses, 1, 0, 2, 4), range_of(counts, 1, 0, SE, 4), range_of(score_sums, 1, 0, SE, 4), range_of(kept, 1, 0, num_sequences, 4),
                            range_of(scratch, 1, 0, (long long)scratch_bytes(g.E, t), 1), range_of(logits, T, row_stride, g.E, es),
                            range_of(topk_ids, 1, 0, (long long)T * g.k, 4), range_of(mask, 1, 0, T, 1), range_of(offsets, 1, 0, num_sequences + 1ll, 4)};
    constexpr int kWritten = 5;
    for (int i = 0; i < kWritten; ++i)
        for (int j = i + 1; j < (int)(sizeof ranges / sizeof *ranges); ++j)
            if (overlap(ranges[i], ranges[j])) return EXMOE_ERR_ARG;
    BalanceArgs a{logits, row_stride, topk_ids, mask, offsets, num_sequences, T, g.E, g.k, g.sigmoid, t.rows, t.tiles, losses, counts, score_sums, kept};
    double* d = static_cast<double*>(scratch);
    const size_t n = (size_t)t.tiles;
    a.tile_loss = d;
    a.tile_z = d + n;
    a.joined = d + 2 * n;
    a.part_sums = reinterpret_cast<float*>(a.joined + 2 * kJoinCtas);
    a.part_counts = reinterpret_cast<int32_t*>(a.part_sums + 2 * n * g.E);
    a.part_kept = a.part_counts + 2 * n * g.E;
    a.tile_kept = a.part_kept + 2 * n;
    a.tile_some = a.tile_kept + n;
    a.tile_open = a.tile_some + n;
    cudaStream_t st = (cudaStream_t)stream;
    const bool fours = in_fours(logits, row_stride, T, g.E, es);
    if (type == EXMOE_F32) return fours ? launch_balance<float, 4>(a, t.wide, st) : launch_balance<float, 1>(a, t.wide, st);
    return fours ? launch_balance<__nv_bfloat16, 4>(a, t.wide, st) : launch_balance<__nv_bfloat16, 1>(a, t.wide, st);
}

extern "C" int exmoe_gate_backward(const exmoe_shape* shape, const exmoe_gate* gate, const void* logits, int type, int64_t row_stride, const int32_t* topk_ids,
                                   const float* d_weights, const float* d_losses, const int32_t* counts, const int32_t* kept, const uint8_t* mask,
                                   const int32_t* offsets, int num_sequences, int T, void* d_logits, int64_t d_row_stride, void* stream) {
    GateArgs g;
    const int rc = check_loss(shape, gate, type, row_stride, T, num_sequences, offsets, &g);
    if (rc) return rc;
    if (d_row_stride < 0 || (T > 1 && d_row_stride < g.E) || (d_losses && (!counts || !kept))) return EXMOE_ERR_ARG;
    if (T == 0) return EXMOE_OK;
    if (!logits || !d_logits || (d_weights && !topk_ids)) return EXMOE_ERR_ARG;
    const int es = type == EXMOE_F32 ? 4 : 2;
    if (!aligned(es, logits, d_logits) || !aligned(4, topk_ids, d_weights, d_losses, counts, kept, offsets)) return EXMOE_ERR_ARG;
    const Range out = range_of(d_logits, T, d_row_stride, g.E, es);
    const long long TK = (long long)T * g.k;
    if (overlap(out, range_of(logits, T, row_stride, g.E, es)) || overlap(out, range_of(topk_ids, 1, 0, TK, 4)) || overlap(out, range_of(d_weights, 1, 0, TK, 4)) ||
        overlap(out, range_of(d_losses, 1, 0, 2, 4)) || overlap(out, range_of(counts, 1, 0, (long long)num_sequences * g.E, 4)) ||
        overlap(out, range_of(kept, 1, 0, num_sequences, 4)) || overlap(out, range_of(mask, 1, 0, T, 1)) || overlap(out, range_of(offsets, 1, 0, num_sequences + 1ll, 4)))
        return EXMOE_ERR_ARG;
    const BackwardArgs a{logits, row_stride, d_row_stride, d_logits, topk_ids, d_weights, d_losses, counts, kept, mask, offsets, num_sequences, T, g.E, g.k, 0,
                         g.sigmoid, g.renorm, g.scale};
    cudaStream_t st = (cudaStream_t)stream;
    const bool fours = in_fours(logits, row_stride, T, g.E, es) && in_fours(d_logits, d_row_stride, T, g.E, es);
    if (type == EXMOE_F32) return fours ? launch_backward<float, 4>(a, st) : launch_backward<float, 1>(a, st);
    return fours ? launch_backward<__nv_bfloat16, 4>(a, st) : launch_backward<__nv_bfloat16, 1>(a, st);
}

}  // namespace exmoe
