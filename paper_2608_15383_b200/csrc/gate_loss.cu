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

template <typename Z> __device__ __forceinline__ float to_float(Z v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

// A team of L lanes per row, each with V experts in runs of W: expert (j L + lane) W + i.  Up to 32 lanes they are (part of) a warp, beyond
// that the whole CTA.
template <int L>
struct Team {
    static constexpr bool kCta = L > 32;
    static constexpr int kThreads = kCta ? L : 512, kWarps = kThreads / 32, kTeams = kThreads / L;
    int lane, index;                   // in the team; of the team in its CTA
    float* room;                       // [2 kWarps], for teams of several warps
    __device__ Team(float* r) : lane((int)threadIdx.x % L), index((int)threadIdx.x / L), room(r) {}
    __device__ __forceinline__ void sync() const {
        if constexpr (kCta) __syncthreads();
        else __syncwarp();
    }
    __device__ __forceinline__ float max(float v) const {
#pragma unroll
        for (int m = (kCta ? 32 : L) / 2; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, m));
        if constexpr (kCta) {
            __syncthreads();
            if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = v;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWarps; ++w) v = fmaxf(v, room[w]);
        }
        return v;
    }
    __device__ __forceinline__ void sum2(float& a, float& b) const {
#pragma unroll
        for (int m = (kCta ? 32 : L) / 2; m >= 1; m >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, m);
            b += __shfl_xor_sync(0xffffffffu, b, m);
        }
        if constexpr (kCta) {
            __syncthreads();
            if ((threadIdx.x & 31) == 0) {
                room[threadIdx.x >> 5] = a;
                room[kWarps + (threadIdx.x >> 5)] = b;
            }
            __syncthreads();
            a = b = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                a += room[w];
                b += room[kWarps + w];
            }
        }
    }
    __device__ __forceinline__ bool any(bool v) const {                    // of the team's warp, or of the CTA: enough to agree on a way
        if constexpr (kCta) return __syncthreads_or(v);
        else return __any_sync(0xffffffffu, v);
    }
};

// A row's logits, -infinity behind the last expert.
template <typename Z, int W, int L, int V>
__device__ __forceinline__ void load_row(const Z* row, int E, int lane, float (&v)[V]) {
#pragma unroll
    for (int j = 0; j < V / W; ++j) {
        const int e = (j * L + lane) * W;
        if constexpr (W == 1) {
            v[j] = e < E ? to_float(row[e]) : -INFINITY;
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
            } else {
                v[4 * j] = v[4 * j + 1] = v[4 * j + 2] = v[4 * j + 3] = -INFINITY;
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

// A sigmoid times exp(-c) (see the top; c <= 0), and 1 - sigmoid.
__device__ __forceinline__ float scaled_sigmoid(float z, float c, float& rest) {
    const float u = expf(-fabsf(z)), inv = __fdividef(1.f, 1.f + u);
    rest = z >= 0.f ? u * inv : inv;
    if (z != z) rest = z;
    return (c < 0.f ? expf(z - c) : z >= 0.f ? 1.f : u) * inv;
}
// The logarithm of a row's sum of exponentials; 0 for a row without any expert left.
__device__ __forceinline__ float log_sum(float base, float sum) { return sum == 0.f ? 0.f : base + logf(sum); }
__device__ __forceinline__ float inverse(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }

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
    int32_t* tile_open;                // [tiles] the sequence that begins in it and goes on behind it, or -1
    int32_t* joined_some;              // [2 kJoinCtas]
};

__device__ __forceinline__ double loss_factor(int E, int k, int n) { return n ? (double)E / ((double)k * n * n) : 0.0; }

__device__ __forceinline__ void cluster_sync() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The sum of a value over the CTA, for thread 0, in a fixed order.
__device__ __forceinline__ double cta_sum(double v, double* room) {
    v = warp_sum_f64(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < (int)blockDim.x >> 5; ++w) v += room[w];
    return v;
}

struct Open { int tile, last, s; };                                       // a sequence, its first and last tile
constexpr int kMostTiles = 8 * kSms;
constexpr size_t join_smem(int threads) { return (size_t)(threads / 32) * (32 * 8 + 4) + 16 + 2 * kMostTiles * sizeof(Open); }

// Second step: the sequences that tiles share, and the losses.  By the CTAs of one cluster.
__device__ void join_tiles(const BalanceArgs& a, int cta, int ctas, unsigned char* smem) {
    __shared__ double room[32];
    const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 31, warp = tid >> 5, warps = threads >> 5;
    float* red_sum = reinterpret_cast<float*>(smem);                       // [warps][32]
    int32_t* red_count = reinterpret_cast<int32_t*>(red_sum + 32 * warps); // [warps][32]
    int32_t* red_kept = red_count + 32 * warps;                            // [warps]
    Open* open = reinterpret_cast<Open*>(red_kept + ((warps + 3) & ~3));   // [kMostTiles]
    Open* ordered = open + kMostTiles;                                     // [kMostTiles]
    constexpr int kFew = 16;                                               // tiles of a sequence that one warp adds up
    const int chunks = (a.E + 31) / 32;
    double loss = 0.0;
    int some = 0, bad = 0;
    // the sequences that go on behind the tile they begin in: few, and those over many tiles
    __shared__ int n_open, n_long;
    if (tid == 0) n_open = n_long = 0;
    __syncthreads();
    for (int tile = tid; tile < a.tiles; tile += threads) {
        const int s = __ldcg(a.tile_open + tile);
        if (s < 0) continue;
        const int last = (min(max(a.offsets ? __ldcg(a.offsets + s + 1) : a.T, 1), a.T) - 1) / a.rows;
        const bool far = last - tile >= kFew;
        const int at = far ? kMostTiles - 1 - atomicAdd(&n_long, 1) : atomicAdd(&n_open, 1);
        open[at] = Open{tile, last, s};
    }
    __syncthreads();
    // (in the order of their tiles, so that every call adds up alike)
    const auto in_order = [&](Open* list, int n) {
        for (int i = tid; i < n; i += threads) {
            int before = 0;
            for (int j = 0; j < n; ++j) before += list[j].tile < list[i].tile;
            ordered[(int)(list - open) + before] = list[i];
        }
    };
    in_order(open, n_open);
    in_order(open + kMostTiles - n_long, n_long);
    __syncthreads();
    auto finish = [&](int s, int c, float sum, int count, int n) {         // by one warp
        const int e = 32 * c + lane;
        if (e < a.E) {
            a.sums[(size_t)s * a.E + e] = sum;
            a.counts[(size_t)s * a.E + e] = count;
            loss += (double)count * (double)sum * loss_factor(a.E, a.k, n);
        }
        if (c == 0 && lane == 0) {
            a.kept[s] = n;
            some += n > 0;
        }
    };
    const auto add_tiles = [&](const Open& o, int c, int first, int step, float& sum, int& count, int& n) {
        const int e = min(32 * c + lane, a.E - 1);
        sum = 0.f;
        count = n = 0;
#pragma unroll 8
        for (int t = o.tile + first; t <= o.last; t += step) {
            const size_t at = 2 * (size_t)t + (t == o.tile);
            sum += __ldcg(a.part_sums + at * a.E + e);
            count += __ldcg(a.part_counts + at * a.E + e);
            n += __ldcg(a.part_kept + at);
        }
    };
    for (int i = cta * warps + warp; i < n_open * chunks; i += ctas * warps) {     // over few tiles: a warp per 32 experts
        const Open o = ordered[i / chunks];
        float sum;
        int count, n;
        add_tiles(o, i % chunks, 0, 1, sum, count, n);
        finish(o.s, i % chunks, sum, count, n);
    }
    for (int i = cta; i < n_long * chunks; i += ctas) {                    // over many: the CTA's warps share its tiles
        const Open o = ordered[kMostTiles - n_long + i / chunks];
        const int c = i % chunks;
        float sum;
        int count, n;
        add_tiles(o, c, warp, warps, sum, count, n);
        red_sum[32 * warp + lane] = sum;
        red_count[32 * warp + lane] = count;
        if (lane == 0) red_kept[warp] = n;
        __syncthreads();
        if (warp == 0) {
            for (int w = 1; w < warps; ++w) {
                sum += red_sum[32 * w + lane];
                count += red_count[32 * w + lane];
                n += red_kept[w];
            }
            finish(o.s, c, sum, count, n);
        }
        __syncthreads();
    }
    if (a.offsets)
        for (int s = cta * threads + tid; s < a.S; s += ctas * threads) {
            const int from = __ldcg(a.offsets + s), to = __ldcg(a.offsets + s + 1);
            bad |= from < 0 || from > to || to > a.T;
        }
    bad = __syncthreads_or(bad);
    loss = cta_sum(loss, room);
    const double all_some = cta_sum((double)some, room);
    if (tid == 0) {
        __stcg(a.joined + cta, loss);
        __stcg(a.joined_some + cta, (int)all_some);
        __stcg(a.joined_some + kJoinCtas + cta, bad);
    }
    cluster_sync();
    if (cta) return;
    double z = 0.0, n = 0.0, in_tiles = 0.0, n_seq = 0.0;
    for (int t = tid; t < a.tiles; t += threads) {
        in_tiles += __ldcg(a.tile_loss + t);
        z += __ldcg(a.tile_z + t);
        n += (double)__ldcg(a.tile_kept + t);
        n_seq += (double)__ldcg(a.tile_some + t);
    }
    in_tiles = cta_sum(in_tiles, room);
    z = cta_sum(z, room);
    n = cta_sum(n, room);
    n_seq = cta_sum(n_seq, room);
    if (tid == 0) {
        int wrong = 0;
        for (int c = 0; c < ctas; ++c) {
            in_tiles += __ldcg(a.joined + c);
            n_seq += (double)__ldcg(a.joined_some + c);
            wrong |= __ldcg(a.joined_some + kJoinCtas + c);
        }
        a.losses[0] = wrong ? NAN : n_seq > 0 ? (float)(in_tiles / n_seq) : 0.f;
        a.losses[1] = wrong ? NAN : n > 0 ? (float)(z / n) : 0.f;
    }
}

__global__ void __launch_bounds__(kJoinThreads)
balance_join_kernel(const __grid_constant__ BalanceArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    grid_dependency_wait();
    grid_launch_dependents();
    join_tiles(a, (int)blockIdx.x, (int)gridDim.x, smem);
}

template <int L, int V>
constexpr size_t balance_smem() { return (size_t)(Team<L>::kCta ? 1 : Team<L>::kWarps) * L * V * 4 + (size_t)L * V * 4; }

// First step: a CTA per tile.  FUSED: the grid is one cluster, which goes on with the second.
template <typename Z, int W, int L, int V, bool FUSED>
__global__ void __launch_bounds__(Team<L>::kThreads)
balance_kernel(const __grid_constant__ BalanceArgs a) {
    using TM = Team<L>;
    extern __shared__ __align__(16) unsigned char smem[];
    float* red = reinterpret_cast<float*>(smem);                           // [warp][L V] column sums
    int32_t* hist = reinterpret_cast<int32_t*>(red + (TM::kCta ? 1 : TM::kWarps) * L * V);   // [L V]
    __shared__ float room[2 * TM::kWarps];
    __shared__ double room64[32];
    __shared__ int32_t window[kWindow + 1];
    __shared__ int n_kept;
    const TM team(room);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, E = a.E, k = a.k;
    const int t0 = (int)min((long long)a.T, (long long)blockIdx.x * a.rows), t1 = (int)min((long long)a.T, (long long)t0 + a.rows);
    const bool last = (int)blockIdx.x == a.tiles - 1;
    for (int e = tid; e < L * V; e += TM::kThreads) hist[e] = 0;
    if (tid == 0) n_kept = 0;
    grid_dependency_wait();
    grid_launch_dependents();
    const Z* z = static_cast<const Z*>(a.z);
    double loss = 0.0, squares = 0.0;
    int some = 0, total = 0, open = -1;                                    // of the tile (the same in all threads)
    int s = a.offsets ? first_ending_at(a.offsets, a.S, t0, lane) : 0, in_window = kWindow;
    for (; s < a.S; ++s, ++in_window) {
        int from = 0, to = a.T;
        if (a.offsets) {
            if (in_window == kWindow) {
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
        for (long long base = (long long)lo + (TM::kCta ? 0 : warp * (32 / L)); base < hi; base += TM::kTeams) {
            const long long t = base + (TM::kCta ? 0 : lane / L);
            const bool on = t < hi && (!a.mask || a.mask[t]);
            if constexpr (TM::kCta) {
                if (!on) continue;
            }
            float v[V];
            if (on) {
                load_row<Z, W, L, V>(z + t * a.ld, E, team.lane, v);
                for (int j = team.lane; j < k; j += L) {
                    const int id = a.ids[t * k + j];
                    if ((unsigned)id < (unsigned)E) atomicAdd(hist + id, 1);
                }
                mine += team.lane == 0;
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = -INFINITY;
            }
            float mx = v[0];
#pragma unroll
            for (int j = 1; j < V; ++j) mx = fmaxf(mx, v[j]);
            mx = team.max(mx);
            const float top = mx == -INFINITY ? 0.f : mx;
            float sum = 0.f, scores = 0.f;
            if (a.sigmoid) {
                const float c = fminf(top, 0.f);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float rest;
                    sum += expf(v[j] - top);
                    v[j] = scaled_sigmoid(v[j], c, rest);
                    scores += v[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    v[j] = expf(v[j] - top);
                    sum += v[j];
                }
            }
            team.sum2(sum, scores);
            const float inv = inverse(a.sigmoid ? scores : sum), lse = log_sum(top, sum);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] = fmaf(v[j], inv, acc[j]);
            if (team.lane == 0) sq = fmaf(lse, lse, sq);
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
        const double factor = whole ? loss_factor(E, k, n) : 0.0;
        for (int e = tid; e < E; e += TM::kThreads) {
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < (TM::kCta ? 1 : TM::kWarps); ++w) sum += red[w * L * V + e];
            const int count = hist[e];
            sums[e] = sum;
            counts[e] = count;
            hist[e] = 0;
            if (whole) loss += (double)count * (double)sum * factor;
        }
        if (tid == 0) (whole ? a.kept : a.part_kept)[at] = n;
        total += n;
        if (whole) some += n > 0;
        else if (from >= t0) open = s;
        __syncthreads();
        if (tid == 0) n_kept = 0;
        __syncthreads();
    }
    loss = cta_sum(loss, room64);
    squares = cta_sum(squares, room64);
    if (tid == 0) {
        a.tile_loss[blockIdx.x] = loss;
        a.tile_z[blockIdx.x] = squares;
        a.tile_kept[blockIdx.x] = total;
        a.tile_some[blockIdx.x] = some;
        a.tile_open[blockIdx.x] = open;
    }
    if constexpr (FUSED) {
        __threadfence();
        cluster_sync();
        join_tiles(a, (int)blockIdx.x, (int)gridDim.x, smem);
    }
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
template <typename Z, int W, int L, int V>
__global__ void __launch_bounds__(Team<L>::kThreads)
gate_backward_kernel(const __grid_constant__ BackwardArgs a) {
    using TM = Team<L>;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float room[2 * TM::kWarps];
    __shared__ double room64[32];
    __shared__ float loss_scale[2];
    const TM team(room);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, E = a.E, k = a.k;
    float* row_add = reinterpret_cast<float*>(smem) + team.index * L * V;
    for (int i = tid; i < TM::kTeams * L * V; i += TM::kThreads) reinterpret_cast<float*>(smem)[i] = 0.f;
    grid_dependency_wait();
    grid_launch_dependents();
    if (a.d_losses) {                                                      // S' and N
        double n = 0.0, some = 0.0;
        for (int s = tid; s < a.S; s += TM::kThreads) {
            const int m = a.kept[s];
            n += m;
            some += m > 0;
        }
        n = cta_sum(n, room64);
        some = cta_sum(some, room64);
        if (tid == 0) {
            loss_scale[0] = some > 0 ? (float)(a.d_losses[0] * (double)E / (some * k)) : 0.f;
            loss_scale[1] = n > 0 ? (float)(2.0 * a.d_losses[1] / n) : 0.f;
        }
    }
    __syncthreads();
    const long long unit = TM::kCta ? blockIdx.x : (long long)blockIdx.x * TM::kWarps + warp;
    const long long t_begin = unit * a.rows, t_end = min((long long)a.T, t_begin + a.rows);
    const bool losses = a.d_losses != nullptr;
    const float balance = losses ? loss_scale[0] : 0.f, z_scale = losses ? loss_scale[1] : 0.f;
    const Z* z = static_cast<const Z*>(a.z);
    float g[V];                                                            // G / balance of the sequence
#pragma unroll
    for (int j = 0; j < V; ++j) g[j] = 0.f;
    int s = -1, s_from = 0, s_to = 0;
    if (losses && t_begin < t_end) s = a.offsets ? first_ending_at(a.offsets, a.S, (int)t_begin + 1, lane) - 1 : -1;
    for (long long base = t_begin; base < t_end; base += TM::kCta ? 1 : 32 / L) {
        const long long t = base + (TM::kCta ? 0 : lane / L);
        const bool in = t < t_end, on = in && (!a.mask || a.mask[t]);
        float v[V];
        if (on) load_row<Z, W, L, V>(z + t * a.ld, E, team.lane, v);
        else
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = -INFINITY;
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
        float mx = v[0];
#pragma unroll
        for (int j = 1; j < V; ++j) mx = fmaxf(mx, v[j]);
        mx = team.max(mx);
        const float top = mx == -INFINITY ? 0.f : mx, c = a.sigmoid ? fminf(top, 0.f) : 0.f;
        float dz[V];
        float sum = 0.f, dot = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            dz[j] = expf(v[j] - top);
            sum += dz[j];
            dot = fmaf(dz[j], g[j], dot);
        }
        team.sum2(sum, dot);
        const float inv = inverse(sum), lse = log_sum(top, sum);
        // what is to be added at the chosen ones, and (softmax) the sum of p d
        float chosen = 0.f;
        if (a.d_weights) {
            float most = -INFINITY;
            if (a.renorm) {
                if (on)
                    for (int j = team.lane; j < k; j += L) {
                        const int id = a.ids[t * k + j];
                        if ((unsigned)id < (unsigned)E) most = fmaxf(most, to_float(z[t * a.ld + id]));
                    }
                most = team.max(most);
            }
            const float least = most == -INFINITY ? 0.f : a.sigmoid ? fminf(most, 0.f) : most;
            float shares = 0.f, d_sum = 0.f;
            bool twice = false;
            if (on)
                for (int j = team.lane; j < k; j += L) {
                    const int id = a.ids[t * k + j];
                    if ((unsigned)id >= (unsigned)E) continue;
                    const float zj = to_float(z[t * a.ld + id]), d = a.scale * a.d_weights[t * k + j];
                    float rest;
                    const float share = !a.renorm && !a.sigmoid ? expf(zj - top) * inv : a.sigmoid ? scaled_sigmoid(zj, a.renorm ? least : 0.f, rest) : expf(zj - least);
                    shares += share;
                    d_sum = fmaf(share, d, d_sum);
                    row_add[id] = __int_as_float(j + 1);
                }
            team.sum2(shares, d_sum);
            team.sync();
            if (on)
                for (int j = team.lane; j < k; j += L) {
                    const int id = a.ids[t * k + j];
                    if ((unsigned)id < (unsigned)E) twice |= __float_as_int(row_add[id]) != j + 1;
                }
            twice = team.any(twice);                                       // an expert that is named twice: one after the other
            if (twice) {
                if (on)
                    for (int j = team.lane; j < k; j += L) {
                        const int id = a.ids[t * k + j];
                        if ((unsigned)id < (unsigned)E) row_add[id] = 0.f;
                    }
                team.sync();
            }
            const float share_inv = a.renorm ? inverse(shares) : 1.f, mean = a.renorm ? d_sum * share_inv : 0.f;
            if (!a.renorm && !a.sigmoid) chosen = d_sum;
            if (on)
                for (int j = twice ? (team.lane ? k : 0) : team.lane; j < k; j += twice ? 1 : L) {
                    const int id = a.ids[t * k + j];
                    if ((unsigned)id >= (unsigned)E) continue;
                    const float zj = to_float(z[t * a.ld + id]), d = a.scale * a.d_weights[t * k + j];
                    float rest = 1.f;
                    const float share = !a.renorm && !a.sigmoid ? expf(zj - top) * inv : a.sigmoid ? scaled_sigmoid(zj, a.renorm ? least : 0.f, rest) : expf(zj - least);
                    const float add = share * share_inv * rest * (d - mean);
                    row_add[id] = twice ? row_add[id] + add : add;
                }
            team.sync();
        }
        if (a.sigmoid) {
            float scores = 0.f;
            dot = 0.f;
            const float zl = counts ? z_scale * lse * inv : 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float rest;
                const float sg = scaled_sigmoid(v[j], c, rest);
                scores += sg;
                dot = fmaf(sg, g[j], dot);
            }
            team.sum2(scores, dot);
            const float sinv = counts ? inverse(scores) : 0.f, mean = dot * sinv;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float rest;
                const float sg = scaled_sigmoid(v[j], c, rest);
                dz[j] = fmaf(dz[j], zl, sg * sinv * rest * (g[j] - mean));
            }
        } else {
            const float zl = counts ? z_scale * lse : 0.f, mean = dot * inv, on_g = counts ? 1.f : 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) dz[j] = dz[j] * inv * (on_g * (g[j] - mean) + zl - chosen);
        }
        if (a.d_weights) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int e = (j / W * L + team.lane) * W + j % W;
                dz[j] += row_add[e];
            }
            team.sync();
            if (on)
                for (int j = team.lane; j < k; j += L) {
                    const int id = a.ids[t * k + j];
                    if ((unsigned)id < (unsigned)E) row_add[id] = 0.f;
                }
            team.sync();
        }
        if (in) store_row<Z, W, L, V>(static_cast<Z*>(a.out) + t * a.ld_out, E, team.lane, dz);
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------

struct Tiling { int rows, tiles; bool fused; };
// Small calls are one cluster, whose CTAs take a tile each and then join them; others a tile per CTA that the chip holds at once.
Tiling tiling(int T, int E) {
    const int at_once = E <= 64 ? 64 : E <= 128 ? 32 : E <= 512 ? 16 : 1;  // rows that a CTA has in hand
    const int most = kSms * (E <= 512 ? 2 : E <= 1024 ? 8 : 2);
    const long long small = T / (2 * at_once);
    if (small <= 8) {
        int ctas = 1;
        while (ctas < 8 && ctas * 2 <= small) ctas *= 2;
        const int rows = std::max(1, (T + ctas - 1) / ctas);
        return {rows, ctas, true};
    }
    const int rows = std::max(2 * at_once, (int)(((long long)T + most - 1) / most));
    return {rows, (int)(((long long)T + rows - 1) / rows), false};
}
size_t scratch_bytes(int E, const Tiling& t) {
    return 8 * (2 * (size_t)t.tiles + 2 * kJoinCtas) + 4 * (4 * (size_t)t.tiles * E + 2 * (size_t)t.tiles + 3 * (size_t)t.tiles + 2 * kJoinCtas);
}

template <typename Z, int W, int L, int V>
int launch_balance(const BalanceArgs& a, bool fused, cudaStream_t st) {
    static SmemOnce once[2];
    constexpr size_t smem = balance_smem<L, V>(), fused_smem = std::max(smem, join_smem(Team<L>::kThreads));
    if (fused) return launch(balance_kernel<Z, W, L, V, true>, (unsigned)a.tiles, Team<L>::kThreads, a.tiles, fused_smem, once[0], st, a);
    const int rc = launch(balance_kernel<Z, W, L, V, false>, (unsigned)a.tiles, Team<L>::kThreads, 1, smem, once[1], st, a);
    if (rc) return rc;
    static SmemOnce join;
    return launch(balance_join_kernel, kJoinCtas, kJoinThreads, kJoinCtas, join_smem(kJoinThreads), join, st, a);
}
template <typename Z, int W>
int launch_balance(const BalanceArgs& a, bool fused, cudaStream_t st) {
    if (a.E <= 64) return launch_balance<Z, W, 8, 8>(a, fused, st);
    if (a.E <= 128) return launch_balance<Z, W, 16, 8>(a, fused, st);
    if (a.E <= 256) return launch_balance<Z, W, 32, 8>(a, fused, st);
    if (a.E <= 512) return launch_balance<Z, W, 32, 16>(a, fused, st);
    if (a.E <= 1024) return launch_balance<Z, W, 128, 8>(a, fused, st);
    return launch_balance<Z, W, 512, 8>(a, fused, st);
}

template <typename Z, int W, int L, int V>
int launch_backward(BackwardArgs a, cudaStream_t st) {
    using TM = Team<L>;
    static SmemOnce once;
    // rows per warp (CTA): as many as leave every SM four CTAs
    constexpr int at_once = TM::kCta ? 1 : 32 / L;
    const long long units = (long long)kSms * 4 * (TM::kCta ? 1 : TM::kWarps);
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
    *bytes = scratch_bytes(shape->num_experts, tiling(T, shape->num_experts));
    return EXMOE_OK;
}

extern "C" int exmoe_balance_loss(const exmoe_shape* shape, const exmoe_gate* gate, const void* logits, int type, int64_t row_stride, const int32_t* topk_ids,
                                  const uint8_t* mask, const int32_t* offsets, int num_sequences, int T, float* losses, int32_t* counts, float* score_sums,
                                  int32_t* kept, void* scratch, void* stream) {
    GateArgs g;
    const int rc = check_loss(shape, gate, type, row_stride, T, num_sequences, offsets, &g);
    if (rc) return rc;
    if ((T && (!logits || !topk_ids)) || !losses || !counts || !score_sums || !kept || !scratch) return EXMOE_ERR_ARG;
    const int es = type == EXMOE_F32 ? 4 : 2;
    if (!aligned(es, logits) || !aligned(4, topk_ids, offsets, losses, counts, score_sums, kept) || !aligned(8, scratch)) return EXMOE_ERR_ARG;
    const Tiling t = tiling(T, g.E);
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
    a.joined_some = a.tile_open + n;
    cudaStream_t st = (cudaStream_t)stream;
    const bool fours = in_fours(logits, row_stride, T, g.E, es);
    if (type == EXMOE_F32) return fours ? launch_balance<float, 4>(a, t.fused, st) : launch_balance<float, 1>(a, t.fused, st);
    return fours ? launch_balance<__nv_bfloat16, 4>(a, t.fused, st) : launch_balance<__nv_bfloat16, 1>(a, t.fused, st);
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
