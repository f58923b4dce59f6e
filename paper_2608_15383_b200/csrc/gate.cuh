// The choice of a gate (exmoe_gate) from a token's logits, shared by the kernels that end in it.
#pragma once
#include <algorithm>

#include "common.cuh"
#include "frag.cuh"

namespace exmoe {

struct GateArgs {
    int E, k, G, size, top_groups;     // experts, choices, groups, experts per group, groups kept (G where there are no groups)
    bool sigmoid, top2, renorm;
    float scale;
    const float* balance;              // [E] or null
    int lanes, log_lanes;              // lanes per group where a warp looks at all of them: 32 / (groups rounded up to a power of two)
    int turns;                         // ceil(size / lanes)
    int log_run;                       // a group is 2^log_run lanes' experts where a lane holds choose_fast's run of them; -1: it is not
    float inv_size;                    // 1 / size
};
constexpr int kFastExperts = 512, kFastChoices = 32;                       // what choose_fast takes
// What it leaves where it cannot decide: a bit per expert whose logit decides, the groups kept, and what is to be done with these logits
constexpr int kTodoKept = kFastExperts / 32, kTodoStage = kTodoKept + 1, kTodoWords = kTodoKept + 2;
enum { GATE_EXPERTS = 0, GATE_ALL = 1, GATE_GROUPS = 2 };
enum { GATE_NEW = 0, GATE_DECIDED = 1, GATE_DONE = -1, GATE_WAITS = -2 };  // how a choice begins, and what go_on says besides

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

// The groups that keep their experts (a bit each), from lane o's value of group o.
template <typename T>
__device__ __forceinline__ unsigned kept_groups(const GateArgs& g, T value, int lane) {
    int before = 0;
#pragma unroll 4
    for (int o = 0; o < g.G; ++o) {
        const T v = __shfl_sync(0xffffffffu, value, o);
        before += v > value || (v == value && o < lane);
    }
    return __ballot_sync(0xffffffffu, lane < g.G && before < g.top_groups);
}
__device__ __forceinline__ int group_of(const GateArgs& g, int e) { return (int)(((float)e + 0.5f) * g.inv_size); }
__device__ __forceinline__ bool in_kept(const GateArgs& g, unsigned kept, int e) { return kept >> group_of(g, e) & 1u; }
// The largest and second largest of group `lane`'s values v [E]; a NaN is none.
template <typename T>
__device__ __forceinline__ void two_largest(const GateArgs& g, const T* v, int lane, T& a, T& b) {
    const int grp = lane >> g.log_lanes, sub = lane & (g.lanes - 1);
    a = b = -INFINITY;
    if (grp < g.G)
        for (int i = 0, at = grp % g.turns; i < g.turns; ++i, at = at + 1 == g.turns ? 0 : at + 1) {     // groups start apart: other banks
            const int idx = sub + (at << g.log_lanes);
            T x = idx < g.size ? v[grp * g.size + idx] : -INFINITY;
            if (x != x) x = -INFINITY;
            b = max(b, min(a, x));
            a = max(a, x);
        }
    for (int m = g.lanes / 2; m >= 1; m /= 2) {
        const T oa = __shfl_xor_sync(0xffffffffu, a, m), ob = __shfl_xor_sync(0xffffffffu, b, m);
        b = max(max(b, ob), min(a, oa));
        a = max(a, oa);
    }
    a = __shfl_sync(0xffffffffu, a, (lane << g.log_lanes) & 31);
    b = __shfl_sync(0xffffffffu, b, (lane << g.log_lanes) & 31);
}

// The whole choice in binary64, by one warp.  z: the token's logits, key: room for as many integers (both in shared memory).
static __device__ __noinline__ void choose_exact(const GateArgs& g, const double* z, unsigned long long* key, int lane, int32_t* ids, float* weights) {
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
        double a, b;
        two_largest(g, g.top2 ? c : by, lane, a, b);
        const double value = g.top2 && b > kMasked ? a + b : a;
        kept = kept_groups(g, value, lane);
        __syncwarp();
    }
    for (int e = lane; e < g.E; e += 32) key[e] = !grouped || in_kept(g, kept, e) ? order_key(by[e]) : 0ull;
    double top = kMasked;                                                  // of the chosen
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
        top = fmax(top, z[e]);
        if (lane == 0) {
            ids[j] = e;
            key[e] = 0ull;
        }
        __syncwarp();
    }
    double f = 1.0;
    if (g.renorm) {
        if (!g.sigmoid && inv == inv && top > kMasked) {                   // relative to the largest chosen: the others may all be below 2^-1074 of the largest of all
            mx = top;
            inv = 1.0;
        }
        double total = 0.0;
        for (int j = lane; j < g.k; j += 32) total += score(z[ids[j]]);
        total = warp_sum_f64(total);
        f = total == 0.0 ? 0.0 : 1.0 / total;
    }
    for (int j = lane; j < g.k; j += 32) weights[j] = (float)(score(z[ids[j]]) * f * (double)g.scale);
}

// ---- the choice in binary32, with what it cannot decide left to choose_exact -------------------------------------------------
// The logits are within dz + rel |z| of the true ones (for what follows, within dz), and a score computed from them within a few roundings of the true one.  With
// |ds/dz| <= 1/4 for a sigmoid and |ds_e| <= 2 s_e (1 - s_e) dz <= dz / 2 for a softmax whose logits are all off by dz at most (0.26 and 0.55
// with the terms of second order, for dz <= 0.05) two choice values that are further apart than `near` below are in their true
// order.  Where a decision rests on a smaller distance, the experts that it concerns are marked, to be looked at again.
__device__ __forceinline__ uint32_t order_key(float v) {                   // as above; no NaN comes here; 0: cannot be chosen
    const uint32_t b = __float_as_uint(v + 0.f);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ float warp_max(float v) {                        // a NaN is left out
    float m;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
    return m;
}
__device__ __forceinline__ float warp_sum_f32(float s) {
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
    return s;
}
__device__ __forceinline__ float sigmoid(float z) {
    const float e = expf(-fabsf(z));
    return (z >= 0.f ? 1.f : e) / (1.f + e);
}
// rel: |z| s (1 - s) < 0.23 for a sigmoid; in a softmax logits 100 below the largest have no part
__device__ __forceinline__ float bound_of(const GateArgs& g, float dz, float rel, float mx) { return dz + (g.sigmoid ? rel : rel * (fabsf(mx) + 100.f)); }
__device__ __forceinline__ float quick_sigmoid(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }
// exp(z - top): the rounding of the difference, 2^-24 of it, is put back
__device__ __forceinline__ float exp_below(float z, float top) {
    const float d = z - top, back = d + top;
    const float err = (z - back) + ((back - d) - top);
    const float e = expf(d);
    return d > -INFINITY ? fmaf(e, err, e) : 0.f;
}

// The weight of a chosen expert's logit, by the lanes that hold one (`chosen`); mx: the largest logit of all, sum: of the exponentials below
// it.  False: too small for binary32, which holds a sigmoid of 2^-126 and less with few bits or none; beside a sum of 1e-8 and more that is nothing.
__device__ __forceinline__ bool choice_weight(const GateArgs& g, float z, bool chosen, float mx, float sum, float& s) {
    if (g.sigmoid) {
        s = sigmoid(z);
    } else {
        const float top = g.renorm ? warp_max(chosen ? z : -INFINITY) : mx;
        s = top > -INFINITY ? exp_below(z, top) : 0.f;
        if (!g.renorm) s /= sum;
    }
    if (g.renorm) {
        const float total = warp_sum_f32(chosen ? s : 0.f);
        if (g.sigmoid && total < 1e-8f) return false;                      // nothing left, or nearly
        s = total > 0.f ? s / total : 0.f;
    }
    s *= g.scale;
    return true;
}

// What few tokens come to is kept out of the way of what all of them do (registers, instruction cache).
// Experts of group o whose value is at least lane o's `from` are marked.
static __device__ __noinline__ void mark_from(const GateArgs& g, uint32_t* todo, const float* v, float from, int lane) {
    for (int e0 = 0; e0 < g.E; e0 += 32) {
        const int e = e0 + lane;
        const float t = __shfl_sync(0xffffffffu, from, group_of(g, min(e, g.E - 1)));
        const unsigned m = __ballot_sync(0xffffffffu, e < g.E && v[e] >= t);
        if (lane == 0) todo[e0 >> 5] |= m;
    }
    __syncwarp();
}
// k rounds of arg-max over v [E]: lane j gets the j-th choice (-1: none).  False: two of them, or the last and the next, are too close.
template <int PER>
static __device__ __noinline__ bool choose_rounds(const GateArgs& g, const float* v, unsigned kept, float near0, float near1, int lane, int& mine) {
    const bool grouped = g.top_groups < g.G, exact = near0 == 0.f;
    uint32_t key[PER];                                                     // of experts lane, lane + 32, ...
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = lane + 32 * i;
        key[i] = e < g.E && (!grouped || in_kept(g, kept, e)) ? order_key(v[e]) : 0u;
    }
    float prev = 0.f;
    for (int j = 0; j <= g.k; ++j) {
        uint32_t top = 0;
        int be = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (key[i] > top) {                                            // ascending experts: the first maximum wins
                top = key[i];
                be = lane + 32 * i;
            }
        const uint32_t most = __reduce_max_sync(0xffffffffu, top);
        if (!most) break;                                                  // no other expert can be chosen
        const int e = (int)__reduce_min_sync(0xffffffffu, top == most ? (unsigned)be : 0x7fffffffu);
        const float x = key_value(most);
        if (!exact && j > 0 && x > -INFINITY && prev - x <= near0 + near1 * (fabsf(prev) + fabsf(x))) return false;
        prev = x;
        if (j == lane && j < g.k) mine = e;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (e == lane + 32 * i) key[i] = 0u;
    }
    return true;
}

// The candidates among which GATE_EXPERTS marks the near-ties, for finish_choice: expert | rank << 9, the largest logit of all, and the sum of
// the exponentials below it.
struct Picks {
    unsigned short at[32];
    int n;
    float mx, sum;
};
static_assert(kFastExperts <= 512 && kFastChoices <= 32, "a candidate's sixteen bits");
// What a warp needs in shared memory for a token's choice.
template <int PER>
struct __align__(16) ChoiceRoom {
    float z[32 * PER];                                                     // logits, -infinity behind the last
    float c[32 * PER];                                                     // choice values
    int expert[32];                                                        // candidates
    uint32_t todo[kTodoWords];
    Picks picks;
};
template <int PER>
__device__ __forceinline__ void load_run(const float* p, float (&v)[PER]) {
    if constexpr (PER == 2) {
        const float2 a = *reinterpret_cast<const float2*>(p);
        v[0] = a.x, v[1] = a.y;
    } else {
#pragma unroll
        for (int i = 0; i < PER; i += 4) {
            const float4 a = *reinterpret_cast<const float4*>(p + i);
            v[i] = a.x, v[i + 1] = a.y, v[i + 2] = a.z, v[i + 3] = a.w;
        }
    }
}
template <int PER>
__device__ __forceinline__ void store_run(float* p, const float (&v)[PER]) {
    if constexpr (PER == 2) {
        *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
    } else {
#pragma unroll
        for (int i = 0; i < PER; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    }
}

// All logits are to be computed again.
template <int PER>
__device__ __forceinline__ void choose_all(const GateArgs& g, ChoiceRoom<PER>& room, int lane) {
    for (int i = lane; 32 * i < g.E; i += 32) room.todo[i] = g.E - 32 * i >= 32 ? 0xffffffffu : (1u << (g.E - 32 * i)) - 1u;
    if (lane == 0) room.todo[kTodoStage] = GATE_ALL;
    __syncwarp();
}

// By one warp; lane l holds the PER experts from PER l on; `balance`: g.balance padded to 32 PER, or null; at most kFastChoices choices.
// `mode`: GATE_NEW; GATE_DECIDED: the groups are those of todo[kTodoKept].  True: nothing is written, and `todo` says what is to be done.
// The choice itself: the k-th largest of the lanes' largest values is no more than the k-th largest value, so what is not below
// it (by more than `near`) are all candidates, k and a few more; they go to a lane each, which counts those before its own.  (Instead
// of k rounds of arg-max, which took twice the instructions.)
template <int PER>
__device__ __forceinline__ bool choose_fast(const GateArgs& g, ChoiceRoom<PER>& room, const float* balance, float dz, float rel, int lane, int mode,
                                            int32_t* ids, float* weights) {
    const bool grouped = g.top_groups < g.G, by_score = balance || (grouped && g.top2);
    float by[PER], other[PER];                                             // what orders the experts; scores where these are not it
    load_run<PER>(room.z + PER * lane, by);
    float mx = -INFINITY, any = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        mx = fmaxf(mx, by[i]);
        any += by[i];                                                      // a NaN where there is one, or infinities of both signs
    }
    mx = warp_max(mx);
    const float dzs = bound_of(g, dz, rel, mx);
    bool odd = __any_sync(0xffffffffu, any != any) || !(fabsf(mx) < INFINITY) || !(dzs <= 0.05f);
    float sum = 1.f;
    // branches around loops that all lanes take alike, not choices per expert: both sides of these would be computed
    if (!odd && !g.sigmoid && (by_score || !g.renorm)) {
        float part[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) part[i] = other[i] = expf(by[i] - mx);
#pragma unroll
        for (int n = PER / 2; n >= 1; n /= 2)
#pragma unroll
            for (int i = 0; i < n; ++i) part[i] += part[i + n];
        sum = warp_sum_f32(part[0]);
    }
    // quick_sigmoid is within 3.5e-7 of the true one (__expf's argument off by 2^-23 |z|, its result by 2^-22 of itself, each times s (1 - s); the quotient
    // by 2^-22 s), a probability p = p_max exp(-a) (a off by 2^-24 of itself, a exp(-a) < 0.37; up to 25 roundings in exponentials, sum and quotient) within
    // 2e-6 p_max; c itself rounds once more.  s (1 - s) is no more than 1/4, in a softmax no more than p_max either: with a hundred experts values
    // lie p_max / 10 and less apart, and 1/4 would have most tokens' logits computed again.
    const float p_max = 1.f / sum;
    const float slope_near = g.sigmoid ? 2.f * 0.26f : 2.f * 2.2f * fminf(0.25f, p_max), round_near = g.sigmoid ? 7e-7f : 4e-6f * p_max;
    const float score_near = slope_near * dzs + round_near;
    const float near0 = balance ? score_near : 2.f * dz, near1 = balance ? 1.2e-7f : rel;                // near = near0 + near1 (|a| + |b|)
    if (!odd && by_score) {
        if (g.sigmoid) {
#pragma unroll
            for (int i = 0; i < PER; ++i) other[i] = quick_sigmoid(by[i]);
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) other[i] *= p_max;
        }
        if (balance) {
            float bias[PER];
            load_run<PER>(balance + PER * lane, bias);
            float all = 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                other[i] += bias[i];
                all += fabsf(bias[i]);
            }
            odd = __any_sync(0xffffffffu, !(all < INFINITY));
        }
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (by[i] == -INFINITY) other[i] = -INFINITY;
        store_run<PER>(room.c + PER * lane, other);
        if (balance)
#pragma unroll
            for (int i = 0; i < PER; ++i) by[i] = other[i];
        __syncwarp();
    }
    int stage = odd ? GATE_ALL : GATE_EXPERTS;
    unsigned kept = mode == GATE_NEW ? 0xffffffffu : room.todo[kTodoKept];
    if (lane < kTodoKept) room.todo[lane] = 0;
    __syncwarp();
    bool marked = false;
    if (grouped && mode == GATE_NEW && !odd) {
        float a, b;
        if (g.log_run >= 0) {
            a = b = -INFINITY;
            if (by_score) {
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    b = fmaxf(b, fminf(a, other[i]));
                    a = fmaxf(a, other[i]);
                }
            } else {                                                       // the largest is all that is asked for
#pragma unroll
                for (int i = 0; i < PER; ++i) a = fmaxf(a, by[i]);
            }
            for (int m = 1 << g.log_run >> 1; m >= 1; m >>= 1) {
                const float oa = __shfl_xor_sync(0xffffffffu, a, m), ob = __shfl_xor_sync(0xffffffffu, b, m);
                b = fmaxf(fmaxf(b, ob), fminf(a, oa));
                a = fmaxf(a, oa);
            }
            a = __shfl_sync(0xffffffffu, a, (lane << g.log_run) & 31);
            b = __shfl_sync(0xffffffffu, b, (lane << g.log_run) & 31);
        } else {
            two_largest(g, by_score ? room.c : room.z, lane, a, b);
        }
        const float value = g.top2 && b > -INFINITY ? a + b : a;
        kept = kept_groups(g, value, lane);
        const bool real = lane < g.G, keep = kept >> lane & 1u;
        // the smallest value kept against the largest dropped; a masked group's -infinity is exact
        const float low = -warp_max(real && keep ? -value : -INFINITY), high = warp_max(real && !keep ? value : -INFINITY);
        const float near_v = by_score ? score_near : 2.f * dz, rel_v = by_score ? 2.4e-7f : rel;
        const float near = (g.top2 ? 2.f : 1.f) * near_v + rel_v * (fabsf(low) + fabsf(high));
        if (near > 0.f && high > -INFINITY && low - high <= near) {
            // the groups on the border, and of each the experts that may be its largest (two)
            const bool border = real && (keep ? value <= high + near : value >= low - near);
            const float least = g.top2 && b > -INFINITY ? b : a;
            mark_from(g, room.todo, by_score ? room.c : room.z, border ? least - near_v - 2.f * rel_v * fabsf(least) : INFINITY, lane);
            stage = GATE_GROUPS;
        }
    }
    if (stage == GATE_EXPERTS) {
        const bool exact = near0 == 0.f;
        const bool lane_in = !grouped || g.log_run < 0 || (kept >> (lane >> g.log_run) & 1u);
        if (grouped && g.log_run < 0)
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (!in_kept(g, kept, min(PER * lane + i, g.E - 1))) by[i] = -INFINITY;
        float best = -INFINITY;
        if (lane_in)
#pragma unroll
            for (int i = 0; i < PER; ++i) best = fmaxf(best, by[i]);
        float from = -INFINITY, largest = 0.f;
        for (int j = 0; j < g.k; ++j) {                                    // equal largest values go together: the bound is only lower
            from = warp_max(best);
            if (j == 0) largest = from;
            if (best == from) best = -INFINITY;
        }
        const bool few = from == -INFINITY;                                // lanes with experts that can be chosen: all of these are candidates
        if (few && largest > -INFINITY) {
            float least = INFINITY;
            if (lane_in)
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (by[i] > -INFINITY) least = fminf(least, by[i]);
            from = -warp_max(-least);
        }
        // the same for all pairs of candidates: these lie between the two
        const float near = near0 + (from > -INFINITY ? 2.f * near1 * fmaxf(fabsf(largest), fabsf(from)) : 0.f);
        if (!exact && !few) from -= near;
        unsigned mine = 0;                                                 // candidates of this lane, a bit each
        if (lane_in)
#pragma unroll
            for (int i = 0; i < PER; ++i) mine |= by[i] >= from ? 1u << i : 0u;
        int n = 0, at = 0;                                                 // of all, before this lane's
        const unsigned lt = (1u << lane) - 1u;
        for (int c = __popc(mine);; --c) {
            const unsigned m = __ballot_sync(0xffffffffu, c > 0);
            if (!m) break;
            n += __popc(m);
            at += __popc(m & lt);
        }
        if (n >= g.k && n <= 32 && from > -INFINITY) {
            for (; mine; mine &= mine - 1) room.expert[at++] = PER * lane + __ffs(mine) - 1;       // in ascending experts
            __syncwarp();
            const int e = lane < n ? room.expert[lane] : 0;
            const float v = lane < n ? (balance ? room.c : room.z)[e] : -INFINITY;
            int before = 0, close = 0;
            float close_by = near;
            if (exact) {
#pragma unroll 4
                for (int j = 0; j < n; ++j) {
                    const float o = __shfl_sync(0xffffffffu, v, j);
                    before += o > v || (o == v && j < lane);
                }
            } else {
                // The candidates' own slopes: they lie where a sigmoid is flat.  A logit of z is off by dz + rel |z| where this has dz + rel: what
                // 2 rel (|z| - 1.06) s (1 - s) lacks is below 3.7e-8, and round_near is 7.3e-8 and more above what two quick_sigmoids need at any z.
                if (balance) {
                    float slope = 0.f;
                    if (lane < n) {
                        const float p = g.sigmoid ? quick_sigmoid(room.z[e]) : expf(room.z[e] - mx) / sum;
                        slope = (g.sigmoid ? p : 2.f * p) * (1.f - p);
                    }
                    close_by = near - near0 + 2.f * 1.06f * dzs * (warp_max(slope) + 1e-5f * (g.sigmoid ? 1.f : p_max)) + round_near;
                }
#pragma unroll 4
                for (int j = 0; j < n; ++j) {
                    const float o = __shfl_sync(0xffffffffu, v, j);
                    before += o > v || (o == v && j < lane);
                    close += fabsf(o - v) <= close_by;                     // itself among them
                }
            }
            const bool chosen = lane < n && before < g.k;
            if (!exact) {
                const float last = __shfl_sync(0xffffffffu, v, __ffs(__ballot_sync(0xffffffffu, lane < n && before == g.k - 1)) - 1);
                if (lane < n && (chosen ? close > 1 : v >= last - close_by)) {
                    atomicOr(&room.todo[e >> 5], 1u << (e & 31));
                    marked = true;
                }
            }
            if (!__any_sync(0xffffffffu, marked)) {
                float s;
                if (choice_weight(g, room.z[e], chosen, mx, sum, s)) {
                    if (chosen) {
                        ids[before] = e;
                        weights[before] = s;
                    }
                    return false;
                }
                stage = GATE_ALL;
            } else {
                room.picks.at[lane] = (unsigned short)(e | before << 9);
                if (lane == 0) {
                    room.picks.n = n;
                    room.picks.mx = mx;
                    room.picks.sum = sum;
                }
            }
        } else {                                                           // many equal values, or few logits that are not -infinity
            int at = -1;
            if (choose_rounds<PER>(g, balance ? room.c : room.z, kept, near0, near1, lane, at)) {
                float s;
                if (choice_weight(g, room.z[max(at, 0)], at >= 0, mx, sum, s)) {
                    if (at >= 0) {
                        ids[lane] = at;
                        weights[lane] = s;
                    }
                    return false;
                }
            }
            stage = GATE_ALL;
        }
    }
    if (!g.sigmoid && balance && stage == GATE_GROUPS) stage = GATE_ALL;   // a softmax with a bias: all logits enter every choice value
    __syncwarp();
    if (lane == 0) {
        room.todo[kTodoKept] = kept;
        room.todo[kTodoStage] = stage;
    }
    if (stage == GATE_ALL) choose_all<PER>(g, room, lane);
    __syncwarp();
    return true;
}

// A marked expert's logit: from z64, or z itself where that is exact (z64 null).
__device__ __forceinline__ double marked_logit(const double* z64, const float* z, int e) { return z64 ? z64[e] : (double)z[e]; }
// The groups kept, from the exact logits of the marked experts, for choose_fast to go on from there; v [E]: room, may be z64.
template <int PER>
static __device__ __noinline__ void choose_groups(const GateArgs& g, ChoiceRoom<PER>& room, const double* z64, double* v, int lane) {
    const bool by_score = g.balance || g.top2;
    float mx = -INFINITY, sum = 0.f;
    if (!g.sigmoid && by_score) {                                          // a common factor of all
        for (int e = lane; e < g.E; e += 32) mx = fmaxf(mx, room.z[e]);
        mx = warp_max(mx);
        for (int e = lane; e < g.E; e += 32) sum += expf(room.z[e] - mx);
        sum = warp_sum_f32(sum);
    }
    for (int e = lane; e < g.E; e += 32) {
        const bool m = room.todo[e >> 5] >> (e & 31) & 1u;
        double x = m ? marked_logit(z64, room.z, e) : (double)room.z[e];
        if (by_score && x > -INFINITY) {
            if (m)
                x = g.sigmoid ? 1.0 / (1.0 + exp(-x)) : exp(x - (double)mx) / (double)sum;
            else
                x = (double)(g.sigmoid ? quick_sigmoid((float)x) : expf((float)x - mx) / sum);
            if (g.balance) x += (double)g.balance[e];
        }
        v[e] = x;
    }
    __syncwarp();
    double a, b;
    two_largest(g, v, lane, a, b);
    const unsigned kept = kept_groups(g, g.top2 && b > -INFINITY ? a + b : a, lane);
    if (lane == 0) room.todo[kTodoKept] = kept;
    __syncwarp();
}

// The choice among the candidates, whose marked ones' logits are exact in z64 (or z, z64 null), z being up to date: each keeps its rank among the unmarked
// ones, from which it is far enough, and the marked ones are ranked among themselves.  False: that does not decide, and everything is to be computed again.
// It may not for a softmax with a bias: p_e = exp(z_e - mx) / sum with a sum of logits that are off by dz, which is itself off by kSumRel (below)
// of itself, leaves c_a - c_b off by (dz + kSumRel) |p_a - p_b|: also where the logits are exact, as given ones are.
// (The whole of choose_fast once more took 10 thousand cycles of gate_8192 where this takes a third.)
// kSumRel: choose_fast's sum in units of 2^-24: expf 4, its argument (in the mean over the probabilities, up to ln 512 of them) 6.3, 4 additions in a lane and 5
// over the lanes: 19.3, or 1.2e-6.
constexpr double kSumRel = 2e-6;
template <int PER>
static __device__ __noinline__ bool finish_choice(const GateArgs& g, ChoiceRoom<PER>& room, const float* balance, const double* z64, float dz, float rel, int lane, int32_t* ids, float* weights) {
    const int n = room.picks.n, e = lane < n ? room.picks.at[lane] & 511 : 0, was = lane < n ? room.picks.at[lane] >> 9 : 32;
    const float mx = room.picks.mx, sum = room.picks.sum;
    const bool m = lane < n && (room.todo[e >> 5] >> (e & 31) & 1u), soft = balance && !g.sigmoid;
    double w = 0.0, b = 0.0;
    if (m) {
        w = marked_logit(z64, room.z, e);
        if (balance) {
            b = (double)balance[e];
            w = w == -INFINITY ? w : (g.sigmoid ? 1.0 / (1.0 + exp(-w)) : exp(w - (double)mx) / (double)sum) + b;
        }
    }
    int before = was;
    bool unsure = false;
    for (unsigned left = __ballot_sync(0xffffffffu, m); left; left &= left - 1) {
        const int j = __ffs(left) - 1;                                     // ascending experts
        const double o = __shfl_sync(0xffffffffu, w, j);
        const int o_was = __shfl_sync(0xffffffffu, was, j);
        if (m) before += (int)(o > w || (o == w && j < lane)) - (int)(o_was < was);
        if (soft) {
            const double ob = __shfl_sync(0xffffffffu, b, j);
            unsure |= m && j != lane && w > -INFINITY && o > -INFINITY && fabs(o - w) <= (1.1 * (double)bound_of(g, dz, rel, mx) + kSumRel) * fabs((o - ob) - (w - b)) + 1e-12;
        }
    }
    const bool chosen = lane < n && before < g.k;
    float s = 0.f;
    if (!__any_sync(0xffffffffu, unsure && before <= g.k) && choice_weight(g, room.z[e], chosen, mx, sum, s)) {
        if (chosen) {
            ids[before] = e;
            weights[before] = s;
        }
        return true;
    }
    if (lane == 0) room.todo[kTodoStage] = GATE_ALL;
    choose_all<PER>(g, room, lane);
    return false;
}
// After choose_fast's `true`, the marked logits being in z64 (room for all): the mode in which it goes on, GATE_DONE, or GATE_WAITS for what
// is marked now.  The logits in `room` are brought up to date.
template <int PER>
__device__ __forceinline__ int go_on(const GateArgs& g, ChoiceRoom<PER>& room, const float* balance, double* z64, float dz, float rel, int lane, int32_t* ids, float* weights) {
    const uint32_t stage = room.todo[kTodoStage];
    if (stage == GATE_ALL) {
        choose_exact(g, z64, reinterpret_cast<unsigned long long*>(room.z), lane, ids, weights);       // z and c
        return GATE_DONE;
    }
    for (int b = 0; 32 * b < g.E; ++b)
        if (room.todo[b] >> lane & 1u) room.z[32 * b + lane] = (float)z64[32 * b + lane];
    __syncwarp();
    if (stage == GATE_EXPERTS) return finish_choice<PER>(g, room, balance, z64, dz, rel, lane, ids, weights) ? GATE_DONE : GATE_WAITS;
    choose_groups<PER>(g, room, z64, z64, lane);
    return GATE_DECIDED;
}

// ---- what the kernels share --------------------------------------------------------------------------------------------
constexpr int kGateSmemMax = 200 * 1024, kSms = 148;
// Squares below 2^-149 are lost from a norm, and products below 2^-126 may be from a logit; where a norm has come out so small that this matters, it is taken
// to be this: 2^-24 of two such norms' product is more than 102,400 products of 2^-126.  A row of zeros, or a
// router of zeros, has exact logits and a bound of 0; where a norm has come out as 0, the numbers tell (logits that all come out as 0 do not: sums may
// cancel).  The form for few tokens does not look at the router's: computing all logits again is quicker there than reading it once more.
constexpr float kLeastSquare = 1e-25f;
__device__ __forceinline__ float least_of(float sum) { return sum == 0.f ? 0.f : fmaxf(sum, kLeastSquare); }
// Whether one of chunks lane, lane + step, ... of eight BF16 numbers is not all zeros, for any lane of the warp.
__device__ __forceinline__ bool any_number(const uint4* p, int chunks, int lane, int step) {
    bool any = false;
#pragma unroll 1
    for (int i = lane; i < chunks; i += step) {
        const uint4 v = p[i];
        any |= ((v.x | v.y | v.z | v.w) & 0x7fff7fffu) != 0u;
    }
    return __any_sync(0xffffffffu, any);
}
// Bias and addend: 2^-24 (|sum before| + |z|), with |sum before| <= 2 |z| + 16.  The logits of a row of zeros are its bias or its addend, exact unless it has both.
constexpr float kAddedRel = 3.f * 0x1p-24f;

__device__ __forceinline__ void unpack8(const uint4& a, float (&x)[8]) {
    const uint32_t r[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(r[i] << 16);
        x[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ float dot8(const float (&w)[8], const float (&x)[8]) {        // two chains of four
    float d = 0.f, e = 0.f;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        d = fmaf(w[n], x[n], d);
        e = fmaf(w[n + 4], x[n + 4], e);
    }
    return d + e;
}
__device__ __forceinline__ float square8(const uint4& a) {
    float x[8];
    unpack8(a, x);
    return dot8(x, x);
}
// What chunks `from` .. `to` - 1 of eight numbers add to a logit, by one warp in binary64.
static __device__ __noinline__ double logit_wide(const uint4* x, const uint4* w, int from, int to, int lane) {
    double s = 0.0;
#pragma unroll 1
    for (int i = from + lane; i < to; i += 32) {
        float a[8], b[8];
        unpack8(w[i], a);
        unpack8(x[i], b);
#pragma unroll
        for (int n = 0; n < 8; ++n) s += (double)a[n] * (double)b[n];
    }
    return warp_sum_f64(s);
}
// Products of BF16 values are exact in binary32 between 2^-126 and 2^128.  Above, a sum of them is an infinity or a NaN; below, they are off by 2^-150, which a
// sum of 2^-66 and more does not hold.
__device__ __forceinline__ bool needs_wide(double s) { return !(fabs(s) >= 0x1p-66 && fabs(s) < (double)INFINITY); }
// The same with products in binary32; WIDE: by logit_wide where the sum needs it, otherwise the caller sees to that.  Conversions to binary64 bound it (16 a cycle
// and SM), half as many as there.
template <bool WIDE>
static __device__ __noinline__ double logit_f64(const uint4* x, const uint4* w, int from, int to, int lane) {
    constexpr int U = 2;                                                   // chunks at a time (little code: it is mostly cold), the next ones in flight
    double s[4 * U] = {};
    uint4 wv[U], xv[U];
    auto fetch = [&](int i0) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int i = i0 + 32 * j + lane;
            wv[j] = xv[j] = make_uint4(0, 0, 0, 0);
            if (i < to) {
                wv[j] = w[i];
                xv[j] = x[i];
            }
        }
    };
    fetch(from);
#pragma unroll 1
    for (int i0 = from; i0 < to; i0 += 32 * U) {
        float p[U][8];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const uint32_t a[4] = {wv[j].x, wv[j].y, wv[j].z, wv[j].w}, b[4] = {xv[j].x, xv[j].y, xv[j].z, xv[j].w};
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                p[j][2 * n] = __uint_as_float(a[n] << 16) * __uint_as_float(b[n] << 16);
                p[j][2 * n + 1] = __uint_as_float(a[n] & 0xffff0000u) * __uint_as_float(b[n] & 0xffff0000u);
            }
        }
        fetch(i0 + 32 * U);
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int j = 0; j < U; ++j) s[4 * j + n % 4] += (double)p[j][n];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] += s[4 + j];
    const double sum = warp_sum_f64((s[0] + s[1]) + (s[2] + s[3]));
    return WIDE && needs_wide(sum) ? logit_wide(x, w, from, to, lane) : sum;
}
// Into how many parts (a power of two, up to eight) the warps of a CTA share the sums of `items` logits: no more than `most` parts in all.
__device__ __forceinline__ int log_parts(int items, int most) {
    return items * 8 <= most ? 3 : items * 4 <= most ? 2 : items * 2 <= most ? 1 : 0;
}
// The marked experts, a word of 32 per lane, and how many there are up to it.
struct Marked {
    unsigned word;
    int up_to;
    __device__ __forceinline__ Marked(const uint32_t* todo, int words, int lane) {
        word = lane < words ? todo[lane] : 0u;
        up_to = __popc(word);
#pragma unroll
        for (int m = 1; m < 32; m <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, up_to, m);
            if (lane >= m) up_to += o;
        }
    }
    __device__ __forceinline__ int count() const { return __shfl_sync(0xffffffffu, up_to, 31); }
};

// every form is a programmatic dependent of the kernel before it in the stream (it waits for it before it reads anything)
template <typename... P, typename... A>
int launch(void (*kern)(P...), unsigned ctas, int threads, int cluster, size_t smem, SmemOnce& once, cudaStream_t st, const A&... args) {
    if (!allow_smem(kern, std::max(kGateSmemMax, (int)smem), once)) return EXMOE_ERR_CUDA;
    cudaLaunchConfig_t lc{};
    lc.gridDim = dim3(ctas);
    lc.blockDim = dim3((unsigned)threads);
    lc.dynamicSmemBytes = smem;
    lc.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = cluster > 1 ? 2 : 1;
#ifdef EXMOE_DISABLE_PDL
    lc.attrs = attr + 1;
    --lc.numAttrs;
#endif
    if (cudaLaunchKernelEx(&lc, kern, args...) != cudaSuccess) {
        cudaGetLastError();
        return EXMOE_ERR_CUDA;
    }
    count_launch();
    return EXMOE_OK;
}

// Many tokens, at most 256 experts: the logits on tensor cores (gate_tc.cu).
int launch_gate_tc(const __nv_bfloat16* x, const __nv_bfloat16* w, const float* bias, const float* addend, int T, int H, const GateArgs& g, int32_t* ids,
                   float* weights, cudaStream_t st);
int launch_gate_tc_stuck(const __nv_bfloat16* x, const __nv_bfloat16* w, int T, int H, const GateArgs& g, int32_t* ids, float* weights, cudaStream_t st);

}  // namespace exmoe
