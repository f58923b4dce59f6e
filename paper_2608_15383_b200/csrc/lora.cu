// Low-rank adapters of many requests beside a shared projection: out_t = base_t + scale_a * B_a (A_a x_t), a the adapter of
// token t.  exmoe_lora_plan groups the tokens by adapter once per step, exmoe_lora runs one projection's adapters over the groups.
#include <algorithm>

#include "common.cuh"

namespace exmoe {

namespace {

constexpr int kMaxAdapters = 1024, kMaxRank = 128;
constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32;
constexpr int kLoraThreads = 256, kLoraWarps = kLoraThreads / 32;

// A plan: header, tiles, then the tokens grouped by adapter (ascending, those without one last; inside a group ascending tokens).
// A tile is a run of at most kTileRows rows of one group.
constexpr int kTileRows = 64;
constexpr int kPlanMagic = 0x4c6f5241;
enum { LP_MAGIC = 0, LP_TOKENS = 1, LP_ADAPTERS = 2, LP_TILES = 3, LP_STATUS = 4, LP_WORDS = 16 };
struct LoraTile { int adapter, row0, nrows, pad; };                        // adapter -1: none
__host__ __device__ inline int plan_tiles(int T, int n) {                  // most tiles of a plan
    const int groups = T < n + 1 ? T : n + 1;
    return T / kTileRows + groups;
}

__global__ void __launch_bounds__(kPlanThreads)
lora_plan_kernel(const int32_t* ids, int T, int n, int32_t* plan) {
    extern __shared__ int32_t sm[];
    int32_t* hist = sm;                                                    // [warp][n + 1]: this warp's tokens of a group, then those of the warps before it
    int32_t* count = hist + kPlanWarps * (n + 1);                          // [n + 1]
    int32_t* first = count + n + 1;                                        // [n + 1] first row of a group
    int32_t* tile0 = first + n + 1;                                        // [n + 1] its first tile
    __shared__ int bad;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned lt = (1u << lane) - 1u;
    LoraTile* tiles = reinterpret_cast<LoraTile*>(plan + LP_WORDS);
    int32_t* perm = plan + LP_WORDS + 4 * plan_tiles(T, n);
    for (int i = tid; i < kPlanWarps * (n + 1); i += kPlanThreads) hist[i] = 0;
    if (tid == 0) bad = 0;
    __syncthreads();
    const int per = ((T + kPlanWarps - 1) / kPlanWarps + 31) & ~31;
    const int t_begin = min(T, warp * per), t_end = min(T, t_begin + per);
    int32_t* mine = hist + warp * (n + 1);
    auto group_of = [&](int t) {
        if (t >= t_end) return n + 1;
        const int id = ids[t];
        return id >= 0 && id < n ? id : n;
    };
    for (int t0 = t_begin; t0 < t_end; t0 += 32) {
        const int b = group_of(t0 + lane);
        const unsigned same = __match_any_sync(0xffffffffu, b);
        if (b == n && ids[t0 + lane] != -1) bad = 1;
        if (b <= n && !(same & lt)) mine[b] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    for (int b = tid; b <= n; b += kPlanThreads) {
        int run = 0;
        for (int w = 0; w < kPlanWarps; ++w) {
            const int c = hist[w * (n + 1) + b];
            hist[w * (n + 1) + b] = run;
            run += c;
        }
        count[b] = run;
    }
    __syncthreads();
    if (warp == 0) {
        int rows = 0, nt = 0;
        for (int b0 = 0; b0 <= n; b0 += 32) {
            const int c = b0 + lane <= n ? count[b0 + lane] : 0, tl = (c + kTileRows - 1) / kTileRows;
            int ic = c, it = tl;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int oc = __shfl_up_sync(0xffffffffu, ic, d), ot = __shfl_up_sync(0xffffffffu, it, d);
                if (lane >= d) {
                    ic += oc;
                    it += ot;
                }
            }
            if (b0 + lane <= n) {
                first[b0 + lane] = rows + ic - c;
                tile0[b0 + lane] = nt + it - tl;
            }
            rows += __shfl_sync(0xffffffffu, ic, 31);
            nt += __shfl_sync(0xffffffffu, it, 31);
        }
        if (lane == 0) {
            plan[LP_MAGIC] = kPlanMagic;
            plan[LP_TOKENS] = T;
            plan[LP_ADAPTERS] = n;
            plan[LP_TILES] = nt;
            plan[LP_STATUS] = bad ? EXMOE_ERR_BAD_ADAPTER_ID : EXMOE_OK;
        }
    }
    __syncthreads();
    for (int b = tid; b <= n; b += kPlanThreads)
        for (int i = 0; i * kTileRows < count[b]; ++i)
            tiles[tile0[b] + i] = LoraTile{b < n ? b : -1, first[b] + i * kTileRows, min(kTileRows, count[b] - i * kTileRows), 0};
    for (int t0 = t_begin; t0 < t_end; t0 += 32) {
        const int b = group_of(t0 + lane);
        const unsigned same = __match_any_sync(0xffffffffu, b);
        if (b <= n) perm[first[b] + mine[b] + __popc(same & lt)] = t0 + lane;
        __syncwarp();
        if (b <= n && !(same & lt)) mine[b] += __popc(same);
        __syncwarp();
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
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void store(float* p, float v) { *p = v; }
__device__ __forceinline__ void store(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

// whether the plan is one for this call; a wrong one is reported and nothing else is done
__device__ __forceinline__ bool plan_fits(const LoraArgs& p) {
    if (p.plan[LP_MAGIC] == kPlanMagic && p.plan[LP_TOKENS] == p.T && p.plan[LP_ADAPTERS] == p.n) return true;
    if (blockIdx.x == 0 && threadIdx.x == 0) p.plan[LP_STATUS] = EXMOE_ERR_STATE;
    return false;
}

// One CTA per tile, row by row.
template <typename O>
__global__ void __launch_bounds__(kLoraThreads)
lora_tile_kernel(LoraArgs p) {
    __shared__ float v[kMaxRank];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (!plan_fits(p) || (int)blockIdx.x >= p.plan[LP_TILES]) return;
    const LoraTile tile = reinterpret_cast<const LoraTile*>(p.plan + LP_WORDS)[blockIdx.x];
    const int32_t* perm = p.plan + LP_WORDS + 4 * plan_tiles(p.T, p.n);
    for (int i = 0; i < tile.nrows; ++i) {
        const long long t = perm[tile.row0 + i];
        const O* base = p.base ? (const O*)p.base + t * p.ld_base : nullptr;
        O* out = (O*)p.out + t * p.ld_out;
        if (tile.adapter < 0) {
            for (int c = tid; c < p.N; c += kLoraThreads) out[c] = base ? base[c] : O(0.f);
            continue;
        }
        const __nv_bfloat16* x = p.x + t * p.ld_x;
        for (int j = warp; j < p.r; j += kLoraWarps) {
            const __nv_bfloat16* a = p.a + ((size_t)tile.adapter * p.r + j) * p.K;
            float s = 0.f;
            for (int k = lane; k < p.K; k += 32) s = fmaf(__bfloat162float(a[k]), __bfloat162float(x[k]), s);
#pragma unroll
            for (int m = 16; m >= 1; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
            if (lane == 0) v[j] = s;
        }
        __syncthreads();
        const float scale = p.scale[tile.adapter];
        for (int c = tid; c < p.N; c += kLoraThreads) {
            const __nv_bfloat16* b = p.b + ((size_t)tile.adapter * p.N + c) * p.r;
            float s = 0.f;
            for (int j = 0; j < p.r; ++j) s = fmaf(__bfloat162float(b[j]), v[j], s);
            store(out + c, fmaf(scale, s, base ? to_float(base[c]) : 0.f));
        }
        __syncthreads();
    }
}

int check_plan(int T, int n) {
    if (T < 0) return EXMOE_ERR_ARG;
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
    if ((!adapter_ids && T) || !plan || (reinterpret_cast<uintptr_t>(plan) & 15)) return EXMOE_ERR_ARG;
    const size_t smem = 4 * (size_t)(kPlanWarps + 3) * (num_adapters + 1);
    static SmemOnce once;
    if (!allow_smem(lora_plan_kernel, 4 * (kPlanWarps + 3) * (kMaxAdapters + 1), once)) return EXMOE_ERR_CUDA;
    lora_plan_kernel<<<1, kPlanThreads, smem, (cudaStream_t)stream>>>(adapter_ids, T, num_adapters, (int32_t*)plan);
    if (cudaGetLastError() != cudaSuccess) return EXMOE_ERR_CUDA;
    count_launch();
    return EXMOE_OK;
}

extern "C" int exmoe_lora_plan_status(const void* plan) {
    if (!plan) return EXMOE_ERR_ARG;
    int32_t head[LP_WORDS];
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(head, plan, sizeof head, cudaMemcpyDeviceToHost) != cudaSuccess) return EXMOE_ERR_CUDA;
    return head[LP_MAGIC] == kPlanMagic ? head[LP_STATUS] : EXMOE_ERR_STATE;
}

extern "C" int exmoe_lora(const exmoe_lora_shape* shape, void* plan, const void* x, int64_t ld_x, const void* a, const void* b,
                          const float* scale, int T, const void* base, int64_t ld_base, void* out, int64_t ld_out, int type,
                          void* stream) {
    if (!shape || T < 0 || (type != EXMOE_F32 && type != EXMOE_BF16)) return EXMOE_ERR_ARG;
    const int n = shape->num_adapters, K = shape->d_in, N = shape->d_out, r = shape->rank;
    if (n < 1 || n > kMaxAdapters || K <= 0 || K % 8 || N <= 0 || r <= 0 || r % 8 || r > kMaxRank) return EXMOE_ERR_SHAPE;
    if (T == 0) return EXMOE_OK;
    if (!plan || !x || !a || !b || !scale || !out) return EXMOE_ERR_ARG;
    if (ld_x < K || ld_x % 8 || ld_out < N || (base && ld_base < N)) return EXMOE_ERR_ARG;
    if ((reinterpret_cast<uintptr_t>(plan) | reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) & 15)
        return EXMOE_ERR_ARG;
    const long long es = type == EXMOE_F32 ? 4 : 2;
    auto range = [](const void* p, long long rows, long long ld, long long width, long long es) {
        return Range{reinterpret_cast<uintptr_t>(p), rows, ld * es, width * es};
    };
    size_t plan_size = 0;
    exmoe_lora_plan_bytes(T, n, &plan_size);
    const Range o = range(out, T, ld_out, N, es), bs = range(base, T, ld_base, N, es);
    if ((!(base == out && ld_base == ld_out) && overlap(o, bs)) || overlap(o, range(x, T, ld_x, K, 2)) || overlap(o, range(a, 1, 0, (long long)n * r * K, 2)) ||
        overlap(o, range(b, 1, 0, (long long)n * r * N, 2)) || overlap(o, range(scale, 1, 0, n, 4)) || overlap(o, range(plan, 1, 0, (long long)plan_size, 1)))
        return EXMOE_ERR_ARG;
    const LoraArgs args{(int32_t*)plan, (const __nv_bfloat16*)x, (const __nv_bfloat16*)a, (const __nv_bfloat16*)b, scale, base, out,
                        ld_x, ld_base, ld_out, T, n, K, N, r};
    const unsigned ctas = (unsigned)plan_tiles(T, n);
    if (type == EXMOE_F32)
        lora_tile_kernel<float><<<ctas, kLoraThreads, 0, (cudaStream_t)stream>>>(args);
    else
        lora_tile_kernel<__nv_bfloat16><<<ctas, kLoraThreads, 0, (cudaStream_t)stream>>>(args);
    if (cudaGetLastError() != cudaSuccess) return EXMOE_ERR_CUDA;
    count_launch();
    return EXMOE_OK;
}

}  // namespace exmoe
