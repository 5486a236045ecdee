// Norms of queries and keys for each head with the rotation by position, packed or on the way into a paged cache, and their
// gradients (include/ttc_attention.h, ttc_heads_* and ttc_pages_append), for gfx950 (MI355X).
//
// A unit is two vectors of V elements, the two sides of V rotations: elements u*V of the first half of the rotated part and the same of the second, or
// neighbours; behind the rotated part simply the next two vectors.  A lane has the same unit of every head that it meets, so that its angles' sines and
// cosines are made once a token and its weights are loaded once a launch; no lane needs another's elements but for the sums over a head.
#include <type_traits>

#include "ttc_attention_internal.h"
#include "ttc_moves_device.h"
#include "ttc_records.h"

namespace ttc {
namespace {

// cos and sin of `turn` * 2^-64 turns: the nearest quarter turn by integers, exactly, then the two series on the rest, at most pi/4 away: their first
// terms left out are below 2^-29.
__device__ __forceinline__ void unit_circle(uint64_t turn, float* c, float* s)
{
    const uint32_t top = (uint32_t)(turn >> 32), quarter = (top + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(top - (quarter << 30)) * 1.46291807926715968e-9f;      // 2 pi / 2^32
    const float y = x * x;
    float sine = __builtin_fmaf(y, 2.75573192e-6f, -1.98412698e-4f);
    sine = __builtin_fmaf(y, sine, 8.33333333e-3f);
    sine = __builtin_fmaf(y, sine, -1.66666667e-1f);
    sine = __builtin_fmaf(x * y, sine, x);
    float cosine = __builtin_fmaf(y, -2.75573192e-7f, 2.48015873e-5f);
    cosine = __builtin_fmaf(y, cosine, -1.38888889e-3f);
    cosine = __builtin_fmaf(y, cosine, 4.16666667e-2f);
    cosine = __builtin_fmaf(y, cosine, -0.5f);
    cosine = __builtin_fmaf(y, cosine, 1.f);
    const float a = quarter & 1 ? sine : cosine, b = quarter & 1 ? cosine : sine;
    *c = (quarter + 1) & 2 ? -a : a;
    *s = quarter & 2 ? -b : b;
}

// Sum over the 2^log lanes that share a head.
__device__ __forceinline__ float over_head(float v, int log)
{
    for (int i = 0; i < log; ++i) v += __shfl_xor(v, 1 << i);
    return v;
}

struct Unit {
    uint32_t a, b;                         // its two vectors' first elements
    bool     has_a, has_b, turned;
};

template <int V> __device__ __forceinline__ Unit unit_of(const HeadsArgs& p, uint32_t u)
{
    const uint32_t half = p.rotated / 2;
    Unit r;
    if (p.paired) {
        r.a = 2 * V * u;
        r.b = r.a + V;
        r.turned = r.a < p.rotated;
    } else if (u * V < half) {
        r.a = u * V;
        r.b = half + u * V;
        r.turned = true;
    } else {
        r.a = p.rotated + 2 * (u * V - half);
        r.b = r.a + V;
        r.turned = false;
    }
    r.has_a = r.a < p.dim;
    r.has_b = r.b < p.dim;
    return r;
}

// A lane's units, with what it knows of them for a whole launch, and for a token.
template <int V, int N> struct Lane {
    Unit     unit[N];
    uint64_t turn[N][V];
    float    cosine[N][V], sine[N][V];
    __device__ __forceinline__ void start(const HeadsArgs& p, uint32_t lane)
    {
        // by the segment that the launch filled: indexed by lane, the parameter itself would be copied to memory first
        const __attribute__((address_space(4))) char* args = (const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr();
        const __attribute__((address_space(4))) uint64_t* turns = (const __attribute__((address_space(4))) uint64_t*)(args + offsetof(HeadsArgs, turns));
#pragma unroll
        for (int n = 0; n < N; ++n) {
            unit[n] = unit_of<V>(p, lane + ((uint32_t)n << p.lanes_log));
            // paired: pairs a/2 ...; else the pair is its first element
            const uint32_t first = p.paired ? unit[n].a / 2 : unit[n].a;
#pragma unroll
            for (int j = 0; j < V; ++j) turn[n][j] = unit[n].turned ? turns[first + j] : 0;
        }
    }
    __device__ __forceinline__ void token(uint32_t position)
    {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int j = 0; j < V; ++j) unit_circle(turn[n][j] * position, &cosine[n][j], &sine[n][j]);
    }
    // x[n] is unit n's 2 V elements; back: by the negative angle
    __device__ __forceinline__ void rotate(float (*x)[2 * V], int paired, bool back) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float c = cosine[n][j], s = back ? -sine[n][j] : sine[n][j];
                if (V > 1 && paired) {
                    const float a = x[n][2 * j], b = x[n][2 * j + 1];
                    x[n][2 * j] = __builtin_fmaf(a, c, -(b * s));
                    x[n][2 * j + 1] = __builtin_fmaf(b, c, a * s);
                } else {
                    const float a = x[n][j], b = x[n][V + j];
                    x[n][j] = __builtin_fmaf(a, c, -(b * s));
                    x[n][V + j] = __builtin_fmaf(b, c, a * s);
                }
            }
    }
};

template <typename T, int V> struct Raw { Vec<T, V> a, b; };

template <typename T, int V> __device__ __forceinline__ Raw<T, V> load_unit(const T* p, const Unit& u, bool here)
{
    Raw<T, V> r = {};
    if (here && u.has_a) r.a = load_vec<T, V, false>(p + u.a);
    if (here && u.has_b) r.b = load_vec<T, V, false>(p + u.b);
    return r;
}
template <typename T, int V> __device__ __forceinline__ void widen_unit(const Raw<T, V>& r, float* x)
{
    widen(r.a, x);
    widen(r.b, x + V);
}
template <typename T, int V> __device__ __forceinline__ void store_unit(T* p, const Unit& u, bool here, const float* x)
{
    Vec<T, V> r;
    if (here && u.has_a) { narrow(x, r); store_vec<T, V, false>(p + u.a, r); }
    if (here && u.has_b) { narrow(x + V, r); store_vec<T, V, false>(p + u.b, r); }
}

// A lane's share of the weights, 1 where there are none (and behind the end).
template <int V, int N> __device__ __forceinline__ void load_weights(const float* w, const Lane<V, N>& lane, float (*x)[2 * V])
{
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            x[n][j] = w && lane.unit[n].has_a ? w[lane.unit[n].a + j] : 1.f;
            x[n][V + j] = w && lane.unit[n].has_b ? w[lane.unit[n].b + j] : 1.f;
        }
}

struct Place {                             // of a wavefront's item
    uint32_t token, group, end;
    int32_t  position;
};
__device__ __forceinline__ Place place_of(const HeadsArgs& p, uint32_t item)
{
    Place r;
    r.token = fdiv(item, p.split_div);
    r.group = (item - r.token * p.split_div.div) * p.per_wave;
    const uint32_t all = p.q_groups + p.k_groups + p.v_groups;
    r.end = r.group + p.per_wave < all ? r.group + p.per_wave : all;
    r.position = p.positions ? p.positions[r.token] : 0;
    return r;
}

constexpr int kBatch = 4;                  // groups whose loads are under way together

// C: the cache's element type, or void for packed results.
template <typename C> struct Cached { static constexpr bool value = true; };
template <> struct Cached<void> { static constexpr bool value = false; };

// One head's vector into the cache.
template <typename T, typename C, int V, int N>
__device__ __forceinline__ void store_cached(void* cache, int64_t at, float scale, const Lane<V, N>& lane, bool here, float (*x)[2 * V], int lanes_log)
{
    if constexpr (std::is_same<C, q4>::value) {
        static_assert(N == 1 && V == 8, "words of eight codes");
        const Unit& u = lane.unit[0];
        RecordRange range;
        if (u.has_a) range.take(x[0], V);
        if (u.has_b) range.take(x[0] + V, V);
        const Record rec = range.record(lanes_log);
        uint8_t* to = static_cast<uint8_t*>(cache) + at;
        if (here) {
            if (u.a == 0) store_word(to, rec.head());
            if (u.has_a) store_word(to + kRecordHead + u.a / 2, rec.codes(x[0]));
            if (u.has_b) store_word(to + kRecordHead + u.b / 2, rec.codes(x[0] + V));
        }
    } else if constexpr (std::is_same<C, f8>::value) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const Unit& u = lane.unit[n];
            Vec<f8, V> r;
            f8* to = static_cast<f8*>(cache) + at;
            if (here && u.has_a) { narrow_scaled(x[n], scale, r); store_vec<f8, V, false>(to + u.a, r); }
            if (here && u.has_b) { narrow_scaled(x[n] + V, scale, r); store_vec<f8, V, false>(to + u.b, r); }
        }
    } else {
#pragma unroll
        for (int n = 0; n < N; ++n) store_unit<T, V>(static_cast<T*>(cache) + at, lane.unit[n], here, x[n]);
    }
}

template <typename T, typename C, int V, int N>
__global__ __launch_bounds__(kHeadsThreads) void heads_kernel(HeadsArgs p)
{
    const uint32_t wave = blockIdx.x * (kHeadsThreads / kWave) + threadIdx.x / kWave, waves = gridDim.x * (kHeadsThreads / kWave);
    const uint32_t in_head = threadIdx.x & ((1u << p.lanes_log) - 1), sub = (threadIdx.x & (kWave - 1)) >> p.lanes_log, each = kWave >> p.lanes_log;
    const uint32_t items = p.tokens * p.split_div.div;
    Lane<V, N> lane;
    lane.start(p, in_head);
    float weight[2][N][2 * V];
    if (p.norm) {
        load_weights<V, N>(p.q_weight, lane, weight[0]);
        load_weights<V, N>(p.k_weight, lane, weight[1]);
    }
    const float each_element = 1.f / (float)p.dim;
    for (uint32_t item = __builtin_amdgcn_readfirstlane(wave); item < items; item += waves) {
        const Place at = place_of(p, item);
        if (at.position < 0) continue;
        lane.token((uint32_t)at.position);
        uint32_t slot = 0;
        int64_t in_cache = 0;
        bool kept = true;
        if constexpr (Cached<C>::value) {
            slot = (uint32_t)p.slots[at.token];
            kept = slot < p.slot_count;
            const uint32_t page = kept ? fdiv(slot, p.page) : 0, inside = kept ? slot - page * p.page.div : 0;
            in_cache = (int64_t)page * p.stride_page + (int64_t)inside * p.stride_slot;
        }
        // queries, then keys, then values: the groups of a kind that are this wavefront's
        auto run = [&](auto kind_of, uint32_t first, uint32_t groups, const void* from, int64_t ld, uint32_t heads) {
            const uint32_t lo = at.group > first ? at.group - first : 0, hi = at.end > first ? (at.end - first < groups ? at.end - first : groups) : 0;
            constexpr int kind = decltype(kind_of)::value;
            const T* row = static_cast<const T*>(from) + (int64_t)at.token * ld;
            for (uint32_t g0 = lo; g0 < hi; g0 += kBatch) {
                Raw<T, V> raw[kBatch][N];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    const uint32_t head = (g0 + i) * each + sub;
                    const bool here = g0 + i < hi && head < heads;
#pragma unroll
                    for (int n = 0; n < N; ++n) raw[i][n] = load_unit<T, V>(row + (int64_t)head * p.dim, lane.unit[n], here);
                }
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    if (g0 + i >= hi) break;
                    const uint32_t head = (g0 + i) * each + sub;
                    const bool here = head < heads;
                    float x[N][2 * V];
#pragma unroll
                    for (int n = 0; n < N; ++n) widen_unit<T, V>(raw[i][n], x[n]);
                    if constexpr (kind < 2) {
                        if (p.norm) {
                            float sum = 0.f;
#pragma unroll
                            for (int n = 0; n < N; ++n)
#pragma unroll
                                for (int j = 0; j < 2 * V; ++j) sum = __builtin_fmaf(x[n][j], x[n][j], sum);
                            const float r = 1.f / __builtin_sqrtf(__builtin_fmaf(over_head(sum, p.lanes_log), each_element, p.eps));
#pragma unroll
                            for (int n = 0; n < N; ++n)
#pragma unroll
                                for (int j = 0; j < 2 * V; ++j) x[n][j] = x[n][j] * r * weight[kind][n][j];
                        }
                        lane.rotate(x, p.paired, false);
                    }
                    if constexpr (kind == 0 || !Cached<C>::value) {
                        T* to = static_cast<T*>(kind == 0 ? p.q_out : p.k_out) + (int64_t)at.token * (kind == 0 ? p.ld_qo : p.ld_ko) + (int64_t)head * p.dim;
#pragma unroll
                        for (int n = 0; n < N; ++n) store_unit<T, V>(to, lane.unit[n], here, x[n]);
                    } else {
                        const float* scales = kind == 1 ? p.k_scale : p.v_scale;
                        const float scale = std::is_same<C, f8>::value && scales && here ? scales[head] : 1.f;
                        store_cached<T, C, V, N>(kind == 1 ? p.k_out : p.v_out, in_cache + (int64_t)head * p.stride_head, scale, lane, here, x, p.lanes_log);
                    }
                }
            }
        };
        run(std::integral_constant<int, 0>{}, 0, p.q_groups, p.q, p.ld_q, p.q_heads);
        if (!kept) continue;
        run(std::integral_constant<int, 1>{}, p.q_groups, p.k_groups, p.k, p.ld_k, p.kv_heads);
        if constexpr (Cached<C>::value) run(std::integral_constant<int, 2>{}, p.q_groups + p.k_groups, p.v_groups, p.v, p.ld_v, p.kv_heads);
    }
}

// The backward pass.  The weights' gradients are summed by every lane over its tokens and heads, by a workgroup over its lanes that have the same
// elements, and over the workgroups by grad_sum_kernel, all in an order that the sizes alone give.
template <typename T, int V, int N>
__global__ __launch_bounds__(kHeadsThreads) void heads_grad_kernel(HeadsArgs p)
{
    constexpr int kWaves = kHeadsThreads / kWave;
    __shared__ float sums[kWaves][2][TTC_HEADS_MAX_DIM];
    const uint32_t wave = blockIdx.x * kWaves + threadIdx.x / kWave, waves = gridDim.x * kWaves;
    const uint32_t in_head = threadIdx.x & ((1u << p.lanes_log) - 1), sub = (threadIdx.x & (kWave - 1)) >> p.lanes_log, each = kWave >> p.lanes_log;
    const uint32_t items = p.tokens * p.split_div.div;
    Lane<V, N> lane;
    lane.start(p, in_head);
    float weight[2][N][2 * V], total[2][N][2 * V] = {};
    if (p.norm) {
        load_weights<V, N>(p.q_weight, lane, weight[0]);
        load_weights<V, N>(p.k_weight, lane, weight[1]);
    }
    const float each_element = 1.f / (float)p.dim;
    for (uint32_t item = __builtin_amdgcn_readfirstlane(wave); item < items; item += waves) {
        const Place at = place_of(p, item);
        if (at.position < 0) continue;
        lane.token((uint32_t)at.position);
        auto run = [&](auto kind_of, uint32_t first, uint32_t groups, const void* from, int64_t ld, const void* dfrom, int64_t ldd, void* out, int64_t ldo, uint32_t heads) {
            constexpr int kind = decltype(kind_of)::value;
            const uint32_t lo = at.group > first ? at.group - first : 0, hi = at.end > first ? (at.end - first < groups ? at.end - first : groups) : 0;
            const T* row = static_cast<const T*>(from) + (int64_t)at.token * ld;
            const T* drow = static_cast<const T*>(dfrom) + (int64_t)at.token * ldd;
            T* to = static_cast<T*>(out) + (int64_t)at.token * ldo;
            constexpr int kPairs = 2;
            for (uint32_t g0 = lo; g0 < hi; g0 += kPairs) {
                Raw<T, V> raw[kPairs][N], draw[kPairs][N];
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    const uint32_t head = (g0 + i) * each + sub;
                    const bool here = g0 + i < hi && head < heads;
#pragma unroll
                    for (int n = 0; n < N; ++n) {
                        draw[i][n] = load_unit<T, V>(drow + (int64_t)head * p.dim, lane.unit[n], here);
                        raw[i][n] = load_unit<T, V>(row + (int64_t)head * p.dim, lane.unit[n], here && p.norm);
                    }
                }
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    if (g0 + i >= hi) break;
                    const uint32_t head = (g0 + i) * each + sub;
                    const bool here = head < heads;
                    float x[N][2 * V], g[N][2 * V];
#pragma unroll
                    for (int n = 0; n < N; ++n) {
                        widen_unit<T, V>(draw[i][n], g[n]);
                        widen_unit<T, V>(raw[i][n], x[n]);
                    }
                    lane.rotate(g, p.paired, true);
                    if (p.norm) {
                        float square = 0.f, both = 0.f;
#pragma unroll
                        for (int n = 0; n < N; ++n)
#pragma unroll
                            for (int j = 0; j < 2 * V; ++j) {
                                square = __builtin_fmaf(x[n][j], x[n][j], square);
                                both = __builtin_fmaf(x[n][j] * weight[kind][n][j], g[n][j], both);
                            }
                        const float r = 1.f / __builtin_sqrtf(__builtin_fmaf(over_head(square, p.lanes_log), each_element, p.eps));
                        const float mean = over_head(both, p.lanes_log) * each_element * r;       // of g * x / s
#pragma unroll
                        for (int n = 0; n < N; ++n)
#pragma unroll
                            for (int j = 0; j < 2 * V; ++j) {
                                const float hat = x[n][j] * r;
                                total[kind][n][j] = __builtin_fmaf(hat, g[n][j], total[kind][n][j]);
                                g[n][j] = r * __builtin_fmaf(g[n][j], weight[kind][n][j], -(hat * mean));
                            }
                    }
#pragma unroll
                    for (int n = 0; n < N; ++n) store_unit<T, V>(to + (int64_t)head * p.dim, lane.unit[n], here, g[n]);
                }
            }
        };
        run(std::integral_constant<int, 0>{}, 0, p.q_groups, p.q, p.ld_q, p.dq_out, p.ld_dqo, p.q_out, p.ld_qo, p.q_heads);
        run(std::integral_constant<int, 1>{}, p.q_groups, p.k_groups, p.k, p.ld_k, p.dk_out, p.ld_dko, p.k_out, p.ld_ko, p.kv_heads);
    }
    if (!p.partial) return;
    const int mine = threadIdx.x / kWave;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind)
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) {
                float v = total[kind][n][j];
                for (int i = p.lanes_log; i < 6; ++i) v += __shfl_xor(v, 1 << i);
                const uint32_t column = j < V ? lane.unit[n].a + j : lane.unit[n].b + j - V;
                if (sub == 0 && (j < V ? lane.unit[n].has_a : lane.unit[n].has_b)) sums[mine][kind][column] = v;
            }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 2 * p.dim; i += kHeadsThreads) {
        const uint32_t kind = i >= p.dim, column = i - kind * p.dim;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += sums[w][kind][column];
        p.partial[(int64_t)blockIdx.x * 2 * p.dim + i] = v;
    }
}

struct SumArgs {
    const float* partial;
    float       *q, *k;
    uint32_t     rows, dim;
};
constexpr int kSumColumns = 16, kSumRows = 16;

__global__ __launch_bounds__(kSumColumns * kSumRows) void grad_sum_kernel(SumArgs p)
{
    __shared__ float sums[kSumRows][kSumColumns];
    const uint32_t c = threadIdx.x % kSumColumns, r = threadIdx.x / kSumColumns, i = blockIdx.x * kSumColumns + c;
    float v = 0.f;
    if (i < 2 * p.dim) {
#pragma unroll 8
        for (uint32_t j = r; j < p.rows; j += kSumRows) v += p.partial[(int64_t)j * 2 * p.dim + i];
    }
    sums[r][c] = v;
    __syncthreads();
    if (r != 0 || i >= 2 * p.dim) return;
    v = 0.f;
#pragma unroll
    for (int j = 0; j < kSumRows; ++j) v += sums[j][c];
    float* out = i < p.dim ? p.q : p.k;
    if (out) out[i < p.dim ? i : i - p.dim] = v;
}

template <typename T, typename C> const void* heads_fn(int vec)
{
    constexpr int V = std::is_same<C, q4>::value ? 8 : 16 / (int)sizeof(T);
    if (vec == V) return reinterpret_cast<const void*>(&heads_kernel<T, C, V, 1>);
    if constexpr (std::is_same<C, q4>::value) return nullptr;
    else return reinterpret_cast<const void*>(&heads_kernel<T, C, 1, 4>);
}
template <typename T> const void* heads_fn(int vec, int cache)
{
    return cache < 0 ? heads_fn<T, void>(vec) : cache == TTC_F8 ? heads_fn<T, f8>(vec) : cache == TTC_Q4 ? heads_fn<T, q4>(vec) : heads_fn<T, T>(vec);
}
template <typename T> const void* grad_fn(int vec)
{
    constexpr int V = 16 / (int)sizeof(T);
    return vec == V ? reinterpret_cast<const void*>(&heads_grad_kernel<T, V, 1>) : reinterpret_cast<const void*>(&heads_grad_kernel<T, 1, 4>);
}

}  // namespace

int launch_heads(const HeadsArgs& a, void* stream)
{
    HeadsArgs p = a;
    const HeadsShape s = cut_heads(p);
    const void* fn = p.dtype == TTC_F32 ? heads_fn<float>(s.vec, p.cache_dtype) : p.dtype == TTC_BF16 ? heads_fn<__bf16>(s.vec, p.cache_dtype)
                                        : heads_fn<_Float16>(s.vec, p.cache_dtype);
    return fn ? launch_blocks(fn, (uint64_t)s.groups, kHeadsThreads, 0, &p, stream) : TTC_ERR_INTERNAL;
}

int launch_heads_grad(const HeadsArgs& a, void* stream)
{
    HeadsArgs p = a;
    const HeadsShape s = cut_heads(p);
    if (p.tokens) {
        const void* fn = p.dtype == TTC_F32 ? grad_fn<float>(s.vec) : p.dtype == TTC_BF16 ? grad_fn<__bf16>(s.vec) : grad_fn<_Float16>(s.vec);
        const int st = launch_blocks(fn, (uint64_t)s.groups, kHeadsThreads, 0, &p, stream);
        if (st != TTC_OK) return st;
    }
    if (!p.dq_weight && !p.dk_weight) return TTC_OK;
    SumArgs q = {p.partial, p.dq_weight, p.dk_weight, p.tokens ? (uint32_t)s.groups : 0, p.dim};
    return launch_blocks(reinterpret_cast<const void*>(&grad_sum_kernel), (2 * p.dim + kSumColumns - 1) / kSumColumns, kSumColumns * kSumRows, 0, &q, stream);
}

}  // namespace ttc
