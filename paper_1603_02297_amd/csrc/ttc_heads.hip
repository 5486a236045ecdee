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
constexpr float kTurn = 1.46291807926715968e-9f, kTurnLow = -4.070940268e-17f;      // 2 pi / 2^32, as two
__device__ __forceinline__ void unit_circle(uint64_t turn, float* c, float* s)
{
    const uint32_t top = (uint32_t)(turn >> 32), quarter = (top + 0x20000000u) >> 30;
    const int32_t rest = (int32_t)(top - (quarter << 30));
    const float f = (float)rest, x = f * kTurn;
    // what the two roundings left out of it
    const float less = __builtin_fmaf((float)(rest - (int32_t)f), kTurn, __builtin_fmaf(f, kTurnLow, __builtin_fmaf(f, kTurn, -x)));
    const float y = x * x;
    float sine = __builtin_fmaf(y, 2.75573192e-6f, -1.98412698e-4f);
    sine = __builtin_fmaf(y, sine, 8.33333333e-3f);
    sine = __builtin_fmaf(y, sine, -1.66666667e-1f);
    sine = __builtin_fmaf(x * y, sine, less) + x;
    float cosine = __builtin_fmaf(y, -2.75573192e-7f, 2.48015873e-5f);
    cosine = __builtin_fmaf(y, cosine, -1.38888889e-3f);
    cosine = __builtin_fmaf(y, cosine, 4.16666667e-2f);
    cosine = __builtin_fmaf(y, cosine, -0.5f);
    cosine = __builtin_fmaf(y, cosine, -(x * less)) + 1.f;
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
    uint32_t a, b;                         // its two vectors' first elements; where it has none, others of the head, which are loaded and not used
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
    r.a = r.has_a ? r.a : 0;
    r.b = r.has_b ? r.b : r.a;
    return r;
}

// What a workgroup keeps of the call: angles and weights (1 where there are none).
struct Kept {
    uint64_t turns[TTC_HEADS_MAX_ROTATED / 2];
    float    weights[2][TTC_HEADS_MAX_DIM];
    __device__ __forceinline__ void fill(const HeadsArgs& p)
    {
        // by the segment that the launch filled: indexed by lane, the parameter itself would be copied to memory first
        const __attribute__((address_space(4))) char* args = (const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr();
        const __attribute__((address_space(4))) uint64_t* from = (const __attribute__((address_space(4))) uint64_t*)(args + offsetof(HeadsArgs, turns));
        for (uint32_t i = threadIdx.x; i < p.rotated / 2; i += kHeadsThreads) turns[i] = from[i];
        if (p.norm)
            for (uint32_t i = threadIdx.x; i < p.dim; i += kHeadsThreads) {
                weights[0][i] = p.q_weight ? p.q_weight[i] : 1.f;
                weights[1][i] = p.k_weight ? p.k_weight[i] : 1.f;
            }
        __syncthreads();
    }
};

// A wavefront's accesses of LDS happen in order: only the compiler has to keep it.
__device__ __forceinline__ void wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// 1 / sqrt(x), to a unit; the instruction takes numbers below the normal range for 0.
__device__ __forceinline__ float inverse_root(float x)
{
    const bool tiny = x < 0x1p-64f;
    const float z = tiny ? x * 0x1p64f : x, r = __builtin_amdgcn_rsqf(z);
    const float better = __builtin_fmaf(r * 0.5f, __builtin_fmaf(-(z * r), r, 1.f), r);       // a step of Newton's
    return (z > 0.f && z < __builtin_inff() ? better : r) * (tiny ? 0x1p32f : 1.f);
}

// A lane's units, the same of every head, and their rotation at a token's position.
template <int V, int N> struct Lane {
    Unit  unit[N];
    float cosine[N][V], sine[N][V];
    __device__ __forceinline__ Lane(const HeadsArgs& p, uint32_t lane)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) unit[n] = unit_of<V>(p, lane + ((uint32_t)n << p.lanes_log));
    }
    // A wavefront's lanes make the rotations, one or two each, and exchange them by LDS: every lane by itself would make those of its units for each of the
    // heads that are under way at a time again, a fifth of all instructions.
    __device__ __forceinline__ void token(const HeadsArgs& p, const Kept& kept, float2* circle, uint32_t position)
    {
        wave_order();                       // the last token's have been read
        for (uint32_t i = threadIdx.x & (kWave - 1); i < p.rotated / 2; i += kWave) {
            float2 c;
            unit_circle(kept.turns[i] * position, &c.x, &c.y);
            circle[i] = c;
        }
        wave_order();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            // paired: pairs a/2 ...; else the pair is its first element
            const uint32_t first = unit[n].turned ? p.paired ? unit[n].a / 2 : unit[n].a : 0;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float2 c = circle[first + j];
                cosine[n][j] = unit[n].turned ? c.x : 1.f;
                sine[n][j] = unit[n].turned ? c.y : 0.f;
            }
        }
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
    __device__ __forceinline__ void weights(const float* kept, float (*w)[2 * V]) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                w[n][j] = kept[unit[n].a + j];
                w[n][V + j] = kept[unit[n].b + j];
            }
    }
};

// Loads go without conditions around them: under one, the compiler would wait for each before the next.  What lanes without an element of their own have
// loaded is made 0, where there are such lanes (!full).
template <typename T, int V> struct Raw { Vec<T, V> a, b; };

template <typename T, int V> __device__ __forceinline__ Raw<T, V> load_unit(const T* p, const Unit& u)
{
    return {load_vec<T, V, false>(p + u.a), load_vec<T, V, false>(p + u.b)};
}
template <typename T, int V> __device__ __forceinline__ void widen_unit(const Raw<T, V>& r, const Unit& u, bool full, bool here, float* x)
{
    widen(r.a, x);
    widen(r.b, x + V);
    if (!full) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            x[j] = here && u.has_a ? x[j] : 0.f;
            x[V + j] = here && u.has_b ? x[V + j] : 0.f;
        }
    }
}
template <bool NT, typename T, int V> __device__ __forceinline__ void store_unit(T* p, const Unit& u, bool here, const float* x)
{
    Vec<T, V> a, b;
    narrow(x, a);
    narrow(x + V, b);
    if (here && u.has_a) store_vec<T, V, NT>(p + u.a, a);
    if (here && u.has_b) store_vec<T, V, NT>(p + u.b, b);
}

// What one lane reads for all of them, by a scalar load: it does not wait for the vector loads and stores under way.
__device__ __forceinline__ int32_t scalar(const int32_t* p, uint32_t i) { return ((const __attribute__((address_space(4))) int32_t*)p)[i]; }

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
    r.position = p.positions ? scalar(p.positions, r.token) : 0;
    return r;
}

// The way of a wavefront over its items, group by group.
struct Step {
    uint32_t item, group;
    Place    at;
    bool     first;                        // of its item: the angles are another token's
};
__device__ __forceinline__ void settle(const HeadsArgs& p, uint32_t items, uint32_t waves, Step& s)        // on the first item from s.item on that is no padding
{
    for (; s.item < items; s.item += waves) {
        const Place at = place_of(p, s.item);
        if (at.position < 0) continue;
        s.at = at;
        s.group = at.group;
        s.first = true;
        break;
    }
}
__device__ __forceinline__ Step after(const HeadsArgs& p, uint32_t items, uint32_t waves, Step s)          // behind the last one: that one again, and no item
{
    if (s.item >= items) return s;
    s.first = false;
    if (s.group + 1 < s.at.end) ++s.group;
    else {
        s.item += waves;
        settle(p, items, waves, s);
    }
    return s;
}

// Groups whose loads are under way together: a token's, as a rule.
constexpr int kBatch = 4, kGradBatch = 2;
__device__ const float kOne = 1.f;

// C: the cache's element type, or void for packed results.
template <typename C> struct Cached { static constexpr bool value = true; };
template <> struct Cached<void> { static constexpr bool value = false; };

// One head's vector into the cache.
template <typename T, typename C, int V, int N, bool NT>
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
            if (here && u.has_a) { narrow_scaled(x[n], scale, r); store_vec<f8, V, NT>(to + u.a, r); }
            if (here && u.has_b) { narrow_scaled(x[n] + V, scale, r); store_vec<f8, V, NT>(to + u.b, r); }
        }
    } else {
#pragma unroll
        for (int n = 0; n < N; ++n) store_unit<NT, T, V>(static_cast<T*>(cache) + at, lane.unit[n], here, x[n]);
    }
}

// Bound by memory: 16384 tokens of 32 + 8 heads of 128 bf16 (336 MB) 66 us a call, 5.1 TB/s (55 where half of it is in the last-level
// cache); 21300 tokens into 8 bits, queries packed beside them (480 MB), 95.  Into
// 4 bits a vector's extremes and codes take the time: 6900 tokens of 28 + 4 heads of 64 17 us, where the bytes take 9.  A decoding step (64 to 128 tokens) is 4.4 to 4.6 us of latency.
template <typename T, typename C, int V, int N, bool NT>
__global__ __launch_bounds__(kHeadsThreads, 4) void heads_kernel(HeadsArgs p)
{
    __shared__ Kept kept;
    __shared__ float2 circle[kHeadsThreads / kWave][TTC_HEADS_MAX_ROTATED / 2];
    constexpr int kLoads = N == 1 ? kBatch : 2;
    const uint32_t wave = blockIdx.x * (kHeadsThreads / kWave) + threadIdx.x / kWave, waves = gridDim.x * (kHeadsThreads / kWave);
    const uint32_t in_head = threadIdx.x & ((1u << p.lanes_log) - 1), sub = (threadIdx.x & (kWave - 1)) >> p.lanes_log, each = kWave >> p.lanes_log;
    const uint32_t items = p.tokens * p.split_div.div, q_end = p.q_groups, k_end = q_end + p.k_groups;
    Lane<V, N> lane(p, in_head);
    const float each_element = 1.f / (float)p.dim;
    Raw<T, V> raw[kLoads][N];
    float scale_of[kLoads];                // beside them: a load between stores waits for those
    // groups g0 ... of an item
    auto load = [&](const Place& at, uint32_t g0) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint32_t g = g0 + i;
            if (g >= at.end) break;
            const bool q = g < q_end, k = g < k_end;
            const T* row = static_cast<const T*>(q ? p.q : k ? p.k : p.v) + (int64_t)at.token * (q ? p.ld_q : k ? p.ld_k : p.ld_v);
            const uint32_t head = (q ? g : k ? g - q_end : g - k_end) * each + sub, last = (q ? p.q_heads : p.kv_heads) - 1;
#pragma unroll
            for (int n = 0; n < N; ++n) raw[i][n] = load_unit<T, V>(row + (int64_t)(head < last ? head : last) * p.dim, lane.unit[n]);
            if constexpr (std::is_same<C, f8>::value) {
                const float* scales = q ? nullptr : k ? p.k_scale : p.v_scale;
                scale_of[i] = *(scales ? scales + (head < last ? head : last) : &kOne);
            }
        }
    };
    kept.fill(p);
    for (uint32_t item = __builtin_amdgcn_readfirstlane(wave); item < items; item += waves) {
        const Place at = place_of(p, item);
        if (at.position < 0) continue;
        load(at, at.group);
        int64_t in_cache = 0;
        bool slotted = true;
        if constexpr (Cached<C>::value) {
            const uint32_t slot = (uint32_t)scalar(p.slots, at.token);
            slotted = slot < p.slot_count;
            const uint32_t page = slotted ? fdiv(slot, p.page) : 0, inside = slotted ? slot - page * p.page.div : 0;
            in_cache = (int64_t)page * p.stride_page + (int64_t)inside * p.stride_slot;
        }
        lane.token(p, kept, circle[threadIdx.x / kWave], (uint32_t)at.position);
        // queries, then keys, then values
        const uint32_t end = slotted ? at.end : at.end < q_end ? at.end : q_end;
        for (uint32_t g0 = at.group; g0 < end; g0 += kLoads) {
            if (g0 != at.group) load(at, g0);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const uint32_t g = g0 + i;
                if (g >= end) break;
                auto run = [&](auto kind_of) {
                    constexpr int kind = decltype(kind_of)::value;
                    const uint32_t head = (kind == 0 ? g : kind == 1 ? g - q_end : g - k_end) * each + sub;
                    const bool here = head < (kind == 0 ? p.q_heads : p.kv_heads);
                    float x[N][2 * V];
#pragma unroll
                    for (int n = 0; n < N; ++n) widen_unit<T, V>(raw[i][n], lane.unit[n], p.full, here, x[n]);
                    if constexpr (kind < 2) {
                        if (p.norm) {
                            float w[N][2 * V], sum = 0.f;
                            lane.weights(kept.weights[kind], w);
#pragma unroll
                            for (int n = 0; n < N; ++n)
#pragma unroll
                                for (int j = 0; j < 2 * V; ++j) sum = __builtin_fmaf(x[n][j], x[n][j], sum);
                            const float r = inverse_root(__builtin_fmaf(over_head(sum, p.lanes_log), each_element, p.eps));
#pragma unroll
                            for (int n = 0; n < N; ++n)
#pragma unroll
                                for (int j = 0; j < 2 * V; ++j) x[n][j] = x[n][j] * r * w[n][j];
                        }
                        lane.rotate(x, p.paired, false);
                    }
                    if constexpr (kind == 0 || !Cached<C>::value) {
                        T* to = static_cast<T*>(kind == 0 ? p.q_out : p.k_out) + (int64_t)at.token * (kind == 0 ? p.ld_qo : p.ld_ko) + (int64_t)head * p.dim;
#pragma unroll
                        for (int n = 0; n < N; ++n) store_unit<NT, T, V>(to, lane.unit[n], here, x[n]);
                    } else {
                        const float scale = std::is_same<C, f8>::value ? scale_of[i] : 1.f;
                        store_cached<T, C, V, N, NT>(kind == 1 ? p.k_out : p.v_out, in_cache + (int64_t)head * p.stride_head, scale, lane, here, x, p.lanes_log);
                    }
                };
                if (g < q_end) run(std::integral_constant<int, 0>{});
                else if (!Cached<C>::value || g < k_end) run(std::integral_constant<int, 1>{});
                else if constexpr (Cached<C>::value) run(std::integral_constant<int, 2>{});
            }
        }
    }
}

// The backward pass.  The weights' gradients are summed by every lane over its tokens and heads, by a workgroup over its lanes that have the same
// elements, and over the workgroups by grad_sum_kernel, all in an order that the sizes alone give.  Bound by memory: 8192 tokens of 32 + 8 heads of 128 bf16 (252 MB)
// 59 us a call, of which the sums over the workgroups are 5.  A group's place is loaded again as soon as it has been widened, before anything is stored: loads
// of two groups once those before are stored take 62.8.  (Forward, where more is under way, the same takes 67 for 66 us, and 101 for 96 into 8 bits.)
template <typename T, int V, int N, bool NT>
__global__ __launch_bounds__(kHeadsThreads, 2) void heads_grad_kernel(HeadsArgs p)
{
    constexpr int kWaves = kHeadsThreads / kWave, kLoads = N == 1 ? kGradBatch : 1;
    __shared__ Kept kept;
    __shared__ float2 circle[kHeadsThreads / kWave][TTC_HEADS_MAX_ROTATED / 2];
    __shared__ float sums[kWaves][2][TTC_HEADS_MAX_DIM];
    const uint32_t wave = blockIdx.x * kWaves + threadIdx.x / kWave, waves = gridDim.x * kWaves;
    const uint32_t in_head = threadIdx.x & ((1u << p.lanes_log) - 1), sub = (threadIdx.x & (kWave - 1)) >> p.lanes_log, each = kWave >> p.lanes_log;
    const uint32_t items = p.tokens * p.split_div.div, q_end = p.q_groups;
    Lane<V, N> lane(p, in_head);
    float total[2][N][2 * V] = {};
    const float each_element = 1.f / (float)p.dim;
    Raw<T, V> raw[kLoads][N], draw[kLoads][N];
    auto load = [&](int i, const Step& s) {
        const bool q = s.group < q_end;
        const T* row = static_cast<const T*>(q ? p.q : p.k) + (int64_t)s.at.token * (q ? p.ld_q : p.ld_k);
        const T* drow = static_cast<const T*>(q ? p.dq_out : p.dk_out) + (int64_t)s.at.token * (q ? p.ld_dqo : p.ld_dko);
        const uint32_t head = (q ? s.group : s.group - q_end) * each + sub, last = (q ? p.q_heads : p.kv_heads) - 1;
        const int64_t from = (int64_t)(head < last ? head : last) * p.dim;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            draw[i][n] = load_unit<T, V>(drow + from, lane.unit[n]);
            raw[i][n] = load_unit<T, V>(row + from, lane.unit[n]);       // without a norm: the gradients again
        }
    };
    kept.fill(p);
    Step step[kLoads];
    step[0].item = __builtin_amdgcn_readfirstlane(wave);
    settle(p, items, waves, step[0]);
    bool more = step[0].item < items;
    if (more) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            if (i) step[i] = after(p, items, waves, step[i - 1]);
            load(i, step[i]);
        }
    }
    while (more) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const Step now = step[i];
            if (now.item >= items) { more = false; break; }
            if (now.first) lane.token(p, kept, circle[threadIdx.x / kWave], (uint32_t)now.at.position);
            const uint32_t g = now.group, head = (g < q_end ? g : g - q_end) * each + sub;
            const bool here = head < (g < q_end ? p.q_heads : p.kv_heads);
            float x[N][2 * V], d[N][2 * V];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                widen_unit<T, V>(draw[i][n], lane.unit[n], p.full, here, d[n]);
                widen_unit<T, V>(raw[i][n], lane.unit[n], p.full, here, x[n]);
            }
            step[i] = after(p, items, waves, step[(i + kLoads - 1) % kLoads]);
            load(i, step[i]);
            auto run = [&](auto kind_of) {
                constexpr int kind = decltype(kind_of)::value;
                lane.rotate(d, p.paired, true);
                if (p.norm) {
                    float w[N][2 * V], square = 0.f, both = 0.f;
                    lane.weights(kept.weights[kind], w);
#pragma unroll
                    for (int n = 0; n < N; ++n)
#pragma unroll
                        for (int j = 0; j < 2 * V; ++j) {
                            square = __builtin_fmaf(x[n][j], x[n][j], square);
                            both = __builtin_fmaf(x[n][j] * w[n][j], d[n][j], both);
                        }
                    // a lane without a head has zeros, whose root is that of eps alone: without one it is infinite, and would be in the sums
                    const float root = inverse_root(__builtin_fmaf(over_head(square, p.lanes_log), each_element, p.eps)), r = here ? root : 0.f;
                    const float mean = over_head(both, p.lanes_log) * each_element * r;       // of g * x / s
#pragma unroll
                    for (int n = 0; n < N; ++n)
#pragma unroll
                        for (int j = 0; j < 2 * V; ++j) {
                            const float hat = x[n][j] * r;
                            total[kind][n][j] = __builtin_fmaf(hat, d[n][j], total[kind][n][j]);
                            d[n][j] = r * __builtin_fmaf(d[n][j], w[n][j], -(hat * mean));
                        }
                }
                T* to = static_cast<T*>(kind == 0 ? p.q_out : p.k_out) + (int64_t)now.at.token * (kind == 0 ? p.ld_qo : p.ld_ko) + (int64_t)head * p.dim;
#pragma unroll
                for (int n = 0; n < N; ++n) store_unit<NT, T, V>(to, lane.unit[n], here, d[n]);
            };
            if (g < q_end) run(std::integral_constant<int, 0>{});
            else run(std::integral_constant<int, 1>{});
        }
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
    __shared__ double sums[kSumRows][kSumColumns];
    const uint32_t c = threadIdx.x % kSumColumns, r = threadIdx.x / kSumColumns, i = blockIdx.x * kSumColumns + c;
    double v = 0.0;                          // 512 sums of much the same size: their roundings would be most of the error
    if (i < 2 * p.dim) {
#pragma unroll 8
        for (uint32_t j = r; j < p.rows; j += kSumRows) v += p.partial[(int64_t)j * 2 * p.dim + i];
    }
    sums[r][c] = v;
    __syncthreads();
    if (r != 0 || i >= 2 * p.dim) return;
    v = 0.0;
#pragma unroll
    for (int j = 0; j < kSumRows; ++j) v += sums[j][c];
    float* out = i < p.dim ? p.q : p.k;
    if (out) out[i < p.dim ? i : i - p.dim] = (float)v;
}

template <typename T, typename C> const void* heads_fn(int vec, bool nt)
{
    constexpr int V = std::is_same<C, q4>::value ? 8 : 16 / (int)sizeof(T);
    if (vec == V) return nt ? reinterpret_cast<const void*>(&heads_kernel<T, C, V, 1, true>) : reinterpret_cast<const void*>(&heads_kernel<T, C, V, 1, false>);
    if constexpr (std::is_same<C, q4>::value) return nullptr;
    else return reinterpret_cast<const void*>(&heads_kernel<T, C, 1, kHeadsRounds, false>);
}
template <typename T> const void* heads_fn(int vec, int cache, bool nt)
{
    return cache < 0 ? heads_fn<T, void>(vec, nt) : cache == TTC_F8 ? heads_fn<T, f8>(vec, nt) : cache == TTC_Q4 ? heads_fn<T, q4>(vec, nt) : heads_fn<T, T>(vec, nt);
}
template <typename T> const void* grad_fn(int vec, bool nt)
{
    constexpr int V = 16 / (int)sizeof(T);
    return vec != V ? reinterpret_cast<const void*>(&heads_grad_kernel<T, 1, kHeadsRounds, false>) : nt ? reinterpret_cast<const void*>(&heads_grad_kernel<T, V, 1, true>)
                                                                                            : reinterpret_cast<const void*>(&heads_grad_kernel<T, V, 1, false>);
}

// Results of this many bytes are stored with the non-temporal hint.
constexpr int64_t kStreamResults = int64_t(16) << 20;
bool streams(const HeadsArgs& p)
{
    return (int64_t)p.tokens * ((p.q ? p.q_heads : 0) + (p.k ? p.kv_heads : 0)) * p.dim * elem_bytes(p.dtype) >= kStreamResults;
}

}  // namespace

int launch_heads(const HeadsArgs& a, void* stream)
{
    HeadsArgs p = a;
    const HeadsShape s = cut_heads(p, kHeadsGroups);
    const bool nt = streams(p);
    const void* fn = p.dtype == TTC_F32 ? heads_fn<float>(s.vec, p.cache_dtype, nt) : p.dtype == TTC_BF16 ? heads_fn<__bf16>(s.vec, p.cache_dtype, nt)
                                        : heads_fn<_Float16>(s.vec, p.cache_dtype, nt);
    return fn ? launch_blocks(fn, (uint64_t)s.groups, kHeadsThreads, 0, &p, stream) : TTC_ERR_INTERNAL;
}

int launch_heads_grad(const HeadsArgs& a, void* stream)
{
    HeadsArgs p = a;
    const HeadsShape s = cut_heads(p, kGradGroups);
    const bool nt = streams(p);
    if (p.tokens) {
        const void* fn = p.dtype == TTC_F32 ? grad_fn<float>(s.vec, nt) : p.dtype == TTC_BF16 ? grad_fn<__bf16>(s.vec, nt) : grad_fn<_Float16>(s.vec, nt);
        const int st = launch_blocks(fn, (uint64_t)s.groups, kHeadsThreads, 0, &p, stream);
        if (st != TTC_OK) return st;
    }
    if (!p.dq_weight && !p.dk_weight) return TTC_OK;
    SumArgs q = {p.partial, p.dq_weight, p.dk_weight, p.tokens ? (uint32_t)s.groups : 0, p.dim};
    return launch_blocks(reinterpret_cast<const void*>(&grad_sum_kernel), (2 * p.dim + kSumColumns - 1) / kSumColumns, kSumColumns * kSumRows, 0, &q, stream);
}

}  // namespace ttc
