// Rows sorted by expert, and back (include/ttc_moves.h, ttc_route_*), for gfx950 (MI355X).
//
// The sort is a stable counting sort of the assignments by expert.  A wavefront ranks 64 assignments at a time: one
// ballot per bit of the expert's number leaves every lane with the lanes that chose the same expert, the lanes before
// it among those are its rank, and a counter per wavefront and expert in LDS carries on to the next 64.  No atomics on
// what is returned: the order is the assignments' own, on every run.
//
// The moves walk over tokens, not over sorted rows: a token's row is read once and written topk times (gather), topk
// rows are read and one is written (combine), and the gradient does both in one pass, dy's vector being in registers
// when the dot product with the expert's row wants it.  All are bound by memory.
#include "ttc_moves_device.h"

namespace ttc {

// ---------------------------------------------------------------------------------
// The sort
// ---------------------------------------------------------------------------------
namespace {

// expert of assignment a, or `experts` for nowhere
__device__ __forceinline__ uint32_t expert_of(const SortArgs& p, uint32_t a)
{
    const uint32_t t = fdiv(a, p.topk_div), k = a - t * (uint32_t)p.topk;
    const int64_t at = (int64_t)t * p.ld_ids + k;
    const int64_t id = p.id_bytes == 8 ? static_cast<const int64_t*>(p.ids)[at] : (int64_t)static_cast<const int32_t*>(p.ids)[at];
    const uint64_t e = (uint64_t)id - (uint64_t)p.first;
    return e < (uint64_t)p.experts ? (uint32_t)e : (uint32_t)p.experts;
}

// Sum of v over the threads before this one; *all is the sum over all.  `part` holds a value per wavefront.
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t* part, uint32_t* all)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
    auto add = [](uint32_t a, uint32_t b) { return a + b; };
    const uint32_t s = over_lanes(v, add);
    if (lane == kWave - 1) part[wave] = s;
    __syncthreads();
    const uint32_t w = over_lanes(lane < waves ? part[lane] : 0, add);         // the wavefronts' sums, summed by every wavefront for itself
    *all = __shfl(w, waves - 1);
    const uint32_t before = __shfl(w, wave > 0 ? wave - 1 : 0);
    return (wave > 0 ? before : 0) + s - v;
}

__device__ __forceinline__ uint32_t padded(uint32_t count, uint32_t align) { return (count + align - 1) / align * align; }

constexpr int kExpertBits = 11;            // TTC_ROUTE_MAX_EXPERTS itself (nowhere) takes them all
static_assert((TTC_ROUTE_MAX_EXPERTS >> kExpertBits) == 0, "every expert and nowhere have a number of kExpertBits bits");

// A workgroup's chunk: every assignment's rank among those of its expert in the chunk, and the experts' counts.
// ALONE: the chunk is all there is, and the result is finished here.  Otherwise ranks are left in `position` and counts
// in `hist` for place_kernel.
// LDS: one word per wavefront, the experts' first rows, counters [waves][experts] (16 bits: a chunk holds at most 8192 ids).
template <int B, bool ALONE>
__global__ __launch_bounds__(kSortThreads) void sort_kernel(SortArgs p)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const int waves = blockDim.x / kWave, wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
    const int experts = p.experts;
    uint32_t* part = reinterpret_cast<uint32_t*>(lds);
    uint32_t* row = part + kSortThreads / kWave;
    volatile uint16_t* counter = reinterpret_cast<volatile uint16_t*>(row + experts);
    const uint32_t chunk = blockIdx.x;
    uint32_t e[B], rank[B];
    const uint64_t start = ((uint64_t)chunk * waves + wave) * (B * kWave) + lane;
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const uint64_t a = start + b * kWave;
        e[b] = a < p.n ? expert_of(p, (uint32_t)a) : (uint32_t)experts;
    }
    for (int i = threadIdx.x; i < waves * experts; i += blockDim.x) counter[i] = 0;
    if (p.source)                           // -1 everywhere; the rows that hold an assignment are written after it
        for (uint64_t i = (uint64_t)chunk * blockDim.x + threadIdx.x; i < p.rows; i += (uint64_t)gridDim.x * blockDim.x) p.source[i] = -1;
    __syncthreads();
    volatile uint16_t* mine = counter + wave * experts;
    const int bits = 32 - __clz(experts);   // experts itself (nowhere) has to be told apart, too
#pragma unroll
    for (int b = 0; b < B; ++b) {
        uint64_t same = ~uint64_t(0);
#pragma unroll
        for (int i = 0; i < kExpertBits; ++i) {
            if (i >= bits) continue;
            const bool set = (e[b] >> i) & 1;
            const uint64_t with = __ballot(set);
            same &= set ? with : ~with;
        }
        const uint32_t before = (uint32_t)__popcll(same & ((uint64_t(1) << lane) - 1));
        rank[b] = 0;
        if (e[b] < (uint32_t)experts) {
            const uint32_t base = mine[e[b]];
            rank[b] = base + before;
            __builtin_amdgcn_wave_barrier();
            if (before == 0) mine[e[b]] = (uint16_t)(base + (uint32_t)__popcll(same));
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    // one thread per expert: its counters become sums over the wavefronts before
    uint32_t total = 0;
    if ((int)threadIdx.x < experts) {
        uint16_t* column = const_cast<uint16_t*>(counter) + threadIdx.x;
        uint32_t held[kSortThreads / kWave];
#pragma unroll
        for (int w = 0; w < kSortThreads / kWave; ++w) held[w] = w < waves ? column[w * experts] : 0;
#pragma unroll
        for (int w = 0; w < kSortThreads / kWave; ++w) {
            if (w < waves) column[w * experts] = (uint16_t)total;
            total += held[w];
        }
    }
    if (ALONE) {
        uint32_t all;
        const uint32_t first = sum_before(padded(total, (uint32_t)p.align), part, &all);
        if ((int)threadIdx.x < experts) {
            row[threadIdx.x] = first;
            p.offsets[threadIdx.x] = (int32_t)first;
            p.counts[threadIdx.x] = (int32_t)total;
        }
        if (threadIdx.x == 0) p.offsets[experts] = (int32_t)all;
    } else if ((int)threadIdx.x < experts) {
        p.hist[(int64_t)chunk * experts + threadIdx.x] = (int32_t)total;
    }
    __syncthreads();
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const uint64_t a = start + b * kWave;
        if (a >= p.n) continue;
        const bool here = e[b] < (uint32_t)experts;
        uint32_t at = 0;
        if (here) at = rank[b] + mine[e[b]] + (ALONE ? row[e[b]] : 0u);
        p.position[a] = here ? (int32_t)at : -1;
        if (ALONE && here && p.source) p.source[at] = (int32_t)a;
    }
}

// Counts of the chunks before, per expert, in place; totals behind the last chunk.  Only where sort_adds() says no:
// 64 experts a workgroup, the chunks in as many ranges as it has wavefronts.
__global__ __launch_bounds__(kSortThreads) void sum_kernel(int32_t* hist, int64_t chunks, int experts)
{
    __shared__ int32_t range_sum[kSortThreads / kWave][kWave];
    const int e = blockIdx.x * kWave + (threadIdx.x & (kWave - 1)), range = threadIdx.x / kWave, ranges = kSortThreads / kWave;
    const int64_t each = (chunks + ranges - 1) / ranges, lo = range * each, hi = lo + each < chunks ? lo + each : chunks;
    int32_t s = 0;
    if (e < experts)
        for (int64_t g = lo; g < hi; ++g) s += hist[g * experts + e];
    range_sum[range][threadIdx.x & (kWave - 1)] = s;
    __syncthreads();
    if (e >= experts) return;
    int32_t before = 0;
    for (int r = 0; r < range; ++r) before += range_sum[r][threadIdx.x & (kWave - 1)];
    for (int64_t g = lo; g < hi; ++g) {
        const int32_t c = hist[g * experts + e];
        hist[g * experts + e] = before;
        before += c;
    }
    if (range == ranges - 1) hist[chunks * experts + e] = before;
}

// Ranks within a chunk become rows.  SUMMED: sum_kernel has been over the counts; otherwise every workgroup adds up
// those of the other chunks by itself (up to 256 KB out of L2), which saves a launch.
template <int B, bool SUMMED>
__global__ __launch_bounds__(kSortThreads) void place_kernel(SortArgs p, int32_t chunks)
{
    extern __shared__ __align__(16) unsigned char lds[];
    uint32_t* part = reinterpret_cast<uint32_t*>(lds);
    uint32_t* row = part + kSortThreads / kWave;
    uint32_t* sums = row + p.experts;       // totals; only where not SUMMED
    const int experts = p.experts, chunk = blockIdx.x;
    // what the last step needs, on its way while the counts are added up
    uint32_t expert[B], rank[B];
    const uint64_t start = ((uint64_t)chunk * B) * blockDim.x + threadIdx.x;
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const uint64_t a = start + (uint64_t)b * blockDim.x;
        expert[b] = a < p.n ? expert_of(p, (uint32_t)a) : (uint32_t)experts;
        rank[b] = a < p.n ? (uint32_t)p.position[a] : 0;
    }
    uint32_t total = 0, before = 0;
    if (SUMMED) {
        if ((int)threadIdx.x < experts) {
            total = (uint32_t)p.hist[(int64_t)chunks * experts + threadIdx.x];
            before = (uint32_t)p.hist[(int64_t)chunk * experts + threadIdx.x];
        }
    } else {
        for (int i = threadIdx.x; i < experts; i += blockDim.x) row[i] = sums[i] = 0;
        __syncthreads();
        int log = 0;
        while ((1 << log) < experts) ++log;
        const int e = threadIdx.x & ((1 << log) - 1), lanes = (int)blockDim.x >> log;
        if (e < experts) {
            uint32_t t = 0, b = 0;
#pragma unroll 8
            for (int g = threadIdx.x >> log; g < chunks; g += lanes) {
                const uint32_t c = (uint32_t)p.hist[(int64_t)g * experts + e];
                t += c;
                b += g < chunk ? c : 0;
            }
            atomicAdd(&sums[e], t);          // whole numbers: the order does not matter
            atomicAdd(&row[e], b);
        }
        __syncthreads();
        if ((int)threadIdx.x < experts) {
            total = sums[threadIdx.x];
            before = row[threadIdx.x];
        }
    }
    uint32_t all;
    const uint32_t first = sum_before(padded(total, (uint32_t)p.align), part, &all);
    if ((int)threadIdx.x < experts) {
        row[threadIdx.x] = first + before;
        if (chunk == 0) {
            p.offsets[threadIdx.x] = (int32_t)first;
            p.counts[threadIdx.x] = (int32_t)total;
        }
    }
    if (chunk == 0 && threadIdx.x == 0) p.offsets[experts] = (int32_t)all;
    __syncthreads();
#pragma unroll
    for (int b = 0; b < B; ++b) {
        if (expert[b] >= (uint32_t)experts) continue;               // its position is -1 already
        const uint64_t a = start + (uint64_t)b * blockDim.x;
        const uint32_t at = rank[b] + row[expert[b]];
        p.position[a] = (int32_t)at;
        if (p.source) p.source[at] = (int32_t)a;
    }
}

template <int B> int launch_sort_blocks(const SortArgs& p, const SortShape& s, void* stream)
{
    const size_t head = sizeof(uint32_t) * (size_t)(kSortThreads / kWave + p.experts);
    const size_t lds = head + sizeof(uint16_t) * (size_t)(s.threads / kWave) * (size_t)p.experts;
    if constexpr (B <= kSortOneBlocks)
        if (s.chunks == 1) return launch_blocks(reinterpret_cast<const void*>(&sort_kernel<B, true>), 1, s.threads, lds, const_cast<SortArgs*>(&p), stream);
    hipStream_t st = (hipStream_t)stream;
    SortArgs a = p;
    int64_t chunks64 = s.chunks;
    int32_t chunks = (int32_t)s.chunks;
    int experts = p.experts;
    void* sort_args[] = {&a};
    void* sum_args[] = {&a.hist, &chunks64, &experts};
    void* place_args[] = {&a, &chunks};
    const bool summed = !sort_adds(s.chunks, p.experts);
    if (hipLaunchKernel(reinterpret_cast<const void*>(&sort_kernel<B, false>), dim3((uint32_t)chunks), dim3(s.threads), sort_args, lds, st) != hipSuccess) return TTC_ERR_HIP;
    if (summed && hipLaunchKernel(reinterpret_cast<const void*>(&sum_kernel), dim3((uint32_t)((experts + kWave - 1) / kWave)), dim3(kSortThreads), sum_args, 0, st) != hipSuccess)
        return TTC_ERR_HIP;
    const void* place = summed ? reinterpret_cast<const void*>(&place_kernel<B, true>) : reinterpret_cast<const void*>(&place_kernel<B, false>);
    const size_t place_lds = head + (summed ? 0 : sizeof(uint32_t) * (size_t)experts);
    return hipLaunchKernel(place, dim3((uint32_t)chunks), dim3(s.threads), place_args, place_lds, st) == hipSuccess ? TTC_OK : TTC_ERR_HIP;
}

}  // namespace

int launch_sort(const SortArgs& a, const SortShape& s, void* stream)
{
    switch (s.blocks) {
    case 1: return launch_sort_blocks<1>(a, s, stream);
    case 2: return launch_sort_blocks<2>(a, s, stream);
    case 4: return launch_sort_blocks<4>(a, s, stream);
    default: return launch_sort_blocks<8>(a, s, stream);
    }
}

// ---------------------------------------------------------------------------------
// The moves.  A row is `vecs` vectors of 16 bytes, the last of which may be cut.  2^lanes_log lanes (at most a
// wavefront, fewer where the row is shorter) take one vector each, `parts` such groups make a row.
// ---------------------------------------------------------------------------------
namespace {

template <typename T> struct RowVec { static constexpr int value = 16 / (int)sizeof(T); };

struct MoveArgs {
    RowArgs  r;
    uint32_t vec;                          // elements of a vector
    uint32_t lanes_log, parts, vecs;
    uint32_t lanes;                        // the gradient's lanes for a token
    FastDiv  parts_div;
    uint32_t units;                        // tokens * parts
    uint32_t blocks, total;                // workgroups over the units, and with those after them that clear padding
    uint32_t pad_parts;                    // workgroups per expert for its padding
};

// Padding rows of expert `e`: those of its segment that hold no token, cleared by `pad_parts` workgroups.
template <typename T, int V, bool NT> __device__ __forceinline__ void clear_padding(const MoveArgs& p, uint32_t block)
{
    if (block >= p.total) return;
    const uint32_t index = block - p.blocks;
    const uint32_t e = index / p.pad_parts, part = index - e * p.pad_parts;
    const int64_t end = p.r.offsets[e + 1], first = (int64_t)p.r.offsets[e] + p.r.counts[e];
    const int64_t lo = first < 0 ? 0 : first, hi = end < (int64_t)p.r.row_count ? end : (int64_t)p.r.row_count;
    if (lo >= hi) return;
    const uint64_t vectors = (uint64_t)(hi - lo) * p.vecs;
    const Vec<T, V> zero = {};
    for (uint64_t i = (uint64_t)part * blockDim.x + threadIdx.x; i < vectors; i += (uint64_t)p.pad_parts * blockDim.x) {
        const uint64_t row = i / p.vecs;
        const MovePlace at = row_place<V>((uint32_t)(i - row * p.vecs), p.r.width);
        store_vec<T, V, NT>(static_cast<T*>(p.r.y) + (lo + (int64_t)row) * p.r.ld_y + at.at, zero);
    }
}

// This lane's token and vector; false if it has none.  WHOLE: a wavefront has one token, which the compiler is told.
template <bool WHOLE> __device__ __forceinline__ bool lane_place(const MoveArgs& p, uint32_t block, uint32_t* token, uint32_t* vec)
{
    const uint32_t unit = block * (kMoveThreads >> p.lanes_log) + (threadIdx.x >> p.lanes_log);
    if (unit >= p.units) return false;
    uint32_t t = fdiv(unit, p.parts_div);
    const uint32_t part = unit - t * p.parts;
    if (WHOLE) t = __builtin_amdgcn_readfirstlane(t);
    *token = t;
    *vec = (part << p.lanes_log) + (threadIdx.x & ((1u << p.lanes_log) - 1));
    return *vec < p.vecs;
}

// GROUP choices (2, 4 or 8, by topk: 4096 x 2 rows of 1001 f32, combine and gradient 33.4 us in groups of eight, 29.2 of two; 700 x 4 of bf16
// 13.1 of eight, 12.4 of four) of a token from k0 on: the rows they point to, kNowhere where there is none, and their
// weights, 0 there.  All loads are under way together, none hangs on a branch: indices past the last choice read the
// last one again.  Where the wavefront has one token they are scalar loads; the compiler would not make them by itself, for all it
// knows the kernel's stores could change the map, and with vector loads that each wait for the one before
// the gather of 32 tokens took 3.6 us instead of 2.9.
constexpr uint32_t kNowhere = ~0u;
template <typename V> using Constant = const V __attribute__((address_space(4)))*;
template <int GROUP, bool WHOLE> struct Choices {
    uint32_t at[GROUP];
    float    w[GROUP];

    // load, then check: what else is to be loaded goes between them
    template <bool WEIGHTS> __device__ __forceinline__ void load(const RowArgs& r, uint32_t token, int k0)
    {
        const uint64_t a = (uint64_t)token * (uint32_t)r.topk;
#pragma unroll
        for (int k = 0; k < GROUP; ++k) {
            const uint64_t i = a + (uint32_t)(k0 + k < r.topk ? k0 + k : r.topk - 1);
            at[k] = (uint32_t)(WHOLE ? ((Constant<int32_t>)r.position)[i] : r.position[i]);
            w[k] = 1.f;
            if (WEIGHTS) w[k] = WHOLE ? ((Constant<float>)r.weights)[i] : r.weights[i];
        }
    }
    __device__ __forceinline__ void check(const RowArgs& r, int k0)
    {
#pragma unroll
        for (int k = 0; k < GROUP; ++k)
            if (k0 + k >= r.topk || at[k] >= r.row_count) {
                at[k] = kNowhere;
                w[k] = 0.f;
            }
    }
    __device__ __forceinline__ bool any() const
    {
        bool a = false;
#pragma unroll
        for (int k = 0; k < GROUP; ++k) a |= at[k] != kNowhere;
        return a;
    }
    __device__ __forceinline__ void load(const RowArgs& r, uint32_t token, int k0)
    {
        if (r.weights) load<true>(r, token, k0); else load<false>(r, token, k0);
        check(r, k0);
    }
};

template <typename T, int V, int GROUP, bool WHOLE, bool NT, bool WEIGHTS>
__global__ __launch_bounds__(kMoveThreads) void gather_kernel(MoveArgs p)
{
    const uint32_t b = block_id();
    if (b >= p.blocks) { clear_padding<T, V, NT>(p, b); return; }
    uint32_t t, vec;
    if (!lane_place<WHOLE>(p, b, &t, &vec)) return;
    const MovePlace place = row_place<V>(vec, p.r.width);
    const uint32_t c = place.at;
    Choices<GROUP, WHOLE> q;
    q.template load<WEIGHTS>(p.r, t, 0);
    const T* from = static_cast<const T*>(p.r.x) + (int64_t)t * p.r.ld_x + c;
    Vec<T, V> x;
    if (!NT) x = load_vec<T, V, false>(from);
    q.check(p.r, 0);
    if (NT) {
        if (p.r.topk <= GROUP && !q.any()) return;
        x = load_vec<T, V, false>(from);
    }
    arrive(x);
    for (int k0 = 0; k0 < p.r.topk; k0 += GROUP) {
        if (k0 > 0) {
            q.template load<WEIGHTS>(p.r, t, k0);
            q.check(p.r, k0);
        }
#pragma unroll
        for (int k = 0; k < GROUP; ++k) {
            if (q.at[k] == kNowhere) continue;
            T* to = static_cast<T*>(p.r.y) + (int64_t)q.at[k] * p.r.ld_y + c;
            if (WEIGHTS) {
                float f[V];
                widen(x, f);
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] *= q.w[k];
                Vec<T, V> r;
                narrow(f, r);
                store_vec<T, V, NT>(to, r);
            } else {
                store_vec<T, V, NT>(to, x);
            }
        }
    }
}
template <typename T, int V, int GROUP, bool WHOLE, bool NT> constexpr auto gather_plain = &gather_kernel<T, V, GROUP, WHOLE, NT, false>;
template <typename T, int V, int GROUP, bool WHOLE, bool NT> constexpr auto gather_weighted = &gather_kernel<T, V, GROUP, WHOLE, NT, true>;

template <typename T, int V, int GROUP, bool WHOLE, bool NT>
__global__ __launch_bounds__(kMoveThreads) void combine_kernel(MoveArgs p)
{
    touch<MoveArgs>();
    uint32_t t, vec;
    if (!lane_place<WHOLE>(p, block_id(), &t, &vec)) return;
    const MovePlace place = row_place<V>(vec, p.r.width);
    const uint32_t c = place.at;
    const T* rows = static_cast<const T*>(p.r.rows) + c;
    float sum[V] = {};
    for (int k0 = 0; k0 < p.r.topk; k0 += GROUP) {
        Choices<GROUP, WHOLE> q;
        q.load(p.r, t, k0);
        Vec<T, V> x[GROUP];
#pragma unroll
        for (int k = 0; k < GROUP; ++k) {
            x[k] = {};
            if (q.at[k] != kNowhere) x[k] = load_vec<T, V, NT>(rows + (int64_t)q.at[k] * p.r.ld_rows);
        }
#pragma unroll
        for (int k = 0; k < GROUP; ++k) {   // 0 * 0 where there is none
            float f[V];
            widen(x[k], f);
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] = __builtin_fmaf(q.w[k], f[i], sum[i]);
        }
    }
    T* to = static_cast<T*>(p.r.y) + (int64_t)t * p.r.ld_y + c;
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] *= p.r.alpha;
    Vec<T, V> r;
    if (p.r.beta != 0.f) {
        // a moved vector leaves what it shares to its neighbour, who may have been here already
        float f[V];
        widen(place.back > 0 ? load_end<T, V>(to, place.back) : load_vec<T, V, NT>(to), f);
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] = __builtin_fmaf(p.r.beta, f[i], sum[i]);
        narrow(sum, r);
        if (place.back > 0) {
            store_end<T, V>(to, r, place.back);
            return;
        }
    } else {
        narrow(sum, r);
    }
    store_vec<T, V, NT>(to, r);
}

// The gradient: `lanes` lanes walk over a whole row, because the dot products need all of it: a power of two up to a wavefront,
// several tokens to a workgroup, or a whole workgroup of several wavefronts.  Their partial sums
// meet by shuffles inside a wavefront and through LDS between wavefronts, always in the same order.
// Wavefronts of a workgroup at most (beyond that they go round): 8, four from kGradMany tokens on, where five to seven of them would leave
// slots of a compute unit empty and the many waits show that half the rows nowhere cause.  This kernel's us with 8 and 4, bf16:
//   3878 x 5 rows of 2112, one of two ranks 36.9, 22.3; 2844 x 5 of 2880 30.3, 21.4; 1996 x 5 of 4104 28.6, 24.9; all rows here 1024 x 8 of 4608 35.8,
//   33.7, of 4104 34.8, 34.0, but 8192 x 4 of 4100 112, 122; below 100 x 4 rows of 8192 6.7, 7.8; 4 x 8 of 4096 5.0, 5.6; 500 x 4 of 4097 9.8, 9.6;
//   900 x 5 of 4104, one of two ranks 16.5, 14.5.
constexpr int kGradWaves = 8, kGradWavesMany = 4, kGradMany = 1024;
template <typename T, int V, int GROUP, bool WHOLE, bool NT>
__global__ __launch_bounds__(WHOLE ? kGradWaves * kWave : kMoveThreads) void combine_grad_kernel(MoveArgs p)
{
    touch<MoveArgs>();
    __shared__ float dots[kGradWaves][GROUP];
    const uint32_t b = block_id();
    if (b >= p.blocks) { clear_padding<T, V, NT>(p, b); return; }
    const uint32_t lanes = p.lanes, lane = WHOLE && lanes > kWave ? threadIdx.x : threadIdx.x & (lanes - 1);
    uint32_t token = WHOLE && lanes > kWave ? b : b * (kMoveThreads / lanes) + threadIdx.x / lanes;
    if (WHOLE) token = __builtin_amdgcn_readfirstlane(token);
    const bool some = token < p.r.tokens;
    const uint32_t t = some ? token : 0;
    const uint64_t a = (uint64_t)t * (uint32_t)p.r.topk;
    const T* dy = static_cast<const T*>(p.r.x) + (int64_t)t * p.r.ld_x;
    for (int k0 = 0; k0 < p.r.topk; k0 += GROUP) {
        Choices<GROUP, WHOLE> q;
        q.load(p.r, t, k0);                 // lanes past the last token look at the first one's, and do nothing with them
        float dot[GROUP];
#pragma unroll
        for (int k = 0; k < GROUP; ++k) {
            if (!some) q.at[k] = kNowhere;
            q.w[k] *= p.r.alpha;
            dot[k] = 0.f;
        }
        if (q.any())                        // a token whose choices are all nowhere reads nothing
            for (uint32_t vec = lane; vec < p.vecs; vec += lanes) {
                const MovePlace place = row_place<V>(vec, p.r.width);
                const uint32_t c = place.at;
                Vec<T, V> d = load_vec<T, V, false>(dy + c), x[GROUP];
#pragma unroll
                for (int k = 0; k < GROUP; ++k) {
                    x[k] = {};
                    if (p.r.dweights && q.at[k] != kNowhere) x[k] = load_vec<T, V, NT>(static_cast<const T*>(p.r.rows) + (int64_t)q.at[k] * p.r.ld_rows + c);
                }
                float g[V], own[V];         // what a moved vector shares is its neighbour's to add
                const Keep<T, V> keep(place.back);
                widen(d, g);
                keep(d);
                widen(d, own);
#pragma unroll
                for (int k = 0; k < GROUP; ++k) {
                    if (q.at[k] == kNowhere) continue;
                    if (p.r.y) {
                        float f[V];
#pragma unroll
                        for (int i = 0; i < V; ++i) f[i] = q.w[k] * g[i];
                        Vec<T, V> r;
                        narrow(f, r);
                        store_vec<T, V, NT>(static_cast<T*>(p.r.y) + (int64_t)q.at[k] * p.r.ld_y + c, r);
                    }
                    if (p.r.dweights) {
                        float f[V];
                        keep(x[k]);
                        widen(x[k], f);
#pragma unroll
                        for (int i = 0; i < V; ++i) dot[k] = __builtin_fmaf(own[i], f[i], dot[k]);
                    }
                }
            }
        if (!p.r.dweights) continue;
        uint32_t last = 0;                  // the lane of a wavefront, or of a smaller group, that has the sum
        if (WHOLE) {
            last = kWave - 1;
#pragma unroll
            for (int k = 0; k < GROUP; ++k) dot[k] = sum_in_last_lane(dot[k]);
        } else {
            for (uint32_t d = lanes / 2; d > 0; d /= 2)
#pragma unroll
                for (int k = 0; k < GROUP; ++k) dot[k] += __shfl_xor(dot[k], (int)d);
        }
        if (WHOLE && lanes > kWave) {
            __syncthreads();                // the sums of the choices before have been read
            if ((threadIdx.x & (kWave - 1)) == last)
#pragma unroll
                for (int k = 0; k < GROUP; ++k) dots[threadIdx.x / kWave][k] = dot[k];
            __syncthreads();
            if (lane < GROUP && some && k0 + (int)lane < p.r.topk) {
                float s = 0.f;
                for (uint32_t w0 = 0; w0 < lanes / kWave; ++w0) s += dots[w0][lane];
                p.r.dweights[a + k0 + lane] = p.r.alpha * s;
            }
        } else if (some && lane == last) {
#pragma unroll
            for (int k = 0; k < GROUP; ++k)
                if (k0 + k < p.r.topk) p.r.dweights[a + k0 + k] = p.r.alpha * dot[k];
        }
    }
}

template <typename T> MoveArgs move_args(const RowArgs& r)
{
    MoveArgs p = {};
    p.r = r;
    p.vec = r.width < (uint32_t)RowVec<T>::value ? 1 : RowVec<T>::value;
    p.vecs = (r.width + p.vec - 1) / p.vec;
    p.lanes_log = (uint32_t)log2_ceil(p.vecs < (uint32_t)kWave ? p.vecs : (uint32_t)kWave);
    p.parts = (p.vecs + (1u << p.lanes_log) - 1) >> p.lanes_log;
    p.parts_div = make_fastdiv(p.parts);
    p.pad_parts = 1;
    return p;
}

// Non-temporal accesses to the sorted rows, by their size: what will not stay in the last-level cache anyhow does better
// without pushing the rest out.  Kernel times at 4096 bf16, 256 to 8192 tokens, three sets of tensors in turn, with the hint and without:
//   gather (stores of rows; x stays plain): 8 choices, 512 tokens 7.4, 8.0 us; 2048: 25.3, 30.0; 8192: 98, 118
//   combine (rows and y): 8 choices, 1024 tokens 13.8, 12.8; 2048: 26.2, 30.8; 8192: 104, 117
//   gradient (rows and drows; dy stays plain), 4 choices: 512 tokens 9.1, 8.3; 1024: 15.3, 15.2, and the combine behind it, which finds its rows still
//   in the cache or not, 7.5, 11.4; 8192: 101, 105
constexpr uint64_t kStreamGather = uint64_t(32) << 20, kStreamCombine = uint64_t(96) << 20, kStreamGrad = uint64_t(24) << 20;
template <typename T> bool streams(const RowArgs& r, uint64_t from) { return (uint64_t)r.tokens * r.topk * r.width * sizeof(T) >= from; }

typedef void (*MoveKernel)(MoveArgs);
struct Kernels {
    MoveKernel k[3][2][2];                 // [two, four, more choices][whole wavefronts][non-temporal]
    MoveKernel narrow;                     // rows shorter than a vector, element by element
};
inline const void* pick(const MoveArgs& p, bool nt, const Kernels& of)
{
    if (p.vec == 1) return reinterpret_cast<const void*>(of.narrow);
    return reinterpret_cast<const void*>(of.k[p.r.topk <= 2 ? 0 : p.r.topk <= 4 ? 1 : 2][p.lanes_log == 6][nt]);
}

#define TTC_KERNELS(kernel)                                                                                             \
    {{{{kernel<T, V, 2, false, false>, kernel<T, V, 2, false, true>}, {kernel<T, V, 2, true, false>, kernel<T, V, 2, true, true>}}, \
      {{kernel<T, V, 4, false, false>, kernel<T, V, 4, false, true>}, {kernel<T, V, 4, true, false>, kernel<T, V, 4, true, true>}}, \
      {{kernel<T, V, 8, false, false>, kernel<T, V, 8, false, true>}, {kernel<T, V, 8, true, false>, kernel<T, V, 8, true, true>}}}, \
     kernel<T, 1, 8, false, false>}
template <typename T> struct kernels_of {
    static constexpr int V = RowVec<T>::value;
    static constexpr Kernels gather = TTC_KERNELS(gather_plain), gather_weights = TTC_KERNELS(gather_weighted), combine = TTC_KERNELS(combine_kernel), combine_grad = TTC_KERNELS(combine_grad_kernel);
};

// Workgroups over the units, and behind them those that clear padding: one per expert and 32 KB that it may have to clear.
template <typename T> int launch_units(const void* fn, MoveArgs& p, int threads, uint64_t units, uint64_t per_block, bool padding, size_t lds, void* stream)
{
    uint64_t blocks = (units + per_block - 1) / per_block, pads = 0;
    if (units > INT32_MAX) return TTC_ERR_OVERFLOW;
    p.units = (uint32_t)units;
    p.blocks = (uint32_t)blocks;
    if (padding && p.r.align > 1) {
        const uint64_t bytes = (uint64_t)(p.r.align - 1) * p.r.width * sizeof(T), parts = (bytes + 32767) / 32768;
        p.pad_parts = (uint32_t)(parts < 64 ? parts : 64);
        pads = (uint64_t)p.r.experts * p.pad_parts;
    }
    p.total = (uint32_t)(blocks + pads);
    return launch_blocks(fn, blocks + pads, threads, lds, &p, stream);
}

template <typename T> int launch_gather_type(const RowArgs& r, void* stream)
{
    MoveArgs p = move_args<T>(r);
    // Six workgroups to a compute unit instead of eight where three choices or more write their rows at once.  4096 bf16 with the sort, us,
    // eight, six, four, three workgroups: 16384 x 3 rows 104, 99, 99, 105; 16384 x 4 135, 127, 123, 123; half of them nowhere 74, 73, 79, 89;
    // 16384 x 8, three of four nowhere 79, 80, 93, 107.  Two choices 144, 144, 150, 164: left alone.
    // Rows that start inside a 64-byte unit go without the hint: 4097 bf16 160 us with it, 150 without.
    const bool nt = streams<T>(r, kStreamGather) && ((uint64_t)r.ld_y * sizeof(T) | (uintptr_t)r.y) % 64 == 0;
    const size_t lds = nt && r.topk >= 3 ? lds_for(6) : 0;
    const void* fn = pick(p, nt, r.weights ? kernels_of<T>::gather_weights : kernels_of<T>::gather);
    return launch_units<T>(fn, p, kMoveThreads, (uint64_t)r.tokens * p.parts, kMoveThreads >> p.lanes_log, true, lds, stream);
}

template <typename T> int launch_combine_type(const RowArgs& r, void* stream)
{
    MoveArgs p = move_args<T>(r);
    const void* fn = pick(p, streams<T>(r, kStreamCombine), kernels_of<T>::combine);
    return launch_units<T>(fn, p, kMoveThreads, (uint64_t)r.tokens * p.parts, kMoveThreads >> p.lanes_log, false, 0, stream);
}

template <typename T> int launch_grad_type(const RowArgs& r, void* stream)
{
    MoveArgs p = move_args<T>(r);
    p.lanes = 1u << p.lanes_log;
    int threads = kMoveThreads;
    if (p.vecs > (uint32_t)kWave) {         // as few rounds as that many wavefronts need, and then no more wavefronts than those rounds
        const uint32_t most = r.tokens >= kGradMany ? kGradWavesMany : kGradWaves;
        const uint32_t pieces = (p.vecs + kWave - 1) / kWave, rounds = (pieces + most - 1) / most;
        p.lanes = (pieces + rounds - 1) / rounds * kWave;
        threads = (int)p.lanes;
    }
    const void* fn = pick(p, streams<T>(r, kStreamGrad), kernels_of<T>::combine_grad);
    return launch_units<T>(fn, p, threads, r.tokens, (uint64_t)threads / p.lanes, r.y != nullptr, 0, stream);
}

}  // namespace

#define TTC_BY_ROW_TYPE(launch, a, stream)                  \
    switch ((a).dtype) {                                    \
    case TTC_F32:  return launch<float>(a, stream);         \
    case TTC_BF16: return launch<__bf16>(a, stream);        \
    case TTC_F16:  return launch<_Float16>(a, stream);      \
    default:       return TTC_ERR_UNSUPPORTED_DTYPE;        \
    }

int launch_gather(const RowArgs& a, void* stream) { TTC_BY_ROW_TYPE(launch_gather_type, a, stream) }
int launch_combine(const RowArgs& a, void* stream) { TTC_BY_ROW_TYPE(launch_combine_type, a, stream) }
int launch_combine_grad(const RowArgs& a, void* stream) { TTC_BY_ROW_TYPE(launch_grad_type, a, stream) }

}  // namespace ttc
