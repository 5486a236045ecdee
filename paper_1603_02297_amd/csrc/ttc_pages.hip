// Pages of a cache (include/ttc_moves.h, ttc_pages_*), for gfx950 (MI355X): block tables and slots from request
// lengths, and the moves of keys and values by those slots.
#include "ttc_moves_device.h"
#include "ttc_records.h"

namespace ttc {

// ---------------------------------------------------------------------------------
// The map.  Two prefix sums over the requests (listed positions, pages taken), then every listed position by itself: its
// request by bisection, its page from the table where the request held it already, from the free list where not.
// Nothing that one lane writes is read by another, so that one launch does it: every workgroup makes the prefix sums for
// itself as long as they fit its LDS (they are a few KB out of L2).
// ---------------------------------------------------------------------------------
namespace {

constexpr int kMapThreads = 1024;          // largest workgroup
// Requests whose sums every workgroup makes for itself (16 bytes of LDS each, 64 KB is what a launch has without asking): 1200 5.1 us that
// way, 8.8 with a launch for the sums; 4000 7.2 and 11.0.
constexpr int kMapRequests = 4000;

// sums stop at 2^31-1; adding up this way is associative, too
__device__ __forceinline__ uint32_t capped(uint32_t a, uint32_t b) { return a + b < 0x7fffffffu ? a + b : 0x7fffffffu; }

constexpr int kMapFew = 1 << 18;           // 200,000 positions of 2000 requests 6.2 us with one per lane, 9.4 with four; 1,000,000 14.4 and 11.0

struct Request {
    uint32_t first, have, listed, taken;   // first listed position, pages held, positions listed, pages to take
};

__device__ __forceinline__ uint32_t blocks_of(uint32_t length, const FastDiv& page) { return length ? fdiv(length - 1, page) + 1 : 0; }

__device__ __forceinline__ Request request(const MapArgs& p, int r)
{
    const int32_t c = p.cached[r], f = p.fresh[r];
    const uint32_t cached = c < 0 ? 0 : (uint32_t)c, end = capped(cached, f < 0 ? 0 : (uint32_t)f);
    Request q;
    q.first = cached;
    if (p.first) {
        const int32_t b = p.first[r];
        q.first = b < 0 ? 0 : (uint32_t)b < cached ? (uint32_t)b : cached;
    }
    q.have = blocks_of(cached, p.page);
    q.listed = end - q.first;
    q.taken = blocks_of(end, p.page) - q.have;
    return q;
}

struct Two { uint32_t a, b; };

// Sums over the threads before this one, and over all; `part` holds two words per wavefront.
__device__ __forceinline__ Two sums_before(Two v, uint32_t (*part)[2], Two* all)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
    const Two s = {over_lanes(v.a, capped), over_lanes(v.b, capped)};
    if (lane == kWave - 1) { part[wave][0] = s.a; part[wave][1] = s.b; }
    __syncthreads();
    // the wavefronts' sums, summed by every wavefront for itself
    const Two w = {over_lanes(lane < waves ? part[lane][0] : 0, capped), over_lanes(lane < waves ? part[lane][1] : 0, capped)};
    all->a = __shfl(w.a, waves - 1);
    all->b = __shfl(w.b, waves - 1);
    const uint32_t a = __shfl_up(s.a, 1), b = __shfl_up(s.b, 1);               // the lanes before in this wavefront
    const uint32_t wa = __shfl(w.a, wave > 0 ? wave - 1 : 0), wb = __shfl(w.b, wave > 0 ? wave - 1 : 0);
    return {capped(wave > 0 ? wa : 0, lane > 0 ? a : 0), capped(wave > 0 ? wb : 0, lane > 0 ? b : 0)};
}

// Both prefix sums of all requests, each thread over up to four neighbouring ones at a time: put(r, sums before r, request r),
// and at last put(requests, sums of all, nothing).
template <typename Put> __device__ __forceinline__ void sum_requests(const MapArgs& p, uint32_t (*part)[2], Put put)
{
    constexpr int kNeighbours = 4;
    const int each = p.requests > (int)blockDim.x ? kNeighbours : 1;
    Two carry = {0, 0};
    for (int64_t base = 0; base < p.requests; base += (int64_t)blockDim.x * each) {
        const int64_t lo = base + (int64_t)threadIdx.x * each;
        Request q[kNeighbours];
        Two mine = {0, 0};
#pragma unroll
        for (int j = 0; j < kNeighbours; ++j) {
            q[j] = {};
            if (j < each && lo + j < p.requests) q[j] = request(p, (int)(lo + j));
            mine.a = capped(mine.a, q[j].listed);
            mine.b = capped(mine.b, q[j].taken);
        }
        if (base > 0) __syncthreads();      // the last round's sums have been read
        Two all, at = sums_before(mine, part, &all);
        at.a = capped(at.a, carry.a);
        at.b = capped(at.b, carry.b);
#pragma unroll
        for (int j = 0; j < kNeighbours; ++j) {
            if (j >= each || lo + j >= p.requests) continue;
            put((int)(lo + j), at, q[j]);
            at.a = capped(at.a, q[j].listed);
            at.b = capped(at.b, q[j].taken);
        }
        carry.a = capped(carry.a, all.a);
        carry.b = capped(carry.b, all.b);
    }
    if (threadIdx.x == 0) put(p.requests, carry, Request{});
}

__global__ __launch_bounds__(1024) void starts_kernel(MapArgs p)
{
    __shared__ uint32_t part[1024 / kWave][2];
    sum_requests(p, part, [&](int r, Two s, const Request&) { p.starts[r] = (int32_t)s.a; p.page_starts[r] = (int32_t)s.b; });
}

// FUSED: makes the sums itself, and keeps what else it needs of the requests beside them; otherwise starts_kernel has left
// the sums where they belong.
template <int EACH, bool FUSED>
__global__ __launch_bounds__(kMapThreads) void map_kernel(MapArgs p)
{
    extern __shared__ uint32_t sums[];      // FUSED: starts, page_starts, first listed positions, pages held
    __shared__ uint32_t part[kMapThreads / kWave][2];
    const int n = p.requests + 1;
    const uint32_t* starts = FUSED ? sums : reinterpret_cast<const uint32_t*>(p.starts);
    const uint32_t* page_starts = FUSED ? sums + n : reinterpret_cast<const uint32_t*>(p.page_starts);
    const uint32_t block = block_id();
    if (FUSED) {
        sum_requests(p, part, [&](int r, Two s, const Request& q) {
            sums[r] = s.a;
            sums[n + r] = s.b;
            sums[2 * n + r] = q.first;
            sums[3 * n + r] = q.have;
            if (block == 0) { p.starts[r] = (int32_t)s.a; p.page_starts[r] = (int32_t)s.b; }
        });
        __syncthreads();
    }
    const uint64_t i0 = ((uint64_t)block * blockDim.x + threadIdx.x) * EACH;
    if (i0 >= (uint64_t)p.tokens) return;
    // the last request that starts at or before i0: requests that list nothing share a start with the next
    int lo = 0, hi = p.requests;            // starts[lo] <= i0 < starts[hi], or past the end
    if (i0 >= starts[p.requests]) lo = p.requests;
    else if (p.tokens > 0) {                // first guess: as if all listed the same number, which in a decoding step they do
        const int guess = (int)(i0 * (uint64_t)p.requests / starts[p.requests]);
        if (starts[guess] <= i0) lo = guess;
        if (starts[guess + 1] > i0) hi = guess + 1;
    }
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (starts[mid] <= i0) lo = mid; else hi = mid;
    }
    int r = lo;
    uint32_t first = 0, have = 0;
    auto take = [&] {
        if (r >= p.requests) return;
        if (FUSED) {
            first = sums[2 * n + r];
            have = sums[3 * n + r];
        } else {
            const Request q = request(p, r);
            first = q.first;
            have = q.have;
        }
    };
    take();
    const int count = (uint64_t)p.tokens - i0 < EACH ? (int)((uint64_t)p.tokens - i0) : EACH;
    // where every position's page is found, then the pages themselves: their loads are in flight together
    const int32_t* from[EACH];
    int32_t* entry[EACH];
    int32_t inside[EACH], at[EACH], who[EACH];
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        from[j] = nullptr;
        entry[j] = nullptr;
        inside[j] = 0;
        at[j] = who[j] = -1;
        const uint32_t i = (uint32_t)i0 + j;
        if (j >= count) continue;
        if (r < p.requests && i >= starts[r + 1]) {
            do ++r; while (r < p.requests && i >= starts[r + 1]);
            take();
        }
        if (r >= p.requests) continue;
        const uint32_t pos = first + (i - starts[r]), block_no = fdiv(pos, p.page);
        inside[j] = (int32_t)(pos - block_no * p.page.div);
        at[j] = (int32_t)pos;
        who[j] = r;
        if ((int64_t)block_no >= p.ld_table) continue;
        int32_t* e = p.table + (int64_t)r * p.ld_table + block_no;
        if (block_no < have) {
            from[j] = e;
        } else {
            const uint64_t pick = (uint64_t)page_starts[r] + (block_no - have);
            if (pick < (uint64_t)p.free_count) from[j] = p.free_list + pick;
            if (inside[j] == 0) entry[j] = e;           // the first token of a page enters it
        }
    }
    int32_t page[EACH];
#pragma unroll
    for (int j = 0; j < EACH; ++j) page[j] = from[j] ? *from[j] : -1;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        if (j >= count) continue;
        if ((uint32_t)page[j] >= p.pages) page[j] = -1;
        if (entry[j]) *entry[j] = page[j];
        p.slots[i0 + j] = page[j] >= 0 ? (int32_t)((uint32_t)page[j] * p.page.div + (uint32_t)inside[j]) : -1;
        if (p.positions) p.positions[i0 + j] = at[j];
        if (p.owner) p.owner[i0 + j] = who[j];
    }
}

}  // namespace

// One listed position per lane while that is a launch of few workgroups; four where there are many, so that fewer of
// them make the sums.
int launch_map(const MapArgs& a, void* stream)
{
    MapArgs p = a;
    const bool fused = p.requests <= kMapRequests, few = p.tokens <= kMapFew;
    const int threads = fused && p.requests > 256 ? kMapThreads : 256;
    const uint64_t per_block = (uint64_t)threads * (few ? 1 : 4);
    const uint64_t blocks = ((uint64_t)p.tokens + per_block - 1) / per_block;
    if (fused) {
        const size_t lds = 4 * sizeof(uint32_t) * (size_t)(p.requests + 1);
        const void* fn = few ? reinterpret_cast<const void*>(&map_kernel<1, true>) : reinterpret_cast<const void*>(&map_kernel<4, true>);
        return launch_blocks(fn, blocks ? blocks : 1, threads, lds, &p, stream);
    }
    const int st = launch_blocks(reinterpret_cast<const void*>(&starts_kernel), 1, 1024, 0, &p, stream);
    const void* fn = few ? reinterpret_cast<const void*>(&map_kernel<1, false>) : reinterpret_cast<const void*>(&map_kernel<4, false>);
    return st != TTC_OK ? st : launch_blocks(fn, blocks, threads, 0, &p, stream);
}

// ---------------------------------------------------------------------------------
// Keys and values into and out of the cache.  A lane moves one vector of a token's keys and the same one of its values; the
// vectors of a token are numbered through its heads, tokens follow each other, so that no lane is idle whatever the
// number of heads and their size.
// ---------------------------------------------------------------------------------
namespace {

struct PlaceArgs {
    SlotArgs s;
    uint32_t units;                        // tokens * heads * vecs
    uint32_t vecs;                         // vectors of a head
    FastDiv  token_div, head_div;          // by heads * vecs, by vecs
    uint32_t near;                         // workgroups before this one are numbered by near_block
};

// Sixteen bytes a lane of the type outside the cache.  With 32 (f32 as two accesses of 16 bytes, and 8 bytes of an 8-bit cache), keys and values of
// 28,448 tokens of 8 heads of 128: f32 out of an 8-bit cache (291 MB) 88 us instead of 52, into it 55 and 52; out of one of f32 (466 MB) 90 and 75, into it 107
// and 79; 55,472 tokens of bf16 out of 8 bits (341 MB) 76 and 57, into them 63 and 59.
template <typename T> struct SlotVec { static constexpr int value = 16 / (int)sizeof(T); };

template <typename T, typename C, bool WRITE> struct SlotTypes { typedef T from; typedef C to; };
template <typename T, typename C> struct SlotTypes<T, C, false> { typedef C from; typedef T to; };

// Into the narrower cache.
template <typename From, int V>
__device__ __forceinline__ void convert_in(const Vec<From, V>& x, float scale, Vec<f8, V>& r)
{
    float f[V];
    widen(x, f);
    narrow_scaled(f, scale, r);
}

// And out of it.
template <typename From, typename To, int V>
__device__ __forceinline__ void convert_out(const Vec<From, V>& x, float scale, Vec<To, V>& r)
{
    float f[V];
    widen(x, f);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] *= scale;
    narrow(f, r);
}

// Workgroups go to the eight dies in turn, each with an L2 of its own.  A head whose elements end inside a line shares it with the next
// slot's, and a token's heads, where the cache is ordered by head, are lines far apart that only the tokens after it use up: on different
// dies such a line moves several times.  So kNear successive workgroups go to the same die.  15 heads of 80, bf16 and an 8-bit cache by head,
// keys and values of 41,239 tokens (297 MB) out of it 69.4 us with runs of 1, 59.8 of 16, 58.7 of 64, 58.9 of 256.
constexpr uint32_t kDies = 8, kNear = 64;
__device__ __forceinline__ uint32_t near_block(uint32_t near)
{
    const uint32_t b = block_id(), in = b % (kDies * kNear);
    return b < near ? b - in + in % kDies * kNear + in / kDies : b;
}

template <typename T, typename C, int V, bool WRITE, bool NTL, bool NTS>
__global__ __launch_bounds__(kMoveThreads) void slots_kernel(PlaceArgs p)
{
    touch<PlaceArgs>();
    constexpr bool same = sizeof(T) == sizeof(C);
    typedef typename SlotTypes<T, C, WRITE>::from From;
    typedef typename SlotTypes<T, C, WRITE>::to To;
    const uint32_t unit = near_block(p.near) * kMoveThreads + threadIdx.x;
    if (unit >= p.units) return;
    const uint32_t token = fdiv(unit, p.token_div), in_token = unit - token * p.token_div.div;
    const uint32_t head = fdiv(in_token, p.head_div), vec = in_token - head * p.vecs;
    const MovePlace place = row_place<V>(vec, p.s.dim);
    const uint32_t c = place.at;
    const uint32_t slot = (uint32_t)p.s.slots[token];
    const bool here = slot < p.s.slot_count;
    if (WRITE && !here) return;
    const uint32_t page = here ? fdiv(slot, p.s.page) : 0, inside = here ? slot - page * p.s.page.div : 0;
    const int64_t in_cache = (int64_t)page * p.s.stride_page + (int64_t)inside * p.s.stride_slot + (int64_t)head * p.s.stride_head + c;
    const int64_t packed = (int64_t)head * p.s.dim + c;
    const int64_t at_k = (int64_t)token * p.s.ld_k + packed, at_v = (int64_t)token * p.s.ld_v + packed;
    const bool both = p.s.v_out != nullptr;
    Vec<From, V> k = {}, v = {};
    if (here) {
        k = load_vec<From, V, NTL>(static_cast<const From*>(p.s.k) + (WRITE ? at_k : in_cache));
        if (both) v = load_vec<From, V, NTL>(static_cast<const From*>(p.s.v) + (WRITE ? at_v : in_cache));
    }
    To* to_k = static_cast<To*>(p.s.k_out) + (WRITE ? in_cache : at_k);
    To* to_v = static_cast<To*>(p.s.v_out) + (WRITE ? in_cache : at_v);
    if constexpr (same) {
        store_vec<To, V, NTS>(to_k, k);
        if (both) store_vec<To, V, NTS>(to_v, v);
    } else {
        const float scale_k = p.s.k_scale ? p.s.k_scale[head] : 1.f, scale_v = p.s.v_scale ? p.s.v_scale[head] : 1.f;
        Vec<To, V> r = {};
        auto convert = [](const Vec<From, V>& x, float scale, Vec<To, V>& y) {
            if constexpr (WRITE) convert_in(x, scale, y); else convert_out(x, scale, y);
        };
        if (here) convert(k, scale_k, r);       // nowhere: zero, whatever the scale
        store_vec<To, V, NTS>(to_k, r);
        if (both) {
            if (here) convert(v, scale_v, r);
            store_vec<To, V, NTS>(to_v, r);
        }
    }
}

// Non-temporal hints by the bytes moved, stores from 16 MB, loads from 256 MB on.  Measured with 8 heads of 128 bf16 into (out of) pages of
// bf16, without hints, stores only, both: 44 MB 8.0, 8.1, 9.4 us (7.9, 7.8, 9.1); 175 MB 35.3, 29.5, 31.5 (36.2, 27.4, 29.5); 700 MB
// 122, 114, 115 (127, 117, 113); with an 8-bit cache 33 MB 8.2, 8.0, 7.9 (7.1, 6.0, 8.0); 524 MB 98, 95, 99 (97, 89, 88).
constexpr uint64_t kStreamStores = uint64_t(16) << 20, kStreamLoads = uint64_t(256) << 20;

template <typename T, typename C, bool WRITE> int launch_slots_types(const SlotArgs& a, void* stream)
{
    constexpr int V = SlotVec<T>::value;
    PlaceArgs p = {};
    p.s = a;
    const bool narrow = a.dim < (uint32_t)V;            // element by element
    p.vecs = narrow ? a.dim : (a.dim + V - 1) / V;
    const uint32_t per_token = a.heads * p.vecs;        // heads * dim < 2^30
    p.token_div = make_fastdiv(per_token);
    p.head_div = make_fastdiv(p.vecs);
    // lane numbers stay below 2^31: very long lists go in several launches
    const uint32_t most = (uint32_t)INT32_MAX / per_token;
    for (uint64_t done = 0; done < a.tokens; done += most) {
        const uint32_t tokens = a.tokens - done < most ? (uint32_t)(a.tokens - done) : most;
        p.s.slots = a.slots + done;
        const int64_t skip_k = (int64_t)done * a.ld_k * (int64_t)sizeof(T), skip_v = (int64_t)done * a.ld_v * (int64_t)sizeof(T);
        if (WRITE) {
            p.s.k = static_cast<const char*>(a.k) + skip_k;
            if (a.v) p.s.v = static_cast<const char*>(a.v) + skip_v;
        } else {
            p.s.k_out = static_cast<char*>(a.k_out) + skip_k;
            if (a.v_out) p.s.v_out = static_cast<char*>(a.v_out) + skip_v;
        }
        p.units = tokens * per_token;
        const uint64_t bytes = (uint64_t)tokens * a.heads * a.dim * (sizeof(T) + sizeof(C)) * (a.v_out ? 2 : 1);
        // five workgroups to a compute unit instead of eight: 700 MB of bf16 in 115 us instead of 122 (out of the cache 112, 117); an 8-bit cache
        // has less under way and wants them all
        const size_t lds = sizeof(T) == sizeof(C) && bytes >= kStreamLoads ? lds_for(5) : 0;
        // Into the cache, where heads are not whole units of 64 bytes: near each other, and without the hint, so that the L2 joins the parts of
        // a line (as above, 42,668 tokens, 307 MB, 119 us; near each other 92; no hint 72; both 61; 5 heads of 84 fp16 by head, 47, 42, 46 and 40).  Where
        // they are whole, or tokens follow each other closely in the cache at 16 bytes a lane, both lose: 8 heads of 128, 8-bit by head, 58.6 and
        // 61.8; one head of 40 bf16 27.5 and 31.3.  Out of the cache, near each other loses nowhere: 16 heads of 64, 8-bit by head 63.2 and 57.8 us, 8 of
        // 128 bf16 112 and 112.
        const bool whole = ((a.dim | (uint64_t)a.stride_head | (uint64_t)a.stride_slot | (uint64_t)a.stride_page) * sizeof(C)
                            | (uintptr_t)a.k_out | (uintptr_t)a.v_out) % 64 == 0;
        const bool packed = a.stride_slot == (int64_t)a.heads * a.dim && (a.heads == 1 || a.stride_head == (int64_t)a.dim);
        const bool parts = WRITE && !whole && !(sizeof(T) == sizeof(C) && packed);
        const uint64_t blocks = ((uint64_t)p.units + kMoveThreads - 1) / kMoveThreads;
        p.near = bytes >= kStreamStores && (!WRITE || parts) ? (uint32_t)(blocks / (kDies * kNear) * (kDies * kNear)) : 0;
        const bool ntl = bytes >= kStreamLoads, nts = bytes >= kStreamStores && !parts;
        const void* fn = narrow ? reinterpret_cast<const void*>(&slots_kernel<T, C, 1, WRITE, false, false>)
                       : ntl && nts ? reinterpret_cast<const void*>(&slots_kernel<T, C, V, WRITE, true, true>)
                       : ntl ? reinterpret_cast<const void*>(&slots_kernel<T, C, V, WRITE, true, false>)
                       : nts ? reinterpret_cast<const void*>(&slots_kernel<T, C, V, WRITE, false, true>)
                             : reinterpret_cast<const void*>(&slots_kernel<T, C, V, WRITE, false, false>);
        const int st = launch_blocks(fn, blocks, kMoveThreads, lds, &p, stream);
        if (st != TTC_OK) return st;
    }
    return TTC_OK;
}

template <bool WRITE> int launch_slots(const SlotArgs& a, void* stream)
{
    const bool narrow = a.cache_dtype == TTC_F8;
    switch (a.dtype) {
    case TTC_F32:  return narrow ? launch_slots_types<float, f8, WRITE>(a, stream) : launch_slots_types<float, float, WRITE>(a, stream);
    case TTC_BF16: return narrow ? launch_slots_types<__bf16, f8, WRITE>(a, stream) : launch_slots_types<__bf16, __bf16, WRITE>(a, stream);
    case TTC_F16:  return narrow ? launch_slots_types<_Float16, f8, WRITE>(a, stream) : launch_slots_types<_Float16, _Float16, WRITE>(a, stream);
    default:       return TTC_ERR_UNSUPPORTED_DTYPE;
    }
}

}  // namespace

// ---------------------------------------------------------------------------------
// Keys and values into and out of a cache in 4 bits: a lane has eight elements of one head's vector, of the keys and of the values, and as
// many lanes as a vector needs, rounded up to a power of two, find its smallest and largest together.
// ---------------------------------------------------------------------------------
namespace {

struct RecordArgs {
    SlotArgs s;
    uint32_t vectors;                      // tokens * heads
    uint32_t words;                        // of eight codes, of a vector
    int32_t  lanes_log;
    FastDiv  heads;
};

// Records and vectors, a lane eight elements of one.  What 6900 tokens of 4 heads of 64 fp16 take in and out is a launch (4.8 us for 10 MB).
template <typename T, bool WRITE>
__global__ __launch_bounds__(kMoveThreads) void records_kernel(RecordArgs p)
{
    touch<RecordArgs>();
    const uint64_t thread = (uint64_t)block_id() * kMoveThreads + threadIdx.x;
    const uint64_t number = thread >> p.lanes_log;
    const uint32_t word = (uint32_t)thread & ((1u << p.lanes_log) - 1), at = 8 * word;
    const uint32_t vector = number < p.vectors ? (uint32_t)number : 0;
    const uint32_t token = fdiv(vector, p.heads), head = vector - token * p.heads.div;
    const bool mine = number < p.vectors && word < p.words;
    const uint32_t slot = (uint32_t)p.s.slots[token];
    const bool here = slot < p.s.slot_count;
    const uint32_t page = here ? fdiv(slot, p.s.page) : 0, inside = here ? slot - page * p.s.page.div : 0;
    const int64_t record = (int64_t)page * p.s.stride_page + (int64_t)inside * p.s.stride_slot + (int64_t)head * p.s.stride_head;
    const int64_t packed = (int64_t)head * p.s.dim + at, at_k = (int64_t)token * p.s.ld_k + packed, at_v = (int64_t)token * p.s.ld_v + packed;
    const bool both = p.s.v_out != nullptr;
    float x[8];
    if constexpr (WRITE) {
        Vec<T, 8> k = {}, v = {};
        if (mine && here) {
            k = load_vec<T, 8, false>(static_cast<const T*>(p.s.k) + at_k);
            if (both) v = load_vec<T, 8, false>(static_cast<const T*>(p.s.v) + at_v);
        }
        auto put = [&](const Vec<T, 8>& r, void* cache) {
            widen(r, x);
            RecordRange range;
            if (mine) range.take(x, 8);
            const Record made = range.record(p.lanes_log);
            uint8_t* to = static_cast<uint8_t*>(cache) + record;
            if (mine && here) {
                if (word == 0) store_word(to, made.head());
                store_word(to + kRecordHead + at / 2, made.codes(x));
            }
        };
        put(k, p.s.k_out);
        if (both) put(v, p.s.v_out);
    } else {
        if (!mine) return;
        uint32_t k_head = 0, k_word = 0, v_head = 0, v_word = 0;           // nowhere: 0 * 0 + 0
        if (here) {
            const uint8_t* from = static_cast<const uint8_t*>(p.s.k) + record;
            k_head = load_word(from);
            k_word = load_word(from + kRecordHead + at / 2);
            if (both) {
                const uint8_t* v_from = static_cast<const uint8_t*>(p.s.v) + record;
                v_head = load_word(v_from);
                v_word = load_word(v_from + kRecordHead + at / 2);
            }
        }
        Vec<T, 8> r;
        widen_record(k_head, k_word, x);
        narrow(x, r);
        store_vec<T, 8, false>(static_cast<T*>(p.s.k_out) + at_k, r);
        if (both) {
            widen_record(v_head, v_word, x);
            narrow(x, r);
            store_vec<T, 8, false>(static_cast<T*>(p.s.v_out) + at_v, r);
        }
    }
}

template <bool WRITE> int launch_records(const SlotArgs& a, void* stream)
{
    RecordArgs p = {};
    p.s = a;
    p.words = a.dim / 8;
    p.lanes_log = log2_ceil(p.words);
    p.heads = make_fastdiv(a.heads);
    const int eb = elem_bytes(a.dtype);
    // vectors are counted below 2^31: very long lists go in several launches
    const uint32_t most = (uint32_t)INT32_MAX / a.heads;
    for (uint64_t done = 0; done < a.tokens; done += most) {
        const uint32_t tokens = a.tokens - done < most ? (uint32_t)(a.tokens - done) : most;
        p.s.slots = a.slots + done;
        const int64_t skip_k = (int64_t)done * a.ld_k * eb, skip_v = (int64_t)done * a.ld_v * eb;
        if (WRITE) {
            p.s.k = static_cast<const char*>(a.k) + skip_k;
            if (a.v) p.s.v = static_cast<const char*>(a.v) + skip_v;
        } else {
            p.s.k_out = static_cast<char*>(a.k_out) + skip_k;
            if (a.v_out) p.s.v_out = static_cast<char*>(a.v_out) + skip_v;
        }
        p.vectors = tokens * a.heads;
        const void* fn = a.dtype == TTC_F32 ? reinterpret_cast<const void*>(&records_kernel<float, WRITE>)
                       : a.dtype == TTC_BF16 ? reinterpret_cast<const void*>(&records_kernel<__bf16, WRITE>)
                                             : reinterpret_cast<const void*>(&records_kernel<_Float16, WRITE>);
        const int st = launch_blocks(fn, (((uint64_t)p.vectors << p.lanes_log) + kMoveThreads - 1) / kMoveThreads, kMoveThreads, 0, &p, stream);
        if (st != TTC_OK) return st;
    }
    return TTC_OK;
}

}  // namespace

int launch_write(const SlotArgs& a, void* stream) { return a.cache_dtype == TTC_Q4 ? launch_records<true>(a, stream) : launch_slots<true>(a, stream); }
int launch_read(const SlotArgs& a, void* stream) { return a.cache_dtype == TTC_Q4 ? launch_records<false>(a, stream) : launch_slots<false>(a, stream); }

}  // namespace ttc
