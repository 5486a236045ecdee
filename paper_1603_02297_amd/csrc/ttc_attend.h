// Attention of new tokens over the pages of their requests (include/ttc_attention.h, ttc_attend_pages), for gfx950 (MI355X): the kernel, instantiated per
// type of the queries in ttc_attend_f32.hip, ttc_attend_bf16.hip and ttc_attend_f16.hip.
//
// The query heads that share a head of the cache are rows of one matrix product, token by token, so that a position's key and value are fetched once for
// them all.  A wavefront has M = 16 or 32 rows.  It makes scores transposed, S^T = K Q^T, with the M x M matrix instructions: their result has a row in 64 / M lanes
// (its "parts", M lanes apart) and its positions in their registers.  The softmax's maximum and sum are then registers, too (an exchange between a row's
// lanes for the maximum of a tile, one for the sum at the end), and the exponentials are, without a move, what O^T = V^T P^T takes as its right
// operand: a product's order of positions is free as long as both sides have the same one.  V^T is read from the tile by the transposing LDS loads, in that order.
//
//   ROWS 16, 32  few rows to a request (tokens that are generated one by one): the wavefronts of a workgroup have the same rows and every one its own tiles of 32
//                positions (64 over 4 bits with 16 rows and keys out of LDS), in LDS of its own; no barrier until they add up their results.  Bound by the cache's bytes: 64 requests
//                behind 8000 positions, 8 heads of 128 in 16 bits, 367 us, 5.7 TB/s; shares are pieces of these tiles as long for every workgroup, so that lengths do not matter.
//   ROWS 128     prompts: wavefronts have 32 rows each of the same 128 and share the tiles.  Bound by the matrix instructions, and the exponentials beside them: 11900
//                tokens behind up to 2048, 20 heads of 128 for 5, 365 to 410 us, 390 in the median, 930 TFLOP/s (a large product on this card: 1212).  Over 8 bits 355 us, over
//                4 bits, whose codes are widened on the way into LDS, 570.
//   OWN          few rows over narrow caches, where dim is what the kernel is compiled for: a lane has a part of the vectors of positions of its own.  Keys are
//                never in LDS: these parts are what the left operand of S^T holds in a lane, in an order of the dims that the queries follow.  Values are there as the
//                cache has them, and widened behind the transposing loads, which there are for 8 and 4 bits, too
//                (64 requests behind 8000 positions in 8 bits 186 us, 5.6 TB/s; 48 to 32,768 in 4 bits, where a code costs as many instructions as an element does elsewhere, 133 us, 4.3).
//
// A tile's loads are under way while the one before it is used, its entries of the block table one tile earlier.
#pragma once

#include <atomic>
#include <type_traits>

#include "ttc_attention_internal.h"
#include "ttc_moves_device.h"
#include "ttc_records.h"

namespace ttc {
namespace attend {

typedef short Short4 __attribute__((ext_vector_type(4)));
typedef short Short8 __attribute__((ext_vector_type(8)));
typedef int Int2 __attribute__((ext_vector_type(2)));
#define TTC_LDS __attribute__((address_space(3)))

template <int M> struct Result;            // of a product, M x M over the wavefront: register i of a lane is row kGap * (i / 4) + 4 * part + i % 4, its column lane % M
template <> struct Result<32> {
    typedef float type __attribute__((ext_vector_type(16)));
    static constexpr int kRegisters = 16, kGap = 8;
};
template <> struct Result<16> {
    typedef float type __attribute__((ext_vector_type(4)));
    static constexpr int kRegisters = 4, kGap = 16;
};

// What a lane holds of an operand: 16 bytes.
template <typename E> struct Fragment;
template <> struct Fragment<__bf16> { typedef __bf16 type __attribute__((ext_vector_type(8))); };
template <> struct Fragment<_Float16> { typedef _Float16 type __attribute__((ext_vector_type(8))); };
template <> struct Fragment<float> { typedef float type __attribute__((ext_vector_type(4))); };

__device__ __forceinline__ void mul(Fragment<__bf16>::type a, Fragment<__bf16>::type b, Result<32>::type& c) { c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ void mul(Fragment<__bf16>::type a, Fragment<__bf16>::type b, Result<16>::type& c) { c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ void mul(Fragment<_Float16>::type a, Fragment<_Float16>::type b, Result<32>::type& c) { c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ void mul(Fragment<_Float16>::type a, Fragment<_Float16>::type b, Result<16>::type& c) { c = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ void mul(Fragment<float>::type a, Fragment<float>::type b, Result<32>::type& c)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
}
__device__ __forceinline__ void mul(Fragment<float>::type a, Fragment<float>::type b, Result<16>::type& c)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
}

// T: queries and results; C: the cache; DP: dim rounded up to what the kernel is compiled for.
template <typename T, typename C, int DP, int ROWS, bool OWN> struct Plan {
    static constexpr bool FEW = ROWS < 128;
    static constexpr int  M = ROWS < 32 ? 16 : 32, kParts = kWave / M;
    typedef T K;                                                            // keys in LDS
    typedef T V;                                                            // values in LDS, and the exponentials
    static constexpr bool kRecords = std::is_same<C, q4>::value;
    // records as codes (integers that 16 bits hold), step and minimum applied to scores and exponentials; in 32 bits as what they stand for
    static constexpr bool kCodes = kRecords && sizeof(T) == 2;
    static constexpr bool kWide = sizeof(T) == 4;
    // Codes are multiplied by exponentials times steps.  fp16 would lose those of small steps and not hold those of large ones: there the exponentials' reference is the
    // largest exponential times step, and the steps' logarithms lie beside them.
    static constexpr bool kLogs = kCodes && std::is_same<T, _Float16>::value;
    // The reference of the exponentials follows the maximum once that is 2^kSlack above where it would be: results need their largest term near 1 only so far as 32 bits
    // (and 16 for the weights) must hold them.  Followed at once it moves in most tiles, for some row of 32, and costs every element of the result a product each time.
    static constexpr int kSlack = 8, kLift = attend_lift(std::is_same<T, _Float16>::value ? TTC_F16 : TTC_F32);
    static constexpr int  kWaves = FEW && kWide && DP > 128 ? 2 : 4;
    static constexpr int  kThreads = kWaves * kWave;
    static constexpr int  kTeams = FEW ? kWaves : 1;
    static constexpr int  kTeam = FEW ? kWave : kThreads;                    // threads that load a tile together
    static constexpr int  kKeys = (FEW && !(OWN && kRecords && M == 16)) || (kWide && DP > 128) ? 32 : 64;     // positions of a tile
    static constexpr int  kStep = kKeys * kTeams;
    static constexpr int  kChunks = DP / 8;                                  // of eight elements, of a vector
    static constexpr int  kMine = kKeys * kChunks / kTeam;                   // chunks of a tile that a thread loads
    static constexpr bool kAhead = !(FEW && kWide && DP > 128);              // loads of the next tile under way beside the products of this one
    // rows in LDS end 16 and 32 bytes later than their elements, so that eight rows (four, of values) meet all banks
    static constexpr int  kKeyRow = DP * (int)sizeof(K) + 16;
    static constexpr int  kValueRow = OWN ? (kRecords ? DP / 2 : DP) + 8 : DP * (int)sizeof(V) + (kWide ? 16 : 32);
    static constexpr int  kTile = kKeys * ((OWN ? 0 : kKeyRow) + kValueRow) + (kCodes ? (kLogs ? 5 : 4) * kKeys * 4 : 0);
    // The queries' fragments in LDS, the same for all wavefronts, where keys and values on their way take the registers.
    static constexpr bool kQueriesInLds = ROWS == 32 && !OWN && sizeof(C) == 2;
    static constexpr int  kDims = kParts * 16 / (int)sizeof(K);              // of the contracted index, in a fragment over a row's lanes
    static constexpr int  kQueries = kQueriesInLds ? DP / kDims * kWave * 16 : 0;
    static constexpr int  kMergeRows = 8;                                    // of the wavefronts' results that are added up at a time
    static constexpr int  kMergeRow = DP + 4;                                // floats
    static constexpr int  kMerge = FEW ? kWaves * kMergeRows * kMergeRow * 4 + 3 * kWaves * ROWS * 4 : 0;
    // workgroups that share a compute unit, and so its registers
    static constexpr int  kResident = attend_resident(sizeof(T), OWN, kRecords, DP, ROWS);
    // Tiles of a workgroup's in LDS: two where they fit, one written while the other is still read, and one barrier for each instead of two (prompts 450 us; so, and
    // with a reference that moves seldom, 436).
    static constexpr int  kTiles = FEW ? kTeams : kResident * (2 * kTile + 256) <= kMaxLdsBytes ? 2 : 1;
    static constexpr int  kLds = kTile * kTiles + kQueries > kMerge ? kTile * kTiles + kQueries : kMerge;
    static_assert(kResident * (kLds + 256) <= kMaxLdsBytes, "they share its LDS");
    // OWN: the words of a part of a vector, a lane's, and the positions that it has such a part of
    static constexpr bool kCarries = FEW && kAhead;                          // the next piece of work's first tile is loaded beside the end of this one
    static constexpr int  kWords = (kRecords ? DP / 2 : DP * (int)sizeof(C)) / kParts / 4, kPositions = kKeys / M;
    struct Part { uint32_t w[kWords], head; };
    static_assert(kKeys * kChunks % kTeam == 0 && DP % 32 == 0 && kLds <= kMaxLdsBytes, "a tile is loaded in whole chunks");
};

// Eight elements of the cache in registers, as they lie there.
template <typename C> struct Chunk8 { Vec<C, 8> v; };
template <> struct Chunk8<q4> { uint32_t word, head; };

// One load and nothing around it: joined with another path, or under a condition, the compiler would wait for each before the next (700 keys' worth of such
// waits made a decoding step of 96 requests take 390 us instead of 270).  Vectors shorter than a chunk (ELEMENTS) go element by element all the same.
template <typename C, bool ELEMENTS> __device__ __forceinline__ Chunk8<C> load_chunk(const char* vector, uint32_t at, uint32_t dim)
{
    Chunk8<C> r = {};
    if constexpr (std::is_same<C, q4>::value) {
        const uint8_t* p = reinterpret_cast<const uint8_t*>(vector);
        r.head = load_word(p);
        r.word = load_word(p + kRecordHead + at / 2);
    } else {
        const C* p = reinterpret_cast<const C*>(vector) + at;
        if (ELEMENTS && dim < 8) {
            C e[8] = {};
            for (uint32_t i = 0; i < 8; ++i)
                if (i < dim) e[i] = p[i];
            __builtin_memcpy(&r.v, e, sizeof(r.v));
        } else {
            r.v = load_vec<C, 8, false>(p);
        }
    }
    return r;
}

// Whether one of eight elements is an infinity or a NaN.
__device__ __forceinline__ bool any_bad(const Vec<float, 8>& v)
{
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) bad |= (v.w[i] & 0x7f800000u) == 0x7f800000u;
    return bad;
}
__device__ __forceinline__ bool any_bad(const Vec<__bf16, 8>& v)
{
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) bad |= (v.w[i] & 0x7f80u) == 0x7f80u || (v.w[i] & 0x7f800000u) == 0x7f800000u;
    return bad;
}
__device__ __forceinline__ bool any_bad(const Vec<_Float16, 8>& v)
{
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) bad |= (v.w[i] & 0x7c00u) == 0x7c00u || (v.w[i] & 0x7c000000u) == 0x7c000000u;
    return bad;
}
__device__ __forceinline__ bool any_bad(const Vec<f8, 8>& v)
{
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) bad |= (v.w[i] >> (8 * j) & 0x7fu) == 0x7fu;
    return bad;
}
template <typename C> __device__ __forceinline__ bool any_bad(const Chunk8<C>& c) { return any_bad(c.v); }
__device__ __forceinline__ bool any_bad(const Chunk8<q4>& c)
{
    return (c.head & 0x7f80u) == 0x7f80u || (c.head & 0x7f800000u) == 0x7f800000u;
}

// Eight codes as 16 + code, which 16 bits hold.  Scores take the 16 back with the minimum; values have 24 times the sum of their weights, as they were
// rounded, taken back, so that a weight's rounding is off by that of code - 8 times the step.
// A byte's two codes go to the two halves of a word by a product: byte * (2^shift + 2^(shift + 12)).
template <int SHIFT> __device__ __forceinline__ void codes_of(uint32_t word, uint32_t one, uint32_t* w)
{
    asm("" : "+v"(one));                    // an instruction takes one constant from elsewhere than a vector register: the mask
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = (word >> (8 * k) & 0xffu) * (0x1001u << SHIFT) & (0x000f000fu << SHIFT) | one;
}
__device__ __forceinline__ void codes_of(uint32_t word, Vec<__bf16, 8>& r) { codes_of<3>(word, 0x41804180u, r.w); }
__device__ __forceinline__ void codes_of(uint32_t word, Vec<_Float16, 8>& r) { codes_of<6>(word, 0x4c004c00u, r.w); }

__device__ __forceinline__ void widen_eight(const Vec<f8, 8>& c, Vec<float, 8>& r)
{
    float x[8];
    widen(c, x);
    narrow(x, r);
}
__device__ __forceinline__ void widen_eight(const Vec<f8, 8>& c, Vec<__bf16, 8>& r)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        r.w[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c.w[i], 1.f, false));
        r.w[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c.w[i], 1.f, true));
    }
}
__device__ __forceinline__ void widen_eight(const Vec<f8, 8>& c, Vec<_Float16, 8>& r)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        r.w[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)c.w[i], 1.f, false));
        r.w[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)c.w[i], 1.f, true));
    }
}

// A chunk as the tile holds it.  16-bit caches are of the queries' type, and 8 bits widen exactly.
template <typename E, typename C> __device__ __forceinline__ Vec<E, 8> tile_chunk(const Chunk8<C>& c)
{
    Vec<E, 8> r;
    if constexpr (std::is_same<C, q4>::value) {
        if constexpr (sizeof(E) == 4) {
            float x[8];
            widen_record(c.head, c.word, x);
            narrow(x, r);
        } else {
            codes_of(c.word, r);
        }
    } else if constexpr (std::is_same<E, C>::value) {
        r = c.v;
    } else {
        widen_eight(c.v, r);
    }
    return r;
}
template <typename E, typename C> __device__ __forceinline__ typename Fragment<E>::type fragment_of(const Chunk8<C>& c)
{
    static_assert(sizeof(E) == 2, "eight elements a fragment");
    return __builtin_bit_cast(typename Fragment<E>::type, tile_chunk<E>(c));
}
template <typename E, bool WHOLE, typename C> __device__ __forceinline__ void store_chunk(char* lds, const Chunk8<C>& c)
{
    const Vec<E, 8> r = tile_chunk<E>(c);
    if constexpr (WHOLE) {
        typedef uint32_t Word4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int i = 0; i < Vec<E, 8>::kWords / 4; ++i) {
            Word4 w;
            __builtin_memcpy(&w, r.w + 4 * i, 16);
            reinterpret_cast<Word4*>(lds)[i] = w;
        }
    } else {                                // moved back, to any element
        E e[8];
        __builtin_memcpy(e, r.w, sizeof(e));
#pragma unroll
        for (int i = 0; i < 8; ++i) reinterpret_cast<E*>(lds)[i] = e[i];
    }
}

template <bool WAVE> __device__ __forceinline__ void team_sync()
{
    if constexpr (WAVE) {                                                   // a wavefront's LDS accesses happen in order: only the compiler has to keep it
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    } else {
        __syncthreads();
    }
}

// The same for all lanes, which the compiler cannot see.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) { return (uint64_t)uniform((uint32_t)(x >> 32)) << 32 | uniform((uint32_t)x); }

// What one lane reads for all of them, by a scalar load: it does not wait for the vector loads under way.
template <typename X> __device__ __forceinline__ X scalar(const X* p, uint32_t i) { return ((const __attribute__((address_space(4))) X*)p)[i]; }
// Numbers of 64 bits that mostly are of 32.
__device__ __forceinline__ uint64_t quotient(uint64_t a, uint64_t b) { return (a | b) >> 32 ? a / b : (uint32_t)a / (uint32_t)b; }

// Asks for N products with READS reads of LDS each in this order: the reads of four products first, then a product and the next one's reads in turn.  Left alone the
// compiler keeps two reads under way and the products wait for LDS (11900 tokens of prompts 396 us; with it 381; six ahead 382).
template <int N, int READS> __device__ __forceinline__ void feed()
{
    constexpr int kProduct = 0x8, kRead = 0x100, kFirst = 4;
    __builtin_amdgcn_sched_group_barrier(kRead, kFirst * READS, 0);
#pragma unroll
    for (int i = 0; i < N - kFirst; ++i) {
        __builtin_amdgcn_sched_group_barrier(kProduct, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kRead, READS, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kProduct, kFirst, 0);
}

// Some rows of a request's for one head, and some of the positions that they see.
struct Work {
    uint32_t request, row0, rows;          // rows: of the request
    uint32_t first_token;                  // of the request
    uint32_t cached;
    uint32_t lo, hi;
    uint32_t head;
    bool     partial;                      // others have other positions of these rows
    uint32_t partial_row;                  // where row0's result goes then, the others' after it
    uint32_t parts;                        // of these rows, where this is the first; else 0
};

__device__ __forceinline__ uint32_t token_of(const AttendArgs& p, int32_t s) { return s < 0 ? 0u : (uint32_t)s < p.tokens ? (uint32_t)s : p.tokens; }

// The positions that rows first .. last of a request see, within the table.
__device__ __forceinline__ void positions_of(const AttendArgs& p, uint32_t cached, uint32_t first, uint32_t last, uint32_t* bottom, uint32_t* count)
{
    const uint64_t entries = (uint64_t)p.ld_table * p.page.div;
    uint64_t hi = (uint64_t)cached + fdiv(last, p.group_div) + 1;
    hi = hi < entries ? hi : entries;
    const uint32_t top = hi < 0x7fffffffu ? (uint32_t)hi : 0x7fffffffu, from = cached + fdiv(first, p.group_div) + 1;
    *bottom = p.window && from > p.window ? from - p.window : 0;
    *count = top > *bottom ? top - *bottom : 0;
}

// Many rows: a workgroup a tile of rows, and one of `splits` parts of its positions at most.  Tile number `slot` is request r's with starts[r] * group / tile + r <= slot:
// these numbers grow with r, so that the wavefront counts, 64 requests at a time.
__device__ __forceinline__ uint32_t first_slot(const AttendArgs& p, uint32_t r, uint32_t tile) { return token_of(p, p.starts[r]) * p.group / tile + r; }

template <typename P, int TILE> __device__ __forceinline__ bool find_tile(const AttendArgs& p, uint32_t slot, uint32_t split, Work& w)
{
    const uint32_t lane = threadIdx.x & (kWave - 1);
    uint32_t lo = 0, n = p.requests;
    while (n > 1) {
        const uint32_t step = (n + kWave - 1) / kWave, r = lo + lane * step;
        const uint64_t before = __ballot(lane * step < n && first_slot(p, r < p.requests ? r : 0, TILE) <= slot);
        const uint32_t count = (uint32_t)__builtin_popcountll(before);
        if (count == 0) return false;
        lo += (count - 1) * step;
        n = n - (count - 1) * step < step ? n - (count - 1) * step : step;
        if (step == 1) n = 1;
    }
    lo = uniform(lo);
    const uint32_t begin = token_of(p, scalar(p.starts, lo)), end = token_of(p, scalar(p.starts, lo + 1));
    const uint32_t base = begin * p.group / TILE + lo;
    if (slot < base) return false;
    w.request = lo;
    w.first_token = begin;
    w.row0 = (slot - base) * TILE;
    w.rows = end > begin ? (end - begin) * p.group : 0;
    if (w.row0 >= w.rows) return false;
    const int32_t c = scalar(p.cached, lo);
    w.cached = c < 0 ? 0 : (uint32_t)c;
    uint32_t bottom, count;
    positions_of(p, w.cached, w.row0, w.row0 + TILE < w.rows ? w.row0 + TILE - 1 : w.rows - 1, &bottom, &count);
    uint32_t parts = (count + kAttendUnit - 1) / kAttendUnit, each = count;
    parts = parts < p.splits ? parts : p.splits;
    if (parts > 1) {
        each = ((count + parts - 1) / parts + P::kStep - 1) / P::kStep * P::kStep;
        parts = (count + each - 1) / each;
    }
    w.parts = split == 0 ? (parts > 1 ? parts : 1) : 0;
    w.partial = parts > 1;
    if (split >= (parts > 1 ? parts : 1)) return false;
    w.lo = bottom + split * each;
    w.hi = bottom + count - w.lo < each ? bottom + count : w.lo + each;
    return true;
}

// Few rows: a head's work is cut into units, up to kAttendUnit positions of a tile of rows, request by request, tile by tile; of the workgroups that have this head, number g
// has the g-th share of them, equal but for one, whatever the requests' lengths are.  The heads' shares are alike and their workgroups next to each other, so
// that a slot's heads, neighbours in the cache, are fetched at about the same time.  A share begins and ends within a tile's positions as a rule: at
// most two of its results are partial ones, the first (of a tile that begins in another share: place 2 b, of workgroup b) and the last (of one that ends in another: 2 b + 1).
struct Units {
    uint32_t tiles, each;                  // of the request's rows, units of one of them
    uint32_t bottom, count;                // positions that some row sees
    uint32_t begin, rows, cached;
};
template <int TILE> __device__ __forceinline__ Units units_of(const AttendArgs& p, int32_t first, int32_t behind, int32_t c)
{
    Units u = {};
    u.begin = token_of(p, first);
    const uint32_t end = token_of(p, behind);
    if (end <= u.begin) return u;
    u.rows = (end - u.begin) * p.group;
    u.cached = c < 0 ? 0 : (uint32_t)c;
    positions_of(p, u.cached, 0, u.rows - 1, &u.bottom, &u.count);
    u.tiles = (u.rows + TILE - 1) / TILE;
    u.each = u.count > kAttendUnit ? (u.count + kAttendUnit - 1) / kAttendUnit : 1;        // none to see: still a result to write
    return u;
}

struct Shares {
    uint64_t all, each, more;              // units, units of a share, shares that have one more
    __device__ __forceinline__ uint64_t first(uint32_t g) const { return each * g + (g < more ? g : more); }
    __device__ __forceinline__ uint32_t of(uint64_t unit) const
    {
        const uint64_t large = more * (each + 1);
        return (uint32_t)(unit < large ? quotient(unit, each + 1) : more + quotient(unit - large, each));
    }
};

// The request that this workgroup's share begins in, and the unit of it.
struct Start {
    uint32_t request;
    uint64_t unit;
};
template <int TILE, int THREADS> __device__ __forceinline__ bool find_share(const AttendArgs& p, uint32_t g, Shares& s, Start& start)
{
    constexpr int kWaves = THREADS / kWave;
    __shared__ uint64_t totals[kWaves];
    __shared__ uint32_t longest[kWaves];
    __shared__ uint64_t found[2];
    const uint32_t lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const uint32_t each = (p.requests + THREADS - 1) / THREADS, first = threadIdx.x * each, last = first + each < p.requests ? first + each : p.requests;
    uint64_t mine = 0;
    uint32_t most = 1;
    for (uint32_t r = first; r < last; ++r) {
        const Units u = units_of<TILE>(p, p.starts[r], p.starts[r + 1], p.cached[r]);
        mine += (uint64_t)u.tiles * u.each;
        most = u.each > most ? u.each : most;
    }
    uint64_t sum = mine;                    // over this lane and those before it
    for (int i = 1; i < kWave; i <<= 1) {
        const uint64_t before = __shfl_up(sum, i);
        const uint32_t other = __shfl_xor(most, i);
        sum += lane >= (uint32_t)i ? before : 0;
        most = other > most ? other : most;
    }
    if (lane == kWave - 1) { totals[wave] = sum; longest[wave] = most; }
    __syncthreads();
    uint64_t before = 0, all = 0;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
        before += (uint32_t)k < wave ? totals[k] : 0;
        all += totals[k];
        most = longest[k] > most ? longest[k] : most;
    }
    s.all = uniform(all);
    most = uniform(most);
    if (s.all == 0) return false;
    // a tile's positions lie in kAttendMaxParts shares at most
    const uint64_t least = (most + kAttendMaxParts - 2) / (kAttendMaxParts - 1);
    uint64_t shares = quotient(s.all, least);
    const uint32_t most_shares = gridDim.x / p.heads;
    shares = shares < 1 ? 1 : shares < most_shares ? shares : most_shares;
    s.each = quotient(s.all, shares);
    s.more = s.all - s.each * shares;
    if (g >= shares) return false;
    const uint64_t want = s.first(g);
    uint64_t at = before + sum - mine;
    if (want >= at && want < at + mine) {
        for (uint32_t r = first; r < last; ++r) {
            const Units u = units_of<TILE>(p, p.starts[r], p.starts[r + 1], p.cached[r]);
            const uint64_t n = (uint64_t)u.tiles * u.each;
            if (want < at + n) {
                found[0] = r;
                found[1] = want - at;
                break;
            }
            at += n;
        }
    }
    __syncthreads();
    start.request = (uint32_t)uniform(found[0]);
    start.unit = uniform(found[1]);
    return true;
}

// The largest, and the sum, of a row's lanes.
template <typename Join> __device__ __forceinline__ float over_row(float x, bool four, Join join)
{
    auto swap = [&](const auto& r) { return join(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1])); };
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    if (four) {
        const uint32_t c = __builtin_bit_cast(uint32_t, swap(__builtin_amdgcn_permlane16_swap(b, b, false, false)));
        return swap(__builtin_amdgcn_permlane32_swap(c, c, false, false));
    }
    return swap(__builtin_amdgcn_permlane32_swap(b, b, false, false));
}
template <int M> __device__ __forceinline__ float max_of_row(float x) { return over_row(x, M == 16, [](float a, float b) { return __builtin_fmaxf(a, b); }); }
template <int M> __device__ __forceinline__ float sum_of_row(float x) { return over_row(x, M == 16, [](float a, float b) { return a + b; }); }

// The weights of a value's element in the count of what is neither finite: at most 64 of each in a tile.
constexpr int kPlus = 1, kMinus = 128, kNan = 16384;

// A fragment of values taken apart: what is finite, and marks where it is not.
template <typename E> struct Bad;
template <typename E, int EXP, int SIGN, int PLUS, int MINUS, int NAN_> struct Bad16 {
    typedef typename Fragment<E>::type Frag;
    static __device__ __forceinline__ Frag marks(Frag& v)
    {
        const Short8 b = __builtin_bit_cast(Short8, v);
        const Short8 bad = (b & (short)EXP) == (short)EXP, nan = bad & ((b & (short)(0x7fff & ~EXP)) != (short)0), minus = (b & (short)SIGN) != (short)0;
        v = __builtin_bit_cast(Frag, b & ~bad);
        return __builtin_bit_cast(Frag, bad & ((nan & (short)NAN_) | (~nan & ((minus & (short)MINUS) | (~minus & (short)PLUS)))));
    }
};
template <> struct Bad<__bf16> : Bad16<__bf16, 0x7f80, 0x8000, 0x3f80, 0x4300, 0x4680> {};
template <> struct Bad<_Float16> : Bad16<_Float16, 0x7c00, 0x8000, 0x3c00, 0x5800, 0x7400> {};
template <> struct Bad<float> {
    typedef typename Fragment<float>::type Frag;
    static __device__ __forceinline__ Frag marks(Frag& v)
    {
        Frag m;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = v[i];
            m[i] = x != x ? (float)kNan : __builtin_isinf(x) ? (x > 0 ? (float)kPlus : (float)kMinus) : 0.f;
            v[i] = m[i] != 0.f ? 0.f : x;
        }
        return m;
    }
};

// A tile on its way: its keys and values as a thread loads them, which of its positions are there, and the table's entries of the tile after it.
template <typename T, typename C, int DP, int ROWS, bool OWN> struct Flight {
    typedef Plan<T, C, DP, ROWS, OWN> P;
    Chunk8<C> raw_k[OWN ? 1 : P::kMine], raw_v[P::kAhead && !OWN ? P::kMine : 1];
    typename P::Part part_k[P::kPositions], part_v[P::kPositions];
    int64_t  offset;
    uint64_t here;
    int32_t  entry;
};

template <typename T, typename C, int DP, int ROWS, bool OWN> struct Reader {
    typedef Plan<T, C, DP, ROWS, OWN> P;
    typedef Flight<T, C, DP, ROWS, OWN> F;
    const AttendArgs& p;
    uint32_t lane, wave, member;
    __device__ __forceinline__ Reader(const AttendArgs& args, uint32_t thread)
        : p(args), lane(thread & (kWave - 1)), wave(uniform(thread / kWave)), member(P::FEW ? lane : thread) {}

    __device__ __forceinline__ uint32_t first(const Work& w) const { return w.lo + (P::FEW ? wave : 0) * P::kKeys; }
    __device__ __forceinline__ const char* keys_of(const Work& w) const { return static_cast<const char*>(p.k_cache) + (int64_t)w.head * p.stride_head * (int64_t)sizeof(C); }
    __device__ __forceinline__ const char* values_of(const Work& w) const { return static_cast<const char*>(p.v_cache) + (int64_t)w.head * p.stride_head * (int64_t)sizeof(C); }

    // lane j of every wavefront has position j of a tile: its entry of the table, then where its vectors are
    __device__ __forceinline__ int32_t look_up(const Work& w, uint32_t at) const
    {
        const uint32_t key = at + (lane & (P::kKeys - 1));
        return key < w.hi ? p.table[(int64_t)w.request * p.ld_table + fdiv(key, p.page)] : -1;
    }
    static constexpr bool kEven = P::kTeam % P::kChunks == 0;                // a thread's chunks are the same one of vectors a constant apart
    // A thread's chunks of a tile.  The last one of a vector is moved back to end with it, and those behind it are that one again.
    __device__ __forceinline__ uint32_t chunk_of(int i) const
    {
        const uint32_t at = (kEven ? member % P::kChunks : (member + i * P::kTeam) % P::kChunks) * 8, last = p.dim < 8 ? 0 : p.dim - 8;
        return at < last ? at : last;
    }
    __device__ __forceinline__ uint32_t key_of(int i) const { return kEven ? member / P::kChunks + i * (P::kTeam / P::kChunks) : (member + i * P::kTeam) / P::kChunks; }
    __device__ __forceinline__ int64_t place(int64_t offset, uint32_t key) const
    {
        return (int64_t)((uint64_t)(uint32_t)__shfl((uint32_t)(offset >> 32), key) << 32 | (uint32_t)__shfl((uint32_t)offset, key));
    }
    __device__ __forceinline__ void load(const char* cache, int64_t offset, Chunk8<C>* raw) const
    {
#pragma unroll
        for (int i = 0; i < P::kMine; ++i) raw[i] = load_chunk<C, DP == 32>(cache + place(offset, key_of(i)), chunk_of(i), p.dim);
    }
    // OWN: a part of the vector of each of this lane's positions, column + M * b of the tile
    __device__ __forceinline__ void load_parts(const char* cache, int64_t offset, typename P::Part* r) const
    {
        const uint32_t part = lane / P::M, column = lane % P::M;
#pragma unroll
        for (int b = 0; b < P::kPositions; ++b) {
            const char* vector = cache + (P::kPositions > 1 ? place(offset, column + P::M * b) : offset);
            const char* from = vector + (P::kRecords ? kRecordHead : 0) + part * (P::kWords * 4);
            r[b].head = P::kRecords ? load_word(reinterpret_cast<const uint8_t*>(vector)) : 0;
#pragma unroll
            for (int i = 0; i + 4 <= P::kWords; i += 4) {
                const typename Bits<16>::type x = *reinterpret_cast<const typename Bits<16>::type*>(from + 4 * i);
                __builtin_memcpy(r[b].w + i, &x, 16);
            }
            constexpr int kLeft = P::kWords % 4, kDone = P::kWords - kLeft;
            if constexpr ((kLeft & 2) != 0) {
                const typename Bits<8>::type x = *reinterpret_cast<const typename Bits<8>::type*>(from + 4 * kDone);
                __builtin_memcpy(r[b].w + kDone, &x, 8);
            }
            if constexpr ((kLeft & 1) != 0) r[b].w[P::kWords - 1] = load_word(reinterpret_cast<const uint8_t*>(from + 4 * (P::kWords - 1)));
        }
    }
    // The tile at `at`, whose entries are there; and the entries of the one after it.
    __device__ __forceinline__ void follow(const Work& w, uint32_t at, F& f) const
    {
        const uint32_t key = at + (lane & (P::kKeys - 1)), inside = key - fdiv(key, p.page) * p.page.div;
        const bool here = (uint32_t)f.entry < p.pages;
        // not there: the first slot of the cache, whose values become 0 and whose scores are left out
        f.offset = here ? ((int64_t)f.entry * p.stride_page + (int64_t)inside * p.stride_slot) * (int64_t)sizeof(C) : 0;
        f.here = __ballot(here);
        if constexpr (OWN) {
            load_parts(keys_of(w), f.offset, f.part_k);
            load_parts(values_of(w), f.offset, f.part_v);
        } else if constexpr (P::kAhead) {
            load(keys_of(w), f.offset, f.raw_k);
            load(values_of(w), f.offset, f.raw_v);
        }
        f.entry = look_up(w, at + P::kStep);
    }
    // The queries of this lane's row; behind the request's last one, that one again.
    __device__ __forceinline__ void queries(const Work& w, typename Fragment<typename P::K>::type* query) const
    {
        const uint32_t own = w.row0 + (P::FEW ? 0 : wave * P::M) + lane % P::M, row = own < w.rows ? own : w.rows - 1, in = fdiv(row, p.group_div), part = lane / P::M;
        const T* from = static_cast<const T*>(p.q) + (int64_t)(w.first_token + in) * p.ld_q + (int64_t)(w.head * p.group + (row - in * p.group)) * p.dim;
        constexpr int E = 16 / (int)sizeof(T);
        if (p.dim % E == 0) {
#pragma unroll
            for (int i = 0; i < DP / P::kDims; ++i) {
                const uint32_t at = OWN ? part * (DP / P::kParts) + i * E : i * P::kDims + part * E;
                query[i] = __builtin_bit_cast(typename Fragment<typename P::K>::type, load_vec<T, E, false>(from + (at < p.dim ? at : 0)));
            }
        } else {
#pragma unroll
            for (int i = 0; i < DP / P::kDims; ++i)
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    const uint32_t at = i * P::kDims + part * E + j;
                    query[i][j] = from[at < p.dim ? at : 0];
                }
        }
    }
    __device__ __forceinline__ void begin(const Work& w, F& f) const
    {

        f.entry = look_up(w, first(w));
        follow(w, first(w), f);
    }
};

template <typename T, typename C, int DP, int ROWS, bool OWN>
__device__ __forceinline__ void attend_work(const AttendArgs& p, const Work& w, const Work& next, bool more, Flight<T, C, DP, ROWS, OWN>& f, char* lds)
{
    typedef Plan<T, C, DP, ROWS, OWN> P;
    constexpr bool FEW = P::FEW;
    constexpr int M = P::M, kParts = P::kParts, kRegisters = Result<M>::kRegisters, kGap = Result<M>::kGap;
    typedef typename Result<M>::type Acc;
    typedef typename P::K KE;
    typedef typename P::V VE;
    typedef typename Fragment<KE>::type KFrag;
    typedef typename Fragment<VE>::type VFrag;
    constexpr int kBlocks = P::kKeys / M, kSteps = DP / P::kDims, kOut = DP / M;
    uint32_t thread = threadIdx.x;
    asm volatile("" : "+v"(thread));        // what follows from it is found again for every piece of work: kept over them, it would take the registers of the loads
    const uint32_t lane = thread & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(thread / kWave), part = lane / M, column = lane % M;
    const uint32_t head = w.head;
    Reader<T, C, DP, ROWS, OWN> read(p, thread);
    // this lane's row; behind the request's last one, that one again
    const uint32_t own = w.row0 + (FEW ? 0 : wave * M) + column, row = own < w.rows ? own : w.rows - 1;
    const uint32_t in_request = fdiv(row, p.group_div), q_head = head * p.group + (row - in_request * p.group);
    const uint32_t token = w.first_token + in_request, position = w.cached + in_request;
    uint32_t first_row = w.row0 + (FEW ? 0 : wave * M);
    const bool idle = first_row >= w.rows;                                  // no row of this wavefront's is one
    first_row = first_row < w.rows ? first_row : w.rows - 1;
    const uint32_t last_row = first_row + M - 1 < w.rows ? first_row + M - 1 : w.rows - 1;
    const uint32_t lowest = w.cached + fdiv(first_row, p.group_div), highest = w.cached + fdiv(last_row, p.group_div);

    // scores times `scale` are exponents of 2; its sign goes into the queries, so that the largest product has the largest exponent
    float scale = p.scale;
    if (std::is_same<C, f8>::value && p.k_scale) scale *= scalar(p.k_scale, head);
    const uint32_t keep = scale == 0.f ? 0u : ~0u, flip = scale < 0.f ? (sizeof(T) == 2 ? 0x80008000u : 0x80000000u) : 0u;
    scale = scale == 0.f ? 1.f : __builtin_fabsf(scale);
    KFrag query[kSteps];
    read.queries(w, query);
    float query_sum = 0.f;
    {
        constexpr int E = 16 / (int)sizeof(T);
        const KFrag none = {};
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (OWN) continue;
            const uint32_t at = i * P::kDims + part * E;                    // what lies behind the vector's end
            if (at >= p.dim) query[i] = none;
            else if (p.dim % E != 0)
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (at + j >= p.dim) query[i][j] = (T)0.f;
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            uint32_t word[4];
            __builtin_memcpy(word, &query[i], 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) word[j] = (word[j] & keep) ^ flip;
            __builtin_memcpy(&query[i], word, 16);
            if constexpr (P::kCodes) {
#pragma unroll
                for (int j = 0; j < E; ++j) query_sum += (float)query[i][j];
            }
        }
        if (P::kCodes) query_sum = sum_of_row<M>(query_sum);
    }

    char* tile = lds + (FEW ? wave * P::kTile : 0);
    char *keys, *values;
    float *key_step, *key_low, *value_step, *value_low, *value_log;         // kCodes: of kKeys each
    // of a step; results in fp16 see nothing of values below 2^-24
    auto log_of = [](float step) { return __builtin_fminf(__builtin_fmaxf(__builtin_amdgcn_logf(step), -24.f), 100.f); };
    auto use_tile = [&](char* there) {
        keys = there;
        values = there + (OWN ? 0 : P::kKeys * P::kKeyRow);
        key_step = reinterpret_cast<float*>(values + P::kKeys * P::kValueRow);
        key_low = key_step + P::kKeys;
        value_step = key_low + P::kKeys;
        value_low = value_step + P::kKeys;
        value_log = value_low + P::kKeys;
    };
    constexpr bool kTwo = !FEW && P::kTiles == 2, kFed = !FEW && sizeof(T) == 2;
    uint32_t second = 0;
    use_tile(tile);
    // A thread's chunks of a tile.
    const bool whole = p.dim % 8 == 0;
    auto chunk_of = [&](int i) { return read.chunk_of(i); };
    auto key_of = [&](int i) { return read.key_of(i); };
    auto put_keys = [&](const Chunk8<C>* raw) {
        auto all = [&](auto is_whole) {
#pragma unroll
            for (int i = 0; i < P::kMine; ++i) store_chunk<KE, decltype(is_whole)::value>(keys + key_of(i) * P::kKeyRow + chunk_of(i) * sizeof(KE), raw[i]);
        };
        if (whole) all(std::true_type{}); else all(std::false_type{});
        if constexpr (P::kCodes) {
#pragma unroll
            for (int i = 0; i < P::kMine; ++i)
                if (chunk_of(i) == 0) {
                    const float step = __builtin_bit_cast(float, raw[i].head << 16);
                    key_step[key_of(i)] = step;
                    key_low[key_of(i)] = __builtin_fmaf(-16.f, step, __builtin_bit_cast(float, raw[i].head & 0xffff0000u));
                }
        }
    };
    auto put_values = [&](Chunk8<C>* raw, uint64_t there, bool holes, bool look) -> bool {
        bool bad = false;
        if (holes) {
#pragma unroll
            for (int i = 0; i < P::kMine; ++i)
                if (!(there >> key_of(i) & 1)) raw[i] = {};
        }
        if (!P::kCodes && look) {
#pragma unroll
            for (int i = 0; i < P::kMine; ++i) bad |= any_bad(raw[i]);
        }
        auto all = [&](auto is_whole) {
#pragma unroll
            for (int i = 0; i < P::kMine; ++i) store_chunk<VE, decltype(is_whole)::value>(values + key_of(i) * P::kValueRow + chunk_of(i) * sizeof(VE), raw[i]);
        };
        if (whole) all(std::true_type{}); else all(std::false_type{});
        if constexpr (P::kCodes) {
#pragma unroll
            for (int i = 0; i < P::kMine; ++i)
                if (chunk_of(i) == 0) {
                    const float step = __builtin_bit_cast(float, raw[i].head << 16);
                    value_step[key_of(i)] = step;
                    value_low[key_of(i)] = __builtin_fmaf(8.f, step, __builtin_bit_cast(float, raw[i].head & 0xffff0000u));
                    if constexpr (P::kLogs) value_log[key_of(i)] = log_of(step);
                }
        }
        return bad;
    };
    // its eight elements number i, as LDS and the products have them
    auto chunk_of_part = [&](const typename P::Part& r, int i) -> Chunk8<C> {
        Chunk8<C> c;
        if constexpr (P::kRecords) c = {r.w[i], r.head};
        else __builtin_memcpy(&c, r.w + i * (int)sizeof(C) * 2, sizeof(c));
        return c;
    };
    auto put_parts = [&](typename P::Part* r, uint64_t there, bool holes, bool look) -> bool {
        bool bad = false;
#pragma unroll
        for (int b = 0; b < P::kPositions; ++b) {
            if (holes && !(there >> (column + M * b) & 1)) r[b] = {};
            char* to = values + (column + M * b) * P::kValueRow + part * (P::kWords * 4);
            constexpr int kUnit = P::kWords % 2 ? 1 : 2;
#pragma unroll
            for (int i = 0; i < P::kWords; i += kUnit) __builtin_memcpy(__builtin_assume_aligned(to + 4 * i, 4 * kUnit), r[b].w + i, 4 * kUnit);
            if (!P::kCodes && look) {
#pragma unroll
                for (int i = 0; i < DP / kParts / 8; ++i) bad |= any_bad(chunk_of_part(r[b], i));
            }
        }
        return bad;
    };
    auto put_steps = [&](const typename P::Part* k, const typename P::Part* v) {
#pragma unroll
        for (int b = 0; b < P::kPositions; ++b)
            if (part == 0) {
                const uint32_t key = column + M * b;
                const float ks = __builtin_bit_cast(float, k[b].head << 16), vs = __builtin_bit_cast(float, v[b].head << 16);
                key_step[key] = ks;
                key_low[key] = __builtin_fmaf(-16.f, ks, __builtin_bit_cast(float, k[b].head & 0xffff0000u));
                value_step[key] = vs;
                value_low[key] = __builtin_fmaf(8.f, vs, __builtin_bit_cast(float, v[b].head & 0xffff0000u));
                if constexpr (P::kLogs) value_log[key] = log_of(vs);
            }
    };
    char* queries = lds + P::kTile * P::kTiles + lane * 16;
    if constexpr (P::kQueriesInLds) {
        if (wave == 0) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) *reinterpret_cast<KFrag*>(queries + i * kWave * 16) = query[i];
        }
        __syncthreads();
    }
    auto query_of = [&](int i) -> KFrag {
        if constexpr (P::kQueriesInLds) return *reinterpret_cast<const KFrag*>(queries + i * kWave * 16);
        else return query[i];
    };
    // what lies behind the vectors' ends in the tile's rows: 0, once
    if (!OWN && p.dim < DP) {
        for (uint32_t key = read.member / 32; key < P::kKeys; key += P::kTeam / 32)
            for (uint32_t d = p.dim + read.member % 32; d < DP; d += 32) {
                reinterpret_cast<KE*>(keys + key * P::kKeyRow)[d] = (KE)0.f;
                if constexpr (kTwo) reinterpret_cast<KE*>(keys + P::kTile + key * P::kKeyRow)[d] = (KE)0.f;
            }
    }

    Acc out[kOut] = {};
    float top = -__builtin_inff(), sum = 0.f, low_sum = 0.f;                // of this lane's row (sums: its part of the positions); top, the exponentials' reference, times scale
    uint32_t at = read.first(w);
    int32_t next_entry = -1;
    if constexpr (P::kCarries) next_entry = read.look_up(next, read.first(next));
    else read.begin(w, f);
    for (; at < w.hi; at += P::kStep) {
        asm volatile("" : "+v"(read.member));    // places in the tile are found again each time: kept, they would take the registers of the loads
        // positions of the tile that some row of the workgroup's does not see
        const uint32_t end = at + P::kKeys;
        const uint64_t now = f.here;
        constexpr uint64_t kAll = P::kKeys == 64 ? ~0ull : (1ull << P::kKeys) - 1;
        const bool holes = (now & kAll) != kAll;
        const uint32_t tile_lowest = w.cached + fdiv(w.row0, p.group_div);
        const bool look = holes || end > tile_lowest + 1 || (p.window && at + p.window <= w.cached + fdiv(w.row0 + ROWS < w.rows ? w.row0 + ROWS - 1 : w.rows - 1, p.group_div));
        bool bad;
        if constexpr (kTwo) {
            use_tile(tile + second);                                        // last read two tiles ago, before the barrier of the one between
            second ^= (uint32_t)P::kTile;
        } else {
            team_sync<FEW>();                                               // the tile before has been used
        }
        if constexpr (OWN) {
            if constexpr (P::kCodes) put_steps(f.part_k, f.part_v);
            bad = put_parts(f.part_v, now, holes, look);
        } else if constexpr (P::kAhead) {
            put_keys(f.raw_k);
            bad = put_values(f.raw_v, now, holes, look);
            if (at + P::kStep < w.hi) read.follow(w, at + P::kStep, f);
        } else {
            const int64_t offset = f.offset;
            read.load(read.keys_of(w), offset, f.raw_k);
            put_keys(f.raw_k);
            read.load(read.values_of(w), offset, f.raw_k);
            bad = put_values(f.raw_k, now, holes, look);
            if (at + P::kStep < w.hi) read.follow(w, at + P::kStep, f);
        }
        if constexpr (FEW) {
            bad = __ballot(bad) != 0;
            team_sync<FEW>();
        } else if (look) {
            bad = __syncthreads_or(bad);
        } else {
            __syncthreads();
        }
        if (!FEW && (idle || at > highest || (p.window && (uint64_t)end + p.window <= (uint64_t)lowest + 1))) continue;       // nothing that this wavefront's rows see

        Acc score[kBlocks] = {};
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            const char* from = keys + (b * M + column) * P::kKeyRow + part * 16;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                if constexpr (OWN) mul(fragment_of<KE>(chunk_of_part(f.part_k[b], i)), query[i], score[b]);
                else mul(*reinterpret_cast<const KFrag*>(from + i * P::kDims * sizeof(KE)), query_of(i), score[b]);
            }
        }
        if constexpr (kFed) feed<kBlocks * kSteps, 1>();
        if constexpr (OWN)
            if (at + P::kStep < w.hi) read.follow(w, at + P::kStep, f);
        // register i of block b is position M b + kGap (i / 4) + 4 part + i % 4
        if constexpr (P::kCodes) {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int j = 0; j < kRegisters / 4; ++j) {
                    const uint32_t four = b * M + j * kGap + part * 4;
                    const float4 step = *reinterpret_cast<const float4*>(key_step + four), low = *reinterpret_cast<const float4*>(key_low + four);
                    const float steps[4] = {step.x, step.y, step.z, step.w}, lows[4] = {low.x, low.y, low.z, low.w};
#pragma unroll
                    for (int c = 0; c < 4; ++c) score[b][4 * j + c] = __builtin_fmaf(score[b][4 * j + c], steps[c], lows[c] * query_sum);
                }
        }
        const bool masked = holes || end > lowest + 1 || (p.window && at + p.window <= highest);
        uint32_t seen[kBlocks];                                             // bit kGap (i / 4) + i % 4 of block b: what register i is of
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) seen[b] = ~0u;
        if (masked) {
            // positions of the tile up to the row's own, less those before its window, and those that are there
            const uint64_t upto = position < at ? 0 : position - at >= 63 ? ~0ull : (2ull << (position - at)) - 1;
            const uint32_t out_of = p.window && position >= p.window && position - p.window >= at ? (position - p.window - at >= 63 ? 64 : position - p.window - at + 1) : 0;
            const uint64_t sees = upto & now & (out_of >= 64 ? 0 : ~0ull << out_of);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                seen[b] = (uint32_t)(sees >> (M * b)) >> (4 * part);
#pragma unroll
                for (int i = 0; i < kRegisters; ++i) score[b][i] = seen[b] >> (kGap * (i / 4) + i % 4) & 1 ? score[b][i] : -__builtin_inff();
            }
        }
        float most = -__builtin_inff();
        if constexpr (P::kLogs) {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int j = 0; j < kRegisters / 4; ++j) {
                    const float4 log = *reinterpret_cast<const float4*>(value_log + b * M + j * kGap + part * 4);
                    const float logs[4] = {log.x, log.y, log.z, log.w};
#pragma unroll
                    for (int c = 0; c < 4; ++c) most = __builtin_fmaxf(most, __builtin_fmaf(score[b][4 * j + c], scale, logs[c]));
                }
            most = max_of_row<M>(most);
        } else {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int i = 0; i < kRegisters; ++i) most = __builtin_fmaxf(most, score[b][i]);
            most = max_of_row<M>(most) * scale;
        }
        // Maximum and reference by their difference, which is exact where it counts; the sum of reference and slack is not, and fp16 has no weight of 2^16.
        constexpr float kMost = P::kSlack + P::kLift;
        if (__ballot(most - top > kMost)) {
            const float higher = most - top > kMost ? most - P::kLift : top, factor = higher == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(top - higher);
            top = higher;
            sum *= factor;
            low_sum *= factor;
#pragma unroll
            for (int d = 0; d < kOut; ++d) out[d] *= factor;
        }
        const float base = top == -__builtin_inff() ? 0.f : top;
        // A tile's are added up by themselves first: one after the other onto a sum of 1 or more, exponentials below 2^-24 would all be rounded away.
        float tile_sum = 0.f, tile_low = 0.f;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < kRegisters; ++i) {
                score[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(score[b][i], scale, -base));
                tile_sum += score[b][i];
            }
        if constexpr (P::kCodes) {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int j = 0; j < kRegisters / 4; ++j) {
                    const uint32_t four = b * M + j * kGap + part * 4;
                    const float4 step = *reinterpret_cast<const float4*>(value_step + four), low = *reinterpret_cast<const float4*>(value_low + four);
                    const float steps[4] = {step.x, step.y, step.z, step.w}, lows[4] = {low.x, low.y, low.z, low.w};
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        tile_low = __builtin_fmaf(score[b][4 * j + c], masked && !(seen[b] >> (kGap * j + c) & 1) ? 0.f : lows[c], tile_low);
                        score[b][4 * j + c] *= masked && !(seen[b] >> (kGap * j + c) & 1) ? 0.f : steps[c];        // not seen: 0, whatever the record says
                    }
                }
        }
        // O^T += V^T P^T, a fragment's positions at a time
        constexpr int kEach = 16 / (int)sizeof(VE), kTakes = P::kKeys / (kParts * kEach);
        VFrag weight[kTakes];
#pragma unroll
        for (int k = 0; k < kTakes; ++k)
#pragma unroll
            for (int e = 0; e < kEach; ++e) weight[k][e] = (VE)score[(k * kEach + e) / kRegisters][(k * kEach + e) % kRegisters];
        if constexpr (P::kCodes) {
            typedef VE Two __attribute__((ext_vector_type(2)));
            const Two back = {(VE)-24.f, (VE)-24.f};
#pragma unroll
            for (int k = 0; k < kTakes; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const Two two = {weight[k][2 * e], weight[k][2 * e + 1]};
                    if constexpr (P::kLogs) tile_low = __builtin_amdgcn_fdot2(two, back, tile_low, false);
                    else tile_low = __builtin_amdgcn_fdot2_f32_bf16(two, back, tile_low, false);
                }
        }
        sum += tile_sum;
        low_sum += tile_low;
        // the left operands of rows d * M ... of the result
        auto values_of = [&](int d, VFrag* v) {
            const uint32_t in = lane & 15, at_column = d * M + (M == 32 ? (lane >> 4 & 1) * 16 : 0);     // the first of these 16 lanes' columns
            if constexpr (P::kCodes && OWN) {
                // a lane's row of 16 codes, in the order of two fragments; a column of them back
                static_assert(kTakes == 2, "two fragments of eight");
                const char* from = values + ((in >> 3) * 8 * kParts + part * 4 + (in & 3) + (in >> 2 & 1) * kGap) * P::kValueRow + at_column / 2;
                const auto r = __builtin_amdgcn_ds_read_tr4_b64_v2i32((TTC_LDS Int2*)from);
                v[0] = fragment_of<VE>(Chunk8<q4>{(uint32_t)r[0], 0});
                v[1] = fragment_of<VE>(Chunk8<q4>{(uint32_t)r[1], 0});
            } else if constexpr (OWN) {
#pragma unroll
                for (int k = 0; k < kTakes; ++k) {
                    const char* from = values + (k * 8 * kParts + part * 4 + (in >> 1 & 3) + (in >> 3) * kGap) * P::kValueRow + at_column + (in & 1) * 8;
                    const auto r = __builtin_amdgcn_ds_read_tr8_b64_v2i32((TTC_LDS Int2*)from);
                    v[k] = fragment_of<VE>(__builtin_bit_cast(Chunk8<C>, r));
                }
            } else if constexpr (sizeof(VE) == 4) {
#pragma unroll
                for (int k = 0; k < kTakes; ++k) {
                    const char* from = values + (k * 4 * kParts + part * 4) * P::kValueRow + (d * M + column) * 4;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[k][e] = *reinterpret_cast<const float*>(from + e * P::kValueRow);
                }
            } else {
#pragma unroll
                for (int k = 0; k < kTakes; ++k) {
                    // four rows of 16 elements for each 16 lanes, which get a column of them each
                    const char* from = values + (k * 8 * kParts + part * 4 + in / 4) * P::kValueRow + (at_column + (in & 3) * 4) * 2;
                    const Short4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((TTC_LDS Short4*)from), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((TTC_LDS Short4*)(from + kGap * P::kValueRow));
                    v[k] = __builtin_bit_cast(VFrag, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
                }
            }
        };
        if (!P::kCodes && masked && bad) {
            // An infinity or a NaN among the values, which zero weights would not keep from the rows that do not see it: products with what is finite, and a
            // count of the rest for each result, by the rows that see it.
#pragma unroll
            for (int d = 0; d < kOut; ++d) {
                Acc count = {};
                VFrag v[kTakes];
                values_of(d, v);
#pragma unroll
                for (int k = 0; k < kTakes; ++k) {
                    const VFrag marks = Bad<VE>::marks(v[k]);
                    mul(v[k], weight[k], out[d]);
                    VFrag sees;
#pragma unroll
                    for (int e = 0; e < kEach; ++e) {
                        const int b = (k * kEach + e) / kRegisters, i = (k * kEach + e) % kRegisters;
                        sees[e] = (VE)(seen[b] >> (kGap * (i / 4) + i % 4) & 1 ? 1.f : 0.f);
                    }
                    mul(marks, sees, count);
                }
#pragma unroll
                for (int i = 0; i < kRegisters; ++i) {
                    const int n = (int)count[i];
                    const bool plus = n & (kMinus - 1), minus = n & (kNan - kMinus), nan = n >= kNan;
                    out[d][i] += nan || (plus && minus) ? __builtin_nanf("") : plus ? __builtin_inff() : minus ? -__builtin_inff() : 0.f;
                }
            }
        } else {
#pragma unroll
            for (int d = 0; d < kOut; ++d) {
                VFrag v[kTakes];
                values_of(d, v);
#pragma unroll
                for (int k = 0; k < kTakes; ++k) mul(v[k], weight[k], out[d]);
            }
            if constexpr (kFed) feed<kOut * kTakes, 2>();
        }
    }

    // the next piece of work's first tile on its way beside the rest of this one
    if constexpr (P::kCarries)
        if (more) {
            f.entry = next_entry;
            read.follow(next, read.first(next), f);
        }

    sum = sum_of_row<M>(sum);
    low_sum = sum_of_row<M>(low_sum);
    const float v_scale = std::is_same<C, f8>::value && p.v_scale ? scalar(p.v_scale, head) : 1.f;
    // Writes four neighbouring elements of a row's result, normalized: to the result, or to this part's place.
    auto write = [&](uint32_t of, uint32_t to_token, uint32_t to_head, uint32_t d, const float* x) {
        if (d >= p.dim) return;
        const uint32_t left = p.dim - d;
        if (w.partial) {
            float* to = p.partial + (int64_t)(w.partial_row + of - w.row0) * p.dim + d;
            if (left >= 4) { Vec<float, 4> v; narrow(x, v); store_vec<float, 4, false>(to, v); }
            else for (uint32_t i = 0; i < left; ++i) to[i] = x[i];
        } else {
            T* to = static_cast<T*>(p.out) + (int64_t)to_token * p.ld_o + (int64_t)to_head * p.dim + d;
            if (left >= 4) { Vec<T, 4> v; narrow(x, v); store_vec<T, 4, false>(to, v); }
            else for (uint32_t i = 0; i < left; ++i) to[i] = (T)x[i];
        }
    };
    auto write_lse = [&](uint32_t of, uint32_t to_token, uint32_t to_head, float m, float l) {
        const int64_t r = (int64_t)to_token * p.q_heads + to_head;
        const uint32_t place = w.partial_row + of - w.row0;
        if (w.partial) p.partial_sums[place] = {m, l};
        else if (p.lse) p.lse[r] = log_of_sum(m, l, P::kLift);
        if (w.parts && p.parts) {
            p.parts[2 * r] = (int32_t)place;
            p.parts[2 * r + 1] = (int32_t)w.parts;
        }
    };
    if constexpr (FEW) {
        // the wavefronts' results to the largest of their maxima, then added up
        __syncthreads();
        float* merged = reinterpret_cast<float*>(lds);
        float *tops = merged + P::kWaves * P::kMergeRows * P::kMergeRow, *sums = tops + P::kWaves * ROWS, *lows = sums + P::kWaves * ROWS;
        if (part == 0) { tops[wave * ROWS + column] = top; sums[wave * ROWS + column] = sum; lows[wave * ROWS + column] = low_sum; }
        const uint32_t rows = w.rows - w.row0 < ROWS ? w.rows - w.row0 : ROWS;
        for (uint32_t first = 0; first < rows; first += P::kMergeRows) {
            if (first > 0) __syncthreads();
            if (column - first < (uint32_t)P::kMergeRows) {
#pragma unroll
                for (int d = 0; d < kOut; ++d)
#pragma unroll
                    for (int j = 0; j < kRegisters / 4; ++j)
                        *reinterpret_cast<float4*>(merged + (wave * P::kMergeRows + column - first) * P::kMergeRow + d * M + j * kGap + part * 4) =
                            make_float4(out[d][4 * j], out[d][4 * j + 1], out[d][4 * j + 2], out[d][4 * j + 3]);
            }
            __syncthreads();
            const uint32_t some = rows - first < (uint32_t)P::kMergeRows ? rows - first : P::kMergeRows;
            for (uint32_t i = thread; i < some * (DP / 4); i += P::kThreads) {
                const uint32_t r = i / (DP / 4), row_of = first + r, d = i % (DP / 4) * 4;
                float m = -__builtin_inff(), l = 0.f, low = 0.f, x[4] = {};
#pragma unroll
                for (int k = 0; k < P::kWaves; ++k) m = __builtin_fmaxf(m, tops[k * ROWS + row_of]);
#pragma unroll
                for (int k = 0; k < P::kWaves; ++k) {
                    // a wavefront whose tiles none sees has no maximum, and 0 for everything else unless that is NaN
                    const float s = sums[k * ROWS + row_of], t = tops[k * ROWS + row_of], factor = t == -__builtin_inff() ? (s != s ? 1.f : 0.f) : __builtin_amdgcn_exp2f(t - m);
                    const float4 v = *reinterpret_cast<const float4*>(merged + (k * P::kMergeRows + r) * P::kMergeRow + d);
                    const bool any = factor != 0.f;
                    l = any ? __builtin_fmaf(s, factor, l) : l;
                    low = any ? __builtin_fmaf(lows[k * ROWS + row_of], factor, low) : low;
                    x[0] = any ? __builtin_fmaf(v.x, factor, x[0]) : x[0]; x[1] = any ? __builtin_fmaf(v.y, factor, x[1]) : x[1];
                    x[2] = any ? __builtin_fmaf(v.z, factor, x[2]) : x[2]; x[3] = any ? __builtin_fmaf(v.w, factor, x[3]) : x[3];
                }
                const uint32_t in = fdiv(w.row0 + row_of, p.group_div), h = head * p.group + (w.row0 + row_of - in * p.group);
                const float inverse = l == 0.f ? 0.f : v_scale / l;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = (x[j] + low) * inverse;
                write(w.row0 + row_of, w.first_token + in, h, d, x);
                if (d == 0) write_lse(w.row0 + row_of, w.first_token + in, h, m, l);
            }
        }
    } else {
        if (own >= w.rows) return;
        const float inverse = sum == 0.f ? 0.f : v_scale / sum;
#pragma unroll
        for (int d = 0; d < kOut; ++d)
#pragma unroll
            for (int j = 0; j < kRegisters / 4; ++j) {
                float x[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) x[c] = (out[d][4 * j + c] + low_sum) * inverse;
                write(own, token, q_head, d * M + j * kGap + part * 4, x);
            }
        if (part == 0) write_lse(own, token, q_head, top, sum);
    }
}

template <typename T, typename C, int DP, int ROWS, bool OWN>
__global__ __launch_bounds__((Plan<T, C, DP, ROWS, OWN>::kThreads), (Plan<T, C, DP, ROWS, OWN>::kResident)) void attend_kernel(AttendArgs p)
{
    typedef Plan<T, C, DP, ROWS, OWN> P;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Work w;
    Flight<T, C, DP, ROWS, OWN> f;
    if constexpr (!P::FEW) {
        // Heads next to each other, tiles from the last on: those see most, and begin first.  (A head's tiles together, the last head's end alone: 436 us for 396.)
        const uint32_t id = uniform((uint32_t)block_id()), place = id / p.heads, split = place % p.splits;
        if (place / p.splits >= p.slots_of_tiles) return;
        const uint32_t slot = p.slots_of_tiles - 1 - place / p.splits;
        w.head = id - place * p.heads;
        if (!find_tile<P, ROWS>(p, slot, split, w)) return;
        w.partial_row = ((slot * p.heads + w.head) * p.splits + split) * ROWS;
        attend_work<T, C, DP, ROWS, OWN>(p, w, w, false, f, lds);
    } else {
        Shares s;
        Start start;
        const uint32_t g = blockIdx.x / p.heads, head = blockIdx.x - g * p.heads;
        if (!find_share<ROWS, P::kThreads>(p, g, s, start)) return;
        auto units = [&](uint32_t of) { return units_of<ROWS>(p, scalar(p.starts, of), scalar(p.starts, of + 1), scalar(p.cached, of)); };
        uint64_t unit = s.first(g), left = s.first(g + 1) - unit;
        uint32_t r = start.request;
        // Lengths are read again here.  Should another stream have changed them since, which no call may: nothing is followed that they do not allow, and the loop ends.
        if (r >= p.requests) return;
        Units u = units(r);
        uint32_t tile = (uint32_t)quotient(start.unit, u.each > 0 ? u.each : 1), done = (uint32_t)(start.unit - (uint64_t)tile * u.each);
        if (tile >= u.tiles) return;
        // the rows of a tile, and those of their positions that are this share's
        auto piece = [&] {
            Work x;
            const uint32_t rest = u.each - done, take = left < rest ? (uint32_t)left : rest;
            const uint32_t from = done * kAttendUnit, to = (done + take) * kAttendUnit;
            x.request = r;
            x.row0 = tile * ROWS;
            x.rows = u.rows;
            x.first_token = u.begin;
            x.cached = u.cached;
            x.head = head;
            x.lo = u.bottom + (from < u.count ? from : u.count);
            x.hi = u.bottom + (to < u.count ? to : u.count);
            x.partial = take < u.each;
            x.partial_row = (2 * blockIdx.x + (done == 0)) * ROWS;
            x.parts = done ? 0 : x.partial ? s.of(unit + u.each - 1) - g + 1 : 1;
            left -= take;
            unit += take;
            done = 0;
            ++tile;
            return x;
        };
        w = piece();
        if constexpr (P::kCarries) Reader<T, C, DP, ROWS, OWN>(p, threadIdx.x).begin(w, f);
        while (true) {
            bool more = left > 0;
            if (more && tile == u.tiles) {
                tile = 0;
                u.tiles = 0;
                while (u.tiles == 0 && r + 1 < p.requests) u = units(++r);
                more = u.tiles > 0;
            }
            const Work next = more ? piece() : w;
            attend_work<T, C, DP, ROWS, OWN>(p, w, next, more, f, lds);
            if (!more) break;
            __syncthreads();                                                // LDS is used again
            w = next;
        }
    }
}

template <typename T, typename C, int DP, int ROWS, bool OWN> AttendKernel kernel_of()
{
    typedef Plan<T, C, DP, ROWS, OWN> P;
    static std::atomic<uint64_t> raised{0};
    return {reinterpret_cast<const void*>(&attend_kernel<T, C, DP, ROWS, OWN>), P::kThreads, P::kLds, &raised};
}
template <typename T, typename C, int DP> AttendKernel kernel_of(int dim, int rows)
{
    constexpr bool kHalf = attend_half(sizeof(T), std::is_same<C, q4>::value, DP);
    if constexpr (sizeof(T) == 2 && sizeof(C) == 1)
        if (attend_own(sizeof(T), sizeof(C), dim, rows)) {
            if constexpr (kHalf)
                if (rows == 32) return kernel_of<T, C, DP, 32, true>();
            return kernel_of<T, C, DP, 16, true>();
        }
    if constexpr (kHalf)
        if (rows == 32) return kernel_of<T, C, DP, 32, false>();
    return rows == 16 ? kernel_of<T, C, DP, 16, false>() : kernel_of<T, C, DP, 128, false>();
}
template <typename T, typename C> AttendKernel kernel_of(int dim, int rows)
{
    switch (attend_dim(dim)) {
    case 32:  return kernel_of<T, C, 32>(dim, rows);
    case 64:  return kernel_of<T, C, 64>(dim, rows);
    case 96:  return kernel_of<T, C, 96>(dim, rows);
    case 128: return kernel_of<T, C, 128>(dim, rows);
    case 192: return kernel_of<T, C, 192>(dim, rows);
    default:  return kernel_of<T, C, 256>(dim, rows);
    }
}
template <typename T> AttendKernel kernel_of(int cache_dtype, int dim, int rows)
{
    return cache_dtype == TTC_F8 ? kernel_of<T, f8>(dim, rows) : cache_dtype == TTC_Q4 ? kernel_of<T, q4>(dim, rows) : kernel_of<T, T>(dim, rows);
}

}  // namespace attend
}  // namespace ttc
