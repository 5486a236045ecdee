// What the kernels of the moves by data share: 16-byte vectors of the element types, their widening to float and the
// one rounding back, and the launch geometry.
#pragma once

#include <hip/hip_runtime.h>

#include "ttc_moves_internal.h"
#include "ttc_walk.h"

namespace ttc {

struct f8 { uint8_t bits; };               // TTC_F8: four exponent and three mantissa bits, largest value 448

template <int BYTES> struct Bits;          // a lane's access, with the alignment of the element only
template <> struct Bits<4> { typedef uint32_t type __attribute__((aligned(1))); };
template <> struct Bits<8> { typedef uint32_t type __attribute__((ext_vector_type(2), aligned(1))); };
template <> struct Bits<16> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(1))); };

// V elements of type T in registers: 16 or 32 bytes (4 or 8 of the narrowest types), or one element (V = 1: rows shorter than a vector).
// Columns start wherever their leading dimension puts them: gfx950 takes global dwordx2/x4 accesses at any byte, and a
// row that starts inside a 16-byte unit costs no second instruction.
template <typename T, int V> struct Vec {
    static constexpr int kWords = V * (int)sizeof(T) / 4;
    uint32_t w[kWords];
};
template <typename T> struct Vec<T, 1> { T e; };

template <int N> struct Chunk { static constexpr int value = N < 4 ? N : 4; };         // words moved per instruction

// NT: with the non-temporal hint.  One instruction after the other and nothing between them: a path of its own for vectors cut by
// the end of a row, joined with this one, made the compiler wait for every load before it issued the next.
template <typename T, int V, bool NT> __device__ __forceinline__ Vec<T, V> load_vec(const T* p)
{
    Vec<T, V> r;
    if constexpr (V == 1) {
        r.e = *p;
    } else {
        constexpr int C = Chunk<Vec<T, V>::kWords>::value;
        typedef typename Bits<C * 4>::type W;
#pragma unroll
        for (int i = 0; i < Vec<T, V>::kWords / C; ++i) {
            const W* from = reinterpret_cast<const W*>(p) + i;
            const W x = NT ? __builtin_nontemporal_load(from) : *from;
            __builtin_memcpy(r.w + i * C, &x, sizeof(x));
        }
    }
    return r;
}

template <typename T, int V, bool NT> __device__ __forceinline__ void store_vec(T* p, const Vec<T, V>& r)
{
    if constexpr (V == 1) {
        *p = r.e;
    } else {
        constexpr int C = Chunk<Vec<T, V>::kWords>::value;
        typedef typename Bits<C * 4>::type W;
#pragma unroll
        for (int i = 0; i < Vec<T, V>::kWords / C; ++i) {
            W x;
            __builtin_memcpy(&x, r.w + i * C, sizeof(x));
            W* to = reinterpret_cast<W*>(p) + i;
            if (NT) __builtin_nontemporal_store(x, to); else *to = x;
        }
    }
}

// Waits for a vector here, once.  Where stores of it follow on branches, the compiler would wait before each of them, and so for the
// stores before it, too.
template <typename T, int V> __device__ __forceinline__ void arrive(Vec<T, V>& r)
{
    if constexpr (V > 1) {
#pragma unroll
        for (int i = 0; i < Vec<T, V>::kWords; ++i) asm volatile("" : "+v"(r.w[i]));
    }
}

// A lane's place in a row of `width` >= V elements.  The last vector of a row that is no multiple of V is moved back to end with the
// row: it shares its first `back` elements with its neighbour, both read the same and store the same.  (Element by element
// the ends of rows of 4100 bf16 cost a backward pass, gradient and combine, of 8192 x 4 rows 264 us instead of 170.)
struct MovePlace {
    uint32_t at;
    int      back;
};
template <int V> __device__ __forceinline__ MovePlace row_place(uint32_t vec, uint32_t width)
{
    const uint32_t at = vec * V, back = at + V > width ? at + V - width : 0;
    return {at - back, (int)back};
}

// Of a vector that was moved back, the elements that are its own: all but the first `back`.
template <typename T, int V> __device__ __forceinline__ Vec<T, V> load_end(const T* p, int back)
{
    T e[V] = {};
    for (int i = 1; i < V; ++i)
        if (i >= back) e[i] = p[i];
    Vec<T, V> r;
    __builtin_memcpy(&r, e, sizeof(r));
    return r;
}
template <typename T, int V> __device__ __forceinline__ void store_end(T* p, const Vec<T, V>& r, int back)
{
    T e[V];
    __builtin_memcpy(e, &r, sizeof(r));
    for (int i = 1; i < V; ++i)
        if (i >= back) p[i] = e[i];
}
// The vector without its first `back` elements, by masks on whole words: taken apart into elements it would have to have arrived.
template <typename T, int V> struct Keep {
    uint32_t mask[V == 1 ? 1 : V * (int)sizeof(T) / 4];
    __device__ __forceinline__ explicit Keep(int back)
    {
        constexpr int each = 4 / (int)sizeof(T);
        if constexpr (V > 1) {
#pragma unroll
            for (int i = 0; i < Vec<T, V>::kWords; ++i)
                mask[i] = each == 1 ? (i < back ? 0u : ~0u) : (2 * i < back ? 0u : 0xffffu) | (2 * i + 1 < back ? 0u : 0xffff0000u);
        }
    }
    __device__ __forceinline__ void operator()(Vec<T, V>& r) const
    {
        if constexpr (V > 1) {
#pragma unroll
            for (int i = 0; i < Vec<T, V>::kWords; ++i) r.w[i] &= mask[i];
        }
    }
};

// Widening is exact.
__device__ __forceinline__ void widen(const Vec<float, 1>& r, float* x) { *x = r.e; }
__device__ __forceinline__ void widen(const Vec<__bf16, 1>& r, float* x) { *x = (float)r.e; }
__device__ __forceinline__ void widen(const Vec<_Float16, 1>& r, float* x) { *x = (float)r.e; }
__device__ __forceinline__ void widen(const Vec<f8, 1>& r, float* x) { *x = __builtin_amdgcn_cvt_f32_fp8((int)r.e.bits, 0); }
template <int V> __device__ __forceinline__ void widen(const Vec<float, V>& r, float* x)
{
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = __builtin_bit_cast(float, r.w[i]);
}
template <int V> __device__ __forceinline__ void widen(const Vec<__bf16, V>& r, float* x)
{
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        x[2 * i] = __builtin_bit_cast(float, r.w[i] << 16);
        x[2 * i + 1] = __builtin_bit_cast(float, r.w[i] & 0xffff0000u);
    }
}
template <int V> __device__ __forceinline__ void widen(const Vec<_Float16, V>& r, float* x)
{
    typedef _Float16 H2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        const H2 h = __builtin_bit_cast(H2, r.w[i]);
        x[2 * i] = (float)h.x;
        x[2 * i + 1] = (float)h.y;
    }
}
template <int V> __device__ __forceinline__ void widen(const Vec<f8, V>& r, float* x)
{
    typedef float F2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        const F2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)r.w[i], true);
        x[4 * i] = a.x; x[4 * i + 1] = a.y; x[4 * i + 2] = b.x; x[4 * i + 3] = b.y;
    }
}

__device__ __forceinline__ float cut_f8(float x)
{
    const float c = __builtin_fminf(__builtin_fmaxf(x, -448.f), 448.f);
    return x != x ? x : c;
}

// One rounding, to nearest even; in 8 bits what is larger than 448 becomes 448 (the format has no infinity) and a NaN
// stays one.
__device__ __forceinline__ void narrow(const float* x, Vec<float, 1>& r) { r.e = *x; }
__device__ __forceinline__ void narrow(const float* x, Vec<__bf16, 1>& r) { r.e = (__bf16)*x; }
__device__ __forceinline__ void narrow(const float* x, Vec<_Float16, 1>& r) { r.e = (_Float16)*x; }
__device__ __forceinline__ void narrow(const float* x, Vec<f8, 1>& r)
{
    r.e.bits = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(cut_f8(*x), 0.f, 0, false);
}
template <int V> __device__ __forceinline__ void narrow(const float* x, Vec<float, V>& r)
{
#pragma unroll
    for (int i = 0; i < V; ++i) r.w[i] = __builtin_bit_cast(uint32_t, x[i]);
}
template <int V> __device__ __forceinline__ void narrow(const float* x, Vec<__bf16, V>& r)
{
    typedef __bf16 B2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        B2 h;
        h.x = (__bf16)x[2 * i];
        h.y = (__bf16)x[2 * i + 1];
        r.w[i] = __builtin_bit_cast(uint32_t, h);
    }
}
template <int V> __device__ __forceinline__ void narrow(const float* x, Vec<_Float16, V>& r)
{
    typedef _Float16 H2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        H2 h;
        h.x = (_Float16)x[2 * i];
        h.y = (_Float16)x[2 * i + 1];
        r.w[i] = __builtin_bit_cast(uint32_t, h);
    }
}
template <int V> __device__ __forceinline__ void narrow(const float* x, Vec<f8, V>& r)
{
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(cut_f8(x[4 * i]), cut_f8(x[4 * i + 1]), 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(cut_f8(x[4 * i + 2]), cut_f8(x[4 * i + 3]), w, true);
        r.w[i] = (uint32_t)w;
    }
}

// Into 8 bits: x / scale.  Divisions cost a dozen instructions each, enough to bound the kernel by arithmetic (bf16, 682 MB
// in 154 us with them, 124 without; 128 MB by head 24.4 and 21.2; 20 MB 6.9 and 5.9).  With r = 1 / |scale| rounded once, q = x * r is off by two units at most, and q - (q * |scale| - x) * r rounds
// the quotient itself: ties of the 8-bit format, which are quotients that 32 bits hold, stay ties.  Subtracted in that order a remainder of nothing, which is +0,
// leaves q as it is, -0 among others.  q is held to +-512 before that, so that an infinite
// one does not become a NaN; beyond 448 the cut follows anyhow.  A negative scale turns the signs of the result, four at a time.  Scales outside
// 2^-60 .. 2^60, where r or the remainder could leave the normal range, take the division.
__device__ __forceinline__ void turn_signs(Vec<f8, 1>& r) { r.e.bits ^= 0x80; }
template <int V> __device__ __forceinline__ void turn_signs(Vec<f8, V>& r)
{
#pragma unroll
    for (int i = 0; i < V / 4; ++i) r.w[i] ^= 0x80808080u;
}
template <int V> __device__ __forceinline__ void narrow_scaled(const float* x, float scale, Vec<f8, V>& r)
{
    float f[V];
    const float size = __builtin_fabsf(scale);
    if (size >= 0x1p-60f && size <= 0x1p60f) {
        const float inverse = 1.f / size;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float q = __builtin_fminf(__builtin_fmaxf(x[i] * inverse, -512.f), 512.f);
            f[i] = __builtin_fmaf(-__builtin_fmaf(q, size, -x[i]), inverse, q);
        }
        narrow(f, r);
        if (scale < 0.f) turn_signs(r);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = x[i] / scale;
        narrow(f, r);
    }
}

// The logarithm of a sum of exponentials relative to 2^top, which carry 2^lift: as that of small numbers where the scores are small.  -inf where there are none.
__device__ __forceinline__ float log_of_sum(float top, float sum, int lift)
{
    return sum == 0.f ? -__builtin_inff() : (top + (float)lift) * 0.693147180559945f + __builtin_logf(sum * (1.f / (float)(1 << lift)));
}

// Inclusive combination over the lanes of a wavefront, in registers: data-parallel-primitive moves by 1, 2, 4 and 8 lanes inside the
// rows of 16, then the last lane of a row to the next row, then of the first half to the second.  join(a, 0) has to be a.
template <int CONTROL, int ROWS> __device__ __forceinline__ uint32_t moved(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CONTROL, ROWS, 0xf, false);
}
template <typename Join> __device__ __forceinline__ uint32_t over_lanes(uint32_t v, Join join)
{
    v = join(v, moved<0x111, 0xf>(v));      // row_shr:1
    v = join(v, moved<0x112, 0xf>(v));
    v = join(v, moved<0x114, 0xf>(v));
    v = join(v, moved<0x118, 0xf>(v));      // row_shr:8
    v = join(v, moved<0x142, 0xa>(v));      // row_bcast:15 into rows 1 and 3
    return join(v, moved<0x143, 0xc>(v));   // row_bcast:31 into rows 2 and 3
}

__device__ __forceinline__ float sum_in_last_lane(float v)        // lane 63 gets the sum over the wavefront, the others partial sums
{
    auto add = [](uint32_t a, uint32_t b) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b)); };
    return __builtin_bit_cast(float, over_lanes(__builtin_bit_cast(uint32_t, v), add));
}

// Touches every 64-byte line of a kernel's arguments (its first parameter, of type Args) at once: read where they are used, a line after the other,
// each costs the way to memory again.  Kernel times without and with it: one token's combine 2.68 and 2.43 us, 128 tokens into the cache 2.64 and
// 2.48, 600 tokens out of it 2.62 and 2.40, a gradient of 2050 x 2 rows of which a quarter is here 5.6 and 5.7; the gather, the sort and the
// map gain nothing.  It goes by the segment that the launch put them in: the parameter's own address is that of a private copy
// until the compiler has dropped it.
template <typename Args> __device__ __forceinline__ void touch()
{
    constexpr unsigned last = sizeof(Args) / 4 - 1;
    static_assert(last < 64, "four lines are touched here");
    const __attribute__((address_space(4))) uint32_t* words = (const __attribute__((address_space(4))) uint32_t*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : : "s"(words[1]), "s"(words[17 < last ? 17 : last]), "s"(words[33 < last ? 33 : last]), "s"(words[49 < last ? 49 : last]));
}

// A launch dimension may count at most 2^32 work items: blocks beyond 2^20 go into the second dimension.
constexpr uint32_t kGridRow = 1u << 20;
__device__ __forceinline__ uint32_t block_id() { return blockIdx.y * kGridRow + blockIdx.x; }

// LDS that a launch asks for and does not use, so that `workgroups` (3 to 8) of its workgroups share a compute unit: with fewer rows
// under way at a time, HBM stays longer at each.
constexpr size_t lds_for(int workgroups) { return (size_t)(kMaxLdsBytes / (workgroups + 1) + 512) / 512 * 512; }

inline int launch_blocks(const void* fn, uint64_t blocks, int threads, size_t lds, void* args, void* stream)
{
    if (blocks == 0) return TTC_OK;
    const dim3 grid(blocks < kGridRow ? (uint32_t)blocks : kGridRow, (uint32_t)((blocks + kGridRow - 1) / kGridRow));
    void* list[] = {args};
    // the launch's own status: an error left behind by an earlier, unrelated call on this thread is not ours
    return hipLaunchKernel(fn, grid, dim3(threads), list, lds, (hipStream_t)stream) == hipSuccess ? TTC_OK : TTC_ERR_HIP;
}

inline int log2_ceil(uint64_t x)
{
    int l = 0;
    while ((uint64_t(1) << l) < x) ++l;
    return l;
}

}  // namespace ttc
