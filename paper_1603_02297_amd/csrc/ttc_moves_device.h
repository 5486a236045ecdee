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

// V elements of type T in registers.  Columns start wherever their leading dimension puts them: gfx950 takes global
// dwordx2/x4 accesses at any byte, and a row that starts inside a 16-byte unit costs no second instruction.
template <typename T, int V> struct Vec {
    static constexpr int kWords = V * (int)sizeof(T) / 4;
    uint32_t w[kWords];
};

template <int N> struct Chunk;             // words moved per instruction
template <> struct Chunk<1> { static constexpr int value = 1; };
template <> struct Chunk<2> { static constexpr int value = 2; };
template <> struct Chunk<4> { static constexpr int value = 4; };
template <> struct Chunk<8> { static constexpr int value = 4; };

// NT: with the non-temporal hint.
template <typename T, int V, bool NT> __device__ __forceinline__ Vec<T, V> load_vec(const T* p)
{
    constexpr int C = Chunk<Vec<T, V>::kWords>::value;
    typedef typename Bits<C * 4>::type W;
    Vec<T, V> r;
#pragma unroll
    for (int i = 0; i < Vec<T, V>::kWords / C; ++i) {
        const W* from = reinterpret_cast<const W*>(p) + i;
        const W x = NT ? __builtin_nontemporal_load(from) : *from;
        __builtin_memcpy(r.w + i * C, &x, sizeof(x));
    }
    return r;
}

template <typename T, int V, bool NT> __device__ __forceinline__ void store_vec(T* p, const Vec<T, V>& r)
{
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

// The same for the last vector of a row, of which `n` < V elements are there: one by one, so that nothing outside the
// row is touched and no element is written twice.
template <typename T, int V> __device__ __forceinline__ Vec<T, V> load_some(const T* p, int n)
{
    T e[V] = {};
    for (int i = 0; i < V; ++i)
        if (i < n) e[i] = p[i];
    Vec<T, V> r;
    __builtin_memcpy(r.w, e, sizeof(r.w));
    return r;
}

template <typename T, int V> __device__ __forceinline__ void store_some(T* p, const Vec<T, V>& r, int n)
{
    T e[V];
    __builtin_memcpy(e, r.w, sizeof(r.w));
    for (int i = 0; i < V; ++i)
        if (i < n) p[i] = e[i];
}

template <typename T, int V, bool NT> __device__ __forceinline__ Vec<T, V> load_row(const T* p, int n)
{
    return n >= V ? load_vec<T, V, NT>(p) : load_some<T, V>(p, n);
}
template <typename T, int V, bool NT> __device__ __forceinline__ void store_row(T* p, const Vec<T, V>& r, int n)
{
    if (n >= V) store_vec<T, V, NT>(p, r); else store_some<T, V>(p, r, n);
}

// Widening is exact.
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

// One rounding, to nearest even; in 8 bits what is larger than 448 becomes 448 (the format has no infinity) and a NaN
// stays one.
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
__device__ __forceinline__ float cut_f8(float x)
{
    const float c = __builtin_fminf(__builtin_fmaxf(x, -448.f), 448.f);
    return x != x ? x : c;
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

// A launch dimension may count at most 2^32 work items: blocks beyond 2^20 go into the second dimension.
constexpr uint32_t kGridRow = 1u << 20;
__device__ __forceinline__ uint32_t block_id() { return blockIdx.y * kGridRow + blockIdx.x; }

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
