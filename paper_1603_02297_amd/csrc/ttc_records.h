// Vectors in 4 bits (TTC_Q4): a step and a minimum in bf16, then a code of four bits for every element.
#pragma once

#include "ttc_moves_device.h"

namespace ttc {

struct q4 { uint8_t bits; };               // a byte of a record

__device__ __forceinline__ void store_word(uint8_t* p, uint32_t w)
{
    *reinterpret_cast<typename Bits<4>::type*>(p) = w;
}
__device__ __forceinline__ uint32_t load_word(const uint8_t* p)
{
    return *reinterpret_cast<const typename Bits<4>::type*>(p);
}

// (x - low) / step, rounded as the division itself: halves between two codes are quotients that 32 bits hold, and stay halves.  With r = 1 / step rounded
// once, q = d * r is off by two units at most, and q - (q * step - d) * r rounds the quotient; steps outside 2^-60 .. 2^60, where r or the remainder
// could leave the normal range, take the division.
struct Record {
    float step, low, inverse;
    __device__ __forceinline__ uint32_t head() const
    {
        return __builtin_bit_cast(uint32_t, step) >> 16 | (__builtin_bit_cast(uint32_t, low) & 0xffff0000u);
    }
    __device__ __forceinline__ uint32_t codes(const float* x) const       // eight elements, the first in the lowest bits
    {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = x[i] - low, q = d * inverse;
            const float exact = inverse != 0.f ? __builtin_fmaf(-__builtin_fmaf(q, step, -d), inverse, q) : step > 0.f ? d / step : 0.f;
            // a NaN (a record of NaN) becomes 0
            w |= (uint32_t)__builtin_fminf(__builtin_fmaxf(__builtin_rintf(exact), 0.f), 15.f) << (4 * i);
        }
        return w;
    }
};

// The smallest and the largest of a vector's elements, first a lane's own.
struct RecordRange {
    float low = __builtin_inff(), high = -__builtin_inff();
    bool  bad = false;
    __device__ __forceinline__ void take(const float* x, int n)
    {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            low = __builtin_fminf(low, x[i]);
            high = __builtin_fmaxf(high, x[i]);
            bad |= !(__builtin_fabsf(x[i]) <= 3.3895313892515355e38f);       // the largest of bf16; a NaN, which the two above pass over, too
        }
    }
    // over the 2^log lanes that share a vector
    __device__ __forceinline__ Record record(int log)
    {
        float h = bad ? __builtin_inff() : high;
        for (int i = 0; i < log; ++i) {
            low = __builtin_fminf(low, __shfl_xor(low, 1 << i));
            h = __builtin_fmaxf(h, __shfl_xor(h, 1 << i));
        }
        // towards minus infinity, and the step towards plus: magnitudes are cut, or raised to the next
        const uint32_t l = __builtin_bit_cast(uint32_t, low);
        Record r;
        r.low = __builtin_bit_cast(float, (l >> 31 ? l + 0xffffu : l) & 0xffff0000u);
        r.step = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, (h - r.low) / 15.f) + 0xffffu) & 0xffff0000u);
        if (!(r.step < __builtin_inff()) || !(h < __builtin_inff())) r.step = r.low = __builtin_nanf("");
        r.inverse = r.step >= 0x1p-60f && r.step <= 0x1p60f ? 1.f / r.step : 0.f;
        return r;
    }
};

// Eight elements of a record: its head, and the word of their codes.
__device__ __forceinline__ void widen_record(uint32_t head, uint32_t word, float* x)
{
    const float step = __builtin_bit_cast(float, head << 16), low = __builtin_bit_cast(float, head & 0xffff0000u);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf((float)(word >> (4 * i) & 15u), step, low);
}

}  // namespace ttc
