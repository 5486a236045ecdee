// Attention over pages: the launches, and the kernel that joins the parts of a row's positions (see ttc_attend.h).
#include "ttc_attention_internal.h"
#include "ttc_moves_device.h"

namespace ttc {
namespace {

// A wavefront a row: its parts' results, weighted by their share of all exponentials.  Rows of one part have been written, and so have, by
// nobody, those before the first and behind the last request.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs p)
{
    touch<AttendArgs>();
    const uint32_t lane = threadIdx.x & (kWave - 1);
    const uint32_t row = __builtin_amdgcn_readfirstlane(block_id() * (256 / kWave) + threadIdx.x / kWave);
    if (row >= p.tokens * p.q_heads) return;
    const uint32_t token = row / p.q_heads, head = row - token * p.q_heads;
    if ((int64_t)token < p.starts[0] || (int64_t)token >= p.starts[p.requests]) return;
    const uint32_t parts = (uint32_t)p.parts[row];
    if (parts < 2 || parts > p.splits) return;
    const float mine = lane < parts ? p.partial_lse[(int64_t)row * p.splits + lane] : -__builtin_inff();
    float top = mine;
    for (int i = 1; i < kWave; i <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, i));
    const float base = top == -__builtin_inff() ? 0.f : top;
    const float weight = __builtin_amdgcn_exp2f((mine - base) * 1.44269504088896f);
    float sum = weight;
    for (int i = 1; i < kWave; i <<= 1) sum += __shfl_xor(sum, i);
    const float share = sum == 0.f ? 0.f : weight / sum;
    T* out = static_cast<T*>(p.out) + (int64_t)token * p.ld_o + (int64_t)head * p.dim;
    const float* from = p.partial + (int64_t)row * p.splits * p.dim;
    float x[TTC_ATTEND_MAX_DIM / kWave] = {};
    for (uint32_t s = 0; s < parts; ++s) {
        const float f = __shfl(share, s);
        if (f == 0.f) continue;                                             // nothing seen, or nothing left of it
#pragma unroll
        for (int j = 0; j < TTC_ATTEND_MAX_DIM / kWave; ++j)
            if (j * kWave + lane < p.dim) x[j] = __builtin_fmaf(f, from[(int64_t)s * p.dim + j * kWave + lane], x[j]);
    }
#pragma unroll
    for (int j = 0; j < TTC_ATTEND_MAX_DIM / kWave; ++j)
        if (j * kWave + lane < p.dim) out[j * kWave + lane] = (T)x[j];
    if (p.lse && lane == 0) p.lse[row] = sum == 0.f ? -__builtin_inff() : base + __builtin_logf(sum);
}

}  // namespace

int launch_attend(const AttendArgs& a, const AttendShape& s, void* stream)
{
    const AttendKernel k = a.dtype == TTC_F32 ? attend_kernel_f32(a.cache_dtype, (int)a.dim, (int)s.tile) : a.dtype == TTC_BF16 ? attend_kernel_bf16(a.cache_dtype, (int)a.dim, (int)s.tile)
                                                                                                    : attend_kernel_f16(a.cache_dtype, (int)a.dim, (int)s.tile);
    // more than 64 KB of dynamic LDS has to be asked for, once per kernel and device
    if (k.lds > 64 * 1024) {
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return TTC_ERR_HIP;
        if (!((k.raised->load(std::memory_order_acquire) >> dev) & 1u)) {
            if (hipFuncSetAttribute(k.fn, hipFuncAttributeMaxDynamicSharedMemorySize, k.lds) != hipSuccess) return TTC_ERR_HIP;
            k.raised->fetch_or(uint64_t(1) << dev, std::memory_order_release);
        }
    }
    AttendArgs p = a;
    void* list[] = {&p};
    // x: the tiles; y: heads of the cache (at most 65535 by the handle); z: parts
    if (hipLaunchKernel(k.fn, dim3(s.slots, p.heads, p.splits), dim3(k.threads), list, (size_t)k.lds, (hipStream_t)stream) != hipSuccess) return TTC_ERR_HIP;
    if (p.splits < 2) return TTC_OK;
    const void* join = a.dtype == TTC_F32 ? reinterpret_cast<const void*>(&join_kernel<float>) : a.dtype == TTC_BF16 ? reinterpret_cast<const void*>(&join_kernel<__bf16>)
                                                                                              : reinterpret_cast<const void*>(&join_kernel<_Float16>);
    return launch_blocks(join, ((uint64_t)p.tokens * p.q_heads + 3) / 4, 256, 0, &p, stream);
}

}  // namespace ttc
