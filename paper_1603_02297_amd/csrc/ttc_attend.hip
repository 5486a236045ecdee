// Attention over pages: the launches, and the kernel that joins the parts of a row's positions (see ttc_attend.h).
#include "ttc_attention_internal.h"
#include "ttc_moves_device.h"

namespace ttc {
namespace {

// A wavefront a row: its partial results, weighted by their share of all exponentials.  Rows of one part have been written, and so have, by
// nobody, those before the first and behind the last request.  A chain of loads (requests, parts, sums, results) bounds it: 3 us for a token of 8 heads, 7 for 96 of 32.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs p)
{
    touch<AttendArgs>();
    constexpr int kEach = TTC_ATTEND_MAX_DIM / kWave;
    const uint32_t lane = threadIdx.x & (kWave - 1);
    const uint32_t row = __builtin_amdgcn_readfirstlane(block_id() * (256 / kWave) + threadIdx.x / kWave);
    if (row >= p.tokens * p.q_heads) return;
    const uint32_t token = row / p.q_heads, head = row - token * p.q_heads;
    const int32_t begin = p.starts[0], end = p.starts[p.requests], first = p.parts[2 * (int64_t)row], count = p.parts[2 * (int64_t)row + 1];
    if ((int64_t)token < begin || (int64_t)token >= end || count < 2) return;
    // starts that are no sums leave rows that nobody has, whose parts are whatever the workspace held
    const uint32_t parts = (uint32_t)count < kAttendMaxParts ? (uint32_t)count : kAttendMaxParts;
    auto place = [&](uint32_t i) {
        const uint32_t at = (uint32_t)first + (i ? i * p.join_step - p.join_back : 0);
        return at < p.partial_rows ? at : 0;
    };
    float mine[kAttendMaxParts / kWave], top = -__builtin_inff();
#pragma unroll
    for (uint32_t c = 0; c < kAttendMaxParts / kWave; ++c) {
        const uint32_t i = c * kWave + lane;
        mine[c] = i < parts ? p.partial_lse[place(i)] : -__builtin_inff();
        top = __builtin_fmaxf(top, mine[c]);
    }
    for (int i = 1; i < kWave; i <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, i));
    const float base = top == -__builtin_inff() ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (uint32_t c = 0; c < kAttendMaxParts / kWave; ++c) {
        mine[c] = __builtin_amdgcn_exp2f((mine[c] - base) * 1.44269504088896f);
        sum += mine[c];
    }
    for (int i = 1; i < kWave; i <<= 1) sum += __shfl_xor(sum, i);
    const float inverse = sum == 0.f ? 0.f : 1.f / sum;
    float x[kEach] = {};
#pragma unroll
    for (uint32_t c = 0; c < kAttendMaxParts / kWave; ++c) {
        if (c * kWave >= parts) break;
        const uint32_t some = parts - c * kWave < (uint32_t)kWave ? parts - c * kWave : kWave;
#pragma unroll 4
        for (uint32_t s = 0; s < some; ++s) {
            const float f = __shfl(mine[c], s) * inverse;
            const float* from = p.partial + (int64_t)place(c * kWave + s) * p.dim;
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const uint32_t d = j * kWave + lane;
                const float v = from[d < p.dim ? d : 0];
                x[j] = f == 0.f ? x[j] : __builtin_fmaf(f, v, x[j]);        // nothing seen, or nothing left of it
            }
        }
    }
    T* out = static_cast<T*>(p.out) + (int64_t)token * p.ld_o + (int64_t)head * p.dim;
#pragma unroll
    for (int j = 0; j < kEach; ++j)
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
    const int rc = launch_blocks(k.fn, s.tile < (uint32_t)kTileMany ? s.shares : (uint64_t)s.slots * p.heads * p.splits, k.threads, (size_t)k.lds, &p, stream);
    if (rc != TTC_OK || !s.partial_rows) return rc;
    const void* join = a.dtype == TTC_F32 ? reinterpret_cast<const void*>(&join_kernel<float>) : a.dtype == TTC_BF16 ? reinterpret_cast<const void*>(&join_kernel<__bf16>)
                                                                                              : reinterpret_cast<const void*>(&join_kernel<_Float16>);
    return launch_blocks(join, ((uint64_t)p.tokens * p.q_heads + 3) / 4, 256, 0, &p, stream);
}

}  // namespace ttc
