// Attention over pages: the launches, and the kernel that joins the parts of a row's positions (see ttc_attend.h).
#include <type_traits>

#include "ttc_attention_internal.h"
#include "ttc_moves_device.h"

namespace ttc {
namespace {

// A wavefront a row: its partial results, weighted by their share of all exponentials.  Rows of one part have been written, and so have, by
// nobody, those before the first and behind the last request.  A chain of loads (requests, parts, sums, results) bounds it: 3 us for a token of 8 heads.
// So the first parts' results are loaded beside their sums, kBatch of them at a time (96 tokens of 32 heads 5.4 us; four at a time behind the sums 6.8, and 9.9 instead
// of 5.8 where rows have up to 13).
template <typename T, int EACH>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs p)
{
    touch<AttendArgs>();
    constexpr uint32_t kBatch = EACH > 2 ? 8 : 16;
    static_assert(kAttendMaxParts == 2 * kWave, "two to a lane");
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
    PartSum mine[kAttendMaxParts / kWave];
    float top = -__builtin_inff();
#pragma unroll
    for (uint32_t c = 0; c < kAttendMaxParts / kWave; ++c) {
        const uint32_t i = c * kWave + lane;
        mine[c] = p.partial_sums[place(i < parts ? i : 0)];
    }
    float part[kBatch][EACH];
    auto load = [&](uint32_t from) {
#pragma unroll
        for (uint32_t s = 0; s < kBatch; ++s) {
            const float* there = p.partial + (int64_t)place(from + s < parts ? from + s : 0) * p.dim;
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                const uint32_t d = e * kWave + lane;
                part[s][e] = there[d < p.dim ? d : 0];
            }
        }
    };
    load(0);
#pragma unroll
    for (uint32_t c = 0; c < kAttendMaxParts / kWave; ++c) {
        if (c * kWave + lane >= parts) mine[c] = {-__builtin_inff(), 0.f};
        top = __builtin_fmaxf(top, mine[c].top);
    }
    for (int i = 1; i < kWave; i <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, i));
    const float base = top == -__builtin_inff() ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (uint32_t c = 0; c < kAttendMaxParts / kWave; ++c) {
        mine[c].sum *= __builtin_amdgcn_exp2f(mine[c].top - base);
        sum += mine[c].sum;
    }
    for (int i = 1; i < kWave; i <<= 1) sum += __shfl_xor(sum, i);
    const float inverse = sum == 0.f ? 0.f : 1.f / sum;
    float x[EACH] = {};
    for (uint32_t from = 0; from < parts; from += kBatch) {
        if (from) load(from);
#pragma unroll
        for (uint32_t s = 0; s < kBatch; ++s) {
            const uint32_t i = from + s;
            const float weight = __shfl(i < kWave ? mine[0].sum : mine[1].sum, i % kWave) * inverse;          // 0 behind the last part
#pragma unroll
            for (int e = 0; e < EACH; ++e) x[e] = weight == 0.f ? x[e] : __builtin_fmaf(weight, part[s][e], x[e]);        // nothing seen, or nothing left of it
        }
    }
    T* out = static_cast<T*>(p.out) + (int64_t)token * p.ld_o + (int64_t)head * p.dim;
#pragma unroll
    for (int e = 0; e < EACH; ++e)
        if (e * kWave + lane < p.dim) out[e * kWave + lane] = (T)x[e];
    if (p.lse && lane == 0) p.lse[row] = log_of_sum(top, sum, attend_lift(std::is_same<T, _Float16>::value ? TTC_F16 : TTC_F32));
}

template <typename T> const void* join_of(uint32_t dim)
{
    return dim <= 64 ? reinterpret_cast<const void*>(&join_kernel<T, 1>) : dim <= 128 ? reinterpret_cast<const void*>(&join_kernel<T, 2>)
                                                                                       : reinterpret_cast<const void*>(&join_kernel<T, TTC_ATTEND_MAX_DIM / kWave>);
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
    const void* join = a.dtype == TTC_F32 ? join_of<float>(p.dim) : a.dtype == TTC_BF16 ? join_of<__bf16>(p.dim) : join_of<_Float16>(p.dim);
    return launch_blocks(join, ((uint64_t)p.tokens * p.q_heads + 3) / 4, 256, 0, &p, stream);
}

}  // namespace ttc
