// Host part of the moves by data under AddressSanitizer and UndefinedBehaviorSanitizer (see test_moves_host.py): every entry point with
// sizes from nothing to the ends of their types, and launchers in place of the kernels that look at what they are handed.
#include <cinttypes>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "ttc_moves_internal.h"

static int failures = 0;
#define CHECK(x) do { if (!(x)) { std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x); ++failures; } } while (0)
static int launched = 0;

namespace ttc {

int launch_sort(const SortArgs& a, const SortShape& s, void*)
{
    ++launched;
    CHECK(s.threads % kWave == 0 && s.threads <= kSortThreads && s.blocks >= 1 && s.blocks <= kSortBlocks);
    CHECK(s.chunk == (int64_t)s.threads * s.blocks && s.chunks >= 1 && s.chunks <= INT32_MAX);
    CHECK(s.chunks * s.chunk >= (int64_t)a.n && (s.chunks - 1) * s.chunk < (int64_t)a.n + (a.n == 0));
    CHECK(s.threads >= a.experts);                       // a thread for every expert
    CHECK(s.chunks == 1 || s.threads == kSortThreads);
    CHECK(s.chunks > 1 || s.blocks <= kSortOneBlocks);   // the forms that are built
    CHECK(a.n <= INT32_MAX && a.rows >= a.n && a.rows <= INT32_MAX);
    CHECK(s.chunks == 1 || a.hist != nullptr);
    for (uint32_t x : {0u, 1u, a.n / 2, a.n}) CHECK((uint32_t)((((uint64_t)x * a.topk_div.mul) >> 32) + x) >> a.topk_div.shift == x / (uint32_t)a.topk);
    return TTC_OK;
}
static int row_move(const RowArgs& a)
{
    ++launched;
    CHECK(a.tokens >= 1 && a.width >= 1 && a.row_count >= (uint64_t)a.tokens * a.topk && a.position != nullptr);
    return TTC_OK;
}
int launch_gather(const RowArgs& a, void*) { return row_move(a); }
int launch_combine(const RowArgs& a, void*) { return row_move(a); }
int launch_combine_grad(const RowArgs& a, void*) { return row_move(a); }
int launch_map(const MapArgs& a, void*)
{
    ++launched;
    CHECK(a.requests >= 0 && a.tokens >= 0 && a.free_count >= 0 && a.starts && a.page_starts && a.pages >= 1);
    return TTC_OK;
}
static int slot_move(const SlotArgs& a)
{
    ++launched;
    CHECK(a.tokens >= 1 && a.slot_count >= 1 && a.slot_count <= INT32_MAX && a.heads >= 1 && a.dim >= 1 && (uint64_t)a.heads * a.dim <= INT32_MAX / 2);
    // the last element of the last slot is where 64 bits reach
    const __int128 last = (__int128)((a.slot_count - 1) / a.page.div) * a.stride_page + (__int128)(a.page.div - 1) * a.stride_slot + (__int128)(a.heads - 1) * a.stride_head + a.dim - 1;
    CHECK(last >= 0 && last < ((__int128)1 << 60));
    return TTC_OK;
}
int launch_write(const SlotArgs& a, void*) { return slot_move(a); }
int launch_read(const SlotArgs& a, void*) { return slot_move(a); }

}  // namespace ttc

int main()
{
    using namespace ttc;
    const int64_t sizes[] = {INT64_MIN, -1, 0, 1, 2, 3, 63, 64, 1000, 65536, INT32_MAX / 2, INT32_MAX, (int64_t)INT32_MAX + 1, (int64_t)1 << 40, INT64_MAX / 2, INT64_MAX};
    const float half = 0.5f;
    auto at = [](uint64_t place) { return reinterpret_cast<void*>((uintptr_t)(place << 56)); };       // far apart, never read
    for (int dtype : {0, 1, 8, 9, 10, -3})
        for (int64_t width : sizes)
            for (int topk : {-1, 0, 1, 7, 64, 65, INT32_MAX})
                for (int experts : {0, 1, 1024, 1025}) {
                    for (int align : {1, 128, 65536, 65537}) {
                        ttc_route_t r = ttc_route_create(dtype, width, topk, experts, 5, align, 8, &half, nullptr);
                        CHECK((r == nullptr) == (ttc_last_status() != TTC_OK));
                        if (!r) continue;
                        for (int64_t tokens : sizes) {
                            const int64_t rows = ttc_route_rows(r, tokens), work = ttc_route_workspace(r, tokens);
                            CHECK((rows < 0) == (work < 0));
                            for (int64_t ld : {width - 1, width, width + 1, (int64_t)1 << 40, INT64_MAX}) {
                                const int a = ttc_route_gather(r, tokens, at(1), ld, nullptr, (int32_t*)at(2), (int32_t*)at(3), (int32_t*)at(4), at(5), ld, nullptr);
                                const int b = ttc_route_combine(r, tokens, at(1), ld, (float*)at(6), (int32_t*)at(2), at(5), ld, nullptr);
                                const int c = ttc_route_combine_grad(r, tokens, at(1), ld, at(7), ld, (float*)at(6), (int32_t*)at(2), (int32_t*)at(3), (int32_t*)at(4), at(5), ld, (float*)at(8), nullptr);
                                CHECK(rows >= 0 || (a != TTC_OK && b != TTC_OK && c != TTC_OK));
                                CHECK(ld >= width || rows < 0 || (a == TTC_ERR_INVALID_VALUE && b == a && c == a));
                            }
                            const int s = ttc_route_sort(r, tokens, at(1), topk, (int32_t*)at(2), (int32_t*)at(3), (int32_t*)at(4), (int32_t*)at(5), at(6), nullptr);
                            CHECK((rows >= 0) == (s == TTC_OK));
                        }
                        ttc_route_destroy(r);
                    }
                }
    for (int64_t heads : {(int64_t)0, (int64_t)1, (int64_t)8, (int64_t)1 << 20, (int64_t)1 << 40})
        for (int64_t dim : sizes)
            for (int64_t page : sizes)
                for (int64_t pages : sizes)
                    for (int64_t extra : {(int64_t)-1, (int64_t)0, (int64_t)3, (int64_t)1 << 38, INT64_MAX}) {
                        const bool small = dim >= 1 && dim < ((int64_t)1 << 31) && page >= 1 && page < ((int64_t)1 << 31) && heads < ((int64_t)1 << 21);
                        int64_t stride[3] = {extra, extra, extra};
                        if (small && extra < INT64_MAX) {
                            __int128 h = (__int128)dim + extra, s = h * (heads ? heads : 1), p = s * page;
                            stride[0] = (int64_t)h; stride[1] = s < INT64_MAX ? (int64_t)s : INT64_MAX; stride[2] = p < INT64_MAX ? (int64_t)p : INT64_MAX;
                        }
                        ttc_pages_t c = ttc_pages_create(TTC_BF16, TTC_F8, heads, dim, page, pages, extra == 0 ? nullptr : stride);
                        CHECK((c == nullptr) == (ttc_last_status() != TTC_OK));
                        if (!c) continue;
                        for (int64_t tokens : {(int64_t)-1, (int64_t)0, (int64_t)1, (int64_t)INT32_MAX, (int64_t)1 << 33})
                            for (int64_t ld : {heads * dim - 1, heads * dim, INT64_MAX}) {
                                const int w = ttc_pages_write(c, tokens, (int32_t*)at(1), at(2), ld, at(3), ld, at(4), at(5), (float*)at(6), (float*)at(7), nullptr);
                                const int q = ttc_pages_read(c, tokens, (int32_t*)at(1), at(4), at(5), (float*)at(6), (float*)at(7), at(2), ld, at(3), ld, nullptr);
                                CHECK(w == q || w == TTC_ERR_ALIAS || q == TTC_ERR_ALIAS);      // tensors longer than the places are apart
                                CHECK(ld >= heads * dim || w == TTC_ERR_INVALID_VALUE);
                            }
                        for (int64_t n : sizes)
                            (void)ttc_pages_map(c, n, nullptr, (int32_t*)at(1), (int32_t*)at(2), (int32_t*)at(3), n, (int32_t*)at(4), n, n, (int32_t*)at(5), (int32_t*)at(6), (int32_t*)at(7), nullptr, (int32_t*)at(8), nullptr);
                        ttc_pages_destroy(c);
                    }
    CHECK(launched > 1000);
    std::printf(failures ? "%d failures\n" : "moves driver ok (%d launches)\n", failures ? failures : launched);
    return failures != 0;
}
