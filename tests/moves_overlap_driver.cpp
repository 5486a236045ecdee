// What the host checks of the paged cache's moves say about tensors that overlap, against every byte of small ones (see test_moves_overlap.py).
// The launchers only say that the checks were passed.
#include <cstdint>
#include <cstdio>
#include <initializer_list>
#include <random>
#include <set>

#include "ttc_moves_internal.h"

static int failures = 0, accepted = 0, refused = 0;

namespace ttc {
int launch_sort(const SortArgs&, const SortShape&, void*) { return TTC_OK; }
int launch_gather(const RowArgs&, void*) { return TTC_OK; }
int launch_combine(const RowArgs&, void*) { return TTC_OK; }
int launch_combine_grad(const RowArgs&, void*) { return TTC_OK; }
int launch_map(const MapArgs&, void*) { return TTC_OK; }
int launch_write(const SlotArgs&, void*) { return TTC_OK; }
int launch_read(const SlotArgs&, void*) { return TTC_OK; }
}  // namespace ttc

static void* at(uint64_t place) { return reinterpret_cast<void*>((uintptr_t)place); }

static void expect(int status, bool meet, const char* what, int64_t a, int64_t b, int64_t c, int64_t d)
{
    ++(meet ? refused : accepted);
    if (status == (meet ? TTC_ERR_ALIAS : TTC_OK)) return;
    if (++failures < 20) std::printf("%s %lld %lld %lld %lld: status %d, shared %d\n", what, (long long)a, (long long)b, (long long)c, (long long)d, status, meet);
}

int main()
{
    using namespace ttc;
    std::mt19937 rng(7);
    auto pick = [&](int lo, int hi) { return (int64_t)(lo + (int)(rng() % (unsigned)(hi - lo + 1))); };
    const uint64_t base = 1 << 20, far = uint64_t(1) << 30;
    for (int round = 0; round < 300; ++round) {
        const int type = round % 3 == 0 ? TTC_F32 : TTC_BF16, cache = round % 3 == 1 ? TTC_F8 : type;
        const int eb = elem_bytes(type), cb = elem_bytes(cache);
        int64_t extent[3] = {pick(1, 3), pick(1, 4), pick(1, 4)}, stride[3], dim = pick(1, 5);
        int order[3] = {0, 1, 2};
        for (int i = 2; i > 0; --i) std::swap(order[i], order[rng() % (i + 1)]);
        int64_t span = dim;
        for (int i : order) {                             // strides in that order, with gaps now and then
            stride[i] = span * (rng() % 3 ? 1 : pick(1, 3)) + (rng() % 2 ? 0 : pick(0, 7));
            if (extent[i] > 1) span += stride[i] * (extent[i] - 1);
        }
        ttc_pages_t h = ttc_pages_create(type, cache, extent[0], dim, extent[1], extent[2], stride);
        if (!h) { ++failures; std::printf("no handle\n"); continue; }
        std::set<int64_t> held;
        for (int64_t p = 0; p < extent[2]; ++p)
            for (int64_t s = 0; s < extent[1]; ++s)
                for (int64_t e = 0; e < extent[0]; ++e)
                    for (int64_t c = 0; c < dim; ++c) held.insert(p * stride[2] + s * stride[1] + e * stride[0] + c);
        const int64_t row = extent[0] * dim;
        for (int64_t d = -span - 2; d <= span + 2; ++d) { // elements from keys to values
            bool meet = false;
            for (int64_t x : held) meet |= held.count(x + d) != 0;
            expect(ttc_pages_write(h, 3, (int32_t*)at(far), at(2 * far), row, at(3 * far), row, at(base), at(base + d * cb), nullptr, nullptr, nullptr), meet, "cache", d, stride[0], stride[1], stride[2]);
        }
        const int64_t tokens = pick(1, 5), ld = row + pick(0, 2 * (int)row + 3), other = rng() % 4 ? ld : row + pick(0, 9);
        for (int64_t d = -tokens * ld - 3; d <= tokens * ld + 3; ++d) {
            bool meet = false;
            for (int64_t i = 0; i < tokens; ++i)
                for (int64_t j = 0; j < tokens; ++j) {
                    const int64_t between = d + j * other - i * ld;
                    meet |= -row < between && between < row;
                }
            if (ld != other && tokens > 1) {              // two distances in one span are refused whether their rows meet or not
                const int64_t mine = (tokens - 1) * ld + row, yours = (tokens - 1) * other + row;
                meet = d < mine && -d < yours;
            }
            expect(ttc_pages_read(h, tokens, (int32_t*)at(far), at(2 * far), at(3 * far), nullptr, nullptr, at(base), ld, at(base + d * eb), other, nullptr), meet, "packed", d, row, ld, other);
        }
        ttc_pages_destroy(h);
    }
    // tensors without elements, inside of what the call writes
    ttc_pages_t h = ttc_pages_create(TTC_BF16, TTC_BF16, 2, 8, 4, 9, nullptr);
    int32_t *a = (int32_t*)at(base), *b = (int32_t*)at(2 * base), *c = (int32_t*)at(3 * base), *d = (int32_t*)at(4 * base), *e = (int32_t*)at(5 * base);
    expect(ttc_pages_map(h, 4, nullptr, a, b, c, 6, c + 3, 0, 0, d, e, d + 1, d + 2, e + 1, nullptr), false, "no tokens, no free pages", 0, 0, 0, 0);
    expect(ttc_pages_map(h, 4, nullptr, a, b, c, 6, c + 3, 1, 0, d, e, d + 1, d + 2, e + 1, nullptr), true, "a free page", 0, 0, 0, 0);
    expect(ttc_pages_map(h, 4, nullptr, a, b, c, 6, nullptr, 0, 1, d, e, d + 1, nullptr, nullptr, nullptr), true, "a token", 0, 0, 0, 0);
    expect(ttc_pages_map(h, 0, c + 1, c + 2, c + 3, c + 4, 6, nullptr, 0, 30, d, e, c, nullptr, nullptr, nullptr), false, "no requests", 0, 0, 0, 0);
    ttc_pages_destroy(h);
    ttc_route_t r = ttc_route_create(TTC_F32, 8, 2, 40, 0, 1, 8, nullptr, nullptr);
    expect(ttc_route_sort(r, 0, a + 2, 2, a, b, a + 5, b + 6, nullptr, nullptr), false, "nothing to sort", 0, 0, 0, 0);
    expect(ttc_route_sort(r, 1, a + 2, 2, a, b, c, d, nullptr, nullptr), true, "ids", 0, 0, 0, 0);
    ttc_route_destroy(r);
    std::printf(failures ? "%d failures\n" : "overlap driver ok (%d)\n", failures ? failures : accepted + refused);
    return failures != 0 || accepted < 3000 || refused < 3000;
}
