// Host part of the heads and the attention under AddressSanitizer and UndefinedBehaviorSanitizer (see test_attention_host.py): every entry point with
// sizes from nothing to the ends of their types, and launchers in place of the kernels that look at what they are handed.
#include <cstdio>
#include <cstdlib>
#include <initializer_list>

#include "ttc_attention_internal.h"

static int failures = 0, launched = 0;
#define CHECK(x) do { if (!(x)) { if (failures < 20) std::printf("%s:%d: %s\n", __FILE__, __LINE__, #x); ++failures; } } while (0)

namespace ttc {

int launch_sort(const SortArgs&, const SortShape&, void*) { return TTC_OK; }
int launch_gather(const RowArgs&, void*) { return TTC_OK; }
int launch_combine(const RowArgs&, void*) { return TTC_OK; }
int launch_combine_grad(const RowArgs&, void*) { return TTC_OK; }
int launch_map(const MapArgs&, void*) { return TTC_OK; }
int launch_write(const SlotArgs&, void*) { return TTC_OK; }
int launch_read(const SlotArgs&, void*) { return TTC_OK; }

static int heads_move(const HeadsArgs& a, int groups)
{
    ++launched;
    HeadsArgs p = a;
    const HeadsShape s = cut_heads(p, groups);
    const uint32_t all = p.q_groups + p.k_groups + p.v_groups;
    CHECK(s.groups >= (a.tokens ? 1 : 0) && s.groups <= groups);
    CHECK(p.lanes_log >= 0 && p.lanes_log <= 6 && all >= 1 && (uint64_t)p.per_wave * s.splits >= all && (s.splits - 1) * (uint64_t)p.per_wave < all);
    CHECK((__int128)a.tokens * s.splits <= INT32_MAX);                       // items are counted in 32 bits
    // every element of a head has a unit, in no more than four rounds of the lanes
    const uint32_t lanes = 1u << p.lanes_log;
    CHECK(s.vec == 1 ? (uint64_t)lanes * 4 * 2 >= p.dim : (uint64_t)lanes * 2 * (uint32_t)s.vec >= p.dim || p.paired == 0);
    CHECK(a.cache_dtype != TTC_Q4 || s.vec == 8);
    return TTC_OK;
}
int launch_heads(const HeadsArgs& a, void*) { return heads_move(a, kHeadsGroups); }
int launch_heads_grad(const HeadsArgs& a, void*) { return a.tokens ? heads_move(a, kGradGroups) : TTC_OK; }

int launch_attend(const AttendArgs& a, const AttendShape& s, void*)
{
    ++launched;
    CHECK(s.tile == 16 || s.tile == 32 || s.tile == (uint32_t)kTileMany);
    CHECK(s.slots >= 1 && (uint64_t)s.slots * s.tile + s.tile > (uint64_t)a.tokens * a.group);
    CHECK((uint64_t)a.tokens * a.q_heads <= INT32_MAX / 4 && a.q_heads == a.heads * a.group && a.heads <= 65535);
    CHECK(s.partial_rows >= 0 && s.partial_rows <= INT32_MAX && (s.partial_rows == 0) == (a.partial == nullptr));
    if (s.tile < (uint32_t)kTileMany) {
        CHECK(s.shares >= a.heads && s.shares % a.heads == 0 && s.splits == 1);
        CHECK(s.partial_rows == 0 || s.partial_rows == 2 * (int64_t)s.shares * s.tile);
    } else {
        CHECK(s.splits >= 1 && s.splits <= (uint32_t)kAttendMaxSplits && s.splits <= kAttendMaxParts);
        CHECK(s.partial_rows == 0 || s.partial_rows == (int64_t)s.slots * a.heads * s.splits * s.tile);
    }
    return TTC_OK;
}

}  // namespace ttc

int main()
{
    using namespace ttc;
    auto at = [](uint64_t place) { return reinterpret_cast<void*>((uintptr_t)(place << 56)); };       // far apart, never read
    auto f = [&](uint64_t place) { return static_cast<float*>(at(place)); };
    auto n32 = [&](uint64_t place) { return static_cast<int32_t*>(at(place)); };
    const int64_t sizes[] = {INT64_MIN, -1, 0, 1, 3, 17, 64, 96, 128, 256, 257, 512, 513, 70000, (int64_t)1 << 20, ((int64_t)1 << 20) + 1, INT32_MAX, (int64_t)1 << 40, INT64_MAX};
    static double angles[TTC_HEADS_MAX_ROTATED / 2];
    for (int i = 0; i < TTC_HEADS_MAX_ROTATED / 2; ++i) angles[i] = i * 0.37 - 5;
    for (int dtype : {(int)TTC_F32, (int)TTC_BF16, (int)TTC_F16, (int)TTC_F8, -1})
        for (int64_t hq : sizes)
            for (int64_t dim : sizes)
                for (int64_t rotated : {(int64_t)-2, (int64_t)0, (int64_t)2, (int64_t)7, (int64_t)64, (int64_t)256, (int64_t)258})
                    for (int mode = 0; mode < 4; ++mode) {
                        ttc_heads_t h = ttc_heads_create(dtype, hq, 3, dim, rotated, mode & 1, angles, mode & 2, 1e-6f);
                        CHECK((h == nullptr) == (ttc_last_status() != TTC_OK));
                        if (!h) continue;
                        for (int64_t tokens : sizes)
                            for (int64_t ld : {hq * dim - 1, hq * dim, INT64_MAX}) {
                                const int64_t work = ttc_heads_workspace(h, tokens), lk = 3 * dim;
                                const int a = ttc_heads_rotate(h, tokens, n32(1), at(2), ld, at(3), lk, nullptr, nullptr, at(4), hq * dim, at(5), lk, nullptr);
                                const int b = ttc_heads_rotate_grad(h, tokens, n32(1), at(2), hq * dim, at(3), lk, at(4), ld, at(5), lk, nullptr, nullptr, at(6), hq * dim, at(7), lk,
                                                                    mode & 2 ? f(8) : nullptr, nullptr, at(9), nullptr);
                                CHECK(work >= 0 || (a != TTC_OK && b != TTC_OK));
                                CHECK(ld >= hq * dim || work < 0 || a == TTC_ERR_INVALID_VALUE);
                            }
                        for (int cache : {dtype, (int)TTC_F8, (int)TTC_Q4}) {
                            ttc_pages_t p = ttc_pages_create(dtype, cache, 3, dim, 16, 100, nullptr);
                            if (!p) continue;
                            for (int64_t tokens : sizes)
                                (void)ttc_pages_append(p, h, tokens, n32(1), n32(2), at(3), hq * dim, at(4), 3 * dim, at(5), 3 * dim, nullptr, nullptr, at(6), hq * dim, at(7), at(8), nullptr, nullptr, nullptr);
                            ttc_pages_destroy(p);
                        }
                        ttc_heads_destroy(h);
                    }
    for (int64_t heads : {(int64_t)1, (int64_t)2, (int64_t)7, (int64_t)300, (int64_t)65535, (int64_t)65536})
        for (int64_t group : {(int64_t)1, (int64_t)4, (int64_t)33, (int64_t)1 << 19})
            for (int64_t dim : {(int64_t)8, (int64_t)80, (int64_t)128, (int64_t)256, (int64_t)257})
                for (int cache : {(int)TTC_BF16, (int)TTC_F8, (int)TTC_Q4})
                    for (int64_t window : {(int64_t)-1, (int64_t)0, (int64_t)1, (int64_t)5000, INT64_MAX}) {
                        ttc_pages_t p = ttc_pages_create(TTC_BF16, cache, heads, dim, 16, 1000, nullptr);
                        if (!p) continue;
                        ttc_attend_t a = ttc_attend_create(p, heads * group, 0.1, window);
                        CHECK((a == nullptr) == (ttc_last_status() != TTC_OK));
                        ttc_pages_destroy(p);
                        if (!a) continue;
                        const int64_t width = heads * group * dim;
                        for (int64_t requests : sizes)
                            for (int64_t tokens : sizes)
                                for (int64_t blocks : {(int64_t)-1, (int64_t)0, (int64_t)1, (int64_t)100, (int64_t)1 << 27, INT64_MAX}) {
                                    const int64_t work = ttc_attend_workspace(a, requests, tokens, blocks);
                                    const int s = ttc_attend_pages(a, requests, tokens, at(1), width, n32(2), n32(3), n32(4), blocks, at(5), at(6), nullptr, nullptr, at(7), width, f(8), at(9), nullptr);
                                    CHECK(work >= 0 || s == (int)-work);
                                    CHECK(s == TTC_OK || work < 0 || s == TTC_ERR_ALIAS || s == TTC_ERR_OVERFLOW);      // tensors longer than the places are apart
                                }
                        ttc_attend_destroy(a);
                    }
    CHECK(launched > 1000);
    std::printf(failures ? "%d failures\n" : "attention driver ok (%d launches)\n", failures ? failures : launched);
    return failures != 0;
}
