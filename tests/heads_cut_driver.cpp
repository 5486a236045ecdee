// How the heads of a call are cut into lanes' units (ttc_attention.cpp, cut_heads), on the CPU: every element of a head is some unit's, once, and `full` is said
// only where every unit of every lane has both its vectors and every lane of a group a head: kernels then take what a lane has loaded as its own.
#include <cstdio>
#include <initializer_list>
#include <vector>

#include "ttc_attention_internal.h"

namespace ttc {

int launch_sort(const SortArgs&, const SortShape&, void*) { return TTC_OK; }
int launch_gather(const RowArgs&, void*) { return TTC_OK; }
int launch_combine(const RowArgs&, void*) { return TTC_OK; }
int launch_combine_grad(const RowArgs&, void*) { return TTC_OK; }
int launch_map(const MapArgs&, void*) { return TTC_OK; }
int launch_write(const SlotArgs&, void*) { return TTC_OK; }
int launch_read(const SlotArgs&, void*) { return TTC_OK; }
int launch_heads(const HeadsArgs&, void*) { return TTC_OK; }
int launch_heads_grad(const HeadsArgs&, void*) { return TTC_OK; }
int launch_attend(const AttendArgs&, const AttendShape&, void*) { return TTC_OK; }

}  // namespace ttc

int main()
{
    using namespace ttc;
    int failures = 0;
    long full = 0, cuts = 0;
    auto fail = [&](const char* what, const HeadsArgs& a) {
        if (failures++ < 20) std::printf("%s: dtype %d cache %d dim %u rotated %u paired %d heads %u %u\n", what, a.dtype, a.cache_dtype, a.dim, a.rotated, a.paired, a.q_heads, a.kv_heads);
    };
    const int there = 0;
    for (int dtype : {(int)TTC_F32, (int)TTC_BF16, (int)TTC_F16})
        for (int cache : {-1, (int)TTC_Q4})
            for (uint32_t dim = 1; dim <= TTC_HEADS_MAX_DIM; ++dim)
                for (uint32_t rotated = 0; rotated <= dim && rotated <= TTC_HEADS_MAX_ROTATED; rotated += 2)
                    for (int paired = 0; paired < 2; ++paired)
                        for (uint32_t heads : {1u, 6u, 64u}) {
                            if (cache == TTC_Q4 && (dim % 8 || rotated % 16)) continue;
                            HeadsArgs a = {};
                            a.dtype = dtype; a.cache_dtype = cache; a.dim = dim; a.rotated = rotated; a.paired = paired;
                            a.tokens = 5; a.q_heads = heads; a.kv_heads = 64; a.q = a.k = &there;
                            const HeadsShape s = cut_heads(a, kHeadsGroups);
                            const uint32_t v = (uint32_t)s.vec, rounds = v > 1 ? 1 : kHeadsRounds, lanes = 1u << a.lanes_log, half = rotated / 2;
                            std::vector<int> of(dim, 0);
                            bool own = true;
                            for (uint32_t u = 0; u < lanes * rounds; ++u) {
                                uint32_t at, other;
                                if (paired) at = 2 * v * u, other = at + v;
                                else if (u * v < half) at = u * v, other = half + u * v;
                                else at = rotated + 2 * (u * v - half), other = at + v;
                                for (uint32_t first : {at, other}) {
                                    if (first >= dim) { own = false; continue; }
                                    for (uint32_t i = first; i < first + v; ++i)
                                        if (i < dim) ++of[i];
                                        else fail("a vector beyond the head", a);
                                }
                            }
                            for (int n : of)
                                if (n != 1) { fail("elements of no unit or of two", a); break; }
                            own = own && heads % (64 / lanes) == 0;
                            if (a.full && !own) fail("full, and lanes have nothing of their own", a);
                            if (!a.full && own) fail("not full, and every lane has its own", a);
                            full += a.full;
                            ++cuts;
                        }
    if (full == 0 || full == cuts) ++failures;
    std::printf(failures ? "%d failures\n" : "heads cut ok (%d)\n", failures);
    return failures != 0;
}
