// Host part of the heads and the attention (include/ttc_attention.h): handles, sizes, and the checks of every call.
// No HIP here: what passes these checks goes to the launchers in ttc_heads.hip and ttc_attend.hip.
#include <algorithm>
#include <cmath>
#include <new>

#include "ttc_attention_internal.h"
#include "ttc_moves_checks.h"

namespace ttc {

HeadsShape cut_heads(HeadsArgs& a, int groups)
{
    HeadsShape s = {};
    const uint32_t wide = a.cache_dtype == TTC_Q4 ? 8 : 16 / elem_bytes(a.dtype), half = a.rotated / 2, rest = a.dim - a.rotated;
    // whole vectors on both sides of every unit, or element by element
    const bool whole = a.paired ? a.rotated % (2 * wide) == 0 && a.dim % wide == 0 : half % wide == 0 && rest % wide == 0;
    const uint32_t vec = whole ? wide : 1;
    const uint32_t units = a.paired ? (a.dim + 2 * vec - 1) / (2 * vec) : half / vec + (rest + 2 * vec - 1) / (2 * vec);
    a.lanes_log = 0;
    while ((1u << a.lanes_log) < units && a.lanes_log < 6) ++a.lanes_log;
    const uint32_t each = 64u >> a.lanes_log;
    a.full = units == (vec > 1 ? 1u : (uint32_t)kHeadsRounds) << a.lanes_log && a.dim % (2 * vec) == 0 && (a.paired || rest % (2 * vec) == 0) && (!a.q || a.q_heads % each == 0) && ((!a.k && !a.v) || a.kv_heads % each == 0);
    a.q_groups = a.q ? (a.q_heads + each - 1) / each : 0;
    a.k_groups = a.k ? (a.kv_heads + each - 1) / each : 0;
    a.v_groups = a.v ? (a.kv_heads + each - 1) / each : 0;
    // a wavefront for each token as long as that fills the launch, else its groups spread over several
    const uint32_t all = std::max<uint32_t>(a.q_groups + a.k_groups + a.v_groups, 1);
    const int64_t waves = (int64_t)groups * (kHeadsThreads / kWave), per = kHeadsThreads / kWave;
    const int64_t splits = std::min<int64_t>(std::max<int64_t>(waves / std::max<uint32_t>(a.tokens, 1), 1), all);
    a.per_wave = (uint32_t)((all + splits - 1) / splits);
    s.vec = (int)vec;
    s.splits = (all + a.per_wave - 1) / a.per_wave;
    a.split_div = make_fastdiv(s.splits);
    s.groups = (int)std::min<int64_t>(((int64_t)a.tokens * s.splits + per - 1) / per, groups);
    return s;
}

AttendShape attend_shape(const ttc_attend_s* a, int64_t requests, int64_t tokens, int64_t longest)
{
    AttendShape s = {};
    const int64_t heads = a->heads, rows = tokens * (a->q_heads / heads);
    // Rows of a tile, from how many rows a request has of a head on average.  Tiles of 16 and 32 rows: each wavefront has positions of its own; of many: each has rows
    // of its own, and all share the positions in LDS.  32 requests behind 8000 positions, heads of 128, in us with tiles of 16, 32 and many: 32 rows 232, 233, 246; 48
    // rows 570, 265, 222.  Codes of 4 bits, once widened in LDS, cost most with many (heads of 256, 48 rows: 449, 345, 643), and so do products in 32 bits (2000
    // positions, heads of 128, 48 rows: 282, 240, 320).  Where 32 rows do not fit the registers, 32 rows take 697 in tiles of 16 and 417 in many, in 32 bits 288 and 452.
    const int bytes = elem_bytes(a->dtype);
    const bool records = a->cache_dtype == TTC_Q4;
    if (rows <= 16 * requests) s.tile = 16;
    else if (attend_half(bytes, records, attend_dim((int)a->dim))) s.tile = rows <= (bytes == 4 || records ? 48 : 32) * requests ? 32 : kTileMany;
    else s.tile = bytes == 4 && rows <= 32 * requests ? 16 : kTileMany;
    // request r's tiles are numbered from starts[r] * group / tile + r on: always enough, and found without a sum over the requests
    s.slots = (uint32_t)(rows / s.tile + requests);
    const int64_t groups = std::max<int64_t>((int64_t)s.slots * heads, 1), units = std::max<int64_t>((longest + kAttendUnit - 1) / kAttendUnit, 1);
    if (s.tile < kTileMany) {
        // As many shares as workgroups fit the device at a time: 64 requests of 8000 positions in 16 bits take 5.7 TB/s, and less with one and a half, two or four
        // times as many.
        const int64_t most = 256 * attend_resident(bytes, attend_own(bytes, elem_bytes(a->cache_dtype), (int)a->dim, (int)s.tile), records, (int)a->dim, (int)s.tile);
        const int64_t each = std::max<int64_t>(most / heads, 1);               // of a head
        s.shares = (uint32_t)(heads * (s.slots >= each / units ? std::min<int64_t>(each, s.slots * units) : s.slots * units));
        s.splits = 1;
        s.partial_rows = units > 1 ? 2 * (int64_t)s.shares * s.tile : 0;
    } else {
        // where tiles alone do not fill the device, several workgroups share a tile's positions
        s.splits = (uint32_t)std::min<int64_t>({std::max<int64_t>(1024 / groups, 1), units, kAttendMaxSplits});
        s.partial_rows = s.splits > 1 ? groups * s.splits * s.tile : 0;
    }
    return s;
}

namespace {

constexpr int64_t kGradPartials = kGradGroups;

// Whether two tensors of `tokens` rows, wa and wb bytes long and lda and ldb elements apart, share a byte.  Rows of one distance are told apart exactly; of two
// distances in one span they are taken to meet.
bool rows_meet(const void* a, int64_t lda, int64_t wa, uint64_t span_a, const void* b, int64_t ldb, int64_t wb, uint64_t span_b, int64_t tokens, int eb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    if (!a || !b || !(x < y + span_b && y < x + span_a)) return false;
    if (tokens == 1 || lda != ldb) return true;
    const int64_t apart = (int64_t)(y - x), row = lda * eb, step = apart / row - (apart % row < 0);
    for (int64_t t = step; t <= step + 1; ++t) {
        const int64_t d = apart - t * row;  // from a's row to b's
        if (-tokens < t && t < tokens && -wb < d && d < wa) return true;
    }
    return false;
}

// One packed tensor of a call.
struct Rows {
    const void* p;
    int64_t     ld, width;                 // elements
    bool        written;
    int         in_place_of;               // index of the tensor that it may be, or -1
    uint64_t    span;
};

// Leading dimensions, spans, alignment, and that nothing written shares an element with another (but in its place).
template <int N> int check_rows(Rows (&r)[N], int64_t tokens, int eb)
{
    for (Rows& x : r)
        if (x.p && x.ld < x.width) return TTC_ERR_INVALID_VALUE;
    for (Rows& x : r)
        if (x.p && !span_bytes(tokens, x.ld, x.width, eb, &x.span)) return TTC_ERR_OVERFLOW;
    for (Rows& x : r)
        if (x.p && (uintptr_t)x.p % (uintptr_t)eb) return TTC_ERR_MISALIGNED;
    for (int i = 0; i < N; ++i)
        for (int j = 0; j < N; ++j) {
            if (i == j || !r[i].p || !r[j].p || !r[i].written) continue;
            if (r[i].in_place_of == j && r[i].p == r[j].p && r[i].ld == r[j].ld) continue;
            if (rows_meet(r[i].p, r[i].ld, r[i].width * eb, r[i].span, r[j].p, r[j].ld, r[j].width * eb, r[j].span, tokens, eb)) return TTC_ERR_ALIAS;
        }
    return TTC_OK;
}

// What is read or written beside the packed tensors: aligned, and apart from them where either is written.
struct Beside {
    const void* p;
    uint64_t    bytes;
    int         align;
    bool        written;
};
template <int N, int M> int check_beside(const Rows (&r)[N], const Beside (&b)[M])
{
    for (const Beside& x : b)
        if (x.p && (uintptr_t)x.p % (uintptr_t)x.align) return TTC_ERR_MISALIGNED;
    auto meet = [](const void* a, uint64_t an, const void* c, uint64_t cn) {
        return a && c && an && cn && (uintptr_t)a < (uintptr_t)c + cn && (uintptr_t)c < (uintptr_t)a + an;
    };
    for (int i = 0; i < M; ++i) {
        for (const Rows& x : r)
            if ((x.written || b[i].written) && meet(b[i].p, b[i].bytes, x.p, x.span)) return TTC_ERR_ALIAS;
        for (int j = 0; j < M; ++j)
            if (i != j && b[i].written && meet(b[i].p, b[i].bytes, b[j].p, b[j].bytes)) return TTC_ERR_ALIAS;
    }
    return TTC_OK;
}

HeadsArgs heads_args(const ttc_heads_s* h, int64_t tokens)
{
    HeadsArgs a = {};
    a.tokens = (uint32_t)tokens;
    a.q_heads = (uint32_t)h->q_heads;
    a.kv_heads = (uint32_t)h->kv_heads;
    a.dim = (uint32_t)h->dim;
    a.rotated = (uint32_t)h->rotated;
    a.dtype = h->dtype;
    a.cache_dtype = -1;
    a.paired = h->paired;
    a.norm = h->norm;
    a.eps = h->eps;
    std::copy(h->turns, h->turns + h->rotated / 2, a.turns);
    return a;
}

// Tokens times groups of heads are counted in 32 bits.
bool countable(const ttc_heads_s* h, int64_t tokens) { return tokens <= INT32_MAX && (__int128)tokens * (h->q_heads + 2 * h->kv_heads) <= INT32_MAX; }

// Rows of all heads are counted in 32 bits, and so are the tiles of them: as many as rows and requests of every head of the cache at most.
bool attend_sizes(const ttc_attend_s* a, int64_t requests, int64_t tokens, int64_t ld_table)
{
    return requests <= INT32_MAX / 4 && tokens <= INT32_MAX / 4 && (__int128)tokens * a->q_heads <= INT32_MAX / 4 &&
           (__int128)requests * a->heads + tokens * a->q_heads <= INT32_MAX && ld_table <= (int64_t)1 << 40;
}

// Positions that the rows of a tile see together, at most.
int64_t longest_context(const ttc_attend_s* a, int64_t tokens, int64_t ld_table)
{
    int64_t n;
    if (__builtin_mul_overflow(ld_table, a->page, &n)) n = INT32_MAX;
    n = std::min<int64_t>(n, INT32_MAX);
    return a->window ? std::min<int64_t>(n, a->window + std::max<int64_t>(tokens, kTileMany)) : n;
}

// An angle as a fraction of a turn in units of 2^-64, whole turns dropped.
uint64_t turn_of(double angle)
{
    const long double turns = (long double)angle / (2 * 3.14159265358979323846264338327950288L), part = turns - std::floor(turns);
    const long double scaled = std::floor(part * 18446744073709551616.0L + 0.5L);
    return scaled >= 18446744073709551616.0L ? 0 : (uint64_t)scaled;
}

}  // namespace
}  // namespace ttc

using namespace ttc;

extern "C" {

ttc_heads_t ttc_heads_create(int dtype, int64_t q_heads, int64_t kv_heads, int64_t dim, int64_t rotated, int paired, const double* angles,
                             int norm, float eps)
{
    int st = TTC_OK;
    if (!row_type(dtype)) st = TTC_ERR_UNSUPPORTED_DTYPE;
    else if (q_heads < 1 || kv_heads < 1 || dim < 1 || dim > TTC_HEADS_MAX_DIM || rotated < 0 || rotated > dim || rotated > TTC_HEADS_MAX_ROTATED || rotated % 2 ||
             (norm && !(eps >= 0.f && std::isfinite(eps))))
        st = TTC_ERR_INVALID_VALUE;
    else if (q_heads > (int64_t)1 << 20 || kv_heads > (int64_t)1 << 20) st = TTC_ERR_OVERFLOW;
    else if (rotated && !angles) st = TTC_ERR_NULL_POINTER;
    for (int64_t i = 0; st == TTC_OK && i < rotated / 2; ++i)
        if (!std::isfinite(angles[i])) st = TTC_ERR_INVALID_VALUE;
    ttc_heads_s* h = st == TTC_OK ? new (std::nothrow) ttc_heads_s : nullptr;
    if (st == TTC_OK && !h) st = TTC_ERR_ALLOC;
    if (h) {
        *h = {dtype, q_heads, kv_heads, dim, rotated, paired != 0, norm != 0, norm ? eps : 0.f, {}};
        for (int64_t i = 0; i < rotated / 2; ++i) h->turns[i] = turn_of(angles[i]);
    }
    set_last_status(st);
    return h;
}

int ttc_heads_destroy(ttc_heads_t heads)
{
    delete heads;
    return TTC_OK;
}

int ttc_heads_rotate(ttc_heads_t heads, int64_t tokens, const int32_t* positions, const void* q, int64_t ldq, const void* k, int64_t ldk,
                     const float* q_weight, const float* k_weight, void* q_out, int64_t ld_qo, void* k_out, int64_t ld_ko, void* stream)
{
    if (!heads) return TTC_ERR_NULL_POINTER;
    if (tokens < 0 || ((q_weight || k_weight) && !heads->norm)) return TTC_ERR_INVALID_VALUE;
    if (!countable(heads, tokens)) return TTC_ERR_OVERFLOW;
    const int64_t wq = heads->q_heads * heads->dim, wk = heads->kv_heads * heads->dim;
    if ((q && (ldq < wq || ld_qo < wq)) || (k && (ldk < wk || ld_ko < wk))) return TTC_ERR_INVALID_VALUE;
    if (tokens == 0) return TTC_OK;
    if (!q != !q_out || !k != !k_out || (!q && !k) || (heads->rotated && !positions)) return TTC_ERR_NULL_POINTER;
    const int eb = elem_bytes(heads->dtype);
    Rows rows[] = {{q, ldq, wq, false, -1, 0}, {k, ldk, wk, false, -1, 0}, {q_out, ld_qo, wq, true, 0, 0}, {k_out, ld_ko, wk, true, 1, 0}};
    int st = check_rows(rows, tokens, eb);
    const uint64_t bw = 4 * (uint64_t)heads->dim;
    if (st == TTC_OK)
        st = check_beside(rows, {Beside{positions, 4 * (uint64_t)tokens, 4, false}, {q ? q_weight : nullptr, bw, 4, false}, {k ? k_weight : nullptr, bw, 4, false}});
    if (st != TTC_OK) return st;
    HeadsArgs a = heads_args(heads, tokens);
    a.q = q; a.k = k; a.q_out = q_out; a.k_out = k_out;
    a.ld_q = ldq; a.ld_k = ldk; a.ld_qo = ld_qo; a.ld_ko = ld_ko;
    a.q_weight = q_weight; a.k_weight = k_weight; a.positions = positions;
    return launch_heads(a, stream);
}

int64_t ttc_heads_workspace(ttc_heads_t heads, int64_t tokens)
{
    if (!heads) return -TTC_ERR_NULL_POINTER;
    if (tokens < 0) return -TTC_ERR_INVALID_VALUE;
    if (!countable(heads, tokens)) return -TTC_ERR_OVERFLOW;
    return heads->norm && tokens ? kGradPartials * 2 * heads->dim * (int64_t)sizeof(float) : 0;
}

int ttc_heads_rotate_grad(ttc_heads_t heads, int64_t tokens, const int32_t* positions, const void* dq_out, int64_t ld_dqo, const void* dk_out,
                          int64_t ld_dko, const void* q, int64_t ldq, const void* k, int64_t ldk, const float* q_weight, const float* k_weight,
                          void* dq, int64_t ld_dq, void* dk, int64_t ld_dk, float* dq_weight, float* dk_weight, void* workspace, void* stream)
{
    if (!heads) return TTC_ERR_NULL_POINTER;
    if (tokens < 0 || ((q_weight || k_weight || dq_weight || dk_weight) && !heads->norm)) return TTC_ERR_INVALID_VALUE;
    if (!countable(heads, tokens)) return TTC_ERR_OVERFLOW;
    const int64_t wq = heads->q_heads * heads->dim, wk = heads->kv_heads * heads->dim;
    const bool norm = heads->norm;
    if ((dq_out && (ld_dqo < wq || ld_dq < wq || (norm && ldq < wq))) || (dk_out && (ld_dko < wk || ld_dk < wk || (norm && ldk < wk)))) return TTC_ERR_INVALID_VALUE;
    const bool sums = dq_weight || dk_weight;
    if (tokens && (!dq_out != !dq || !dk_out != !dk || (!dq && !dk) || (norm && dq && !q) || (norm && dk && !k) || (heads->rotated && !positions) || (sums && !workspace)))
        return TTC_ERR_NULL_POINTER;
    if ((dq_weight && !dq && tokens) || (dk_weight && !dk && tokens)) return TTC_ERR_NULL_POINTER;
    const int eb = elem_bytes(heads->dtype);
    const uint64_t bw = 4 * (uint64_t)heads->dim;
    Rows rows[] = {{norm && dq ? q : nullptr, ldq, wq, false, -1, 0}, {norm && dk ? k : nullptr, ldk, wk, false, -1, 0}, {dq_out, ld_dqo, wq, false, -1, 0},
                   {dk_out, ld_dko, wk, false, -1, 0}, {dq, ld_dq, wq, true, 2, 0}, {dk, ld_dk, wk, true, 3, 0}};
    int st = tokens ? check_rows(rows, tokens, eb) : TTC_OK;
    const int64_t work = sums && tokens ? ttc_heads_workspace(heads, tokens) : 0;
    if (st == TTC_OK)
        st = check_beside(rows, {Beside{positions, 4 * (uint64_t)tokens, 4, false}, {q_weight, bw, 4, false}, {k_weight, bw, 4, false}, {dq_weight, bw, 4, true},
                                 {dk_weight, bw, 4, true}, {work ? workspace : nullptr, (uint64_t)work, 4, true}});
    if (st != TTC_OK || (tokens == 0 && !sums)) return st;
    HeadsArgs a = heads_args(heads, tokens);
    a.q = dq ? (norm ? q : dq_out) : nullptr; a.k = dk ? (norm ? k : dk_out) : nullptr;
    a.ld_q = norm ? ldq : ld_dqo; a.ld_k = norm ? ldk : ld_dko;
    a.dq_out = dq_out; a.dk_out = dk_out; a.ld_dqo = ld_dqo; a.ld_dko = ld_dko;
    a.q_out = dq; a.k_out = dk; a.ld_qo = ld_dq; a.ld_ko = ld_dk;
    a.q_weight = q_weight; a.k_weight = k_weight; a.positions = positions;
    a.dq_weight = dq_weight; a.dk_weight = dk_weight;
    a.partial = sums ? static_cast<float*>(workspace) : nullptr;
    return launch_heads_grad(a, stream);
}

int ttc_pages_append(ttc_pages_t pages, ttc_heads_t heads, int64_t tokens, const int32_t* slots, const int32_t* positions, const void* q, int64_t ldq,
                     const void* k, int64_t ldk, const void* v, int64_t ldv, const float* q_weight, const float* k_weight, void* q_out, int64_t ld_qo,
                     void* k_cache, void* v_cache, const float* k_scale, const float* v_scale, void* stream)
{
    if (!pages || !heads) return TTC_ERR_NULL_POINTER;
    if (pages->dtype != heads->dtype || pages->dim != heads->dim || pages->heads != heads->kv_heads) return TTC_ERR_INVALID_VALUE;
    if (pages->cache_dtype == TTC_Q4 && heads->rotated % 16) return TTC_ERR_INVALID_VALUE;
    if (tokens < 0 || ((q_weight || k_weight) && !heads->norm) || ((k_scale || v_scale) && pages->cache_dtype != TTC_F8)) return TTC_ERR_INVALID_VALUE;
    if (!countable(heads, tokens)) return TTC_ERR_OVERFLOW;
    const int64_t wq = heads->q_heads * heads->dim, wk = heads->kv_heads * heads->dim;
    if ((q && (ldq < wq || ld_qo < wq)) || ldk < wk || ldv < wk) return TTC_ERR_INVALID_VALUE;
    if (tokens == 0) return TTC_OK;
    if (!slots || !q != !q_out || !k || !v || !k_cache || !v_cache || (heads->rotated && !positions)) return TTC_ERR_NULL_POINTER;
    const int eb = elem_bytes(heads->dtype), cb = elem_bytes(pages->cache_dtype);
    Rows rows[] = {{q, ldq, wq, false, -1, 0}, {k, ldk, wk, false, -1, 0}, {v, ldv, wk, false, -1, 0}, {q_out, ld_qo, wq, true, 0, 0}};
    int st = check_rows(rows, tokens, eb);
    const uint64_t bw = 4 * (uint64_t)heads->dim, bs = 4 * (uint64_t)heads->kv_heads, bc = (uint64_t)pages->span * cb, bt = 4 * (uint64_t)tokens;
    // keys and values of the cache may be parts of one tensor: each against everything else, and the two for sharing elements
    for (const void* cache : {(const void*)k_cache, (const void*)v_cache})
        if (st == TTC_OK)
            st = check_beside(rows, {Beside{cache, bc, cb, true}, {slots, bt, 4, false}, {positions, bt, 4, false}, {q ? q_weight : nullptr, bw, 4, false},
                                     {k_weight, bw, 4, false}, {k_scale, bs, 4, false}, {v_scale, bs, 4, false}});
    if (st == TTC_OK) {
        Level level[3];
        int levels = 0;
        for (const Level& l : {Level{pages->stride_head, pages->heads}, {pages->stride_slot, pages->page}, {pages->stride_page, pages->pages}})
            if (l.extent > 1) level[levels++] = {l.stride * cb, l.extent};
        std::sort(level, level + levels, [](const Level& a, const Level& b) { return a.stride > b.stride; });
        if (k_cache == v_cache || share(k_cache, v_cache, bc, level, levels, pages->vec * cb)) st = TTC_ERR_ALIAS;
    }
    if (st != TTC_OK) return st;
    HeadsArgs a = heads_args(heads, tokens);
    a.q = q; a.k = k; a.v = v; a.q_out = q_out; a.k_out = k_cache; a.v_out = v_cache;
    a.ld_q = ldq; a.ld_k = ldk; a.ld_v = ldv; a.ld_qo = ld_qo;
    a.q_weight = q_weight; a.k_weight = k_weight; a.k_scale = k_scale; a.v_scale = v_scale;
    a.positions = positions; a.slots = slots;
    a.stride_head = pages->stride_head; a.stride_slot = pages->stride_slot; a.stride_page = pages->stride_page;
    a.slot_count = (uint32_t)(pages->page * pages->pages);
    a.page = pages->page_div;
    a.cache_dtype = pages->cache_dtype;
    return launch_heads(a, stream);
}

ttc_attend_t ttc_attend_create(ttc_pages_t pages, int64_t q_heads, double scale, int64_t window)
{
    int st = TTC_OK;
    if (!pages) st = TTC_ERR_NULL_POINTER;
    else if (pages->dim > TTC_ATTEND_MAX_DIM || q_heads < 1 || q_heads % pages->heads || window < 0 || !std::isfinite((float)(scale * 1.4426950408889634)))
        st = TTC_ERR_INVALID_VALUE;
    else if (q_heads > (int64_t)1 << 20 || pages->heads > 65535) st = TTC_ERR_OVERFLOW;
    ttc_attend_s* a = st == TTC_OK ? new (std::nothrow) ttc_attend_s : nullptr;
    if (st == TTC_OK && !a) st = TTC_ERR_ALLOC;
    if (a)
        *a = {pages->dtype, pages->cache_dtype, q_heads, pages->heads, pages->dim, pages->page, pages->pages, pages->vec, pages->span,
              pages->stride_head, pages->stride_slot, pages->stride_page, (float)(scale * 1.4426950408889634), std::min<int64_t>(window, INT32_MAX), pages->page_div};
    set_last_status(st);
    return a;
}

int ttc_attend_destroy(ttc_attend_t attend)
{
    delete attend;
    return TTC_OK;
}

int64_t ttc_attend_workspace(ttc_attend_t attend, int64_t requests, int64_t tokens, int64_t ld_table)
{
    if (!attend) return -TTC_ERR_NULL_POINTER;
    if (requests < 0 || tokens < 0 || ld_table < 0) return -TTC_ERR_INVALID_VALUE;
    if (!attend_sizes(attend, requests, tokens, ld_table)) return -TTC_ERR_OVERFLOW;
    if (requests == 0 || tokens == 0) return 0;
    const AttendShape s = attend_shape(attend, requests, tokens, longest_context(attend, tokens, ld_table));
    return s.partial_rows ? s.partial_rows * (attend->dim + 2) * 4 + tokens * attend->q_heads * 8 : 0;
}

int ttc_attend_pages(ttc_attend_t attend, int64_t requests, int64_t tokens, const void* q, int64_t ldq, const int32_t* starts, const int32_t* cached,
                     const int32_t* table, int64_t ld_table, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                     void* out, int64_t ldo, float* lse, void* workspace, void* stream)
{
    const int64_t work = ttc_attend_workspace(attend, requests, tokens, ld_table);
    if (work < 0) return (int)-work;
    const int64_t row = attend->q_heads * attend->dim;
    if (ldq < row || ldo < row || ((k_scale || v_scale) && attend->cache_dtype != TTC_F8)) return TTC_ERR_INVALID_VALUE;
    if (requests == 0 || tokens == 0) return TTC_OK;
    if (!q || !starts || !cached || (ld_table && !table) || !k_cache || !v_cache || !out || (work && !workspace)) return TTC_ERR_NULL_POINTER;
    const int eb = elem_bytes(attend->dtype), cb = elem_bytes(attend->cache_dtype);
    uint64_t table_bytes;
    if (!span_bytes(requests, ld_table, ld_table, 4, &table_bytes)) return TTC_ERR_OVERFLOW;
    Rows rows[] = {{q, ldq, row, false, -1, 0}, {out, ldo, row, true, -1, 0}};
    int st = check_rows(rows, tokens, eb);
    const uint64_t bc = (uint64_t)attend->span * cb, bs = 4 * (uint64_t)attend->heads;
    if (st == TTC_OK)
        st = check_beside(rows, {Beside{starts, 4 * (uint64_t)requests + 4, 4, false}, {cached, 4 * (uint64_t)requests, 4, false}, {table, table_bytes, 4, false},
                                 {k_cache, bc, cb, false}, {v_cache, bc, cb, false}, {k_scale, bs, 4, false}, {v_scale, bs, 4, false},
                                 {lse, 4 * (uint64_t)(tokens * attend->q_heads), 4, true}, {work ? workspace : nullptr, (uint64_t)work, 16, true}});
    if (st != TTC_OK) return st;
    const int64_t group = attend->q_heads / attend->heads;
    const AttendShape s = attend_shape(attend, requests, tokens, longest_context(attend, tokens, ld_table));
    AttendArgs a = {};
    a.q = q; a.k_cache = k_cache; a.v_cache = v_cache; a.out = out; a.lse = lse;
    if (work) {
        a.partial = static_cast<float*>(workspace);
        a.partial_sums = reinterpret_cast<PartSum*>(a.partial + s.partial_rows * attend->dim);
        a.parts = reinterpret_cast<int32_t*>(a.partial_sums + s.partial_rows);
    }
    a.k_scale = k_scale; a.v_scale = v_scale;
    a.starts = starts; a.cached = cached; a.table = table;
    a.ld_q = ldq; a.ld_o = ldo; a.ld_table = ld_table;
    a.stride_head = attend->stride_head; a.stride_slot = attend->stride_slot; a.stride_page = attend->stride_page;
    a.tokens = (uint32_t)tokens; a.requests = (uint32_t)requests;
    a.q_heads = (uint32_t)attend->q_heads; a.heads = (uint32_t)attend->heads; a.group = (uint32_t)group;
    a.dim = (uint32_t)attend->dim; a.pages = (uint32_t)attend->pages;
    a.splits = s.splits; a.slots_of_tiles = s.slots;
    a.partial_rows = (uint32_t)s.partial_rows;
    a.join_step = s.tile < kTileMany ? 2 * s.tile * (uint32_t)attend->heads : s.tile; a.join_back = s.tile < kTileMany ? s.tile : 0;
    a.window = (uint32_t)attend->window;
    a.page = attend->page_div;
    a.group_div = make_fastdiv((uint32_t)group);
    a.scale = attend->scale;
    a.dtype = attend->dtype; a.cache_dtype = attend->cache_dtype;
    return launch_attend(a, s, stream);
}

}  // extern "C"
