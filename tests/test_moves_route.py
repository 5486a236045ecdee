"""Rows sorted by expert and back (include/ttc_moves.h, ttc_route_*) against plain implementations in 64 bits."""
import numpy as np
import pytest
import torch

import moves_reference as ref
import paper_1603_02297_amd as ttc

gpu = pytest.mark.gpu
DEV = "cuda"


class Route:
    def __init__(self, *args, **kwargs):
        self.h = ttc.ttc_route_create(*args, **kwargs)

    def __enter__(self):
        return self.h

    def __exit__(self, *_):
        ttc.ttc_route_destroy(self.h)


def stream():
    return torch.cuda.current_stream().cuda_stream


def choose(rng, tokens, topk, total, empty=0.1):
    """Distinct experts per token where there are enough, some tokens without any (-1)."""
    if topk <= total:
        ids = np.argsort(rng.random((tokens, total)) - 0.3 * (np.arange(total) % 3 == 0), axis=1)[:, :topk]
    else:
        ids = rng.integers(0, total, (tokens, topk))
    ids[rng.random(tokens) < empty] = -1
    return ids.astype(np.int64)


def run_sort(h, ids, experts, ld=None, source=True):
    """ids: numpy [tokens, topk] of int32 or int64 -> device results."""
    tokens, topk = ids.shape
    ld = ld or topk
    buf = torch.full((max(tokens, 1), ld), 3, dtype=torch.int64 if ids.dtype == np.int64 else torch.int32, device=DEV)
    buf[:tokens, :topk] = torch.from_numpy(ids).to(DEV)
    rows = ttc.ttc_route_rows(h, tokens)
    guard = 77
    out = {"offsets": torch.full((experts + 1 + 4,), guard, dtype=torch.int32, device=DEV), "counts": torch.full((experts + 4,), guard, dtype=torch.int32, device=DEV),
           "position": torch.full((tokens * topk + 4,), guard, dtype=torch.int32, device=DEV), "source": torch.full((rows + 4,), guard, dtype=torch.int32, device=DEV)}
    work = torch.full((ttc.ttc_route_workspace(h, tokens) // 4 + 4,), guard, dtype=torch.int32, device=DEV)
    ttc.ttc_route_sort(h, tokens, buf.data_ptr(), ld, out["offsets"].data_ptr(), out["counts"].data_ptr(), out["position"].data_ptr(),
                       out["source"].data_ptr() if source else 0, work.data_ptr(), stream())
    torch.cuda.synchronize()
    for v in (*out.values(), work):
        assert (v[-4:] == guard).all()                            # nothing past the end
    return out["offsets"][:experts + 1], out["counts"][:experts], out["position"][:tokens * topk].view(tokens, topk), out["source"][:rows]


@gpu
@pytest.mark.parametrize("tokens,topk,experts,first,align,id_type", [
    (0, 2, 8, 0, 1, np.int64), (0, 1, 1, 0, 16, np.int32), (1, 1, 1, 0, 1, np.int32), (1, 8, 64, 0, 1, np.int64), (1, 64, 3, 0, 7, np.int64),
    (63, 1, 5, 0, 1, np.int32), (64, 1, 64, 0, 16, np.int64), (65, 3, 65, 0, 1, np.int64), (128, 8, 1024, 0, 1, np.int64), (341, 3, 7, 2, 128, np.int32),
    (1024, 1, 33, 0, 1, np.int64), (1025, 1, 33, 0, 1, np.int64), (1024, 8, 128, 64, 16, np.int32), (2731, 3, 1000, 0, 3, np.int64),
    (4097, 2, 16, 16, 64, np.int64), (16384, 4, 64, 0, 128, np.int64), (30011, 5, 129, 3, 1, np.int32), (100003, 7, 255, 0, 16, np.int64),
    (140001, 8, 8, 4, 1, np.int64), (140001, 8, 1024, 0, 2, np.int32), (70001, 5, 300, 0, 64, np.int64),
    (341, 6, 40, 0, 1, np.int64), (2049, 1, 2, 0, 1, np.int32), (131073, 1, 17, 0, 1, np.int64), (150000, 8, 40, 0, 1, np.int32),
    (600000, 8, 700, 0, 1, np.int32), (70000, 8, 900, 0, 16, np.int64), (300000, 8, 30, 1, 1, np.int32),
    (20000, 8, 1000, 0, 1, np.int64), (60000, 8, 400, 0, 128, np.int32)])
def test_sort(tokens, topk, experts, first, align, id_type):
    rng = np.random.default_rng(tokens * 31 + topk)
    ids = (choose(rng, tokens, topk, experts + first + 2) if tokens < 20000 else rng.integers(-1, experts + first + 2, (tokens, topk))).astype(id_type)
    ids[rng.random(ids.shape) < 0.02] = np.iinfo(id_type).max     # nowhere, whatever the number
    ids[rng.random(ids.shape) < 0.02] = np.iinfo(id_type).min
    with Route(ttc.TTC_F32, 8, topk, experts, first, align, np.dtype(id_type).itemsize) as h:
        got = run_sort(h, ids, experts, ld=topk + tokens % 3)
        want = ref.sort(ids, first, experts, align, ttc.ttc_route_rows(h, tokens))
        for name, g, w in zip(("offsets", "counts", "position", "source"), got, want):
            assert np.array_equal(g.cpu().numpy(), w), name
        again = run_sort(h, ids, experts, source=False)           # without source, ids dense
        assert all(torch.equal(a, b) for a, b in zip(again[:3], got[:3]))


@gpu
@pytest.mark.parametrize("tokens,same", [(5000, True), (5000, False), (70000, True)])
def test_sort_of_one_expert_and_of_none(tokens, same):
    ids = np.full((tokens, 2), 4 if same else 9, np.int64)        # all to one expert; all to a rank that is not here
    with Route(ttc.TTC_F32, 8, 2, 8, 0, 16, 8) as h:
        got = run_sort(h, ids, 8)
        want = ref.sort(ids, 0, 8, 16, ttc.ttc_route_rows(h, tokens))
        assert all(np.array_equal(g.cpu().numpy(), w) for g, w in zip(got, want))


def columns(rng, n, width, ld, dtype, shift=0):
    """A row-major [n, width] tensor of the type with rows ld apart that starts `shift` elements into its buffer."""
    buf = torch.full((shift + max(n, 1) * ld + 8,), 5.0, dtype=dtype, device=DEV)
    view = buf[shift:shift + max(n, 1) * ld].view(max(n, 1), ld)[:n, :width]
    view.copy_(torch.from_numpy(rng.standard_normal((n, width))).to(DEV))
    return buf, view


def untouched(buf, before, view, written):
    """Only `written` rows of the view may differ from before."""
    mask = torch.zeros_like(buf, dtype=torch.bool)
    inside = torch.as_strided(mask, view.shape, view.stride(), view.storage_offset())
    inside[torch.as_tensor(written, device=DEV, dtype=torch.bool)] = True
    bits = lambda x: x.view(torch.int32 if x.element_size() == 4 else torch.int16)  # noqa: E731: NaN are equal to themselves
    return torch.equal(bits(buf)[~mask], bits(before)[~mask])


SHAPES = [
    # type, tokens, topk, experts, first, align, width, extra ld, shift, weights, alpha, beta
    ("bf16", 1, 8, 16, 0, 1, 2048, 0, 0, True, 1.0, 1.0), ("f32", 33, 2, 4, 0, 8, 64, 0, 0, True, 1.0, 0.0), ("f16", 50, 3, 7, 1, 1, 1001, 3, 1, True, 2.5, 0.5),
    ("bf16", 20, 9, 12, 0, 16, 7, 0, 0, True, 1.0, 0.0), ("f32", 17, 1, 3, 0, 1, 1, 0, 0, False, 1.0, 0.0), ("bf16", 64, 17, 20, 2, 3, 130, 5, 3, True, -1.0, 1.0),
    ("f16", 257, 4, 9, 0, 64, 512, 0, 0, False, 1.0, 0.0), ("f32", 12, 8, 8, 0, 1, 5000, 1, 1, True, 1.0, -2.0), ("bf16", 5, 2, 300, 0, 128, 9000, 0, 0, True, 0.5, 0.0),
    ("f16", 100, 5, 6, 0, 1, 9, 7, 2, True, 1.0, 1.0), ("f32", 9, 6, 40, 10, 5, 260, 0, 0, False, 3.0, 1.0), ("bf16", 40, 3, 5, 0, 2, 16, 0, 0, True, 1.0, 0.0),
    ("bf16", 31, 12, 24, 0, 4, 33, 1, 0, False, 1.0, 0.0), ("f32", 3, 64, 70, 0, 1, 129, 0, 0, True, 1.0, 0.0), ("f32", 6, 3, 4, 0, 1, 4100, 0, 3, True, 1.0, 0.0),
]


@gpu
@pytest.mark.parametrize("kind,tokens,topk,experts,first,align,width,extra,shift,weighted,alpha,beta", SHAPES)
def test_moves(kind, tokens, topk, experts, first, align, width, extra, shift, weighted, alpha, beta):
    rng = np.random.default_rng(width * 7 + tokens)
    code, dtype = ref.TYPES[kind]
    ids = choose(rng, tokens, topk, experts + first + 1, 0.15)
    with Route(code, width, topk, experts, first, align, 8, alpha, beta) as h:
        rows = ttc.ttc_route_rows(h, tokens)
        offsets, counts, position, _ = ref.sort(ids, first, experts, align, rows)
        d_off, d_cnt, d_pos = (torch.from_numpy(x).to(DEV) for x in (offsets, counts, position))
        w = torch.from_numpy(rng.standard_normal((tokens, topk)).astype(np.float32)).to(DEV) if weighted else None
        w64, wp = (ref.wide(w), w.data_ptr()) if weighted else (None, 0)
        live = np.zeros(rows, bool)
        live[position[position >= 0]] = True
        pads = np.zeros(rows, bool)
        pads[:offsets[-1]] = True
        pads &= ~live
        ld = width + extra

        # gather, with and without weights
        _, x = columns(rng, tokens, width, ld, dtype, shift)
        for pointer, factor in ((0, None), (wp, w64)):
            buf, s = columns(rng, rows, width, ld, dtype, shift)
            before = buf.clone()
            ttc.ttc_route_gather(h, tokens, x.data_ptr(), ld, pointer, d_pos.data_ptr(), d_off.data_ptr(), d_cnt.data_ptr(), s.data_ptr(), ld, stream())
            torch.cuda.synchronize()
            got, want = ref.wide(s), np.zeros((rows, width))
            for t in range(tokens):
                for k in range(topk):
                    if position[t, k] >= 0:
                        want[position[t, k]] = ref.wide(x[t]) * (1.0 if factor is None else factor[t, k])
            if factor is None:
                assert np.array_equal(got[live], want[live])
            else:
                ref.assert_close(got[live], want[live], kind, np.abs(want[live]), 1, "weighted gather")
            assert (got[pads] == 0).all()
            assert untouched(buf, before, s, live | pads)

        # combine
        _, s = columns(rng, rows, width, ld, dtype, shift)
        s[torch.from_numpy(~live).to(DEV)] = float("nan")         # padding and what is past the end adds nothing
        buf, y = columns(rng, tokens, width, ld, dtype, shift)
        if not beta:
            y.fill_(float("nan"))                                  # not read
        before, y0 = buf.clone(), ref.wide(y)
        ttc.ttc_route_combine(h, tokens, s.data_ptr(), ld, wp, d_pos.data_ptr(), y.data_ptr(), ld, stream())
        torch.cuda.synchronize()
        want, mag = ref.combine(ref.wide(s), w64, position, alpha, beta, y0 if beta else np.zeros_like(y0))
        ref.assert_close(ref.wide(y), want, kind, mag, topk + 3, "combine")
        assert untouched(buf, before, y, np.ones(tokens, bool))

        # its gradients: both, rows only, weights only
        _, dy = columns(rng, tokens, width, ld, dtype, shift)
        want_rows, want_w, mag_w = ref.combine_grad(ref.wide(dy), np.where(live[:, None], ref.wide(s), 0.0), w64, position, alpha)
        for parts in ("both", "rows", "weights"):
            buf, ds = columns(rng, rows, width, ld, dtype, shift)
            before = buf.clone()
            dw = torch.full((tokens * topk + 4,), 77.0, device=DEV)
            ttc.ttc_route_combine_grad(h, tokens, dy.data_ptr(), ld, s.data_ptr() if parts != "rows" else 0, ld, wp, d_pos.data_ptr(), d_off.data_ptr(), d_cnt.data_ptr(),
                                       ds.data_ptr() if parts != "weights" else 0, ld, dw.data_ptr() if parts != "rows" else 0, stream())
            torch.cuda.synchronize()
            if parts != "weights":
                ref.assert_close(ref.wide(ds)[live], want_rows[live], kind, np.abs(want_rows[live]), 2, "drows")
                assert (ref.wide(ds)[pads] == 0).all()
            assert untouched(buf, before, ds, live | pads if parts != "weights" else np.zeros(rows, bool))
            if parts != "rows":
                # a lane's chain, the shuffles, the wavefronts and the factor alpha: fewer roundings than the terms there are
                ref.assert_close(ref.wide(dw[:tokens * topk]).reshape(tokens, topk), want_w, "f32", mag_w, width + 20, "dweights")
            assert (dw[-4:] == 77).all()


@gpu
@pytest.mark.parametrize("kind,tokens,topk,experts,first,align,width,beta", [
    ("bf16", 3000, 8, 32, 0, 16, 4128, 1.0), ("f32", 6001, 3, 5, 1, 1, 2049, 0.0), ("f16", 4000, 4, 9, 0, 64, 4100, 1.0), ("bf16", 2500, 9, 12, 3, 1, 2880, 0.0),
    ("bf16", 20000, 2, 4, 4, 1, 2056, 0.0), ("f32", 90000, 2, 8, 0, 128, 130, 0.5), ("f16", 200000, 5, 64, 0, 8, 48, 0.0), ("bf16", 1500, 1, 8, 0, 1, 40000, 1.0),
    ("bf16", 5000, 4, 8, 0, 1, 4097, 1.0), ("f16", 3000, 6, 8, 2, 32, 3333, 0.0)])
def test_moves_of_large_batches(kind, tokens, topk, experts, first, align, width, beta):
    """Sizes at which rows are streamed and rows take several rounds, against 64 bits on the GPU; some choices elsewhere, some tokens empty."""
    code, dtype = ref.TYPES[kind]
    rel, tiny = ref.ROUND[kind]
    g = torch.Generator(device=DEV).manual_seed(width)
    ids = torch.rand(tokens, experts + first + 2, generator=g, device=DEV).topk(topk, dim=1).indices.contiguous()
    ids[torch.rand(tokens, generator=g, device=DEV) < 0.1] = -1
    draw = lambda *shape: torch.randn(shape, generator=g, device=DEV).to(dtype)  # noqa: E731
    weights = torch.randn(tokens, topk, generator=g, device=DEV)
    with Route(code, width, topk, experts, first, align, 8, 1.0, beta) as h:
        n = ttc.ttc_route_rows(h, tokens)
        i32 = lambda k: torch.empty(k, dtype=torch.int32, device=DEV)  # noqa: E731
        offsets, counts, position, source, work = i32(experts + 1), i32(experts), i32(tokens * topk), i32(n), i32(ttc.ttc_route_workspace(h, tokens) // 4 + 1)
        ttc.ttc_route_sort(h, tokens, ids.data_ptr(), topk, offsets.data_ptr(), counts.data_ptr(), position.data_ptr(), source.data_ptr(), work.data_ptr(), stream())
        pos = position.view(tokens, topk).long()
        here = pos >= 0
        assert torch.equal(here, (ids >= first) & (ids < first + experts)) and torch.equal(source[pos[here]].long(), torch.nonzero(here.reshape(-1)).reshape(-1))
        x, rows = draw(tokens, width), torch.full((n, width), 3.0, dtype=dtype, device=DEV)
        ttc.ttc_route_gather(h, tokens, x.data_ptr(), width, 0, position.data_ptr(), offsets.data_ptr(), counts.data_ptr(), rows.data_ptr(), width, stream())
        want = torch.where((torch.arange(n, device=DEV) < offsets[-1])[:, None], 0.0, torch.full_like(rows, 3.0))
        want[pos[here]] = x[torch.nonzero(here)[:, 0]]
        assert torch.equal(rows, want)
        del want
        rows = draw(n, width)
        rows[source < 0] = float("nan")
        y = draw(tokens, width)
        exact, mag = beta * y.double(), abs(beta) * y.double().abs()
        for k in range(topk):
            term = torch.where(here[:, k, None], weights[:, k, None].double() * rows[pos[:, k].clamp(min=0)].double(), 0.0)
            exact, mag = exact + term, mag + term.abs()
        ttc.ttc_route_combine(h, tokens, rows.data_ptr(), width, weights.data_ptr(), position.data_ptr(), y.data_ptr(), width, stream())
        err = (topk + 3) * ref.F32 * mag
        assert ((y.double() - exact).abs() <= err * 1.01 + rel * (exact.abs() + err) + tiny).all()
        del exact, mag, err
        dy, drows, dweights = draw(tokens, width), torch.full((n, width), 3.0, dtype=dtype, device=DEV), torch.empty(tokens, topk, device=DEV)
        ttc.ttc_route_combine_grad(h, tokens, dy.data_ptr(), width, rows.data_ptr(), width, weights.data_ptr(), position.data_ptr(), offsets.data_ptr(), counts.data_ptr(),
                                   drows.data_ptr(), width, dweights.data_ptr(), stream())
        assert (drows[(source < 0) & (torch.arange(n, device=DEV) < offsets[-1])] == 0).all() and (drows[int(offsets[-1]):] == 3).all()
        for k in range(topk):
            at, mine = pos[here[:, k], k], dy[here[:, k]].double()
            want = weights[here[:, k], k, None].double() * mine
            assert ((drows[at].double() - want).abs() <= (rel + 2 * ref.F32) * want.abs() * 1.01 + tiny).all()
            product = mine * rows[at].double()
            assert ((dweights[here[:, k], k].double() - product.sum(1)).abs() <= (width + 20) * ref.F32 * product.abs().sum(1)).all()
        assert (dweights[~here] == 0).all()


@gpu
def test_positions_that_point_nowhere_are_not_followed():
    code, dtype = ref.TYPES["bf16"]
    rng = np.random.default_rng(5)
    tokens, topk, width = 40, 4, 136
    with Route(code, width, topk, 8, 0, 1, 8) as h:
        rows = ttc.ttc_route_rows(h, tokens)
        position = np.arange(rows, dtype=np.int32).reshape(tokens, topk)
        for bad in (-1, -2 ** 31, rows, 2 ** 31 - 1):
            position[rng.random(position.shape) < 0.1] = bad
        p = torch.from_numpy(position).to(DEV)
        live = np.zeros(rows, bool)
        good = position[(position >= 0) & (position < rows)]
        live[good] = True
        _, x = columns(rng, tokens, width, width, dtype)
        buf, s = columns(rng, rows, width, width, dtype)
        before = buf.clone()
        ttc.ttc_route_gather(h, tokens, x.data_ptr(), width, 0, p.data_ptr(), 0, 0, s.data_ptr(), width, stream())
        torch.cuda.synchronize()
        assert untouched(buf, before, s, live)
        _, y = columns(rng, tokens, width, width, dtype)
        ttc.ttc_route_combine(h, tokens, s.data_ptr(), width, 0, p.data_ptr(), y.data_ptr(), width, stream())
        want, mag = ref.combine(ref.wide(s), None, position, 1.0, 0.0, np.zeros((tokens, width)))
        ref.assert_close(ref.wide(y), want, "bf16", mag, topk)
        dw = torch.empty(tokens, topk, device=DEV)
        buf, ds = columns(rng, rows, width, width, dtype)
        before = buf.clone()
        ttc.ttc_route_combine_grad(h, tokens, x.data_ptr(), width, s.data_ptr(), width, 0, p.data_ptr(), 0, 0, ds.data_ptr(), width, dw.data_ptr(), stream())
        torch.cuda.synchronize()
        assert untouched(buf, before, ds, live)
        assert (ref.wide(dw)[(position < 0) | (position >= rows)] == 0).all()


@gpu
def test_infinities_and_nan_stay_where_they_are():
    code, dtype = ref.TYPES["f16"]
    with Route(code, 24, 2, 2, 0, 1, 8) as h:
        position = torch.tensor([[0, 2], [1, -1], [-1, -1]], dtype=torch.int32, device=DEV)
        weights = torch.tensor([[1.0, 2.0], [0.5, float("nan")], [float("inf"), 1.0]], device=DEV)       # those of choices that are nowhere do not count
        s = torch.ones(6, 24, dtype=dtype, device=DEV)
        s[0, 3], s[1, 4], s[2, 3], s[2, 5] = float("inf"), float("nan"), -float("inf"), 60000.0
        y = torch.empty(3, 24, dtype=dtype, device=DEV)
        ttc.ttc_route_combine(h, 3, s.data_ptr(), 24, weights.data_ptr(), position.data_ptr(), y.data_ptr(), 24, stream())
        want = np.full((3, 24), 3.0)
        want[1], want[2] = 0.5, 0.0
        want[0, 3], want[1, 4], want[0, 5] = np.nan, np.nan, np.inf                                      # inf - inf; 120001 overflows
        assert np.array_equal(ref.wide(y), want, equal_nan=True)


@gpu
@pytest.mark.parametrize("topk,width", [(2, 96), (9, 257)])
def test_gradient_against_differences(topk, width):
    """combine is linear in the rows and in the weights: a symmetric difference is its derivative up to rounding."""
    rng = np.random.default_rng(topk)
    tokens, experts, alpha = 37, 11, 1.75
    ids = choose(rng, tokens, topk, experts + 3)
    with Route(ttc.TTC_F32, width, topk, experts, 0, 4, 8, alpha, 0.0) as h:
        n = ttc.ttc_route_rows(h, tokens)
        offsets, counts, position, _ = ref.sort(ids, 0, experts, 4, n)
        o, c, p = (torch.from_numpy(x).to(DEV) for x in (offsets, counts, position))
        draw = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(DEV)  # noqa: E731
        rows, weights, dy = draw(n, width), draw(tokens, topk), draw(tokens, width)

        def loss(r, w):
            y = torch.empty(tokens, width, device=DEV)
            ttc.ttc_route_combine(h, tokens, r.data_ptr(), width, w.data_ptr(), p.data_ptr(), y.data_ptr(), width, stream())
            return float((y.double() * dy.double()).sum())

        drows, dweights = torch.zeros(n, width, device=DEV), torch.empty(tokens, topk, device=DEV)
        ttc.ttc_route_combine_grad(h, tokens, dy.data_ptr(), width, rows.data_ptr(), width, weights.data_ptr(), p.data_ptr(), o.data_ptr(), c.data_ptr(),
                                   drows.data_ptr(), width, dweights.data_ptr(), stream())
        live = position >= 0
        for _ in range(4):
            dr, dw, step = draw(n, width), draw(tokens, topk), 0.5
            # every value of y is off by at most (topk + 3) roundings of its terms; two losses, their difference over 2 * step
            _, mag = ref.combine(np.abs(ref.wide(rows)) + step * np.abs(ref.wide(dr)), np.abs(ref.wide(weights)) + step * np.abs(ref.wide(dw)), position, alpha, 0.0, np.zeros((tokens, width)))
            limit = 2 * (topk + 6) * ref.F32 * float((mag * np.abs(ref.wide(dy))).sum()) / (2 * step)
            by_rows = (loss(rows + step * dr, weights) - loss(rows - step * dr, weights)) / (2 * step)
            assert abs(by_rows - float((drows.double() * dr.double()).sum())) <= 2 * limit
            by_weights = (loss(rows, weights + step * dw) - loss(rows, weights - step * dw)) / (2 * step)
            assert abs(by_weights - float((dweights.double() * dw.double())[torch.from_numpy(live).to(DEV)].sum())) <= 2 * limit
        # the gradient of the gather is the combine without weights
        with Route(ttc.TTC_F32, width, topk, experts, 0, 4, 8) as plain:
            x, s, ds, dx = draw(tokens, width), torch.zeros(n, width, device=DEV), draw(n, width), torch.empty(tokens, width, device=DEV)
            ttc.ttc_route_combine(plain, tokens, ds.data_ptr(), width, 0, p.data_ptr(), dx.data_ptr(), width, stream())
            ttc.ttc_route_gather(plain, tokens, x.data_ptr(), width, 0, p.data_ptr(), o.data_ptr(), c.data_ptr(), s.data_ptr(), width, stream())
            left, right = float((s.double() * ds.double()).sum()), float((x.double() * dx.double()).sum())       # <gather(x), ds> = <x, dx>
            assert abs(left - right) <= topk * ref.F32 * float((s.double() * ds.double()).abs().sum())


@gpu
def test_rows_beyond_two_to_the_32_elements():
    """Leading dimensions that put the last rows behind 2^32 elements."""
    code, dtype = ref.TYPES["bf16"]
    tokens, topk, width, ld = 300, 2, 72, 1 << 23
    with Route(code, width, topk, 5, 0, 1, 8) as h:
        n = ttc.ttc_route_rows(h, tokens)
        rng = np.random.default_rng(1)
        position = rng.permutation(n).astype(np.int32).reshape(tokens, topk)
        p = torch.from_numpy(position).to(DEV)
        x = torch.randn(tokens, width, device=DEV).to(dtype)
        big = torch.empty((n - 1) * ld + width, dtype=dtype, device=DEV)
        s = torch.as_strided(big, (n, width), (ld, 1))
        ttc.ttc_route_gather(h, tokens, x.data_ptr(), width, 0, p.data_ptr(), 0, 0, big.data_ptr(), ld, stream())
        assert torch.equal(s[p.long().reshape(-1)], x.repeat_interleave(topk, 0))
        y = torch.empty_like(x)
        ttc.ttc_route_combine(h, tokens, big.data_ptr(), ld, 0, p.data_ptr(), y.data_ptr(), width, stream())
        assert torch.equal(y, x + x)                              # exact: a doubled value
        dw = torch.empty(tokens, topk, device=DEV)
        ttc.ttc_route_combine_grad(h, tokens, x.data_ptr(), width, big.data_ptr(), ld, 0, p.data_ptr(), 0, 0, 0, 0, dw.data_ptr(), stream())
        want = (x.double() ** 2).sum(1, keepdim=True).expand(tokens, topk)
        assert ((dw.double() - want).abs() <= (width + 20) * ref.F32 * want).all()


@gpu
def test_streams_and_graphs():
    """On another stream, and captured: every replay gives what the calls give by themselves."""
    code, dtype = ref.TYPES["bf16"]
    tokens, topk, experts, width, align = 6000, 4, 24, 264, 16
    with Route(code, width, topk, experts, 0, align, 8) as h:
        rng = np.random.default_rng(2)
        n = ttc.ttc_route_rows(h, tokens)
        ids = torch.empty(tokens, topk, dtype=torch.int64, device=DEV)
        x = torch.empty(tokens, width, dtype=dtype, device=DEV)
        weights = torch.rand(tokens, topk, device=DEV)
        i32 = lambda k: torch.zeros(k, dtype=torch.int32, device=DEV)  # noqa: E731

        def buffers():
            return {"offsets": i32(experts + 1), "counts": i32(experts), "position": i32(tokens * topk), "source": i32(n), "work": i32(ttc.ttc_route_workspace(h, tokens) // 4 + 1),
                    "rows": torch.zeros(n, width, dtype=dtype, device=DEV), "y": torch.zeros(tokens, width, dtype=dtype, device=DEV),
                    "drows": torch.zeros(n, width, dtype=dtype, device=DEV), "dw": torch.zeros(tokens, topk, device=DEV)}

        def calls(b):
            q = {k: v.data_ptr() for k, v in b.items()}
            st = stream()
            ttc.ttc_route_sort(h, tokens, ids.data_ptr(), topk, q["offsets"], q["counts"], q["position"], q["source"], q["work"], st)
            ttc.ttc_route_gather(h, tokens, x.data_ptr(), width, 0, q["position"], q["offsets"], q["counts"], q["rows"], width, st)
            ttc.ttc_route_combine(h, tokens, q["rows"], width, weights.data_ptr(), q["position"], q["y"], width, st)
            ttc.ttc_route_combine_grad(h, tokens, q["y"], width, q["rows"], width, weights.data_ptr(), q["position"], q["offsets"], q["counts"], q["drows"], width, q["dw"], st)

        def fill():
            ids.copy_(torch.from_numpy(choose(rng, tokens, topk, experts)))
            x.copy_(torch.randn(tokens, width, device=DEV))

        fill()
        captured, eager = buffers(), buffers()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            calls(captured)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls(captured)
        for _ in range(4):
            fill()
            for b in (captured, eager):
                for k in ("rows", "drows"):
                    b[k].zero_()                                  # rows past the last segment are not written
            graph.replay()
            calls(eager)
            torch.cuda.synchronize()
            for k in captured:
                if k != "work":
                    assert torch.equal(captured[k], eager[k]), k


# ---- refusals: before anything reaches a device -----------------------------------------------------------

def test_create_refuses():
    ok = dict(dtype=ttc.TTC_BF16, width=64, topk=2, experts=8, first=0, align=1, id_bytes=8)
    for change, status in (({"dtype": ttc.TTC_F64}, ttc.TTC_ERR_UNSUPPORTED_DTYPE), ({"dtype": ttc.TTC_F8}, ttc.TTC_ERR_UNSUPPORTED_DTYPE), ({"dtype": -1}, ttc.TTC_ERR_UNSUPPORTED_DTYPE),
                           ({"width": 0}, ttc.TTC_ERR_INVALID_VALUE), ({"width": 1 << 40}, ttc.TTC_ERR_OVERFLOW), ({"topk": 0}, ttc.TTC_ERR_INVALID_VALUE),
                           ({"topk": 65}, ttc.TTC_ERR_INVALID_VALUE), ({"experts": 0}, ttc.TTC_ERR_INVALID_VALUE), ({"experts": 1025}, ttc.TTC_ERR_INVALID_VALUE),
                           ({"first": -1}, ttc.TTC_ERR_INVALID_VALUE), ({"first": 2 ** 63 - 3}, ttc.TTC_ERR_OVERFLOW), ({"align": 0}, ttc.TTC_ERR_INVALID_VALUE),
                           ({"align": 65537}, ttc.TTC_ERR_INVALID_VALUE), ({"id_bytes": 2}, ttc.TTC_ERR_INVALID_VALUE)):
        with pytest.raises(ttc.TtcError) as e:
            ttc.ttc_route_create(**{**ok, **change})
        assert e.value.status == status, change
        assert ttc.ttc_last_status() == status
    ttc.ttc_route_destroy(None)
    for dtype in (ttc.TTC_BF16, ttc.TTC_F16, ttc.TTC_F8):         # the transposition takes none of the types of these moves
        with pytest.raises(ttc.TtcError) as e:
            ttc.ttc_plan_create(dtype, 2, (8, 8), (1, 0))
        assert e.value.status == ttc.TTC_ERR_UNSUPPORTED_DTYPE


def test_sizes():
    with Route(ttc.TTC_F32, 8, 4, 16, 0, 128, 4) as h:
        assert ttc.ttc_route_rows(h, 0) == 0 and ttc.ttc_route_rows(h, 1) == 4 + 4 * 127 and ttc.ttc_route_rows(h, 1000) == 4000 + 16 * 127
        assert ttc.ttc_route_workspace(h, 0) == 0 and 0 < ttc.ttc_route_workspace(h, 1 << 20) < 1 << 20
        for f in (ttc.ttc_route_rows, ttc.ttc_route_workspace):
            for tokens, status in ((-1, ttc.TTC_ERR_INVALID_VALUE), (1 << 29, ttc.TTC_ERR_OVERFLOW), (1 << 62, ttc.TTC_ERR_OVERFLOW)):
                with pytest.raises(ttc.TtcError) as e:
                    f(h, tokens)
                assert e.value.status == status
            with pytest.raises(ttc.TtcError) as e:
                f(None, 3)
            assert e.value.status == ttc.TTC_ERR_NULL_POINTER


A, B, C, D, E, F, G = (0x10000000 * k for k in range(1, 8))      # addresses that no call here dereferences


@pytest.mark.parametrize("change,status", [
    ({"h": None}, ttc.TTC_ERR_NULL_POINTER), ({"tokens": -1}, ttc.TTC_ERR_INVALID_VALUE), ({"tokens": 1 << 40}, ttc.TTC_ERR_OVERFLOW), ({"ldx": 63}, ttc.TTC_ERR_INVALID_VALUE),
    ({"ld_rows": 63}, ttc.TTC_ERR_INVALID_VALUE), ({"x": 0}, ttc.TTC_ERR_NULL_POINTER), ({"position": 0}, ttc.TTC_ERR_NULL_POINTER), ({"rows": 0}, ttc.TTC_ERR_NULL_POINTER),
    ({"offsets": 0}, ttc.TTC_ERR_NULL_POINTER), ({"counts": 0}, ttc.TTC_ERR_NULL_POINTER), ({"x": A + 1}, ttc.TTC_ERR_MISALIGNED), ({"position": C + 2}, ttc.TTC_ERR_MISALIGNED),
    ({"weights": E + 1}, ttc.TTC_ERR_MISALIGNED), ({"rows": A + 64}, ttc.TTC_ERR_ALIAS), ({"rows": C - 64}, ttc.TTC_ERR_ALIAS), ({"ldx": 1 << 61}, ttc.TTC_ERR_OVERFLOW)])
def test_gather_refuses(change, status):
    with Route(ttc.TTC_BF16, 64, 2, 8, 0, 16, 8) as h:
        ok = dict(h=h, tokens=10, x=A, ldx=64, weights=E, position=C, offsets=D, counts=F, rows=B, ld_rows=64)
        with pytest.raises(ttc.TtcError) as e:
            ttc.ttc_route_gather(*{**ok, **change}.values(), None)
        assert e.value.status == status


@pytest.mark.parametrize("change,status", [
    ({"h": None}, ttc.TTC_ERR_NULL_POINTER), ({"tokens": -5}, ttc.TTC_ERR_INVALID_VALUE), ({"ld_ids": 1}, ttc.TTC_ERR_INVALID_VALUE), ({"ids": 0}, ttc.TTC_ERR_NULL_POINTER),
    ({"offsets": 0}, ttc.TTC_ERR_NULL_POINTER), ({"counts": 0}, ttc.TTC_ERR_NULL_POINTER), ({"position": 0}, ttc.TTC_ERR_NULL_POINTER), ({"workspace": 0}, ttc.TTC_ERR_NULL_POINTER),
    ({"ids": A + 4}, ttc.TTC_ERR_MISALIGNED), ({"source": E + 2}, ttc.TTC_ERR_MISALIGNED), ({"position": A}, ttc.TTC_ERR_ALIAS), ({"source": D}, ttc.TTC_ERR_ALIAS), ({"workspace": B}, ttc.TTC_ERR_ALIAS)])
def test_sort_refuses(change, status):
    with Route(ttc.TTC_BF16, 64, 2, 8, 0, 16, 8) as h:
        ok = dict(h=h, tokens=10000, ids=A, ld_ids=2, offsets=B, counts=C, position=D, source=E, workspace=F)
        with pytest.raises(ttc.TtcError) as e:
            ttc.ttc_route_sort(*{**ok, **change}.values(), None)
        assert e.value.status == status


@pytest.mark.parametrize("change,status", [
    ({"h": None}, ttc.TTC_ERR_NULL_POINTER), ({"ldy": 63}, ttc.TTC_ERR_INVALID_VALUE), ({"ld_rows": 10}, ttc.TTC_ERR_INVALID_VALUE), ({"rows": 0}, ttc.TTC_ERR_NULL_POINTER),
    ({"y": 0}, ttc.TTC_ERR_NULL_POINTER), ({"position": 0}, ttc.TTC_ERR_NULL_POINTER), ({"y": A + 128}, ttc.TTC_ERR_ALIAS), ({"y": C - 8}, ttc.TTC_ERR_ALIAS), ({"y": B + 1}, ttc.TTC_ERR_MISALIGNED)])
def test_combine_refuses(change, status):
    with Route(ttc.TTC_F16, 64, 2, 8, 0, 1, 8) as h:
        ok = dict(h=h, tokens=100, rows=A, ld_rows=64, weights=D, position=C, y=B, ldy=64)
        with pytest.raises(ttc.TtcError) as e:
            ttc.ttc_route_combine(*{**ok, **change}.values(), None)
        assert e.value.status == status


@pytest.mark.parametrize("change,status", [
    ({"h": None}, ttc.TTC_ERR_NULL_POINTER), ({"ld_dy": 63}, ttc.TTC_ERR_INVALID_VALUE), ({"ld_rows": 63}, ttc.TTC_ERR_INVALID_VALUE), ({"ld_drows": 1}, ttc.TTC_ERR_INVALID_VALUE),
    ({"dy": 0}, ttc.TTC_ERR_NULL_POINTER), ({"rows": 0}, ttc.TTC_ERR_NULL_POINTER), ({"drows": 0, "dweights": 0}, ttc.TTC_ERR_NULL_POINTER), ({"counts": 0}, ttc.TTC_ERR_NULL_POINTER),
    ({"drows": B}, ttc.TTC_ERR_ALIAS), ({"dweights": D}, ttc.TTC_ERR_ALIAS), ({"dweights": F + 16}, ttc.TTC_ERR_ALIAS), ({"dweights": G + 2}, ttc.TTC_ERR_MISALIGNED)])
def test_combine_grad_refuses(change, status):
    with Route(ttc.TTC_F32, 64, 2, 8, 0, 4, 8) as h:
        ok = dict(h=h, tokens=100, dy=A, ld_dy=64, rows=B, ld_rows=64, weights=C, position=D, offsets=E, counts=E + 4096, drows=F, ld_drows=64, dweights=G)
        with pytest.raises(ttc.TtcError) as e:
            ttc.ttc_route_combine_grad(*{**ok, **change}.values(), None)
        assert e.value.status == status


def test_nothing_to_move_is_no_error():
    with Route(ttc.TTC_F32, 64, 2, 8, 0, 4, 8) as h:
        ttc.ttc_route_gather(h, 0, 0, 64, 0, 0, 0, 0, 0, 64)
        ttc.ttc_route_combine(h, 0, 0, 64, 0, 0, 0, 64)
        ttc.ttc_route_combine_grad(h, 0, 0, 64, 0, 64, 0, 0, 0, 0, 0, 64, 0)
