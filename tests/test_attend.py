"""Attention over the pages of a cache (include/ttc_attention.h, ttc_attend_pages) against a plain implementation in 64 bits."""
import numpy as np
import pytest
import torch

import attention_reference as ref
import moves_reference as moves
import paper_1603_02297_amd as ttc

gpu = pytest.mark.gpu
DEV = "cuda"


class Handle:
    def __init__(self, create, destroy, *args):
        self.h, self.destroy = create(*args), destroy

    def __enter__(self):
        return self.h

    def __exit__(self, *_):
        self.destroy(self.h)


def stream():
    return torch.cuda.current_stream().cuda_stream


def ptr(x):
    return 0 if x is None or x.numel() == 0 else x.data_ptr()


class Problem:
    """Requests over a cache that has been in use: pages in no order, everything else in it other values."""

    def __init__(self, kind, cache, order, hq, hk, dim, page, lengths, seed=0, width=None, pad=0, extra_pages=2):
        g, rng = torch.Generator().manual_seed(seed), np.random.default_rng(seed)
        self.kind, self.cache, self.order, self.hq, self.hk, self.dim, self.page = kind, cache, order, hq, hk, dim, page
        self.dtype, cache_type = ref.TYPES[kind][1], ref.TYPES[cache][1]
        self.cached, fresh = (np.array([x[i] for x in lengths], np.int32) for i in range(2))
        self.starts = np.concatenate([[0], fresh.cumsum()]).astype(np.int32)
        self.tokens = int(self.starts[-1]) + pad
        blocks = [-(-(c + f) // page) for c, f in lengths]
        self.width = max(blocks) + 1 if width is None else width
        self.pages = sum(blocks) + extra_pages
        self.table = np.full((len(lengths), self.width), -1, np.int32)
        order_of = rng.permutation(self.pages).astype(np.int32)
        used = 0
        for r, n in enumerate(blocks):
            n = min(n, self.width)
            self.table[r, :n] = order_of[used:used + n]
            used += n
        rec = self.rec = dim // 2 + 4 if cache == "q4" else dim
        shape = (self.pages, page, hk, rec) if order == "slots" else (self.pages, hk, page, rec)
        self.strides = (rec, hk * rec, page * hk * rec) if order == "slots" else (page * rec, rec, page * hk * rec)
        self.caches = []
        for _ in range(2):
            if cache == "q4":
                x = torch.randint(0, 256, shape, dtype=torch.uint8, generator=g)
                step = (0.15 + 0.1 * torch.rand(shape[:3], generator=g)).to(torch.bfloat16)
                low = (-7 * step.float() + 0.3 * torch.randn(shape[:3], generator=g)).to(torch.bfloat16)
                x[..., :4] = torch.stack([step, low], -1).view(torch.uint8)
            else:
                x = torch.randn(shape, generator=g).to(cache_type)
            self.caches.append(x)
        self.scales = [0.5 + torch.rand(hk, generator=g) if cache == "f8" else None for _ in range(2)]
        self.ldq = hq * dim + 8
        self.q = (1.5 * torch.randn(self.tokens, self.ldq, generator=g)).to(self.dtype)

    def handles(self, scale, window):
        return (Handle(ttc.ttc_pages_create, ttc.ttc_pages_destroy, ref.TYPES[self.kind][0], ref.TYPES[self.cache][0], self.hk, self.dim, self.page, self.pages, self.strides),
                lambda p: Handle(ttc.ttc_attend_create, ttc.ttc_attend_destroy, p, self.hq, scale, window))

    def to_gpu(self):
        d = {k: torch.from_numpy(getattr(self, k)).to(DEV) for k in ("cached", "starts", "table")}
        d["q"] = self.q.to(DEV)
        d["k"], d["v"] = (x.to(DEV) for x in self.caches)
        d["ks"], d["vs"] = (None if x is None else x.to(DEV) for x in self.scales)
        d["out"] = torch.full((self.tokens, self.hq * self.dim + 4), 9.0, dtype=self.dtype, device=DEV)
        d["lse"] = torch.full((self.tokens, self.hq), 9.0, device=DEV)
        return d

    def call(self, attend, d, work, lse=True):
        ttc.ttc_attend_pages(attend, len(self.cached), self.tokens, ptr(d["q"]), self.ldq, ptr(d["starts"]), ptr(d["cached"]), ptr(d["table"]), self.width, ptr(d["k"]), ptr(d["v"]),
                             ptr(d["ks"]), ptr(d["vs"]), ptr(d["out"]), self.hq * self.dim + 4, ptr(d["lse"]) if lse else 0, ptr(work), stream())

    def workspace(self, attend):
        n = ttc.ttc_attend_workspace(attend, len(self.cached), self.tokens, self.width)
        return torch.full((n + 16,), 255, dtype=torch.uint8, device=DEV)

    def run(self, scale, window=0, lse=True):
        pages, attend_of = self.handles(scale, window)
        with pages as p, attend_of(p) as attend:
            d, work = self.to_gpu(), self.workspace(attend)
            self.call(attend, d, work[:-16] if work.numel() > 16 else work[:0], lse)
            torch.cuda.synchronize()
            assert (work[-16:] == 255).all()
        out = moves.wide(d["out"])
        assert (out[:, self.hq * self.dim:] == 9).all()
        return out[:, :self.hq * self.dim].reshape(self.tokens, self.hq, self.dim), moves.wide(d["lse"])

    def values(self, which):
        """[page, slot, head, dim] in 64 bits, and the magnitude that roundings of them are relative to."""
        x = self.caches[which]
        x = x if self.order == "slots" else x.transpose(1, 2)
        if self.cache == "q4":
            step, low, code = ref.from_records(x.contiguous().numpy())
            # products of codes run over 16 + code, their exponentials' roundings over code - 8
            return low + step * code, 40 * np.abs(step) + np.abs(low) if which == 0 else np.broadcast_to(16 * np.abs(step) + np.abs(low), code.shape)
        x = moves.wide(x)
        if self.scales[which] is not None:
            x = x * moves.wide(self.scales[which])[:, None]
        return x, np.abs(x)

    def expect(self, scale, window=0):
        """(out, limit, lse, limit of lse), NaN where a request has no token."""
        k, kmag = self.values(0)
        v, vmag = self.values(1)
        q = moves.wide(self.q)[:, :self.hq * self.dim].reshape(self.tokens, self.hq, self.dim)
        shape = q.shape
        out, limit = np.full(shape, 9.0), np.zeros(shape)
        lse, lse_limit = np.full(shape[:2], 9.0), np.zeros(shape[:2])
        # roundings of a weight to 16 bits; of 4-bit caches to bf16
        u = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -8 if self.cache == "q4" else 2.0 ** -11}[self.kind]
        for r in range(len(self.cached)):
            c, a, b = max(int(self.cached[r]), 0), int(self.starts[r]), int(self.starts[r + 1])
            pos = np.arange(min(c + b - a, self.width * self.page))
            entry = self.table[r, pos // self.page]
            there = (entry >= 0) & (entry < self.pages)
            entry = np.where(there, entry, 0)
            kr, kmr, vr, vmr = (np.broadcast_to(x, v.shape)[entry, pos % self.page] for x in (k, kmag, v, vmag))
            for i in range(b - a):
                sees = there & (pos <= c + i)
                if window:
                    sees &= pos > c + i - window
                for h in range(self.hq):
                    g = h // (self.hq // self.hk)
                    if not sees.any():
                        out[a + i, h], lse[a + i, h] = 0, -np.inf
                        continue
                    with np.errstate(invalid="ignore", over="ignore"):
                        s = scale * (kr[sees, g] @ q[a + i, h])
                        size = abs(scale) * (kmr[sees, g] @ np.abs(q[a + i, h]))
                        m = s.max()
                        p = np.exp(s - m)
                        n = sees.sum()
                        # a score: dim products added up in 32 bits, the scale, the maximum taken away; an exponential is off by that and 2^-22
                        err = (size * (self.dim + 8) * 2.0 ** -23 + np.abs(s).max() * 2.0 ** -22 + 2.0 ** -21).max()
                        w = p / p.sum()
                        out[a + i, h] = w @ vr[sees, g]
                        err32 = (2 * err + u + (n / 16 + 60) * 2.0 ** -23) * (w @ vmr[sees, g])
                        limit[a + i, h] = ref.rounded(out[a + i, h], self.kind, err32)
                        lse[a + i, h] = m + np.log(p.sum())
                        lse_limit[a + i, h] = err + (n / 16 + 60) * 2.0 ** -23 + 2.0 ** -22 * abs(lse[a + i, h])
        return out, limit, lse, lse_limit

    def check(self, scale, window=0):
        out, limit, lse, lse_limit = self.expect(scale, window)
        got, got_lse = self.run(scale, window)
        ref.assert_within(got, out, limit, "out")
        ref.assert_within(got_lse, lse, lse_limit, "lse")


@gpu
@pytest.mark.parametrize("kind,cache,order,hq,hk,dim,page,window,lengths,pad", [
    ("bf16", "bf16", "slots", 8, 2, 128, 16, 0, [(700, 1)], 0), ("bf16", "bf16", "slots", 1, 1, 64, 16, 0, [(0, 1)], 0),
    ("bf16", "bf16", "heads", 4, 4, 128, 7, 0, [(0, 1), (1, 1), (63, 1), (64, 1), (0, 0), (300, 1), (31, 1), (32, 1)], 2),
    ("bf16", "f8", "heads", 8, 1, 128, 64, 0, [(129, 1), (1000, 1), (5, 3)], 0), ("bf16", "q4", "heads", 8, 2, 128, 16, 0, [(500, 1), (33, 1), (0, 2)], 1),
    ("f16", "f16", "slots", 6, 2, 80, 5, 0, [(10, 40), (200, 7), (0, 1), (90, 130)], 3), ("f16", "q4", "slots", 5, 5, 64, 8, 0, [(10, 90), (200, 1)], 0),
    ("f32", "f32", "slots", 4, 2, 96, 16, 0, [(150, 1), (3, 60)], 0), ("f32", "f8", "heads", 10, 5, 80, 24, 50, [(300, 7), (20, 3), (0, 7)], 0),
    ("f32", "q4", "heads", 2, 1, 192, 4, 0, [(70, 2), (0, 40)], 0), ("f32", "f32", "heads", 2, 2, 256, 16, 0, [(70, 1), (5, 1)], 0), ("f32", "f32", "slots", 2, 1, 250, 3, 0, [(9, 70)], 0),
    ("f32", "q4", "slots", 3, 1, 256, 16, 0, [(200, 1), (1, 1)], 0), ("bf16", "bf16", "slots", 3, 3, 256, 32, 0, [(0, 150), (260, 1), (64, 64)], 0),
    ("bf16", "q4", "slots", 2, 2, 256, 16, 0, [(100, 1), (0, 70)], 0), ("bf16", "f8", "slots", 4, 1, 192, 16, 20, [(100, 1), (3, 200)], 0),
    ("f16", "f8", "heads", 3, 1, 17, 3, 0, [(50, 1), (0, 1), (400, 2)], 0), ("bf16", "bf16", "slots", 7, 7, 33, 9, 0, [(11, 150)], 5),
    ("bf16", "bf16", "slots", 40, 1, 64, 16, 0, [(20, 1), (77, 1)], 0), ("bf16", "bf16", "slots", 300, 2, 64, 16, 0, [(40, 2)], 0),
    ("bf16", "bf16", "heads", 16, 4, 128, 32, 128, [(0, 500), (700, 90), (1000, 1)], 0), ("f16", "f16", "slots", 2, 1, 1, 2, 0, [(5, 1), (0, 64)], 0),
    ("bf16", "bf16", "slots", 2, 2, 128, 1, 1, [(300, 1), (2, 70)], 0), ("f16", "q4", "heads", 4, 1, 8, 16, 7, [(300, 100)], 0), ("f16", "q4", "heads", 4, 2, 192, 16, 0, [(300, 1), (128, 30)], 0),
    ("bf16", "q4", "heads", 24, 1, 128, 16, 0, [(300, 1), (65, 1)], 0), ("f16", "f8", "slots", 6, 2, 64, 16, 40, [(300, 9), (65, 8)], 0), ("f16", "q4", "slots", 8, 1, 96, 8, 0, [(200, 3), (65, 4)], 0),
    ("bf16", "f8", "heads", 16, 1, 96, 16, 0, [(99, 1), (129, 1)], 0), ("f16", "f16", "heads", 20, 1, 256, 16, 0, [(99, 1), (129, 1)], 0), ("bf16", "q4", "slots", 3, 1, 32, 16, 0, [(99, 1), (700, 1)], 0),
    ("bf16", "f8", "slots", 3, 1, 32, 16, 9, [(99, 1), (700, 1)], 0), ("bf16", "f8", "slots", 18, 1, 192, 16, 0, [(99, 1), (70, 1)], 0), ("f32", "f32", "slots", 24, 1, 64, 16, 0, [(99, 1), (70, 2)], 0)])
def test_attend(kind, cache, order, hq, hk, dim, page, window, lengths, pad):
    Problem(kind, cache, order, hq, hk, dim, page, lengths, seed=dim + page, pad=pad).check(dim ** -0.5, window)


@gpu
@pytest.mark.parametrize("requests", [65, 200, 4100])
def test_many_requests(requests):
    """Requests beyond one, and beyond 64 x 64, of the search for a tile's request; some bring nothing."""
    rng = np.random.default_rng(requests)
    lengths = [(int(c), int(f)) for c, f in zip(rng.integers(0, 20, requests), rng.integers(0, 3, requests))]
    Problem("bf16", "bf16", "slots", 2, 1, 64, 16, lengths, seed=requests, pad=3).check(0.125)


@gpu
@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "q4"), ("f32", "f8")])
def test_long_contexts_in_parts(kind, cache):
    """Positions shared among workgroups: one request by all of them, several by few; parts that see nothing of a window."""
    Problem(kind, cache, "heads", 4, 2, 64, 64, [(6000, 1)], seed=1).check(0.2)
    Problem(kind, cache, "slots", 2, 1, 64, 16, [(3000, 1), (40, 1), (0, 1), (1500, 2)], seed=2).check(0.2, 700)
    Problem(kind, cache, "slots", 2, 1, 96, 16, [(1200, 90), (40, 100)], seed=3).check(0.1)


@gpu
@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("bf16", "f8"), ("f16", "q4"), ("f32", "f32")])
@pytest.mark.parametrize("lengths", [[(150, 1), (20, 1), (64, 1)], [(100, 120), (0, 140)]])
def test_holes_and_narrow_tables(kind, cache, lengths):
    """Entries that are no page, a request of nothing else, and a table that ends before its requests do: those positions are not there."""
    p = Problem(kind, cache, "heads", 4, 2, 64, 16, lengths, seed=5, width=9)
    p.table[0, 2], p.table[0, 4], p.table[0, 5] = p.pages, -7, 2 ** 31 - 1
    p.table[1, :] = -1
    p.check(0.125)
    p.check(0.125, 30)


@gpu
@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("bf16", "f8"), ("bf16", "q4"), ("f16", "f16"), ("f16", "q4"), ("f32", "f32"), ("f32", "q4")])
@pytest.mark.parametrize("lengths,window", [([(60, 90), (0, 5)], 0), ([(200, 1), (37, 3)], 0), ([(150, 100)], 40), ([(400, 2)], 50)])
def test_what_is_not_seen_has_no_effect(kind, cache, lengths, window):
    """Infinities and NaN at every position that no token sees, and at positions that some tokens see and others do not."""
    p = Problem(kind, cache, "slots", 4, 2, 64, 16, lengths, seed=6)
    rng = np.random.default_rng(7)
    slots = []
    for r, (c, f) in enumerate(lengths):
        for at in range(-(-(c + f) // 16) * 16):
            behind = at >= c + f                                  # the rest of a page
            before = window and at <= c - window
            if behind or before or (at > c and rng.random() < 0.15):
                slots.append(int(p.table[r, at // 16]) * 16 + at % 16)
    used = {int(e) for e in p.table[p.table >= 0]}
    slots += [page * 16 + i for page in range(p.pages) if page not in used for i in range(16)]
    for which, x in enumerate(p.caches):
        flat = x.reshape(p.pages * 16, p.hk, -1)
        for n, s in enumerate(slots):
            bad = [float("nan"), float("inf"), -float("inf")][n % 3 if which else 0]
            if cache == "q4":
                flat[s, n % p.hk, :4] = torch.tensor([bad, 1.0], dtype=torch.bfloat16).view(torch.uint8)
            elif cache == "f8":
                flat.view(torch.uint8)[s, n % p.hk, n % 64] = 0x7f | n % 2 << 7
            else:
                flat[s, n % p.hk, n % 64] = bad
    out, limit, lse, lse_limit = p.expect(0.125, window)
    got, got_lse = p.run(0.125, window)
    assert np.isfinite(got).any() and np.array_equal(np.isnan(lse), np.isnan(got_lse))
    # a row that sees a NaN key is NaN in all; a value that is not finite is in its elements only
    fine = np.isfinite(out)
    assert np.array_equal(fine, np.isfinite(got))
    ref.assert_within(np.where(fine, got, 0), np.where(fine, out, 0), np.where(fine, limit, 0))


@gpu
def test_infinite_values_come_out_with_their_sign():
    p = Problem("bf16", "bf16", "slots", 2, 1, 64, 16, [(10, 60)], seed=8)
    flat = p.caches[1].transpose(1, 2).reshape(-1, 64) if p.order == "heads" else p.caches[1].reshape(-1, 64)
    slot = lambda at: int(p.table[0, at // 16]) * 16 + at % 16  # noqa: E731
    flat[slot(20), 0], flat[slot(30), 1], flat[slot(25), 2], flat[slot(40), 2], flat[slot(33), 3] = float("inf"), -float("inf"), float("inf"), -float("inf"), float("nan")
    out, limit, _, _ = p.expect(0.1)
    got, _ = p.run(0.1)
    ref.assert_within(got, out, limit)
    assert np.isposinf(got[10:, :, 0]).all() and np.isneginf(got[20:, :, 1]).all() and np.isposinf(got[15:30, :, 2]).all() and np.isnan(got[30:, :, 2]).all()


@gpu
@pytest.mark.parametrize("scale", [0.0, -0.25, 3.0])
@pytest.mark.parametrize("cache", ["bf16", "f8", "q4"])
def test_scales(scale, cache):
    """None, a negative one, a large one (weights of one position only); a negative scale of the cache beside it."""
    p = Problem("bf16", cache, "slots", 4, 2, 64, 16, [(100, 1), (0, 40)], seed=9)
    if cache == "f8":
        p.scales[0][1] = -0.7
        p.scales[1][0] = -1.3
    p.check(scale)


@gpu
def test_rows_around_the_requests_are_left_and_bad_starts_stay_inside():
    p = Problem("bf16", "bf16", "slots", 2, 1, 64, 16, [(10, 5), (3, 6)], seed=10, pad=7)
    p.starts = p.starts + 4                                       # four tokens before the first request's
    got, lse = p.run(0.125)
    assert (got[:4] == 9).all() and (got[15:] == 9).all() and (lse[:4] == 9).all() and (lse[15:] == 9).all() and (got[4:15] != 9).any(-1).all()
    for starts in ([-5, 3, 2 ** 31 - 1], [9, 4, 1], [0, -1, -2], [2 ** 31 - 1] * 3):
        p.starts = np.array(starts, np.int32)
        p.cached = np.array([-4, 2 ** 31 - 1], np.int32)
        p.run(0.125)


@gpu
def test_offsets_beyond_32_bits():
    """A cache of 6 GB, of which the last pages are used."""
    pages, page, dim = 23500, 16, 128
    p = Problem("bf16", "bf16", "slots", 2, 1, dim, page, [(100, 1), (40, 20)], seed=11)
    heads = 64
    k, v = (torch.zeros(pages, page, heads, dim, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    assert k.numel() * 2 > 2 ** 32
    at = torch.arange(pages - p.pages, pages)
    for big, small in ((k, p.caches[0]), (v, p.caches[1])):
        big[at.to(DEV), :, heads - 1] = small[:, :, 0].to(DEV)
    want, limit, _, _ = p.expect(0.1)
    table = torch.from_numpy(np.where(p.table >= 0, p.table + pages - p.pages, -1).astype(np.int32)).to(DEV)
    q = torch.zeros(p.tokens, heads * 2 * dim, dtype=torch.bfloat16, device=DEV)
    q[:, -2 * dim:] = p.q[:, :2 * dim].to(DEV)
    out, d = torch.empty_like(q), p.to_gpu()
    with Handle(ttc.ttc_pages_create, ttc.ttc_pages_destroy, ttc.TTC_BF16, ttc.TTC_BF16, heads, dim, page, pages) as c, \
            Handle(ttc.ttc_attend_create, ttc.ttc_attend_destroy, c, 2 * heads, 0.1, 0) as attend:
        work = torch.empty(max(16, ttc.ttc_attend_workspace(attend, 2, p.tokens, p.width)), dtype=torch.uint8, device=DEV)
        ttc.ttc_attend_pages(attend, 2, p.tokens, ptr(q), q.shape[1], ptr(d["starts"]), ptr(d["cached"]), ptr(table), p.width, ptr(k), ptr(v), 0, 0, ptr(out), q.shape[1], 0, ptr(work), stream())
    got = moves.wide(out)[:, -2 * dim:].reshape(want.shape)
    ref.assert_within(got, want, limit)


@gpu
@pytest.mark.parametrize("lengths", [[(900, 1), (30, 1), (400, 1)], [(100, 150), (0, 80)]])
def test_same_bits_again_on_another_stream_and_in_graphs(lengths):
    """Two runs, a run on another stream, and two captured graphs with workspaces of their own, replayed in turn with eager work between."""
    p = Problem("bf16", "bf16", "slots", 4, 1, 64, 16, lengths, seed=12)
    pages, attend_of = p.handles(0.125, 0)
    with pages as c, attend_of(c) as attend:
        d = [p.to_gpu() for _ in range(3)]
        work = [p.workspace(attend) for _ in range(3)]
        p.call(attend, d[0], work[0])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            p.call(attend, d[1], work[1])
        torch.cuda.synchronize()
        assert torch.equal(d[0]["out"], d[1]["out"]) and torch.equal(d[0]["lse"], d[1]["lse"])
        graphs = []
        for i in (1, 2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                p.call(attend, d[i], work[i])
            graphs.append(graph)
        for _ in range(3):
            for i, graph in zip((1, 2), graphs):
                d[i]["out"].fill_(9.0)
                work[i].fill_(255)
                graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(d[0]["out"], d[1]["out"]) and torch.equal(d[0]["out"], d[2]["out"])
            p.call(attend, d[0], work[0])


@gpu
@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "f8"), ("f16", "q4"), ("bf16", "q4"), ("f32", "f32")])
@pytest.mark.parametrize("fresh", [1, 100])
def test_scores_that_rise_along_the_positions(kind, cache, fresh):
    """The largest score so far moves by a little in every tile, and by much at some: each exponential is taken of a difference to some earlier maximum."""
    p = Problem(kind, cache, "slots", 2, 1, 32, 16, [(900, fresh), (40, fresh)], seed=13)
    p.q.fill_(0)
    p.q[:, 0::32] = 1                                             # a score is 16 times the key's first element
    for r in range(2):
        c, f = int(p.cached[r]), int(p.starts[r + 1] - p.starts[r])
        for at in range(c + f):
            x, where = (at % 400) / 128 + 2 * (at // 400), (int(p.table[r, at // 16]), at % 16, 0)
            if cache == "q4":
                p.caches[0][where][:4] = torch.tensor([2.0 ** -7, x], dtype=torch.bfloat16).view(torch.uint8)
                p.caches[0][where][4:] = 0
            else:
                p.caches[0][where][0] = x
    if cache == "f8":
        p.scales[0].fill_(1.0)
    p.check(16.0)


@gpu
@pytest.mark.parametrize("lengths", [[(70, 1), (300, 1)], [(200, 20)], [(30, 100), (0, 64)]])
def test_fp16_over_four_bits_keeps_its_precision(lengths):
    """Steps from 2^-14 to 2^10, exponentials times steps rounded to fp16 and no further."""
    p = Problem("f16", "q4", "slots", 4, 1, 128, 16, lengths, seed=14)
    g = torch.Generator().manual_seed(15)
    shape = p.caches[1].shape[:3]
    step = (2.0 ** torch.randint(-14, 11, shape, generator=g) * (1 + torch.rand(shape, generator=g))).to(torch.bfloat16)
    p.caches[1][..., :4] = torch.stack([step, -7 * step], -1).to(torch.bfloat16).view(torch.uint8)
    out, limit, lse, lse_limit = p.expect(0.01)
    # The limit without the roundings of weights has those to 2^-8 taken out: of w |16 step + min| all told.  In fp16 a weight is off by 2^-11 of itself, or by 2^-25 where
    # that is more: of a scale on which the largest of the row is 1 at least.  A code's factor is 8 + 16 at most beside it.
    step, low, code = ref.from_records(p.caches[1].contiguous().numpy())
    k, _ = p.values(0)
    q = moves.wide(p.q)[:, :4 * 128].reshape(p.tokens, 4, 128)
    for r, (c, f) in enumerate(lengths):
        for i in range(f):
            at = np.arange(c + i + 1)
            entry, slot = p.table[r, at // 16], at % 16
            st, mag = np.abs(step[entry, slot, 0]).reshape(-1), (16 * np.abs(step) + np.abs(low))[entry, slot, 0].reshape(-1)
            t = int(p.starts[r]) + i
            for h in range(4):
                s = 0.01 * (k[entry, slot, 0] @ q[t, h])
                w = np.exp(s - s.max())
                w /= w.sum()
                limit[t, h] -= (2.0 ** -8 - 2.0 ** -11) * (w @ mag) * (1 + 2.0 ** -11)
                limit[t, h] += (len(at) * 24 * 2.0 ** -25 * (w * st).max()) * (1 + 2.0 ** -11)
    got, got_lse = p.run(0.01)
    ref.assert_within(got, out, limit)
    ref.assert_within(got_lse, lse, lse_limit, "lse")


@gpu
@pytest.mark.parametrize("kind,cache,dim", [("bf16", "bf16", 256), ("f16", "f8", 256), ("bf16", "q4", 256), ("f32", "f32", 192), ("f32", "q4", 256), ("bf16", "f8", 200)])
@pytest.mark.parametrize("fresh", [3, 5, 7])
def test_wide_heads_and_tiles_of_every_size(kind, cache, dim, fresh):
    """24, 40 and 56 rows of a request's."""
    Problem(kind, cache, "slots", 8, 1, dim, 16, [(150, fresh), (0, fresh), (31, fresh)], seed=16).check(0.05)


@gpu
def test_first_call_in_a_graph():
    """A kernel that asks for more LDS than every launch may have asks for it on its first call, which may be a captured one."""
    p = Problem("bf16", "bf16", "slots", 6, 1, 200, 16, [(40, 90)], seed=17)
    pages, attend_of = p.handles(0.1, 0)
    with pages as c, attend_of(c) as attend:
        d, eager, work = p.to_gpu(), p.to_gpu(), p.workspace(attend)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            p.call(attend, d, work)
        p.call(attend, eager, work)
        for _ in range(3):
            d["out"].fill_(9.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(d["out"], eager["out"]) and torch.equal(d["lse"], eager["lse"])


@gpu
@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("f16", "q4"), ("f32", "f8")])
@pytest.mark.parametrize("lengths", [[(100, 1), (0, 1)], [(0, 150), (33, 90)]])
def test_rows_at_any_element_and_two_streams_at_once(kind, cache, lengths):
    """Queries and results one element behind an aligned address, rows an odd distance apart; two streams beside each other, with a workspace each."""
    p = Problem(kind, cache, "heads", 4, 2, 64, 16, lengths, seed=18)
    out, limit, _, _ = p.expect(0.125)
    pages, attend_of = p.handles(0.125, 0)
    row = p.hq * p.dim
    q = torch.zeros(p.tokens * (row + 3) + 1, dtype=p.dtype, device=DEV)
    q[1:].view(p.tokens, row + 3)[:, :row] = p.q[:, :row].to(DEV)
    with pages as c, attend_of(c) as attend:
        d, got, works = p.to_gpu(), [torch.full((p.tokens * (row + 5) + 1,), 9.0, dtype=p.dtype, device=DEV) for _ in range(2)], [p.workspace(attend) for _ in range(2)]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        for _ in range(20):
            for s, x, work in zip(streams, got, works):
                with torch.cuda.stream(s):
                    ttc.ttc_attend_pages(attend, len(p.cached), p.tokens, q.data_ptr() + q.element_size(), row + 3, ptr(d["starts"]), ptr(d["cached"]), ptr(d["table"]), p.width,
                                         ptr(d["k"]), ptr(d["v"]), ptr(d["ks"]), ptr(d["vs"]), x.data_ptr() + x.element_size(), row + 5, 0, ptr(work), stream())
        torch.cuda.synchronize()
    for x in got:
        y = moves.wide(x)
        assert y[0] == 9 and (y[1:].reshape(p.tokens, row + 5)[:, row:] == 9).all()
        ref.assert_within(y[1:].reshape(p.tokens, row + 5)[:, :row].reshape(out.shape), out, limit)


@gpu
@pytest.mark.parametrize("lengths", [[(100, 1), (7, 2)], [(10, 150)]])
def test_no_table_at_all(lengths):
    """Tables of no entries: nothing is there, whatever the lengths say."""
    p = Problem("bf16", "bf16", "slots", 2, 1, 64, 16, lengths, seed=19, width=0)
    got, lse = p.run(0.125)
    assert (got == 0).all() and np.isneginf(lse).all()


# ---- refusals: before anything reaches a device -----------------------------------------------------------

V, O, T, N, A, M = (getattr(ttc, "TTC_ERR_" + x) for x in ("INVALID_VALUE", "OVERFLOW", "UNSUPPORTED_DTYPE", "NULL_POINTER", "ALIAS", "MISALIGNED"))


def refused(status, f, *args):
    with pytest.raises(ttc.TtcError) as e:
        f(*args)
    assert e.value.status == status


def pages_of(*args):
    return Handle(ttc.ttc_pages_create, ttc.ttc_pages_destroy, *args)


def test_create_refuses():
    with pages_of(ttc.TTC_BF16, ttc.TTC_BF16, 2, 64, 16, 10) as p, pages_of(ttc.TTC_BF16, ttc.TTC_BF16, 2, 257, 16, 10) as wide, pages_of(ttc.TTC_BF16, ttc.TTC_F8, 70000, 8, 1, 1) as many:
        for args, status in (((0, 4, 1.0), N), ((p, 3, 1.0), V), ((p, 0, 1.0), V), ((p, 4, float("nan")), V), ((p, 4, float("inf")), V), ((p, 4, 1e300), V), ((p, 4, 1.0, -1), V), ((wide, 2, 1.0), V),
                             ((p, 1 << 21, 1.0), O), ((many, 70000, 1.0), O)):
            refused(status, ttc.ttc_attend_create, *args)
            assert ttc.ttc_last_status() == status
        a = ttc.ttc_attend_create(p, 4, -0.5, 1 << 40)
        ttc.ttc_attend_destroy(a)
        ttc.ttc_attend_destroy(None)


def test_attend_refuses():
    Q, S, C, B, K, W, X, L = (i << 40 for i in range(1, 9))
    with pages_of(ttc.TTC_BF16, ttc.TTC_BF16, 2, 64, 16, 10) as p, pages_of(ttc.TTC_BF16, ttc.TTC_F8, 2, 64, 16, 10) as f8, \
            Handle(ttc.ttc_attend_create, ttc.ttc_attend_destroy, p, 4, 0.125, 0) as h, Handle(ttc.ttc_attend_create, ttc.ttc_attend_destroy, f8, 4, 0.125, 0) as h8:
        assert ttc.ttc_attend_workspace(h, 3, 3, 100) > 0 and ttc.ttc_attend_workspace(h, 0, 0, 100) == 0
        ok = [h, 3, 3, Q, 256, S, C, B, 100, K, K + (1 << 20), 0, 0, X, 256, L, W, 0]
        for change, status in (({0: 0}, N), ({1: -1}, V), ({2: -1}, V), ({8: -1}, V), ({1: 1 << 40}, O), ({2: 1 << 40}, O), ({8: 1 << 50}, O), ({4: 255}, V), ({14: 255}, V), ({11: W}, V), ({12: W}, V),
                               ({3: 0}, N), ({5: 0}, N), ({6: 0}, N), ({7: 0}, N), ({9: 0}, N), ({10: 0}, N), ({13: 0}, N), ({16: 0}, N), ({3: Q + 1}, M), ({5: S + 2}, M), ({16: W + 8}, M), ({15: L + 2}, M),
                               ({13: Q}, A), ({13: Q + 512, 14: 512, 4: 300}, A), ({13: K}, A), ({15: X}, A), ({16: X}, A), ({16: K}, A), ({15: W}, A), ({7: X}, A), ({0: h8, 11: X}, A)):
            args = list(ok)
            for k, v in change.items():
                args[k] = v
            refused(status, ttc.ttc_attend_pages, *args)
        ttc.ttc_attend_pages(h, 0, 0, 0, 256, 0, 0, 0, 0, 0, 0, 0, 0, 0, 256, 0, 0)
        ttc.ttc_attend_pages(h, 4, 0, 0, 256, 0, 0, 0, 5, 0, 0, 0, 0, 0, 256, 0, 0)
        refused(N, ttc.ttc_attend_workspace, 0, 1, 1, 1)
        refused(V, ttc.ttc_attend_workspace, h, 1, -1, 1)
        refused(O, ttc.ttc_attend_workspace, h, 1, 1 << 40, 1)
