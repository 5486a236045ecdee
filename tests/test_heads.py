"""Norms of the heads with the rotation by position, their gradients, and the same on the way into the cache (include/ttc_attention.h, ttc_heads_*,
ttc_pages_append) against plain implementations in 64 bits."""
import numpy as np
import pytest
import torch

import attention_reference as ref
import moves_reference as moves
import paper_1603_02297_amd as ttc

gpu = pytest.mark.gpu
DEV = "cuda"

# Roundings of 2^-24 that a result holds at most.  Norm: squares of up to 16 elements a lane, six additions over lanes, a product and the eps, halved by
# the root; the root, the division, two products: 25 / 2 + 4.  Rotation: angle and series are off by 4, two products and their sum.
NORM, TURN = 17, 7


class Handle:
    def __init__(self, create, destroy, *args):
        self.h, self.destroy = create(*args), destroy

    def __enter__(self):
        return self.h

    def __exit__(self, *_):
        self.destroy(self.h)


def heads(*args):
    return Handle(ttc.ttc_heads_create, ttc.ttc_heads_destroy, *args)


def stream():
    return torch.cuda.current_stream().cuda_stream


def ptr(x):
    return 0 if x is None else x.data_ptr()


def packed(g, tokens, widths, dtype, pad=0, offset=0):
    """Parts of one projection, side by side, after `offset` elements and with `pad` unused ones behind each row."""
    row = sum(widths) + pad
    flat = torch.randn(tokens * row + offset, generator=g).to(dtype).to(DEV)
    whole = flat[offset:].view(tokens, row)
    parts, at = [], 0
    for w in widths:
        parts.append(whole[:, at:at + w])
        at += w
    return parts, row


CASES = [  # dtype, tokens, q_heads, kv_heads, dim, rotated, paired, norm, pad, offset
    ("bf16", 1, 1, 1, 64, 64, 0, 1, 0, 0), ("bf16", 5, 32, 8, 128, 128, 0, 1, 0, 0), ("f16", 300, 4, 2, 128, 64, 1, 1, 3, 1), ("f32", 77, 6, 3, 80, 40, 1, 1, 0, 0),
    ("f32", 33, 3, 1, 96, 96, 0, 0, 5, 3), ("bf16", 2500, 2, 1, 64, 32, 0, 1, 0, 0), ("f16", 19, 7, 5, 80, 80, 0, 1, 0, 0), ("bf16", 9, 2, 2, 256, 256, 1, 1, 0, 0),
    ("bf16", 40, 3, 2, 17, 6, 0, 1, 1, 0), ("f32", 11, 2, 1, 1, 0, 0, 1, 0, 0), ("f16", 6, 1, 3, 512, 256, 0, 1, 0, 0), ("f32", 4, 2, 2, 511, 250, 1, 1, 0, 7),
    ("f32", 3, 1, 1, 512, 128, 1, 1, 0, 0), ("bf16", 70, 5, 1, 192, 96, 0, 0, 0, 0), ("bf16", 4700, 9, 1, 128, 128, 0, 1, 0, 0), ("f16", 21, 2, 1, 20, 20, 1, 1, 0, 0)]


def positions_of(tokens, rng, padded=True):
    p = rng.integers(0, 1 << 20, tokens).astype(np.int32)
    p[: min(3, tokens)] = [0, 1, 2 ** 31 - 1][: min(3, tokens)]
    if padded and tokens > 4:
        p[rng.random(tokens) < 0.1] = -1
        p[4] = -2 ** 31
    return p


@gpu
@pytest.mark.parametrize("kind,tokens,hq,hk,dim,rotated,paired,norm,pad,offset", CASES)
def test_rotate(kind, tokens, hq, hk, dim, rotated, paired, norm, pad, offset):
    code, dtype = ref.TYPES[kind]
    g, rng = torch.Generator().manual_seed(tokens), np.random.default_rng(dim)
    (q, k, _), ld = packed(g, tokens, (hq * dim, hk * dim, hk * dim), dtype, pad, offset)
    w = [(1 + 0.2 * torch.randn(dim, generator=g)).to(DEV) if norm and dim != 64 else None for _ in range(2)]
    pos = positions_of(tokens, rng)
    angle = ref.angles(rotated) if rotated else None
    dpos = torch.from_numpy(pos).to(DEV)
    outs = [torch.full((tokens, h * dim + 5), 9.0, dtype=dtype, device=DEV) for h in (hq, hk)]
    with heads(code, hq, hk, dim, rotated, paired, angle, norm, ref.EPS) as h:
        ttc.ttc_heads_rotate(h, tokens, ptr(dpos), ptr(q), ld, ptr(k), ld, ptr(w[0]), ptr(w[1]), ptr(outs[0]), hq * dim + 5, ptr(outs[1]), hk * dim + 5, stream())
        for x, weight, n, out in ((q, w[0], hq, outs[0]), (k, w[1], hk, outs[1])):
            wide = moves.wide(x).reshape(tokens, n, dim)
            want, size = ref.heads(wide, None if weight is None else moves.wide(weight), pos, angle, rotated, paired, norm)
            got = moves.wide(out)
            assert (got[:, n * dim:] == 9).all() and (got[pos < 0] == 9).all()
            keep = pos >= 0
            limit = ref.rounded(want, kind, (NORM * norm + TURN) * ref.F32 * size)
            ref.assert_within(got[:, :n * dim].reshape(want.shape)[keep], want[keep], limit[keep])
        # in place, and one of the two only, give the same bits
        both = q.clone(), k.clone()
        ttc.ttc_heads_rotate(h, tokens, ptr(dpos), ptr(both[0]), hq * dim, 0, 0, ptr(w[0]), 0, ptr(both[0]), hq * dim, 0, 0, stream())
        ttc.ttc_heads_rotate(h, tokens, ptr(dpos), 0, 0, ptr(both[1]), hk * dim, 0, ptr(w[1]), 0, 0, ptr(both[1]), hk * dim, stream())
        for x, out, was, n in ((both[0], outs[0], q, hq), (both[1], outs[1], k, hk)):
            assert torch.equal(x[dpos >= 0], out[:, :n * dim][dpos >= 0]) and torch.equal(x[dpos < 0], was[dpos < 0])


@gpu
@pytest.mark.parametrize("kind,tokens,hq,hk,dim,rotated,paired,norm,pad,offset", CASES)
def test_grad(kind, tokens, hq, hk, dim, rotated, paired, norm, pad, offset):
    code, dtype = ref.TYPES[kind]
    g, rng = torch.Generator().manual_seed(tokens + 1), np.random.default_rng(dim)
    (q, k, _), ld = packed(g, tokens, (hq * dim, hk * dim, hk * dim), dtype, pad, offset)
    (dq_out, dk_out), ldd = packed(g, tokens, (hq * dim, hk * dim), dtype, 2, 0)
    w = [(1 + 0.2 * torch.randn(dim, generator=g)).to(DEV) if norm and dim != 64 else None for _ in range(2)]
    pos = positions_of(tokens, rng)
    angle, dpos, keep = ref.angles(rotated) if rotated else None, torch.from_numpy(pos).to(DEV), pos >= 0
    with heads(code, hq, hk, dim, rotated, paired, angle, norm, ref.EPS) as h:
        def run(weights=True, which="qk"):
            outs = [torch.full((tokens, n * dim + 5), 9.0, dtype=dtype, device=DEV) for n in (hq, hk)]
            dw = [torch.full((dim,), 9.0, device=DEV) if norm and weights else None for _ in range(2)]
            work = torch.empty(max(1, ttc.ttc_heads_workspace(h, tokens)), dtype=torch.uint8, device=DEV).fill_(255)
            a = (ptr(dq_out), ldd, ptr(dk_out), ldd, ptr(q), ld, ptr(k), ld)
            ttc.ttc_heads_rotate_grad(h, tokens, ptr(dpos), *a, ptr(w[0]), ptr(w[1]), ptr(outs[0]), hq * dim + 5, ptr(outs[1]), hk * dim + 5, ptr(dw[0]), ptr(dw[1]),
                                      ptr(work) if norm and weights else 0, stream())
            return outs, dw
        outs, dw = run()
        # additions behind a weight's gradient: a lane's own, one for each of its heads, then lanes, wavefronts, workgroups
        chain = tokens * (hq + hk) / 64 + 10 + 4 + 64 + 16
        for x, dy, weight, n, out, dweight in ((q, dq_out, w[0], hq, outs[0], dw[0]), (k, dk_out, w[1], hk, outs[1], dw[1])):
            wide, wdy = (moves.wide(v).reshape(tokens, n, dim) for v in (x, dy))
            dx, size, total, total_size = ref.heads_grad(wdy[keep], wide[keep], None if weight is None else moves.wide(weight), pos[keep], angle, rotated, paired, norm)
            got = moves.wide(out)
            assert (got[:, n * dim:] == 9).all() and (got[~keep] == 9).all()
            # x/s twice, its mean with a sum over the head, the rotation, and the last two products
            limit = ref.rounded(dx, kind, (2 * NORM * norm + TURN + 28 * norm) * ref.F32 * size)
            ref.assert_within(got[:, :n * dim].reshape(tokens, n, dim)[keep], dx, limit)
            if norm:
                ref.assert_within(moves.wide(dweight), total, (NORM + TURN + 1 + chain) * ref.F32 * total_size)
        again, dw2 = run()
        assert all(torch.equal(a, b) for a, b in zip(outs, again)) and all(a is None or torch.equal(a, b) for a, b in zip(dw, dw2))
        without, _ = run(weights=False)
        assert all(torch.equal(a, b) for a, b in zip(outs, without))


@gpu
@pytest.mark.parametrize("paired,rotated", [(0, 16), (1, 12), (0, 6)])
def test_gradients_against_differences(paired, rotated):
    """The formula's gradients and the kernel's against central differences of the formula."""
    rng = np.random.default_rng(5)
    tokens, n, dim, pos, angle = 3, 2, 16, np.array([0, 7, 1000], np.int32), ref.angles(rotated)
    x, dy = (rng.standard_normal((tokens, n, dim)).astype(np.float32).astype(np.float64) for _ in range(2))
    w = (1 + 0.2 * rng.standard_normal(dim)).astype(np.float32).astype(np.float64)
    f = lambda x, w: (ref.heads(x, w, pos, angle, rotated, paired, 1)[0] * dy).sum()  # noqa: E731
    step, dx, dw = 1e-5, np.empty_like(x), np.empty_like(w)
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = step
        dx[i] = (f(x + e, w) - f(x - e, w)) / (2 * step)
    for i in range(dim):
        e = np.zeros_like(w)
        e[i] = step
        dw[i] = (f(x, w + e) - f(x, w - e)) / (2 * step)
    t = lambda v, *s: torch.from_numpy(v.astype(np.float32).reshape(*s)).to(DEV)  # noqa: E731
    tx, tdy, tw, tpos = t(x, tokens, -1), t(dy, tokens, -1), t(w, -1), torch.from_numpy(pos).to(DEV)
    out, out_w = torch.empty_like(tx), torch.empty(dim, device=DEV)
    with heads(ttc.TTC_F32, n, 1, dim, rotated, paired, angle, 1, ref.EPS) as h:
        work = torch.empty(ttc.ttc_heads_workspace(h, tokens), dtype=torch.uint8, device=DEV)
        ttc.ttc_heads_rotate_grad(h, tokens, ptr(tpos), ptr(tdy), n * dim, 0, 0, ptr(tx), n * dim, 0, 0, ptr(tw), 0, ptr(out), n * dim, 0, 0, ptr(out_w), 0, ptr(work), stream())
    # differences are off by step^2 times a third derivative (below 1e2 here) and by 2^-52 * |f| / step
    assert np.abs(moves.wide(out).reshape(x.shape) - dx).max() < 2e-6 * max(1, np.abs(dx).max()) + 1e-8
    assert np.abs(moves.wide(out_w) - dw).max() < 2e-6 * max(1, np.abs(dw).max()) + 1e-8


@gpu
def test_rotation_far_out_and_of_whole_turns():
    """Positions to 2^31 - 1 and angles of many turns, negative ones among them, against Python's integers: the angle is a double, which is a fraction."""
    from fractions import Fraction
    import math
    angle = [1.0, 2 * math.pi, -3.0, 1e-9, 12345.678, 0.0, 1 / 3, 5e-6]
    pos = np.array([0, 1, 12345, 2 ** 24 + 1, 2 ** 31 - 1], np.int32)
    x = torch.zeros(len(pos), 16)
    x[:, :8] = 1                                                  # (1, 0) turned: cos and sin
    out, dpos = x.to(DEV), torch.from_numpy(pos).to(DEV)
    with heads(ttc.TTC_F32, 1, 1, 16, 16, 0, angle, 0, 0.0) as h:
        ttc.ttc_heads_rotate(h, len(pos), ptr(dpos), ptr(out), 16, 0, 0, 0, 0, ptr(out), 16, 0, 0, stream())
    got = moves.wide(out)
    # 2 pi to 200 bits, by Machin's formula
    def arctan_inverse(n, bits):
        one, total, term, k = 1 << bits, 0, (1 << bits) // n, 1
        while term:
            total += term // k if k % 4 == 1 else -(term // k)
            term //= n * n
            k += 2
        return Fraction(total, one)
    two_pi = 8 * (4 * arctan_inverse(5, 220) - arctan_inverse(239, 220))
    for i, p in enumerate(pos.tolist()):
        for j, a in enumerate(angle):
            turns = Fraction(a) * p / two_pi
            r = float((turns - math.floor(turns)) * two_pi)
            # the angle is rounded to 2^-64 of a turn, or by a long double's 2^-64 of it, before it is multiplied
            slack = p * max(2.0 ** -64, abs(a) / 6 * 2.0 ** -63) * 7
            assert abs(got[i, j] - math.cos(r)) < 5 * ref.F32 + slack and abs(got[i, 8 + j] - math.sin(r)) < 5 * ref.F32 + slack, (p, a)


@gpu
def test_infinities_and_nan_stay_in_their_heads():
    """A head with a NaN becomes NaN, its neighbours do not; without a norm only the pair does."""
    x = torch.ones(2, 3 * 64, dtype=torch.bfloat16, device=DEV)
    x[0, 64 + 5] = float("nan")
    x[1, 7] = float("inf")
    pos = torch.tensor([3, 4], dtype=torch.int32, device=DEV)
    for norm in (0, 1):
        out = torch.empty_like(x)
        with heads(ttc.TTC_BF16, 3, 1, 64, 64, 0, ref.angles(64), norm, ref.EPS) as h:
            ttc.ttc_heads_rotate(h, 2, ptr(pos), ptr(x), 192, 0, 0, 0, 0, ptr(out), 192, 0, 0, stream())
        bad = ~torch.isfinite(out.view(2, 3, 64))
        assert not bad[0, [0, 2]].any() and not bad[1, 1:].any()
        assert bad[0, 1].all() if norm else bad[0, 1].nonzero().flatten().tolist() == [5, 37]
        assert bad[1, 0].any()


@gpu
@pytest.mark.parametrize("kind,cache,order,tokens,hq,hk,dim,rotated,paired,norm,page", [
    ("bf16", "bf16", "slots", 1, 8, 2, 128, 128, 0, 1, 16), ("bf16", "f8", "heads", 50, 4, 4, 64, 64, 0, 1, 8), ("bf16", "q4", "heads", 37, 4, 2, 128, 128, 0, 1, 16),
    ("f16", "f16", "heads", 300, 6, 3, 80, 40, 1, 1, 7), ("f16", "q4", "slots", 70, 2, 1, 80, 16, 1, 0, 5), ("f32", "f32", "slots", 20, 3, 3, 96, 96, 0, 1, 32),
    ("f32", "f8", "heads", 90, 2, 1, 17, 6, 0, 1, 3), ("f32", "q4", "slots", 44, 1, 5, 256, 256, 1, 1, 4), ("f16", "f8", "slots", 2600, 3, 1, 64, 0, 0, 0, 16),
    ("bf16", "q4", "heads", 9, 2, 2, 512, 32, 0, 1, 2)])
def test_append(kind, cache, order, tokens, hq, hk, dim, rotated, paired, norm, page):
    """Queries, keys and values of one projection; slots in no order, some nowhere, padded tokens; the rest of the cache stays as it was."""
    code, dtype = ref.TYPES[kind]
    cache_code, cache_type = ref.TYPES[cache]
    g, rng = torch.Generator().manual_seed(tokens), np.random.default_rng(dim + page)
    (q, k, v), ld = packed(g, tokens, (hq * dim, hk * dim, hk * dim), dtype, 1)
    w = [(1 + 0.2 * torch.randn(dim, generator=g)).to(DEV) if norm else None for _ in range(2)]
    pos, angle = positions_of(tokens, rng), ref.angles(rotated) if rotated else None
    pages, rec = -(-tokens // page) + 2, dim // 2 + 4 if cache == "q4" else dim
    slots = rng.permutation(pages * page)[:tokens].astype(np.int32)
    if tokens > 5:
        slots[rng.random(tokens) < 0.1] = -1
        slots[5] = pages * page
    shape = (pages, page, hk, rec) if order == "slots" else (pages, hk, page, rec)
    strides = (rec, hk * rec, page * hk * rec) if order == "slots" else (page * rec, rec, page * hk * rec)
    caches = [torch.full((*shape,), 77, dtype=torch.uint8, device=DEV).to(cache_type) for _ in range(2)]
    scales = [torch.rand(hk, generator=g).mul(0.05).add(0.01).to(DEV) if cache == "f8" else None for _ in range(2)]
    dpos, dslots = torch.from_numpy(pos).to(DEV), torch.from_numpy(slots).to(DEV)
    q_out = torch.full((tokens, hq * dim), 9.0, dtype=dtype, device=DEV)
    with heads(code, hq, hk, dim, rotated, paired, angle, norm, ref.EPS) as h, \
            Handle(ttc.ttc_pages_create, ttc.ttc_pages_destroy, code, cache_code, hk, dim, page, pages, strides) as p:
        def run(q_in, q_to, *c):
            ttc.ttc_pages_append(p, h, tokens, ptr(dslots), ptr(dpos), ptr(q_in), ld, ptr(k), ld, ptr(v), ld, ptr(w[0]), ptr(w[1]), ptr(q_to), hq * dim, ptr(c[0]), ptr(c[1]),
                                 ptr(scales[0]), ptr(scales[1]), stream())
        run(q, q_out, *caches)
        other = [torch.full((*shape,), 77, dtype=torch.uint8, device=DEV).to(cache_type) for _ in range(2)]
        run(None, None, *other)
    bits = lambda x: x.view(torch.uint8) if cache == "f8" else x  # noqa: E731
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip(caches, other))
    wide = lambda x, n: moves.wide(x).reshape(tokens, n, dim)  # noqa: E731
    weight = [None if x is None else moves.wide(x) for x in w]
    want, size = ref.heads(wide(q, hq), weight[0], pos, angle, rotated, paired, norm)
    got, keep = wide(q_out, hq), pos >= 0
    ref.assert_within(got[keep], want[keep], ref.rounded(want, kind, (NORM * norm + TURN) * ref.F32 * size)[keep], "q")
    assert (got[~keep] == 9).all()
    here = keep & (slots >= 0) & (slots < pages * page)
    for name, x, out, scale, y, ysize in (("k", k, caches[0], scales[0], *ref.heads(wide(k, hk), weight[1], pos, angle, rotated, paired, norm)),
                                          ("v", v, caches[1], scales[1], wide(v, hk), None)):
        err = 0 * y if ysize is None else (NORM * norm + TURN) * ref.F32 * ysize
        by_slot = out if order == "slots" else out.transpose(1, 2)
        flat = by_slot.reshape(pages * page, hk, rec)
        untouched = np.ones(pages * page, bool)
        untouched[slots[here]] = False
        blank = torch.full((1,), 77, dtype=torch.uint8, device=DEV).to(cache_type)
        assert (bits(flat)[torch.from_numpy(untouched).to(DEV)] == bits(blank)).all()
        y, err, held = y[here], err[here], flat[torch.from_numpy(slots[here].astype(np.int64)).to(DEV)]
        if cache == "q4":
            step, low, c = ref.from_records(held.cpu().numpy())
            # minimum and step reach from the smallest to the largest element, and are the nearest of bf16 that do, within what y is off
            e = err.max(-1, keepdims=True) + 2.0 ** -22 * (np.abs(y).max(-1, keepdims=True))
            lo, hi = y.min(-1, keepdims=True), y.max(-1, keepdims=True)
            assert (low <= lo + e).all() and (low >= ref.bf16_towards(lo - e, np.floor)).all()
            assert (low + 15 * step >= hi - 2 * e).all() and (step <= ref.bf16_towards((hi - low + 2 * e) / 15, np.ceil)).all()
            assert (np.abs(low + c * step - y) <= step / 2 + 2 * e).all()
        elif cache == "f8":
            s = moves.wide(scale)[:, None]
            x32 = np.clip(y / s, -448, 448)
            # a value between two of the format's may fall to either within what y is off: at most half a step, 2^-4 of it or 2^-10, and the error itself
            limit = 2.0 ** -4 * np.abs(x32) + 2.0 ** -10 + 1.1 * (err / s + 2.0 ** -23 * np.abs(x32))
            ref.assert_within(moves.wide(held), x32, limit, name)
        else:
            ref.assert_within(moves.wide(held), y, ref.rounded(y, kind, err), name)


@gpu
def test_append_is_rotate_then_write():
    """What goes into a cache of the same type is bit for bit what ttc_heads_rotate makes, written by ttc_pages_write."""
    g = torch.Generator().manual_seed(0)
    tokens, hq, hk, dim = 130, 8, 4, 128
    (q, k, v), ld = packed(g, tokens, (hq * dim, hk * dim, hk * dim), torch.bfloat16)
    w = [(1 + 0.2 * torch.randn(dim, generator=g)).to(DEV) for _ in range(2)]
    pos, slots = torch.arange(500, 500 + tokens, dtype=torch.int32, device=DEV), torch.randperm(160, generator=g)[:tokens].to(torch.int32).to(DEV)
    caches = torch.zeros(4, 10, 16, hk, dim, dtype=torch.bfloat16, device=DEV)
    q1, q2, k2 = (torch.empty(tokens, n * dim, dtype=torch.bfloat16, device=DEV) for n in (hq, hq, hk))
    with heads(ttc.TTC_BF16, hq, hk, dim, dim, 0, ref.angles(dim), 1, ref.EPS) as h, \
            Handle(ttc.ttc_pages_create, ttc.ttc_pages_destroy, ttc.TTC_BF16, ttc.TTC_BF16, hk, dim, 16, 10) as p:
        ttc.ttc_pages_append(p, h, tokens, ptr(slots), ptr(pos), ptr(q), ld, ptr(k), ld, ptr(v), ld, ptr(w[0]), ptr(w[1]), ptr(q1), hq * dim, ptr(caches[0]), ptr(caches[1]), 0, 0, stream())
        ttc.ttc_heads_rotate(h, tokens, ptr(pos), ptr(q), ld, ptr(k), ld, ptr(w[0]), ptr(w[1]), ptr(q2), hq * dim, ptr(k2), hk * dim, stream())
        ttc.ttc_pages_write(p, tokens, ptr(slots), ptr(k2), hk * dim, ptr(v), ld, ptr(caches[2]), ptr(caches[3]), 0, 0, stream())
    assert torch.equal(q1, q2) and torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])


@gpu
def test_on_another_stream_and_in_a_graph():
    """Captured on a stream of its own and replayed three times with eager work between; every replay equals the eager result."""
    g = torch.Generator().manual_seed(0)
    tokens, hq, hk, dim = 600, 4, 2, 64
    (q, k, _), ld = packed(g, tokens, (hq * dim, hk * dim, 0), torch.bfloat16)
    dy = torch.randn(2, tokens, hq * dim, generator=g).to(torch.bfloat16).to(DEV)
    w = torch.ones(dim, device=DEV)
    pos = torch.arange(tokens, dtype=torch.int32, device=DEV)
    with heads(ttc.TTC_BF16, hq, hk, dim, dim, 0, ref.angles(dim), 1, ref.EPS) as h:
        work = torch.empty(ttc.ttc_heads_workspace(h, tokens), dtype=torch.uint8, device=DEV)
        q_out, dq, dw = torch.empty(tokens, hq * dim, dtype=torch.bfloat16, device=DEV), torch.empty(tokens, hq * dim, dtype=torch.bfloat16, device=DEV), torch.empty(dim, device=DEV)

        def step():
            s = torch.cuda.current_stream().cuda_stream
            ttc.ttc_heads_rotate(h, tokens, ptr(pos), ptr(q), ld, 0, 0, ptr(w), 0, ptr(q_out), hq * dim, 0, 0, s)
            ttc.ttc_heads_rotate_grad(h, tokens, ptr(pos), ptr(dy[0]), hq * dim, 0, 0, ptr(q), ld, 0, 0, ptr(w), 0, ptr(dq), hq * dim, 0, 0, ptr(dw), 0, ptr(work), s)
        step()
        torch.cuda.synchronize()
        eager = [x.clone() for x in (q_out, dq, dw)]
        side = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        for _ in range(3):
            for x in (q_out, dq, dw):
                x.zero_()
            work.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((q_out, dq, dw), eager))
            (dy[1] * 2).sum().item()


# ---- refusals: before anything reaches a device -----------------------------------------------------------

V, O, T, N, A, M = (getattr(ttc, "TTC_ERR_" + x) for x in ("INVALID_VALUE", "OVERFLOW", "UNSUPPORTED_DTYPE", "NULL_POINTER", "ALIAS", "MISALIGNED"))


def refused(status, f, *args):
    with pytest.raises(ttc.TtcError) as e:
        f(*args)
    assert e.value.status == status


def test_create_refuses():
    ok = [ttc.TTC_BF16, 8, 2, 64, 4, 0, [1.0, 0.5], 1, 1e-6]
    nan, inf = float("nan"), float("inf")
    for change, status in (({0: ttc.TTC_F64}, T), ({0: ttc.TTC_F8}, T), ({0: ttc.TTC_Q4}, T), ({1: 0}, V), ({2: -1}, V), ({3: 0}, V), ({3: 513}, V), ({3: 2}, V), ({4: 3, 6: [1.0]}, V), ({4: -2, 6: None}, V),
                           ({4: 258, 3: 300, 6: [0.1] * 129}, V), ({6: None}, N), ({6: [1.0, nan]}, V), ({6: [inf, 1.0]}, V), ({8: -1.0}, V), ({8: nan}, V), ({8: inf}, V), ({1: 1 << 21}, O)):
        args = list(ok)
        for k, v in change.items():
            args[k] = v
        refused(status, ttc.ttc_heads_create, *args)
        assert ttc.ttc_last_status() == status
    with pytest.raises(ValueError):
        ttc.ttc_heads_create(ttc.TTC_BF16, 8, 2, 64, 4, 0, [1.0], 1, 1e-6)
    for args in ((ttc.TTC_F32, 1, 1, 1), (ttc.TTC_F16, 1, 1, 64, 64, 1, [2.0] * 32, 0, nan), ok):
        ttc.ttc_heads_destroy(ttc.ttc_heads_create(*args))
    ttc.ttc_heads_destroy(None)


def test_rotate_refuses():
    Q, K, QO, KO, P, W = (i << 40 for i in range(1, 7))
    with heads(ttc.TTC_BF16, 4, 2, 64, 64, 0, ref.angles(64), 1, 1e-6) as h, heads(ttc.TTC_BF16, 4, 2, 64, 64, 0, ref.angles(64), 0, 1e-6) as plain:
        ok = [h, 10, P, Q, 512, K, 512, W, W, QO, 256, KO, 128, 0]
        for change, status in (({0: 0}, N), ({1: -1}, V), ({1: 1 << 31}, O), ({1: 1 << 29}, O), ({2: 0}, N), ({3: 0}, N), ({9: 0}, N), ({5: 0}, N), ({11: 0}, N), ({3: 0, 9: 0, 5: 0, 11: 0}, N),
                               ({4: 255}, V), ({6: 127}, V), ({10: 255}, V), ({12: 127}, V), ({0: plain}, V), ({0: plain, 7: 0}, V), ({3: Q + 1}, M), ({11: KO + 1}, M), ({2: P + 2}, M), ({7: W + 2}, M),
                               ({4: 1 << 62}, O), ({9: Q + 2, 10: 512}, A), ({9: Q, 10: 256}, A), ({9: K - 2}, A), ({11: QO + 100}, A), ({11: QO, 10: 512, 12: 512}, A),
                               ({2: QO + 40}, A), ({7: KO}, A), ({9: Q + 256 * 2 - 2, 10: 512}, A)):
            args = list(ok)
            for k, v in change.items():
                args[k] = v
            refused(status, ttc.ttc_heads_rotate, *args)
        ttc.ttc_heads_rotate(h, 0, 0, 0, 256, 0, 128, 0, 0, 0, 256, 0, 128)


def test_grad_refuses():
    DQ, DK, Q, K, X, Y, P, W, S = (i << 40 for i in range(1, 10))
    with heads(ttc.TTC_F32, 4, 2, 64, 64, 0, ref.angles(64), 1, 1e-6) as h, heads(ttc.TTC_F32, 4, 2, 64, 64, 0, ref.angles(64), 0, 1e-6) as plain:
        ok = [h, 10, P, DQ, 256, DK, 128, Q, 256, K, 128, W, W + 4096, X, 256, Y, 128, W + 8192, W + 16384, S, 0]
        for change, status in (({0: 0}, N), ({1: -1}, V), ({1: 1 << 31}, O), ({2: 0}, N), ({3: 0}, N), ({7: 0}, N), ({9: 0}, N), ({13: 0}, N), ({19: 0}, N), ({4: 255}, V), ({8: 255}, V), ({14: 3}, V), ({16: 127}, V),
                               ({0: plain}, V), ({0: plain, 11: 0, 12: 0}, V), ({3: DQ + 2}, M), ({17: W + 8194}, M), ({13: DQ + 4}, A), ({13: Q}, A), ({15: X + 64}, A), ({17: W}, A), ({17: W + 16384}, A),
                               ({19: W}, A), ({18: S + 64}, A), ({5: 0, 15: 0, 9: 0}, N)):
            args = list(ok)
            for k, v in change.items():
                args[k] = v
            refused(status, ttc.ttc_heads_rotate_grad, *args)
        assert ttc.ttc_heads_workspace(h, 10) > 0 and ttc.ttc_heads_workspace(plain, 10) == 0 and ttc.ttc_heads_workspace(h, 0) == 0
        refused(N, ttc.ttc_heads_workspace, 0, 10)
        refused(V, ttc.ttc_heads_workspace, h, -1)
        refused(O, ttc.ttc_heads_workspace, h, 1 << 40)


def test_append_refuses():
    Q, K, X, C, D, P, S, W = (i << 40 for i in range(1, 9))
    pages = lambda *a: Handle(ttc.ttc_pages_create, ttc.ttc_pages_destroy, *a)  # noqa: E731
    turn = (64, 0, ref.angles(64), 1, 1e-6)
    with heads(ttc.TTC_BF16, 4, 2, 64, *turn) as h, pages(ttc.TTC_BF16, ttc.TTC_BF16, 2, 64, 16, 10) as p, pages(ttc.TTC_F16, ttc.TTC_F16, 2, 64, 16, 10) as half, \
            pages(ttc.TTC_BF16, ttc.TTC_BF16, 2, 128, 16, 10) as wide, pages(ttc.TTC_BF16, ttc.TTC_BF16, 4, 64, 16, 10) as more, pages(ttc.TTC_BF16, ttc.TTC_Q4, 2, 64, 16, 10) as q4, \
            heads(ttc.TTC_BF16, 4, 2, 64, 8, 0, ref.angles(8), 1, 1e-6) as part, pages(ttc.TTC_BF16, ttc.TTC_F8, 2, 64, 16, 10) as f8:
        ok = [p, h, 10, S, P, Q, 512, K, 512, K + 256, 512, W, W, X, 256, C, D, 0, 0, 0]
        for change, status in (({0: 0}, N), ({1: 0}, N), ({0: half}, V), ({0: wide}, V), ({0: more}, V), ({0: q4, 1: part}, V), ({2: -1}, V), ({2: 1 << 31}, O), ({3: 0}, N), ({4: 0}, N), ({5: 0}, N), ({7: 0}, N),
                               ({9: 0}, N), ({13: 0}, N), ({15: 0}, N), ({16: 0}, N), ({17: W}, V), ({0: q4, 17: W}, V), ({6: 255}, V), ({8: 127}, V), ({10: 100}, V), ({14: 255}, V), ({7: K + 1}, M), ({15: C + 1}, M),
                               ({3: S + 1}, M), ({16: C}, A), ({16: C + 64}, A), ({15: K}, A), ({13: K}, A), ({13: C + 128}, A), ({3: C}, A), ({0: f8, 18: D}, A), ({11: D}, A)):
            args = list(ok)
            for k, v in change.items():
                args[k] = v
            refused(status, ttc.ttc_pages_append, *args)
        ttc.ttc_pages_append(p, h, 0, 0, 0, 0, 0, 0, 128, 0, 128, 0, 0, 0, 0, 0, 0)
