"""Plain implementations in 64 bits of the moves whose index map is data, on the CPU with numpy, and what their tests share.
They share no code with the library: loops over assignments, requests and tokens, in the order of the definitions."""
import numpy as np
import torch

import paper_1603_02297_amd as ttc

TYPES = {"f32": (ttc.TTC_F32, torch.float32), "bf16": (ttc.TTC_BF16, torch.bfloat16), "f16": (ttc.TTC_F16, torch.float16), "f8": (ttc.TTC_F8, torch.float8_e4m3fn)}
# half a unit in the last place, relative, and the largest absolute rounding error below the normal range
ROUND = {"f32": (2.0 ** -24, 2.0 ** -150), "bf16": (2.0 ** -8, 2.0 ** -134), "f16": (2.0 ** -11, 2.0 ** -25), "f8": (2.0 ** -4, 2.0 ** -10)}
F32 = 2.0 ** -24


def wide(x):
    return x.detach().cpu().to(torch.float64).numpy()


def sort(ids, first, experts, align, rows):
    """ids [tokens, topk] -> offsets, counts, position [tokens, topk], source [rows]."""
    flat = np.asarray(ids).reshape(-1)
    lists = [[] for _ in range(experts)]
    for a, e in enumerate(flat.tolist()):
        if first <= e < first + experts:
            lists[e - first].append(a)
    offsets, counts = [0], []
    position, source = np.full(flat.size, -1, np.int32), np.full(rows, -1, np.int32)
    for mine in lists:
        at = offsets[-1]
        position[mine] = np.arange(at, at + len(mine))
        source[at:at + len(mine)] = mine
        counts.append(len(mine))
        offsets.append(at + -(-len(mine) // align) * align)
    return np.array(offsets, np.int32), np.array(counts, np.int32), position.reshape(np.shape(ids)), source


def combine(rows, weights, position, alpha, beta, y):
    """(result, sum of the magnitudes that go into it): the second bounds what 32-bit sums may be off."""
    out, mag = np.zeros_like(y), np.zeros_like(y)
    for t in range(position.shape[0]):
        for k in range(position.shape[1]):
            p = position[t, k]
            if 0 <= p < rows.shape[0]:
                term = (weights[t, k] if weights is not None else 1.0) * rows[p]
                out[t] += term
                mag[t] += np.abs(term)
    if beta:
        return alpha * out + beta * y, abs(alpha) * mag + np.abs(beta * y)
    return alpha * out, abs(alpha) * mag


def combine_grad(dy, rows, weights, position, alpha):
    """drows (0 where nothing goes), dweights, and the magnitudes behind dweights."""
    drows, dweights, mag = np.zeros_like(rows), np.zeros(position.shape), np.zeros(position.shape)
    for t in range(position.shape[0]):
        for k in range(position.shape[1]):
            p = position[t, k]
            if 0 <= p < rows.shape[0]:
                drows[p] = alpha * (weights[t, k] if weights is not None else 1.0) * dy[t]
                dweights[t, k] = alpha * np.dot(dy[t], rows[p])
                mag[t, k] = abs(alpha) * np.dot(np.abs(dy[t]), np.abs(rows[p]))
    return drows, dweights, mag


def assert_close(got, want, kind, magnitude=None, roundings=0, what=""):
    """|got - want| within one rounding to `kind` of a value that 32-bit arithmetic made with `roundings` roundings of
    terms whose magnitudes add up to `magnitude`; infinities and NaN in the same places."""
    got, want = np.asarray(got), np.asarray(want)
    assert got.shape == want.shape, what
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), what
    ok = np.isfinite(want)
    rel, tiny = ROUND[kind]
    err32 = 0.0 if magnitude is None else roundings * F32 * magnitude[ok] * 1.01
    limit = err32 + rel * (np.abs(want[ok]) + err32) + tiny
    off = np.abs(got[ok] - want[ok])
    assert (off <= limit).all(), f"{what}: {off.max()} off, {(off - limit).max()} over the limit"


def pages_map(first, cached, fresh, table, free, page, pages, tokens):
    """New table, starts, page_starts, slots, positions, owner, request by request and position by position."""
    table = table.copy()
    starts, page_starts = [0], [0]
    slots, positions, owner = (np.full(tokens, -1, np.int32) for _ in range(3))
    for r in range(len(cached)):
        c, f = max(int(cached[r]), 0), max(int(fresh[r]), 0)
        begin = c if first is None else min(max(int(first[r]), 0), c)
        have, need = -(-c // page), -(-(c + f) // page)
        for at in range(begin, c + f):
            i, b = starts[-1] + at - begin, at // page
            if i >= tokens:
                break
            if b < have:
                entry = int(table[r, b]) if b < table.shape[1] else -1
            else:
                pick = page_starts[-1] + b - have
                entry = int(free[pick]) if pick < len(free) else -1
            if not 0 <= entry < pages:
                entry = -1
            if b >= have and at % page == 0 and b < table.shape[1]:
                table[r, b] = entry
            slots[i] = entry * page + at % page if entry >= 0 and b < table.shape[1] else -1
            positions[i], owner[i] = at, r
        starts.append(starts[-1] + c + f - begin)
        page_starts.append(page_starts[-1] + need - have)
    return table, np.array(starts, np.int32), np.array(page_starts, np.int32), slots, positions, owner


def f8_values():
    """The 256 values of the 8-bit format, by its definition: sign, four exponent bits (bias 7), three mantissa bits."""
    v = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = np.nan if e == 15 and m == 7 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[b] = -x if b & 128 else x
    return v


def to_f8(x):
    """Cut at +-448 and rounded to the nearest of the format's values, to the even one in the middle; NaN stays."""
    x = np.asarray(x, np.float64)
    cut = np.clip(x, -448.0, 448.0)
    exponent = np.floor(np.log2(np.maximum(np.abs(cut), 2.0 ** -6)))
    step = 2.0 ** (exponent - 3)
    return np.where(np.isnan(x), np.nan, np.round(cut / step) * step)
