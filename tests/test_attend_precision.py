"""What attention over pages (include/ttc_attention.h, ttc_attend_pages) keeps of its statistics and weights, where the 64-bit result is known closely enough to tell."""
import math

import numpy as np
import pytest
import torch

import attention_reference as ref
import moves_reference as moves
from test_attend import Problem

gpu = pytest.mark.gpu


def slot_of(p, r, at):
    return p.table[r, at // p.page], at % p.page


def by_position(p, which, r, positions):
    """Elements of the cache [positions, heads, vector] of request r: a copy to be changed, and how to put it back."""
    entry, slot = slot_of(p, r, np.arange(positions))
    x = p.caches[which]
    index = (torch.from_numpy(entry).long(), torch.from_numpy(slot).long())
    if p.order == "heads":
        x = x.transpose(1, 2)
    return x[index].clone(), lambda new: x.index_put_(index, new)


@gpu
@pytest.mark.parametrize("cache", ["f32", "f8"])
@pytest.mark.parametrize("lengths", [[(8000, 1)], [(3000, 20), (5, 1)], [(2500, 90)], [(40, 1), (1500, 1), (0, 3)]])
def test_parts_of_large_scores_are_joined_as_exactly_as_small_ones(cache, lengths):
    """Every score is 2^20: a logarithm of the sum of exponentials has a sixteenth for its last place there, the maximum and the sum by themselves lose nothing."""
    p = Problem("f32", cache, "slots", 4, 2, 64, 16, lengths, seed=31)
    p.q.zero_()
    p.q[:, 0:4 * 64:64] = 2.0 ** 20
    if cache == "f8":
        p.scales = [torch.ones(2), torch.ones(2)]
    for r, (c, f) in enumerate(lengths):
        for which in (0, 1):
            x, put = by_position(p, which, r, c + f)
            x = torch.zeros(x.shape)
            if which == 0:
                x[..., 0] = 1
            else:                                                 # whole numbers that rise along the positions: all sums of them are exact
                at = torch.arange(c + f)[:, None, None]
                x[:] = (8 * at // max(c + f, 1) - 3 + (at + torch.arange(64)) % 2).float()
            put(x.to(p.caches[which].dtype))
    scale = 1 / 1.4426950408889634                                # exponents of 2 are the scores themselves
    got, lse = p.run(scale)
    v = p.values(1)[0]
    for r, (c, f) in enumerate(lengths):
        for i in range(f):
            t, n = int(p.starts[r]) + i, c + i + 1
            entry, slot = slot_of(p, r, np.arange(n))
            for h in range(4):
                values = v[entry, slot, h // 2]
                # all weights are 1: a part's mean has two roundings, and the join 128 parts' products and sums at most, the largest value 5
                assert np.abs(got[t, h] - values.mean(0)).max() <= (128 + 8) * 2.0 ** -24 * 5, (t, h)
                want = 2.0 ** 20 * math.log(2) + math.log(n)
                assert abs(lse[t, h] - want) <= 3 * 2.0 ** -24 * want


def behind_a_large_one(kind, cache, fresh, spread=0.7):
    """64 requests of the same pages, so that a workgroup has all positions of one: position 5 has a weight of 1, 32,768 others some 2^-25 of it each, and together a part of
    the result.  Returns the problem, its scale, and the exponents of 2 and the values of the positions, the same for all heads."""
    dim, heads, requests, positions = 64, 8, 64, 32768
    p = Problem(kind, cache, "slots", heads, heads, dim, 64, [(positions, fresh)], seed=32)
    g = torch.Generator().manual_seed(33)
    total = positions + fresh
    k, put_k = by_position(p, 0, 0, total)
    v, put_v = by_position(p, 1, 0, total)
    scores = -25.05 - spread * torch.rand(total, generator=g)
    scores[5] = 0
    values = (13 if cache == "q4" else 1) + torch.randint(0, 3, (total, dim), generator=g)
    values[5] = 0
    if cache == "q4":
        # keys: a step of 0 and the score as the minimum, all of whose elements meet a query of one 1; values: steps of 1 and minima of 0
        k[..., :4] = torch.stack([torch.zeros(total), scores], -1).to(torch.bfloat16).view(torch.uint8)[:, None]
        v[..., :4] = torch.tensor([1.0, 0.0], dtype=torch.bfloat16).view(torch.uint8)
        code = values.to(torch.uint8)[:, None]
        v[..., 4:] = code[..., 0::2] | code[..., 1::2] << 4
        put_k(k)
        put_v(v)
    else:
        k, v = torch.zeros(k.shape), torch.zeros(v.shape)
        k[:, :, 0:2] = (scores / 2)[:, None, None] if cache != "f8" else torch.tensor([-13.0, 0.0])        # 8 bits hold whole numbers there
        k[5] = 0
        v[:] = values[:, None].float()
        put_k(k.to(p.caches[0].dtype))
        put_v(v.to(p.caches[1].dtype))
        if cache == "f8":
            p.scales = [torch.ones(heads), torch.ones(heads)]
    at = 1 if cache == "q4" else 2                                # elements of a query that are 1; those of 8 bits see scores of -26
    p.tokens, p.cached, p.starts = requests * fresh, np.full(requests, positions, np.int32), np.arange(requests + 1, dtype=np.int32) * fresh
    p.table = np.repeat(p.table, requests, 0)
    p.q = torch.zeros(p.tokens, p.ldq, dtype=p.dtype)
    for i in range(at):
        p.q[:, i:heads * dim:dim] = 1
    entry, slot = slot_of(p, 0, np.arange(total))
    kk, vv = (p.values(i)[0][entry, slot, 0] for i in range(2))
    s = kk[:, :at].sum(1) * (2 if cache == "f8" else 1)
    assert s[5] == 0 and np.delete(s, 5).max() <= -25
    return p, math.log(2) * (2 if cache == "f8" else 1), s, vv


# Of the logarithm of n exponentials' sum, and so of the sum: 32 of them are added up in a lane, then the tiles of 64 positions, then lanes, wavefronts and 128 parts; each is
# off by 2^-20 at most, and so is the logarithm of a number near 1.
def off_of_sum(n):
    return (32 + n / 64 + 140) * 2.0 ** -24 + 2 * 2.0 ** -20


@gpu
@pytest.mark.parametrize("kind,cache", [("f32", "f32"), ("f32", "f8"), ("f32", "q4"), ("bf16", "bf16"), ("bf16", "q4")])
@pytest.mark.parametrize("fresh", [1, 40])
def test_sums_of_many_small_weights_behind_a_large_one(kind, cache, fresh):
    p, scale, s, v = behind_a_large_one(kind, cache, fresh)
    got, lse = p.run(scale)
    for i in range(fresh):
        n = p.cached[0] + i + 1
        w = 2.0 ** s[:n]
        want = (w @ v[:n]) / w.sum()
        for t in range(i, p.tokens, fresh):
            assert np.abs(lse[t] - math.log(w.sum())).max() <= off_of_sum(n), (t, np.abs(lse[t] - math.log(w.sum())).max())
            if kind == "f32":                                     # two products are added to a result at a time; position 5's value is 0
                assert (np.abs(got[t] - want) - ((n / 2 + 60) * 2.0 ** -24 + off_of_sum(n)) * want).max() <= 0, t


@gpu
@pytest.mark.parametrize("kind,cache", [("f16", "f16"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("requests,fresh,where", [(1, 90, 100), (2000, 1, 130)])
def test_scores_whose_neighbours_are_sixteen_apart(kind, cache, requests, fresh, where):
    """Exponents of 2 from 2^27 on: a score that is the next one in 32 bits has 2^16 times the weight of those before it, and comes in a later tile of the same wavefront."""
    cached = 200
    p = Problem(kind, cache, "slots", 1, 1, 64, 16, [(cached, fresh)], seed=34)
    total = cached + fresh
    k, put_k = by_position(p, 0, 0, total)
    v, put_v = by_position(p, 1, 0, total)
    k, v = torch.zeros(k.shape), torch.zeros(v.shape)
    k[..., 0], k[..., 1], v[..., 0] = 2048, 1, 1
    k[where, 0, 1], v[where, 0, 0], v[where, 0, 1] = 2, 0, 1
    put_k(k.to(p.dtype))
    put_v(v.to(p.dtype))
    p.tokens, p.cached, p.starts = requests * fresh, np.full(requests, cached, np.int32), np.arange(requests + 1, dtype=np.int32) * fresh
    p.table = np.repeat(p.table, requests, 0)
    p.q = torch.zeros(p.tokens, p.ldq, dtype=p.dtype)
    p.q[:, 0], p.q[:, 1] = 4096, 1                                # scores of 2^23 + 1, and of 2^23 + 2
    got, _ = p.run(16 * math.log(2))
    for i in range(fresh):
        others = (cached + i) * 2.0 ** -16
        want = np.zeros(64)
        want[:2] = others / (1 + others), 1 / (1 + others)
        # all weights are powers of 2, and their sums whole numbers of 2^-16
        assert np.abs(got[i::fresh, 0] - want).max() <= ref.rounded(1.0, kind, 4 * 2.0 ** -24), (i, got[i, 0, :2], want[:2])


@gpu
@pytest.mark.parametrize("cache", ["f16", "f8", "q4"])
@pytest.mark.parametrize("fresh", [1, 40])
def test_fp16_keeps_many_small_weights_behind_a_large_one(cache, fresh):
    """Weights of less than half of fp16's smallest step beside one of 1."""
    p, scale, s, v = behind_a_large_one("f16", cache, fresh)
    got, lse = p.run(scale)
    for i in range(fresh):
        n = p.cached[0] + i + 1
        w = 2.0 ** s[:n]
        want = (w @ v[:n]) / w.sum()
        # A weight in fp16 is off by 2^-11 of itself, or by half of fp16's smallest step where that is more: 2^-25 of a scale on which the largest is 2^7 at least.  It goes with the
        # value, over 4 bits with code - 8, 8 at most.  Position 5's is a power of 2.  Products are added up 16 at a time and may be cut to 32 bits, over 4 bits those of
        # 16 + code less 24 and more 8: 24 for position 5 alone and 31 of the others.
        small = np.maximum(2.0 ** -11 * w, 2.0 ** -32)[np.arange(n) != 5].sum()
        added = 24 + 31 * (w.sum() - 1) if cache == "q4" else 3 * (w.sum() - 1)
        off = small * (8 if cache == "q4" else 3) + off_of_sum(n) * want + (n / 16 + 60) * 2.0 ** -23 * added
        limit = ref.rounded(want, "f16", off)
        for t in range(i, p.tokens, fresh):
            assert (np.abs(got[t] - want) - limit).max() <= 0, (t, np.abs(got[t] - want).max(), want.max(), limit.max())
            assert np.abs(lse[t] - math.log(w.sum())).max() <= off_of_sum(n)
