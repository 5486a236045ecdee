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
