"""Attention over pages (include/ttc_attention.h, ttc_attend_pages) where requests differ: one with many tokens among many with one, in the tiles of few rows that their
average gives; and fp16 over 4 bits in every form of the kernel, with the limit that fp16 gives."""
import numpy as np
import pytest

import attention_reference as ref
import moves_reference as moves
from test_attend import Problem

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("window", [0, 100])
@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("bf16", "f8"), ("f16", "q4"), ("f32", "f8")])
@pytest.mark.parametrize("group,fresh", [(1, 900), (2, 600)])
def test_one_prompt_among_single_tokens(kind, cache, window, group, fresh):
    """963 rows of 64 requests go in tiles of 16, 1326 in tiles of 32: one request has up to 57 of them, and shares of the positions begin and end in any."""
    rng = np.random.default_rng(group)
    lengths = [(int(c), 1) for c in rng.integers(0, 400, 63)]
    lengths.insert(20, (300, fresh))
    rows = sum(f for _, f in lengths) * group
    assert (group - 1) * 16 * len(lengths) < rows <= group * 16 * len(lengths)
    Problem(kind, cache, "heads", group, 1, 64, 16, lengths, seed=40 + group).check(0.125, window)


@gpu
@pytest.mark.parametrize("dim", [8, 80, 128, 192])
@pytest.mark.parametrize("lengths", [[(70, 1), (300, 1)], [(200, 11)], [(30, 70), (0, 64)]])
def test_fp16_over_four_bits(dim, lengths):
    """Heads that share keys in pairs, keys in LDS and out of it, tiles of 16, 32 and 128 rows: exponentials times steps are rounded to 2^-11 and no further."""
    p = Problem("f16", "q4", "slots", 4, 2, dim, 16, lengths, seed=dim)
    out, limit, lse, lse_limit = p.expect(0.125)
    step, low, _ = ref.from_records(p.caches[1].contiguous().numpy())
    k, _ = p.values(0)
    q = moves.wide(p.q)[:, :4 * dim].reshape(p.tokens, 4, dim)
    for r, (c, f) in enumerate(lengths):
        for i in range(f):
            at = np.arange(c + i + 1)
            entry, slot, t = p.table[r, at // 16], at % 16, int(p.starts[r]) + i
            for h in range(4):
                st, mag = np.abs(step[entry, slot, h // 2, 0]), (16 * np.abs(step) + np.abs(low))[entry, slot, h // 2, 0]
                w = np.exp(0.125 * (k[entry, slot, h // 2] @ q[t, h]))
                w /= w.sum()
                # the limit holds roundings of weights to 2^-8; in their place 2^-11, or half of fp16's smallest step on a scale on which the largest is 2^7 at least, with 24 at most
                limit[t, h] += (2.0 ** -11 - 2.0 ** -8) * (w @ mag) * (1 + 2.0 ** -11) + len(at) * 24 * 2.0 ** -32 * (w * st).max() * (1 + 2.0 ** -11)
    got, got_lse = p.run(0.125)
    ref.assert_within(got, out, limit)
    ref.assert_within(got_lse, lse, lse_limit, "lse")
