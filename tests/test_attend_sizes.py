"""The largest calls of attention over pages (include/ttc_attention.h, ttc_attend_pages): what is refused, and what is not."""
import numpy as np
import pytest
import torch

import moves_reference as moves
import paper_1603_02297_amd as ttc
from test_attend import Handle, ptr, refused, stream

gpu = pytest.mark.gpu
DEV = "cuda"


def handles(heads, dim, page, pages, q_heads, strides=None):
    c = Handle(ttc.ttc_pages_create, ttc.ttc_pages_destroy, ttc.TTC_BF16, ttc.TTC_BF16, heads, dim, page, pages, strides)
    return c, Handle(ttc.ttc_attend_create, ttc.ttc_attend_destroy, c.h, q_heads, 0.3, 0)


@pytest.mark.parametrize("heads,q_heads,requests,tokens,status", [
    (128, 128, 64, 131072, None), (128, 128, 1, 4_000_000, None), (1, 128, 64, 4_194_303, None), (65535, 65535, 24000, 8000, None), (8, 32, 1 << 24, (1 << 24) - 1, None),
    (128, 128, 64, 1 << 23, "O"), (1, 128, 64, 4_194_304, "O"), (65535, 65535, 32768, 8192, "O"), (1, 1, 1 << 29, 1, "O"), (128, 128, 1 << 24, 1, "O")])
def test_sizes(heads, q_heads, requests, tokens, status):
    """2^29 rows of queries and heads, and 2^31 of these and of requests and heads together."""
    cache, attend = handles(heads, 8, 16, 100, q_heads)
    with cache, attend as h:
        if status is None:
            assert ttc.ttc_attend_workspace(h, requests, tokens, 1000) >= 0
        else:
            refused(ttc.TTC_ERR_OVERFLOW, ttc.ttc_attend_workspace, h, requests, tokens, 1000)


@gpu
def test_many_tokens_of_many_heads():
    """131,072 tokens of 128 heads with keys of their own: the same bits as of each half of the heads, and a few results by themselves."""
    requests, fresh, heads, dim, page = 64, 2048, 128, 8, 64
    tokens, pages = requests * fresh, requests * fresh // page
    g = torch.Generator(device=DEV).manual_seed(5)
    q, k, v = (torch.randn(tokens, heads * dim, generator=g, device=DEV).to(torch.bfloat16) for _ in range(3))
    starts = torch.arange(requests + 1, dtype=torch.int32, device=DEV) * fresh
    cached = torch.zeros(requests, dtype=torch.int32, device=DEV)
    table = torch.arange(pages, dtype=torch.int32, device=DEV).view(requests, -1)
    outs = [torch.full_like(q, 9.0) for _ in range(2)]
    for part, out in ((heads, outs[0]), (heads // 2, outs[1])):
        cache, attend = handles(part, dim, page, pages, part, (dim, heads * dim, page * heads * dim))
        with cache, attend as h:
            assert ttc.ttc_attend_workspace(h, requests, tokens, table.shape[1]) == 0
            for at in range(0, heads, part):
                a, b, c, d = (x[:, at * dim:] for x in (q, k, v, out))
                ttc.ttc_attend_pages(h, requests, tokens, ptr(a), heads * dim, ptr(starts), ptr(cached), ptr(table), table.shape[1], ptr(b), ptr(c), 0, 0, ptr(d), heads * dim, 0, 0, stream())
            torch.cuda.synchronize()
    assert torch.equal(*outs)
    rng = np.random.default_rng(6)
    for _ in range(50):
        r, i, h = int(rng.integers(requests)), int(rng.integers(fresh)), int(rng.integers(heads))
        rows, at = slice(r * fresh, r * fresh + i + 1), slice(h * dim, (h + 1) * dim)
        kk, vv, qq = moves.wide(k[rows, at]), moves.wide(v[rows, at]), moves.wide(q[r * fresh + i, at])
        s = 0.3 * (kk @ qq)
        w = np.exp(s - s.max())
        w /= w.sum()
        # a weight's rounding to bf16 and the result's, and 32-bit sums far below both
        limit = (2 * 2.0 ** -8 + 2.0 ** -14) * (w @ np.abs(vv))
        assert (np.abs(moves.wide(outs[0][r * fresh + i, at]) - w @ vv) <= limit).all()
