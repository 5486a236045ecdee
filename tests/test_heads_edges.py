"""Heads (include/ttc_attention.h, ttc_heads_*, ttc_pages_append) at sizes that go element by element and fill a wavefront's lanes all the same: the comparisons of
test_heads.py, with its limits."""
import pytest

import attention_reference as ref
import test_heads

gpu = pytest.mark.gpu

# dtype, tokens, q_heads, kv_heads, dim, rotated, paired, norm, pad, offset: pairs of a head that are a power of two, heads that fill every group of lanes
ELEMENTS = [
    ("f32", 40, 2, 4, 64, 12, 0, 1, 0, 0), ("f32", 5, 4, 2, 64, 6, 1, 1, 1, 0), ("bf16", 300, 8, 4, 32, 4, 0, 1, 0, 0), ("f16", 21, 64, 64, 2, 2, 0, 1, 0, 0),
    ("bf16", 9, 2, 2, 64, 24, 0, 1, 3, 1), ("bf16", 7, 1, 1, 128, 20, 0, 1, 0, 0), ("f16", 33, 1, 3, 512, 6, 0, 1, 0, 0), ("f32", 3, 8, 8, 16, 6, 0, 1, 0, 0), ("bf16", 900, 16, 16, 8, 8, 0, 1, 0, 0)]


@gpu
@pytest.mark.parametrize("case", ELEMENTS, ids=lambda c: "-".join(map(str, c)))
def test_full_lanes_element_by_element(case):
    test_heads.test_rotate(*case)
    test_heads.test_grad(*case)


@gpu
@pytest.mark.parametrize("case", [("bf16", "f8", "slots", 50, 2, 2, 64, 24, 0, 1, 8), ("f32", "f32", "heads", 30, 4, 2, 64, 12, 0, 1, 4), ("f16", "f16", "slots", 70, 8, 8, 16, 6, 1, 1, 16)],
                         ids=lambda c: "-".join(map(str, c)))
def test_full_lanes_into_the_cache(case):
    test_heads.test_append(*case)


@gpu
@pytest.mark.parametrize("hq,hk", [(1, 7), (3, 1), (4, 2), (5, 6)])
@pytest.mark.parametrize("kind,dim,rotated,paired", [("bf16", 64, 64, 0), ("bf16", 128, 128, 0), ("f16", 80, 40, 0), ("f32", 128, 64, 1), ("f32", 64, 12, 0)])
def test_without_an_epsilon(monkeypatch, kind, dim, rotated, paired, hq, hk):
    """eps = 0: lanes of a group without a head hold zeros, whose norm is none."""
    monkeypatch.setattr(ref, "EPS", 0.0)
    test_heads.test_rotate(kind, 37, hq, hk, dim, rotated, paired, 1, 0, 0)
    test_heads.test_grad(kind, 37, hq, hk, dim, rotated, paired, 1, 0, 0)
