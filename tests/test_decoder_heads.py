"""Which heads the example's serving layer (paper_1603_02297_amd/decoder.py) takes: refusals before anything is in the cache, and heads longer than the attention over pages has."""
import pytest
import torch

import paper_1603_02297_amd as ttc
from paper_1603_02297_amd import decoder
from test_decoder import plain_experts

gpu = pytest.mark.gpu


@pytest.mark.parametrize("dim", [16, 288])
def test_heads_that_share_no_keys_evenly_are_refused_before_anything_is_mapped(monkeypatch, dim):
    called = []
    for name in ("ttc_pages_map", "ttc_pages_write", "ttc_pages_append", "ttc_pages_read", "ttc_attend_pages"):
        monkeypatch.setattr(ttc, name, lambda *args, name=name: called.append(name))
    cache = decoder.PagedCache(3, 2, dim, 8, 9, 24, torch.float32, torch.float32, device="cpu")
    w = decoder.weights(32, 3, 2, dim, 4, 16, torch.float32, device="cpu")
    with pytest.raises(ValueError, match="heads"):
        decoder.layer(torch.randn(3, 32), torch.ones(3, dtype=torch.int32), cache, w, 3, 2)
    assert not called and cache.cached.tolist() == [0, 0, 0] and cache.free.numel() == 9


def test_what_the_library_refuses_is_refused_before_anything_is_mapped(monkeypatch):
    called = []
    for name in ("ttc_pages_map", "ttc_pages_write"):
        monkeypatch.setattr(ttc, name, lambda *args, name=name: called.append(name))

    def no(*args):
        raise ttc.TtcError(ttc.TTC_ERR_ALLOC, "ttc_attend_create")
    monkeypatch.setattr(ttc, "ttc_attend_create", no)
    cache = decoder.PagedCache(3, 2, 16, 8, 9, 24, torch.float32, torch.float32, device="cpu")
    with pytest.raises(ttc.TtcError):
        decoder.layer(torch.randn(3, 32), torch.ones(3, dtype=torch.int32), cache, decoder.weights(32, 4, 2, 16, 4, 16, torch.float32, device="cpu"), 4, 2)
    assert not called and cache.cached.tolist() == [0, 0, 0] and cache.free.numel() == 9


@gpu
@pytest.mark.parametrize("rotate", [False, True])
def test_heads_longer_than_the_attention_over_pages_has(rotate):
    """Heads of 288 elements, prompts and single tokens, against a layer that keeps every key and value as a row."""
    torch.manual_seed(16)
    width, heads, kv, dim, experts, topk = 48, 4, 2, 288, 4, 2
    assert dim > ttc.TTC_ATTEND_MAX_DIM
    w = decoder.weights(width, heads, kv, dim, experts, 32, torch.float32)
    w64 = {k: v.double().cpu() for k, v in w.items()}
    held = decoder.PagedCache(3, kv, dim, 8, 30, 64, torch.float32, torch.float32)
    rotation = decoder.Heads(heads, kv, dim, 64, torch.float32, norm=False) if rotate else None
    angle = torch.tensor([10000.0 ** (-2 * i / 64) for i in range(32)], dtype=torch.float64)

    def turn(x, positions):
        if not rotate:
            return x
        x = x.view(x.shape[0], -1, dim)
        t = positions.double()[:, None, None] * angle
        a, b = x[..., :32], x[..., 32:64]
        return torch.cat([a * t.cos() - b * t.sin(), b * t.cos() + a * t.sin(), x[..., 64:]], -1).flatten(1)

    past = [torch.zeros(0, 2 * kv * dim, dtype=torch.float64) for _ in range(3)]
    for lengths in ([17, 0, 8], [1, 5, 1], [0, 0, 0], [1, 1, 0]):
        x = torch.randn(sum(lengths), width)
        got = decoder.layer(x.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), held, w, heads, topk, rotation)
        if not sum(lengths):
            assert got.shape == (0, width)
            continue
        x64 = x.double()
        positions = torch.cat([torch.arange(len(p), len(p) + n) for p, n in zip(past, lengths)])
        q, k, v = (x64 @ w64["qkv"]).split([heads * dim, kv * dim, kv * dim], 1)
        q, k = turn(q, positions), turn(k, positions)
        rows, at = [], 0
        for r, n in enumerate(lengths):
            past[r] = torch.cat([past[r], torch.cat([k[at:at + n], v[at:at + n]], 1)])
            for i in range(n):
                seen = past[r][:len(past[r]) - n + i + 1]
                out = []
                for h in range(heads):
                    g = h // (heads // kv)
                    kk, vv = seen[:, g * dim:(g + 1) * dim], seen[:, (kv + g) * dim:(kv + g + 1) * dim]
                    out.append((kk @ q[at + i, h * dim:(h + 1) * dim] / dim ** 0.5).softmax(0) @ vv)
                rows.append(torch.cat(out))
            at += n
        x64 = x64 + torch.stack(rows) @ w64["out"]
        want = x64 + plain_experts(x64, w64["router"], w64["up"], w64["down"], topk)
        # in 32 bits: chains of a few products over at most 1152 terms, each off by the root of their length in units of 2^-24 as a rule, by 1152 at most: 7e-5
        assert (got.cpu().double() - want).abs().max() <= 3e-4 * want.abs().max()
    assert held.cached.tolist() == [19, 6, 9]
