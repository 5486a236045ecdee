"""The example's heads and its attention over pages (paper_1603_02297_amd/decoder.py) against plain computations in 64 bits, and its checks of arguments."""
import subprocess
import sys

import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_1603_02297_amd as ttc
from paper_1603_02297_amd import decoder
from test_decoder import plain_experts

gpu = pytest.mark.gpu


def plain_heads(x, weight, positions, dim, rotated, eps):
    """[tokens, heads*dim] in 64 bits, differentiable: norm, weights, rotation of the first `rotated` elements of each head, halves apart."""
    x = x.view(x.shape[0], -1, dim)
    x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight
    angle = torch.tensor([10000.0 ** (-2 * i / rotated) for i in range(rotated // 2)], dtype=torch.float64)
    t = positions.double()[:, None, None] * angle
    a, b = x[..., :rotated // 2], x[..., rotated // 2:rotated]
    return torch.cat([a * t.cos() - b * t.sin(), b * t.cos() + a * t.sin(), x[..., rotated:]], -1).flatten(1)


@gpu
@pytest.mark.parametrize("cache", ["f32", "f8", "q4"])
def test_serving_with_rotation(cache):
    """Prompts, then single tokens of some of the requests; heads normed, a part of each rotated; against a layer that keeps every key and value as a row.  In 8 and 4 bits
    that layer keeps what such a cache stands for."""
    torch.manual_seed(14)
    width, heads, kv, dim, rotated, experts, topk = 64, 4, 2, 16, 16, 6, 2
    w = decoder.weights(width, heads, kv, dim, experts, 32, torch.float32)
    w["q_norm"], w["k_norm"] = (1 + 0.2 * torch.randn(dim, device="cuda") for _ in range(2))
    w64 = {k: v.double().cpu() for k, v in w.items()}
    held = decoder.PagedCache(3, kv, dim, 8, 30, 64, torch.float32, {"f32": torch.float32, "f8": torch.float8_e4m3fn, "q4": decoder.FOUR_BITS}[cache])
    rotation = decoder.Heads(heads, kv, dim, rotated, torch.float32)

    def keep(x):                                                  # [tokens, kv*dim]
        if cache == "f8":
            return (x.float() / 0.0625).clamp(-448, 448).to(torch.float8_e4m3fn).double() * 0.0625
        if cache == "q4":
            step, low, code = ref.to_records(x.view(-1, kv, dim).numpy())
            return torch.from_numpy(low + step * code).reshape(x.shape)
        return x

    past = [torch.zeros(0, 2 * kv * dim, dtype=torch.float64) for _ in range(3)]
    for lengths in ([17, 0, 8], [1, 5, 1], [1, 1, 0], [1, 1, 1]):
        x = torch.randn(sum(lengths), width)
        got = decoder.layer(x.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), held, w, heads, topk, rotation)
        x64 = x.double()
        positions = torch.cat([torch.arange(len(p), len(p) + n) for p, n in zip(past, lengths)])
        q, k, v = (x64 @ w64["qkv"]).split([heads * dim, kv * dim, kv * dim], 1)
        q, k = plain_heads(q, w64["q_norm"], positions, dim, rotated, 1e-6), plain_heads(k, w64["k_norm"], positions, dim, rotated, 1e-6)
        rows, at = [], 0
        for r, n in enumerate(lengths):
            past[r] = torch.cat([past[r], torch.cat([keep(k[at:at + n]), keep(v[at:at + n])], 1)])
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
        # in 32 bits: chains of a few products over at most 64 terms, each off by their length in units of 2^-24; in 8 and 4 bits an element on the edge between
        # two values may fall on the other side than here: one step of 2^-3 of it, or of a fifteenth of its vector's range
        limit = {"f32": 1e-4, "f8": 2e-2, "q4": 5e-2}[cache]
        assert (got.cpu().double() - want).abs().max() <= limit * want.abs().max()
    assert held.cached.tolist() == [20, 7, 10]


@gpu
def test_training_the_whole_layer():
    """Values and all gradients in 32 bits against autograd in 64 bits."""
    torch.manual_seed(15)
    width, heads, kv, dim, rotated, experts, topk, lengths = 40, 4, 2, 20, 12, 5, 2, [13, 1, 22]
    names = ("qkv", "out", "router", "up", "down", "q_norm", "k_norm")
    shapes = ((width, (heads + 2 * kv) * dim), (heads * dim, width), (width, experts), (experts, width, 24), (experts, 24, width))
    values = [torch.randn(s, dtype=torch.float64) / s[-2] ** 0.5 for s in shapes] + [1 + 0.2 * torch.randn(dim, dtype=torch.float64) for _ in range(2)]
    x, dy = torch.randn(sum(lengths), width, dtype=torch.float64), torch.randn(sum(lengths), width, dtype=torch.float64).float().double()
    exact = [v.float().double().requires_grad_() for v in (x, *values)]
    mine = [v.detach().float().cuda().requires_grad_() for v in exact]
    got = decoder.train_layer(mine[0], lengths, dict(zip(names, mine[1:])), heads, kv, topk, decoder.Heads(heads, kv, dim, rotated, torch.float32))
    got.backward(dy.float().cuda())
    p = dict(zip(names, exact[1:]))
    positions = torch.cat([torch.arange(n) for n in lengths])
    q, k, v = (exact[0] @ p["qkv"]).split([heads * dim, kv * dim, kv * dim], 1)
    q, k = plain_heads(q, p["q_norm"], positions, dim, rotated, 1e-6), plain_heads(k, p["k_norm"], positions, dim, rotated, 1e-6)
    mixed = []
    for a, b, c in zip(q.split(lengths), k.split(lengths), v.split(lengths)):
        n = a.shape[0]
        qh, kh, vh = (t.view(n, -1, dim).transpose(0, 1) for t in (a, b, c))
        kh, vh = kh.repeat_interleave(heads // kv, 0), vh.repeat_interleave(heads // kv, 0)
        s = (qh @ kh.transpose(1, 2) / dim ** 0.5).masked_fill(torch.ones(n, n).triu(1).bool(), -torch.inf).softmax(-1)
        mixed.append((s @ vh).transpose(0, 1).reshape(n, -1))
    y = exact[0] + torch.cat(mixed) @ p["out"]
    want = y + plain_experts(y, p["router"], p["up"], p["down"], topk)
    want.backward(dy)
    # chains of some ten products over at most 80 terms, each off by their length in units of 2^-24: 1e-4 of the largest value is far above, an error is far beyond
    for name, a, b in (("y", got, want), *((n, m.grad, e.grad) for n, m, e in zip(("x", *names), mine, exact))):
        off = (a.detach().cpu().double() - b.detach()).abs().max()
        assert off <= 1e-4 * b.detach().abs().max(), (name, float(off))


@gpu
def test_gradients_of_the_rotations_gradients_are_refused():
    heads = decoder.Heads(1, 1, 8, 8, torch.float32)
    q, k, w = (torch.randn(*s, device="cuda", requires_grad=True) for s in ((3, 8), (3, 8), (8,)))
    out, _ = decoder.Rotate.apply(q, k, w, w, torch.arange(3, dtype=torch.int32, device="cuda"), heads)
    g, = torch.autograd.grad(out.square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


@gpu
def test_the_command_runs_all_of_it():
    done = subprocess.run([sys.executable, "-m", "paper_1603_02297_amd.decoder", "--steps", "2"], capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stderr[-2000:]
    lines = done.stdout.splitlines()
    assert sum(x.startswith("4 bits") and "[72, 3, 35, 130] tokens held" in x for x in lines) == 1
    assert sum(x.startswith("whole layer, training step") for x in lines) == 2
    assert "nan" not in done.stdout and "inf" not in done.stdout


def test_what_is_not_fit_is_refused_before_anything_is_mapped(monkeypatch):
    called = []
    for name in ("ttc_pages_map", "ttc_pages_write", "ttc_pages_append", "ttc_attend_pages", "ttc_heads_rotate", "ttc_heads_rotate_grad"):
        monkeypatch.setattr(ttc, name, lambda *args: called.append(args))
    c = decoder.PagedCache(3, 2, 4, 8, 9, 24, torch.float32, torch.float32, device="cpu")
    heads, plain = decoder.Heads(4, 2, 4, 4, torch.float32), decoder.Heads(4, 2, 4, 4, torch.float32, norm=False)
    one, k, q, w = torch.ones(3, dtype=torch.int32), torch.ones(3, 8), torch.ones(3, 16), torch.ones(4)
    for args in ((one, k, k, q, None), (one, k, k, None, heads), (one, k, k, q[:, :8], heads), (one, k, k, q.half(), heads), (one, k, k, q[:2], heads), (one, k, k, q, heads, (w[:3], None)),
                 (one, k, k, q, heads, (None, w.double())), (one, k, k, q, plain, (w, None)), (one, k, k, q, heads, (w.to("meta"), None))):
        with pytest.raises(ValueError):
            c.append(*args)
    for args in ((q, one, 4), (q.half(), torch.zeros(4, dtype=torch.int32), 4), (q, torch.zeros(4), 4), (q, torch.zeros(4, dtype=torch.int32), 3)):
        with pytest.raises(ValueError):
            c.attend(*args)
    for args in ((q, k[:2], None, None, one), (q, k, None, None, one.long()), (q, k, None, None, one[:2]), (q[:, :15], k, None, None, one), (q, k, w[:2], None, one)):
        with pytest.raises(ValueError):
            heads.rotate(*args)
    assert not called


def test_a_rotation_of_other_heads_than_the_cache_is_refused_before_anything_is_mapped(monkeypatch):
    called = []
    for name in ("ttc_pages_map", "ttc_pages_append"):
        monkeypatch.setattr(ttc, name, lambda *args: called.append(args))
    one = torch.ones(3, dtype=torch.int32)
    for cache_dtype, dim, others in ((torch.float32, 4, [(4, 1, 4, 4, torch.float32), (2, 2, 8, 4, torch.float32), (4, 2, 4, 4, torch.float16)]), (decoder.FOUR_BITS, 32, [(4, 2, 32, 8, torch.float32)])):
        c = decoder.PagedCache(3, 2, dim, 8, 9, 24, torch.float32, cache_dtype, device="cpu")
        k, q = torch.ones(3, 2 * dim), torch.ones(3, 4 * dim)
        for args in others:
            with pytest.raises(ValueError, match="rotation"):
                c.append(one, k, k, q, decoder.Heads(*args))
    assert not called
