"""The example that uses the moves by data together (paper_1603_02297_amd/decoder.py) against plain computations in 64 bits."""
import subprocess
import sys

import pytest
import torch

gpu = pytest.mark.gpu


def plain_experts(x, router, up, down, topk):
    best, ids = (x @ router).topk(topk, dim=1)
    w = best.softmax(1)
    y = torch.zeros_like(x)
    for t in range(x.shape[0]):
        for k in range(topk):
            e = int(ids[t, k])
            y[t] = y[t] + w[t, k] * (torch.nn.functional.silu(x[t] @ up[e]) @ down[e])
    return y


@gpu
def test_training_the_experts():
    """Values and all gradients of the routed experts in 32 bits, through the moves, against autograd in 64 bits."""
    from paper_1603_02297_amd import decoder
    torch.manual_seed(3)
    tokens, width, hidden, experts, topk = 45, 52, 24, 7, 3
    x, router = torch.randn(tokens, width, dtype=torch.float64), torch.randn(width, experts, dtype=torch.float64) / width ** 0.5
    up, down = torch.randn(experts, width, hidden, dtype=torch.float64) / width ** 0.5, torch.randn(experts, hidden, width, dtype=torch.float64) / hidden ** 0.5
    exact = [p.float().double().requires_grad_() for p in (x, router, up, down)]
    mine = [p.detach().float().cuda().requires_grad_() for p in exact]
    dy = torch.randn(tokens, width, dtype=torch.float64).float().double()
    want = plain_experts(*exact, topk)
    want.backward(dy)
    got = decoder.experts_forward(*mine, topk)
    got.backward(dy.float().cuda())
    # chains of a few products over at most 52 terms, each off by their length in units of 2^-24: 1e-4 of the largest value is far above, an error is far beyond
    for name, a, b in (("y", got, want), *((n, m.grad, e.grad) for n, m, e in zip(("x", "router", "up", "down"), mine, exact))):
        off = (a.detach().cpu().double() - b.detach()).abs().max()
        assert off <= 1e-4 * b.detach().abs().max(), (name, float(off))


@gpu
@pytest.mark.parametrize("cache", ["f32", "f8"])
def test_serving_a_layer(cache):
    """Prompts, then single tokens of some of the requests, over pages in no order; against a layer that keeps every key and value as a row."""
    from paper_1603_02297_amd import decoder
    torch.manual_seed(4)
    width, heads, kv_heads, dim, experts, topk = 64, 4, 2, 16, 6, 2
    w = decoder.weights(width, heads, kv_heads, dim, experts, 32, torch.float32)
    w64 = {k: v.double().cpu() for k, v in w.items()}
    held = decoder.PagedCache(3, kv_heads, dim, 8, 30, 64, torch.float32, torch.float32 if cache == "f32" else torch.float8_e4m3fn)
    past = [torch.zeros(0, 2 * kv_heads * dim, dtype=torch.float64) for _ in range(3)]
    for lengths in ([17, 0, 8], [1, 5, 1], [1, 1, 0], [1, 1, 1]):
        x = torch.randn(sum(lengths), width)
        got = decoder.layer(x.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), held, w, heads, topk)
        x64 = x.double()
        qkv = x64 @ w64["qkv"]
        rows, at = [], 0
        for r, n in enumerate(lengths):
            new = qkv[at:at + n, heads * dim:]
            if cache == "f8":                                     # what the cache holds: cut at +-448 and rounded to four bits, at this scale
                new = (new.float() / 0.0625).clamp(-448, 448).to(torch.float8_e4m3fn).double() * 0.0625
            past[r] = torch.cat([past[r], new])
            for i in range(n):
                seen = past[r][:len(past[r]) - n + i + 1]
                out = []
                for h in range(heads):
                    g = h // (heads // kv_heads)
                    k, v = seen[:, g * dim:(g + 1) * dim], seen[:, (kv_heads + g) * dim:(kv_heads + g + 1) * dim]
                    out.append((k @ qkv[at + i, h * dim:(h + 1) * dim] / dim ** 0.5).softmax(0) @ v)
                rows.append(torch.cat(out))
            at += n
        x64 = x64 + torch.stack(rows) @ w64["out"]
        want = x64 + plain_experts(x64, w64["router"], w64["up"], w64["down"], topk)
        # in 32 bits as above; in 8 bits a key on the edge between two of the format's values may fall on the other side than here: one step of 2^-3 of it
        limit = 1e-4 if cache == "f32" else 2e-2
        assert (got.cpu().double() - want).abs().max() <= limit * want.abs().max()
    assert held.cached.tolist() == [20, 7, 10]


@gpu
def test_the_command_runs():
    done = subprocess.run([sys.executable, "-m", "paper_1603_02297_amd.decoder", "--steps", "2"], capture_output=True, text=True, timeout=100)
    assert done.returncode == 0, done.stderr[-2000:]
    lines = done.stdout.splitlines()
    assert sum("tokens each" in x for x in lines) == 2
    losses = [float(x.rsplit(" ", 1)[1]) for x in lines if x.startswith("training")]
    assert len(losses) == 2 and losses[1] < losses[0]
