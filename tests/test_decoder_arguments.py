"""What the example's classes (paper_1603_02297_amd/decoder.py) hand to the library: addresses and leading dimensions that stay inside the tensors, or an error
before the call."""
import subprocess
import sys

import pytest
import torch

import paper_1603_02297_amd as ttc
from paper_1603_02297_amd import decoder

gpu = pytest.mark.gpu


class Recorder:
    """In place of the library's moves: what they were given."""

    def __init__(self, monkeypatch):
        self.calls = []
        monkeypatch.setattr(decoder, "_stream", lambda: 0)
        for name in ("ttc_route_gather", "ttc_route_combine", "ttc_route_combine_grad"):
            monkeypatch.setattr(ttc, name, lambda *args, name=name: self.calls.append((name, args)))


def routing(tokens, topk, width, rows, dtype=torch.float32):
    """A routing whose maps are of no interest, on the CPU."""
    r = decoder.Routing.__new__(decoder.Routing)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    r.tokens, r.topk, r.width, r.row_count, r.dtype, r.device, r.handle = tokens, topk, width, rows, dtype, torch.device("cpu"), 0
    r.offsets, r.counts, r.position = i32(5), i32(4), i32(tokens, topk)
    return r


def matrices(width):
    """Matrices of 6 rows whose strides are not a dense matrix's: one row for all, one column for all, columns for rows, part of a wider one, every other element."""
    base = torch.arange(400.0)
    return [base[:width].expand(6, width), base[:6, None].expand(6, width), base[:6 * width].view(width, 6).t(), base[:6 * (width + 3)].view(6, width + 3)[:, 1:width + 1],
            base[:12 * width].view(6, 2 * width)[:, ::2], base[:6 * width].view(6, width)]


@pytest.mark.parametrize("width", [1, 2, 17])
def test_addresses_stay_inside_and_mean_the_tensor(monkeypatch, width):
    """What a call would read, by address and leading dimension, is the tensor's own elements."""
    def read(x, ld, address, rows, kept):
        owner = next((t for t in kept if t.untyped_storage().data_ptr() <= address < t.untyped_storage().data_ptr() + t.untyped_storage().nbytes()), None)
        assert owner is not None
        flat = torch.empty(0, dtype=torch.float32).set_(owner.untyped_storage())
        first = (address - owner.untyped_storage().data_ptr()) // 4
        assert first + (rows - 1) * ld + width <= flat.numel()
        assert torch.equal(torch.as_strided(flat, (rows, width), (ld, 1), first), x)

    kept = []
    whole = torch.Tensor.contiguous
    monkeypatch.setattr(torch.Tensor, "contiguous", lambda t: kept.append(whole(t)) or kept[-1])      # copies live as long as the test
    for x in matrices(width):
        kept[:] = [x]
        seen = Recorder(monkeypatch)
        r = routing(6, 2, width, 6)
        r.gather(x)
        r.combine(x, None)
        r.combine_grad(x, x, torch.ones(6, 2))
        (_, g), (_, c), (_, d) = seen.calls
        for address, ld in ((g[2], g[3]), (c[2], c[3]), (d[2], d[3]), (d[4], d[5])):
            read(x, ld, address, 6, kept)


def test_weights_and_their_gradient_are_dense(monkeypatch):
    seen, r = Recorder(monkeypatch), routing(6, 3, 4, 18)
    w = torch.arange(18.0).view(3, 6).t()
    kept, whole = [], torch.Tensor.contiguous
    monkeypatch.setattr(torch.Tensor, "contiguous", lambda t: kept.append(whole(t)) or kept[-1])
    _, dw = r.combine_grad(torch.ones(6, 4), torch.ones(18, 4), w)
    assert dw.is_contiguous() and dw.shape == w.shape
    assert any(t.data_ptr() == seen.calls[0][1][6] and torch.equal(t, w) and t.is_contiguous() for t in kept)


def test_other_types_and_shapes_are_refused(monkeypatch):
    seen, r = Recorder(monkeypatch), routing(6, 2, 8, 12)
    x, rows, w = torch.ones(6, 8), torch.ones(12, 8), torch.ones(6, 2)
    for bad in (x.bfloat16(), x.double(), x[:5], x[:, :7], x.view(48), torch.ones(6, 9), x.to("meta")):
        for call in (lambda: r.gather(bad), lambda: r.combine_grad(bad, rows, w)):
            with pytest.raises(ValueError):
                call()
    for bad in (rows.half(), rows[:11], torch.ones(13, 8), rows[:, 1:]):
        for call in (lambda: r.combine(bad, w), lambda: r.combine_grad(x, bad, w)):
            with pytest.raises(ValueError):
                call()
    for bad in (w.double(), w.bfloat16(), w[:, :1], w[:5], torch.ones(6, 3)):
        for call in (lambda: r.combine(rows, bad), lambda: r.combine_grad(x, rows, bad)):
            with pytest.raises(ValueError):
                call()
    assert not seen.calls


def test_ids_are_whole_numbers_on_the_gpu():
    for ids in (torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4, 2), torch.zeros(4, dtype=torch.int64)):
        with pytest.raises(ValueError):
            decoder.Routing(ids, 4, 8, torch.float32)


@gpu
def test_broadcast_tokens_and_gradients():
    """One token for many, and the gradient of a sum (one number for all): as for the same values written out."""
    torch.manual_seed(5)
    tokens, topk, width, experts = 37, 3, 24, 5
    ids = torch.rand(tokens, experts, device="cuda").topk(topk, dim=1).indices
    for made in (ids, ids.t().contiguous().t(), ids.to(torch.int32)):
        r = decoder.Routing(made, experts, width, torch.float32, align=4)
        weights, one = torch.randn(tokens, topk, device="cuda"), torch.randn(1, width, device="cuda")
        results = []
        for form in (lambda t: t.expand(tokens, width), lambda t: t.expand(tokens, width).contiguous()):
            x, w = one.clone().requires_grad_(), weights.clone().requires_grad_()
            rows = decoder.Gather.apply(form(x), r)
            y = decoder.Combine.apply(rows * 2, w, r)
            scale = form(torch.full((1, 1), 3.0, device="cuda"))
            gx, gw = torch.autograd.grad(y, (x, w), scale)
            results.append((rows, y, gx, gw))
        for a, b in zip(*results):
            assert torch.equal(a, b)
        assert torch.equal(results[0][0][r.position.long().reshape(-1)], one.expand(tokens * topk, width))
    with pytest.raises(ValueError):
        decoder.Routing(torch.zeros(4, 2, device="cuda"), 4, 8, torch.float32)
    with pytest.raises(ValueError):
        r.gather(torch.zeros(tokens, width, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        r.combine(torch.zeros(r.row_count - 1, width, device="cuda"), weights)


# ---- derivatives of derivatives -------------------------------------------------------------------------------

class PlainRouting:
    """The moves of Routing in torch operations on the CPU, detached as the library's calls are."""

    def __init__(self, position, rows):
        self.position, self.rows = position, rows

    def gather(self, x):
        out = torch.zeros(self.rows, x.shape[1], dtype=x.dtype)
        out[self.position.reshape(-1)] = x.detach().repeat_interleave(self.position.shape[1], 0)
        return out

    def combine(self, rows, weights):
        w = torch.ones(self.position.shape, dtype=rows.dtype) if weights is None else weights.detach()
        return (rows.detach()[self.position] * w[:, :, None]).sum(1)

    def combine_grad(self, dy, rows, weights):
        drows = torch.zeros_like(rows)
        drows[self.position.reshape(-1)] = (dy.detach()[:, None, :] * weights.detach()[:, :, None]).reshape(-1, dy.shape[1])
        return drows, (dy.detach()[:, None, :] * rows.detach()[self.position]).sum(2)


def test_derivatives_of_derivatives():
    """First, second and third derivatives through Gather and Combine agree with those through torch's operations."""
    torch.manual_seed(1)
    position = torch.randperm(12).view(6, 2)
    r, up = PlainRouting(position, 12), torch.randn(5, 5, dtype=torch.float64, requires_grad=True)
    x, w = torch.randn(6, 5, dtype=torch.float64, requires_grad=True), torch.randn(6, 2, dtype=torch.float64, requires_grad=True)

    def through(moves):
        rows = decoder.Gather.apply(x, r) if moves else torch.zeros(12, 5, dtype=torch.float64).index_put((position.reshape(-1),), x.repeat_interleave(2, 0))
        rows = torch.tanh(rows @ up)
        y, levels = decoder.Combine.apply(rows, w, r) if moves else (rows[position] * w[:, :, None]).sum(1), []
        value = (y ** 2).sum()
        for _ in range(3):
            levels.append(torch.autograd.grad(value, (x, w, up), create_graph=True))
            value = sum((g ** 2).sum() for g in levels[-1])
        return levels

    for mine, exact in zip(through(True), through(False)):
        assert all(torch.allclose(a, b, rtol=1e-9) for a, b in zip(mine, exact))


@gpu
def test_gradient_of_a_gradient_norm_through_the_experts():
    """In 32 bits through the moves, against torch's operations in 64 bits."""
    from test_decoder import plain_experts
    torch.manual_seed(3)
    tokens, width, hidden, experts, topk = 29, 52, 24, 7, 3
    exact = [torch.randn(tokens, width), torch.randn(width, experts) / width ** 0.5, torch.randn(experts, width, hidden) / width ** 0.5, torch.randn(experts, hidden, width) / hidden ** 0.5]
    mine = [p.cuda().requires_grad_() for p in exact]
    exact = [p.double().requires_grad_() for p in exact]
    results = []
    for f, p in ((plain_experts, exact), (decoder.experts_forward, mine)):
        first = torch.autograd.grad((f(*p, topk) ** 2).sum(), p, create_graph=True)
        results.append(torch.autograd.grad(sum((g ** 2).sum() for g in first), p))
    # chains of products over at most 52 terms and sums over at most 29 tokens, each off by their length in units of 2^-24, some ten of them one
    # after another: below 1e-4 of the largest value; a part that is missing is some tenths of it
    for a, b in zip(*results):
        assert float((b.cpu().double() - a).abs().max()) <= 1e-3 * float(a.abs().max())


# ---- the paged cache: what does not fit changes nothing ----------------------------------------------------------

def filled_cache(device, pages=9, longest=24, dtype=torch.float32):
    """Three requests that hold 20, 0 and 9 tokens in pages of 8."""
    c = decoder.PagedCache(3, 2, 4, 8, pages, longest, dtype, dtype, device=device)
    return c, torch.tensor([20, 0, 9], dtype=torch.int32, device=device)


BAD = [  # fresh, tokens, error
    ([5, 0, 0], 5, RuntimeError), ([0, 25, 0], 25, RuntimeError), ([4, 24, 16], 44, RuntimeError), ([4, 24, 15], 43, RuntimeError), ([2 ** 31 - 1, 2 ** 31 - 1, 2], 0, ValueError), ([1, 1, 1], 2, ValueError),
    ([1, 1, 1], 4, ValueError), ([3, -1, 0], 2, ValueError), ([0, 0, 0], 1, ValueError)]


@pytest.mark.parametrize("fresh,tokens,error", BAD)
def test_what_does_not_fit_the_table_or_the_pages_is_not_appended(monkeypatch, fresh, tokens, error):
    called = []
    for name in ("ttc_pages_map", "ttc_pages_write"):
        monkeypatch.setattr(ttc, name, lambda *args: called.append(args))
    monkeypatch.setattr(decoder, "_stream", lambda: 0)
    c, c.cached = filled_cache("cpu", pages=3 if sum(fresh) == 43 else 99)
    free, cached = c.free.clone(), c.cached.clone()
    with pytest.raises(error) as e:
        c.append(torch.tensor(fresh, dtype=torch.int32), torch.ones(tokens, 8), torch.ones(tokens, 8))
    assert not isinstance(e.value, ttc.TtcError) and not called
    assert torch.equal(c.free, free) and torch.equal(c.cached, cached)


def test_appended_tensors_are_checked(monkeypatch):
    called = []
    for name in ("ttc_pages_map", "ttc_pages_write"):
        monkeypatch.setattr(ttc, name, lambda *args: called.append(args))
    c, _ = filled_cache("cpu")
    one, k = torch.ones(3, dtype=torch.int32), torch.ones(3, 8)
    for fresh, a, b in ((one.long(), k, k), (one[:2], k, k), (one.view(3, 1), k, k), (one, k.half(), k), (one, k, k[:2]), (one, k[:, :7], k), (one, k, torch.ones(3, 9)), (one.to("meta"), k, k)):
        with pytest.raises(ValueError):
            c.append(fresh, a, b)
    assert not called


@gpu
def test_a_cache_filled_to_its_last_place_and_beyond():
    """Up to the table's end everything is kept; one token more is an error that leaves the cache as it was."""
    torch.manual_seed(6)
    c, lengths = filled_cache("cuda")
    draw = lambda n: torch.randn(n, 8, device="cuda")  # noqa: E731
    k, v = draw(29), draw(29)
    c.append(lengths, k, v)
    more = torch.tensor([4, 24, 15], dtype=torch.int32, device="cuda")
    k2, v2 = draw(43), draw(43)
    c.append(more, k2, v2)
    assert c.cached.tolist() == [24, 24, 24] and c.free.numel() == 0

    def check():
        starts, got_k, got_v = c.context()
        assert starts.tolist() == [0, 24, 48, 72]
        for got, a, b in ((got_k, k, k2), (got_v, v, v2)):
            assert torch.equal(got, torch.cat([a[:20], b[:4], b[4:28], a[20:], b[28:]]))

    check()
    for r in range(3):
        fresh = torch.zeros(3, dtype=torch.int32, device="cuda")
        fresh[r] = 1
        with pytest.raises(RuntimeError):
            c.append(fresh, draw(1), draw(1))
    assert c.cached.tolist() == [24, 24, 24] and c.free.numel() == 0
    check()


@gpu
def test_the_command_serves_as_many_steps_as_it_is_asked_for():
    """The cache is sized by the prompts and the steps: 140 steps take the longest request past 256 tokens."""
    done = subprocess.run([sys.executable, "-m", "paper_1603_02297_amd.decoder", "--steps", "140"], capture_output=True, text=True, timeout=110)
    assert done.returncode == 0, done.stderr[-2000:]
    assert done.stdout.count("lengths [210, 141, 173, 268]") == 2


@gpu
def test_a_step_without_tokens():
    """Nothing new for any request: no rows come out, nothing is taken; the next step goes on from there."""
    torch.manual_seed(7)
    w = decoder.weights(32, 2, 1, 16, 4, 16, torch.float32)
    for before in ([0, 0], [9, 3]):
        c = decoder.PagedCache(2, 1, 16, 8, 6, 24, torch.float32, torch.float32)
        step = lambda n: decoder.layer(torch.randn(sum(n), 32, device="cuda"), torch.tensor(n, dtype=torch.int32, device="cuda"), c, w, 2, 2)  # noqa: E731
        step(before)
        free = c.free.clone()
        assert step([0, 0]).shape == (0, 32)
        assert c.cached.tolist() == before and torch.equal(c.free, free)
        assert step([1, 0]).shape == (1, 32) and c.cached.tolist() == [before[0] + 1, before[1]]
    x = torch.zeros(0, 32, device="cuda", requires_grad=True)
    decoder.experts_forward(x, w["router"], w["up"], w["down"], 2).sum().backward()
    assert x.grad.shape == (0, 32)
