"""A decoder layer with routed experts over a paged cache: the moves by data (include/ttc_moves.h) and the attention around them (include/ttc_attention.h) as they
are used together.

    python -m paper_1603_02297_amd.decoder [--steps N]

serves prompts and then single tokens of several requests, and trains the experts on a batch, and the whole layer on packed sequences.  A step of serving:

    request lengths --ttc_pages_map--> block tables, packed offsets, slots, positions --ttc_pages_append (or, without rotation, ttc_pages_write)--> queries,
    and keys and values in their pages --ttc_attend_pages--> attention of the new tokens over the pages
    --> router --ttc_route_sort--> rows by expert --ttc_route_gather--> the experts' products --ttc_route_combine--> residual

Everything else (projections, the experts, attention in training) is plain torch: this is the path that these calls serve, not a model.
"""
from __future__ import annotations

import argparse
import weakref

import torch

import paper_1603_02297_amd as ttc

# the type of a cache in 4 bits: its records are bytes
FOUR_BITS = torch.uint8
CODES = {FOUR_BITS: ttc.TTC_Q4, torch.float32: ttc.TTC_F32, torch.bfloat16: ttc.TTC_BF16, torch.float16: ttc.TTC_F16, torch.float8_e4m3fn: ttc.TTC_F8}


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _ptr(x) -> int:
    return 0 if x is None else x.data_ptr()


def _matrix(x: torch.Tensor, shape, dtype: torch.dtype, device, what: str) -> torch.Tensor:
    """x as the moves take a matrix, by its address and leading dimension alone: of this type and shape, elements of a row next to each other,
    rows apart from each other.  Columns in the place of rows and a row that stands for many (an expanded tensor) are copied out."""
    if x.dtype != dtype or tuple(x.shape) != tuple(shape) or x.device != device:
        raise ValueError(f"{what}: {x.dtype} {list(x.shape)} on {x.device}, wanted {dtype} {list(shape)} on {device}")
    fits = (x.shape[1] <= 1 or x.stride(1) == 1) and (x.shape[0] <= 1 or x.stride(0) >= x.shape[1])
    return x if fits else x.contiguous()


def _rows_apart(x: torch.Tensor) -> int:
    """The leading dimension of such a matrix, which may be part of a wider one."""
    return max(x.stride(0), x.shape[1])


class Routing:
    """The rows of one batch sorted by expert: what ttc_route_sort found, and the moves along it."""

    def __init__(self, ids: torch.Tensor, experts: int, width: int, dtype: torch.dtype, first: int = 0, align: int = 1):
        if ids.dim() != 2 or ids.dtype not in (torch.int32, torch.int64) or not ids.is_cuda:
            raise ValueError(f"ids: {ids.dtype} {list(ids.shape)} on {ids.device}, wanted [tokens, topk] of int32 or int64 on the GPU")
        self.tokens, self.topk = ids.shape
        self.width, self.dtype, self.experts, self.device = width, dtype, experts, ids.device
        ids = _matrix(ids, ids.shape, ids.dtype, ids.device, "ids")
        self.handle = ttc.ttc_route_create(CODES[dtype], width, self.topk, experts, first, align, ids.element_size())
        weakref.finalize(self, ttc.ttc_route_destroy, self.handle)
        self.row_count = ttc.ttc_route_rows(self.handle, self.tokens)
        i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device=self.device)  # noqa: E731
        self.offsets, self.counts, self.position = i32(experts + 1), i32(experts), i32(self.tokens, self.topk)
        work = torch.empty(ttc.ttc_route_workspace(self.handle, self.tokens), dtype=torch.uint8, device=self.device)
        ttc.ttc_route_sort(self.handle, self.tokens, _ptr(ids), _rows_apart(ids), _ptr(self.offsets), _ptr(self.counts), _ptr(self.position), 0, _ptr(work), _stream())

    def _tokens(self, x: torch.Tensor, what: str) -> torch.Tensor:
        return _matrix(x, (self.tokens, self.width), self.dtype, self.device, what)

    def _rows(self, x: torch.Tensor, what: str) -> torch.Tensor:
        return _matrix(x, (self.row_count, self.width), self.dtype, self.device, what)

    def _weights(self, w: torch.Tensor) -> torch.Tensor:
        return _matrix(w, (self.tokens, self.topk), torch.float32, self.device, "weights").contiguous()

    def gather(self, x: torch.Tensor) -> torch.Tensor:
        """Tokens to their rows; rows past the last segment are 0."""
        x = self._tokens(x, "x")
        rows = torch.zeros(self.row_count, self.width, dtype=self.dtype, device=self.device)
        ttc.ttc_route_gather(self.handle, self.tokens, _ptr(x), _rows_apart(x), 0, _ptr(self.position), _ptr(self.offsets), _ptr(self.counts), _ptr(rows), self.width, _stream())
        return rows

    def combine(self, rows: torch.Tensor, weights) -> torch.Tensor:
        rows, weights = self._rows(rows, "rows"), None if weights is None else self._weights(weights)
        y = torch.empty(self.tokens, self.width, dtype=self.dtype, device=self.device)
        ttc.ttc_route_combine(self.handle, self.tokens, _ptr(rows), _rows_apart(rows), _ptr(weights), _ptr(self.position), _ptr(y), self.width, _stream())
        return y

    def combine_grad(self, dy: torch.Tensor, rows: torch.Tensor, weights: torch.Tensor):
        dy, rows, weights = self._tokens(dy, "dy"), self._rows(rows, "rows"), self._weights(weights)
        drows = torch.zeros(self.row_count, self.width, dtype=self.dtype, device=self.device)
        dweights = torch.empty(self.tokens, self.topk, dtype=torch.float32, device=self.device)
        ttc.ttc_route_combine_grad(self.handle, self.tokens, _ptr(dy), _rows_apart(dy), _ptr(rows), _rows_apart(rows), _ptr(weights), _ptr(self.position),
                                   _ptr(self.offsets), _ptr(self.counts), _ptr(drows), self.width, _ptr(dweights), _stream())
        return drows, dweights


class Gather(torch.autograd.Function):
    """Tokens to their rows; the gradient adds the rows up again.  The moves go by address and record no graph of their own, so that every
    backward pass here is written in these functions again and can be differentiated in its turn."""

    @staticmethod
    def forward(ctx, x, routing):
        ctx.routing = routing
        return routing.gather(x)

    @staticmethod
    def backward(ctx, drows):
        return Combine.apply(drows, None, ctx.routing), None


class Combine(torch.autograd.Function):
    """Rows back to their tokens, weighted (weights None: all 1); the gradients of rows and weights in one pass."""

    @staticmethod
    def forward(ctx, rows, weights, routing):
        ctx.routing = routing
        ctx.save_for_backward(rows, weights)
        return routing.combine(rows, weights)

    @staticmethod
    def backward(ctx, dy):
        rows, weights = ctx.saved_tensors
        if weights is None:
            return Gather.apply(dy, ctx.routing), None, None
        return (*CombineGrad.apply(dy, rows, weights, ctx.routing), None)


class CombineGrad(torch.autograd.Function):
    """drows = weights * dy and dweights = <dy, rows>, along the map: both are linear in dy, the one in weights, the other in rows."""

    @staticmethod
    def forward(ctx, dy, rows, weights, routing):
        ctx.routing = routing
        ctx.save_for_backward(dy, rows, weights)
        return routing.combine_grad(dy, rows, weights)

    @staticmethod
    def backward(ctx, to_rows, to_weights):
        dy, rows, weights = ctx.saved_tensors
        back = Combine.apply(to_rows, weights, ctx.routing) + Combine.apply(rows, to_weights, ctx.routing)
        return (back, *CombineGrad.apply(dy, to_rows, to_weights, ctx.routing), None)


def experts_forward(x: torch.Tensor, router: torch.Tensor, up: torch.Tensor, down: torch.Tensor, topk: int, align: int = 16) -> torch.Tensor:
    """x [tokens, width] through the experts that the router chooses: up [experts, width, hidden], down [experts, hidden, width]."""
    logits = x.float() @ router.float()
    best, ids = logits.topk(topk, dim=1)
    routing = Routing(ids, up.shape[0], x.shape[1], x.dtype, align=align)
    rows = Gather.apply(x, routing)
    ends = routing.offsets.tolist()                               # the segments' sizes shape the products
    out = [torch.nn.functional.silu(rows[a:b] @ up[e]) @ down[e] for e, (a, b) in enumerate(zip(ends, ends[1:]))]
    out.append(rows[ends[-1]:])                                   # rows that nothing points to
    return Combine.apply(torch.cat(out), best.softmax(1), routing)


class Heads:
    """Norms of a layer's queries and keys for each head (weights None: no norm), and the rotation of their first `rotated` elements by position."""

    def __init__(self, q_heads: int, kv_heads: int, dim: int, rotated: int, dtype: torch.dtype, norm: bool = True, base: float = 10000.0, eps: float = 1e-6):
        self.q_heads, self.kv_heads, self.dim, self.rotated, self.dtype, self.norm = q_heads, kv_heads, dim, rotated, dtype, norm
        angles = [base ** (-2 * i / rotated) for i in range(rotated // 2)] if rotated else None
        self.handle = ttc.ttc_heads_create(CODES[dtype], q_heads, kv_heads, dim, rotated, 0, angles, int(norm), eps)
        weakref.finalize(self, ttc.ttc_heads_destroy, self.handle)

    def _both(self, q, k, what: str):
        rows = q.shape[0]
        return [_matrix(x, (rows, n * self.dim), self.dtype, q.device, f"{what} of {n} heads") for x, n in ((q, self.q_heads), (k, self.kv_heads))]

    def check(self, positions: torch.Tensor, q: torch.Tensor, weights) -> list:
        """Positions [tokens] int32 and the two weights [dim] float, as the library takes them."""
        if positions.dtype != torch.int32 or tuple(positions.shape) != (q.shape[0],) or positions.device != q.device:
            raise ValueError(f"positions: {positions.dtype} {list(positions.shape)} on {positions.device}, wanted int32 [{q.shape[0]}] on {q.device}")
        for w in weights:
            if w is not None and (not self.norm or w.dtype != torch.float32 or tuple(w.shape) != (self.dim,) or w.device != q.device):
                raise ValueError(f"weights: {w.dtype} {list(w.shape)} on {w.device}, wanted float32 [{self.dim}] on {q.device}, and a norm")
        return [positions.contiguous(), *(None if w is None else w.contiguous() for w in weights)]

    def rotate(self, q, k, q_weight, k_weight, positions):
        q, k = self._both(q, k, "inputs")
        positions, q_weight, k_weight = self.check(positions, q, (q_weight, k_weight))
        q_out, k_out = (torch.zeros(x.shape, dtype=x.dtype, device=x.device) for x in (q, k))      # padding stays 0
        ttc.ttc_heads_rotate(self.handle, q.shape[0], _ptr(positions), _ptr(q), _rows_apart(q), _ptr(k), _rows_apart(k), _ptr(q_weight), _ptr(k_weight),
                             _ptr(q_out), q_out.shape[1], _ptr(k_out), k_out.shape[1], _stream())
        return q_out, k_out

    def rotate_grad(self, dq_out, dk_out, q, k, q_weight, k_weight, positions):
        dq_out, dk_out = self._both(dq_out, dk_out, "gradients")
        q, k = self._both(q, k, "inputs")
        positions, q_weight, k_weight = self.check(positions, q, (q_weight, k_weight))
        dq, dk = (torch.zeros(x.shape, dtype=x.dtype, device=x.device) for x in (q, k))
        dw = [None if w is None else torch.empty_like(w) for w in (q_weight, k_weight)]
        work = torch.empty(ttc.ttc_heads_workspace(self.handle, q.shape[0]), dtype=torch.uint8, device=q.device)
        ttc.ttc_heads_rotate_grad(self.handle, q.shape[0], _ptr(positions), _ptr(dq_out), _rows_apart(dq_out), _ptr(dk_out), _rows_apart(dk_out), _ptr(q), _rows_apart(q),
                                  _ptr(k), _rows_apart(k), _ptr(q_weight), _ptr(k_weight), _ptr(dq), dq.shape[1], _ptr(dk), dk.shape[1], _ptr(dw[0]), _ptr(dw[1]), _ptr(work), _stream())
        return dq, dk, *dw


class Rotate(torch.autograd.Function):
    """Queries and keys through Heads; the gradients of both and of both weights in one pass.  That pass records no graph of its own: a gradient of it is refused."""

    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, positions, heads):
        ctx.heads = heads
        ctx.save_for_backward(q, k, q_weight, k_weight, positions)
        return heads.rotate(q, k, q_weight, k_weight, positions)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq_out, dk_out):
        return (*ctx.heads.rotate_grad(dq_out, dk_out, *ctx.saved_tensors), None, None)


class PagedCache:
    """Keys and values of several requests in pages; the requests' lengths say where everything goes."""

    def __init__(self, requests: int, heads: int, dim: int, page: int, pages: int, longest: int, dtype: torch.dtype, cache_dtype: torch.dtype, device="cuda"):
        self.heads, self.dim, self.page, self.requests, self.device = heads, dim, page, requests, device
        self.dtype = dtype
        self.handle = ttc.ttc_pages_create(CODES[dtype], CODES[cache_dtype], heads, dim, page, pages)
        weakref.finalize(self, ttc.ttc_pages_destroy, self.handle)
        vector = dim // 2 + 4 if cache_dtype == FOUR_BITS else dim
        self.k, self.v = (torch.zeros(pages, page, heads, vector, dtype=torch.uint8, device=device).to(cache_dtype) for _ in range(2))
        self.before, self.attends = torch.zeros(requests, dtype=torch.int32, device=device), {}
        self.scale = torch.full((heads,), 0.0625, device=device) if cache_dtype == torch.float8_e4m3fn else None
        self.table = torch.full((requests, -(-longest // page)), -1, dtype=torch.int32, device=device)
        self.free = torch.randperm(pages, device=device).to(torch.int32)
        self.cached = torch.zeros(requests, dtype=torch.int32, device=device)

    def _map(self, first, fresh, tokens):
        i32 = lambda n: torch.empty(n, dtype=torch.int32, device=self.device)  # noqa: E731
        starts, page_starts, slots, positions = i32(self.requests + 1), i32(self.requests + 1), i32(tokens), i32(tokens)
        ttc.ttc_pages_map(self.handle, self.requests, _ptr(first), _ptr(self.cached), _ptr(fresh), _ptr(self.table), self.table.shape[1], _ptr(self.free),
                          self.free.numel(), tokens, _ptr(starts), _ptr(page_starts), _ptr(slots), _ptr(positions), 0, _stream())
        return starts, slots, positions

    def append(self, fresh: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q=None, rotation: Heads | None = None, weights=(None, None)):
        """fresh [requests]: how many of the packed new tokens are each one's; k, v [tokens, heads*dim].  Returns their packed offsets; with a rotation (and its
        weights) keys go into the cache rotated, and the queries q [tokens, q_heads*dim], rotated, are returned beside them.  What does
        not fit is refused before anything is mapped: a position past the table has no slot, and the write would leave its token out."""
        tokens, device = k.shape[0], self.k.device
        if (q is None) != (rotation is None):
            raise ValueError("queries and a rotation come together")
        k, v = (_matrix(x, (tokens, self.heads * self.dim), self.dtype, device, "keys and values") for x in (k, v))
        if fresh.dtype != torch.int32 or tuple(fresh.shape) != (self.requests,) or fresh.device != device:
            raise ValueError(f"fresh: {fresh.dtype} {list(fresh.shape)} on {fresh.device}, wanted int32 [{self.requests}] on {device}")
        fresh, end, limit = fresh.contiguous(), self.cached.long() + fresh, self.table.shape[1] * self.page
        blocks = lambda n: (n + (self.page - 1)) // self.page  # noqa: E731
        total, negative, over, taken = torch.stack([fresh.sum(), (fresh < 0).any(), (end > limit).sum(), (blocks(end) - blocks(self.cached.long())).sum()]).tolist()
        if negative or total != tokens:
            raise ValueError(f"fresh: {total} tokens, the keys are of {tokens}" if not negative else "fresh: a negative length")
        if over:
            raise RuntimeError(f"{over} requests would hold more than the {limit} tokens that the table has entries for")
        if taken > self.free.numel():
            raise RuntimeError(f"{taken} pages wanted, {self.free.numel()} free")
        if rotation is not None:
            if (rotation.kv_heads, rotation.dim, rotation.dtype) != (self.heads, self.dim, self.dtype) or (self.k.dtype == FOUR_BITS and rotation.rotated % 16):
                raise ValueError(f"a rotation of {rotation.rotated} elements of {rotation.kv_heads} heads of {rotation.dim} {rotation.dtype}, the cache has {self.heads} of {self.dim} "
                                 f"{self.dtype}" + (", and in 4 bits a multiple of 16" if self.k.dtype == FOUR_BITS else ""))
            q = _matrix(q, (tokens, rotation.q_heads * self.dim), self.dtype, device, "queries")
            _, q_weight, k_weight = rotation.check(torch.empty(tokens, dtype=torch.int32, device=device), q, weights)
            turned = torch.empty(tokens, rotation.q_heads * self.dim, dtype=self.dtype, device=device)
        starts, slots, positions = self._map(None, fresh, tokens)
        if rotation is None:
            ttc.ttc_pages_write(self.handle, tokens, _ptr(slots), _ptr(k), _rows_apart(k), _ptr(v), _rows_apart(v), _ptr(self.k), _ptr(self.v),
                                _ptr(self.scale), _ptr(self.scale), _stream())
        else:
            ttc.ttc_pages_append(self.handle, rotation.handle, tokens, _ptr(slots), _ptr(positions), _ptr(q), _rows_apart(q), _ptr(k), _rows_apart(k), _ptr(v), _rows_apart(v),
                                 _ptr(q_weight), _ptr(k_weight), _ptr(turned), turned.shape[1], _ptr(self.k), _ptr(self.v), _ptr(self.scale), _ptr(self.scale), _stream())
        self.free, self.before, self.cached = self.free[taken:].contiguous(), self.cached, self.cached + fresh
        return starts if rotation is None else (starts, turned)

    def attends_of(self, q_heads: int) -> int:
        """The handle of attention of that many query heads over this cache."""
        if q_heads not in self.attends:
            self.attends[q_heads] = ttc.ttc_attend_create(self.handle, q_heads, self.dim ** -0.5)
            weakref.finalize(self, ttc.ttc_attend_destroy, self.attends[q_heads])
        return self.attends[q_heads]

    def attend(self, q: torch.Tensor, starts: torch.Tensor, q_heads: int) -> torch.Tensor:
        """Attention of the tokens that the last append brought, q [tokens, q_heads*dim] at its packed offsets, over the pages of their requests."""
        tokens, width = q.shape[0], q_heads * self.dim
        q = _matrix(q, (tokens, width), self.dtype, self.k.device, "queries")
        if starts.dtype != torch.int32 or tuple(starts.shape) != (self.requests + 1,) or starts.device != q.device:
            raise ValueError(f"starts: {starts.dtype} {list(starts.shape)} on {starts.device}, wanted int32 [{self.requests + 1}] on {q.device}")
        starts = starts.contiguous()
        handle, blocks = self.attends_of(q_heads), self.table.shape[1]
        work = torch.empty(ttc.ttc_attend_workspace(handle, self.requests, tokens, blocks), dtype=torch.uint8, device=q.device)
        out = torch.empty(tokens, width, dtype=self.dtype, device=q.device)
        ttc.ttc_attend_pages(handle, self.requests, tokens, _ptr(q), _rows_apart(q), _ptr(starts), _ptr(self.before), _ptr(self.table), blocks, _ptr(self.k), _ptr(self.v),
                             _ptr(self.scale), _ptr(self.scale), _ptr(out), width, 0, _ptr(work), _stream())
        return out

    def context(self):
        """Every request's keys and values, packed, and their offsets."""
        none, total = torch.zeros_like(self.cached), int(self.cached.sum())
        starts, slots, _ = self._map(none, none, total)
        k, v = (torch.empty(total, self.heads * self.dim, dtype=self.dtype, device=self.device) for _ in range(2))
        ttc.ttc_pages_read(self.handle, total, _ptr(slots), _ptr(self.k), _ptr(self.v), _ptr(self.scale), _ptr(self.scale), _ptr(k), k.shape[1], _ptr(v), v.shape[1], _stream())
        return starts, k, v


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, heads: int, kv_heads: int) -> torch.Tensor:
    """Causal attention of one request's last tokens over its context, in 32 bits: q [new, heads*dim], k and v [all, kv_heads*dim]."""
    new, length, dim = q.shape[0], k.shape[0], k.shape[1] // kv_heads
    by_head = lambda x, n: x.float().view(x.shape[0], n, dim).transpose(0, 1)  # noqa: E731
    kh, vh = (by_head(x, kv_heads).repeat_interleave(heads // kv_heads, 0).contiguous() for x in (k, v))
    scores = by_head(q, heads).contiguous() @ kh.transpose(1, 2).contiguous() / dim ** 0.5
    later = torch.arange(length, device=q.device)[None, :] > torch.arange(length - new, length, device=q.device)[:, None]
    return (scores.masked_fill(later, -torch.inf).softmax(-1) @ vh).transpose(0, 1).reshape(new, heads * dim).to(q.dtype)


def layer(x: torch.Tensor, fresh: torch.Tensor, cache: PagedCache, w: dict, heads: int, topk: int, rotation: Heads | None = None) -> torch.Tensor:
    """One layer over the packed new tokens of all requests.  Heads longer than the attention over pages has read every request's context and attend in plain torch."""
    kv, over_pages = cache.heads * cache.dim, cache.dim <= ttc.TTC_ATTEND_MAX_DIM
    if heads % cache.heads:
        raise ValueError(f"{heads} heads of queries for {cache.heads} heads of keys: wanted a multiple")
    if over_pages:
        cache.attends_of(heads)                                   # what it refuses is refused before anything is in the cache
    q, k, v = (x @ w["qkv"]).split([heads * cache.dim, kv, kv], 1)
    if rotation is None:
        starts = cache.append(fresh, k, v)
    else:
        starts, q = cache.append(fresh, k, v, q, rotation, (w.get("q_norm"), w.get("k_norm")))
    if x.shape[0]:                                                # a step may bring nothing
        if over_pages:
            mixed = cache.attend(q, starts, heads)
        else:
            ends, k, v = cache.context()
            starts, ends = starts.tolist(), ends.tolist()
            mixed = torch.cat([attention(q[a:b], k[c:d], v[c:d], heads, cache.heads) for a, b, c, d in zip(starts, starts[1:], ends, ends[1:]) if b > a])
        x = x + mixed @ w["out"]
    return x + experts_forward(x, w["router"], w["up"], w["down"], topk)


def train_layer(x: torch.Tensor, lengths: list, w: dict, heads: int, kv_heads: int, topk: int, rotation: Heads) -> torch.Tensor:
    """The same layer on packed sequences, to be trained: rotation and experts through the library, attention in plain torch."""
    dim = rotation.dim
    q, k, v = (x @ w["qkv"]).split([heads * dim, kv_heads * dim, kv_heads * dim], 1)
    positions = torch.cat([torch.arange(n, dtype=torch.int32, device=x.device) for n in lengths])
    q, k = Rotate.apply(q, k, w.get("q_norm"), w.get("k_norm"), positions, rotation)
    mixed = [attention(a, b, c, heads, kv_heads) for a, b, c in zip(q.split(lengths), k.split(lengths), v.split(lengths))]
    x = x + torch.cat(mixed) @ w["out"]
    return x + experts_forward(x, w["router"], w["up"], w["down"], topk)


def weights(width: int, heads: int, kv_heads: int, dim: int, experts: int, hidden: int, dtype: torch.dtype, seed: int = 0, device="cuda") -> dict:
    g = torch.Generator(device=device).manual_seed(seed)
    draw = lambda *s: (torch.randn(s, generator=g, device=device) / s[-2] ** 0.5).to(dtype)  # noqa: E731
    return {"qkv": draw(width, (heads + 2 * kv_heads) * dim), "out": draw(heads * dim, width), "router": draw(width, experts),
            "up": draw(experts, width, hidden), "down": draw(experts, hidden, width)}


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=4, help="decoding steps, and training steps")
    steps = ap.parse_args().steps
    width, heads, kv_heads, dim, experts, topk, dtype = 512, 8, 2, 64, 16, 4, torch.bfloat16
    w = weights(width, heads, kv_heads, dim, experts, 1024, dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    prompts, page = [70, 1, 33, 128], 16
    longest, pages = max(prompts) + steps, sum(-(-(n + steps) // page) for n in prompts)
    lengths = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    for cache_dtype in (torch.bfloat16, torch.float8_e4m3fn):
        cache = PagedCache(len(prompts), kv_heads, dim, page, max(pages, 64), longest, dtype, cache_dtype)
        with torch.no_grad():
            y = layer(torch.randn(int(lengths.sum()), width, generator=g, device="cuda").to(dtype), lengths, cache, w, heads, topk)
            print(f"{cache_dtype}: prompts of {lengths.tolist()} tokens, mean square {float(y.float().square().mean()):.3f}, {cache.free.numel()} pages free")
            for _ in range(steps):
                y = layer(torch.randn(4, width, generator=g, device="cuda").to(dtype), torch.ones_like(lengths), cache, w, heads, topk)
        print(f"  {steps} tokens each: lengths {cache.cached.tolist()}, mean square {float(y.float().square().mean()):.3f}, {cache.free.numel()} pages free")
    norms = {"q_norm": torch.ones(dim, device="cuda"), "k_norm": torch.ones(dim, device="cuda")}
    rotation, cache = Heads(heads, kv_heads, dim, dim, dtype), PagedCache(len(prompts), kv_heads, dim, page, max(pages, 64), longest, dtype, FOUR_BITS)
    with torch.no_grad():
        for n in (lengths, *[torch.ones_like(lengths)] * steps):
            y = layer(torch.randn(int(n.sum()), width, generator=g, device="cuda").to(dtype), n, cache, {**w, **norms}, heads, topk, rotation)
    print(f"4 bits, heads normed and rotated: {cache.cached.tolist()} tokens held, mean square {float(y.float().square().mean()):.3f}, {cache.free.numel()} pages free")
    params = {k: w[k].float().requires_grad_() for k in ("router", "up", "down")}
    x = torch.randn(512, width, generator=g, device="cuda")
    target = torch.randn(512, width, generator=g, device="cuda")
    optimizer = torch.optim.Adam(params.values(), lr=1e-3)
    for step in range(steps):
        optimizer.zero_grad()
        loss = (experts_forward(x, params["router"], params["up"], params["down"], topk) - target).square().mean()
        loss.backward()
        optimizer.step()
        print(f"training step {step}: loss {float(loss):.4f}")
    params = {k: v.float().requires_grad_() for k, v in {**w, **norms}.items()}
    optimizer, rotation = torch.optim.Adam(params.values(), lr=1e-3), Heads(heads, kv_heads, dim, dim, torch.float32)
    for step in range(steps):
        optimizer.zero_grad()
        loss = (train_layer(x, [200, 1, 311], params, heads, kv_heads, topk, rotation) - target).square().mean()
        loss.backward()
        optimizer.step()
        print(f"whole layer, training step {step}: loss {float(loss):.4f}")


if __name__ == "__main__":
    main()
