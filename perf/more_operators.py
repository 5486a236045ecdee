"""Performance cases of the way of a layer's queries, keys and values: norms of the heads with the position rotation and their gradient
(ttc_heads_*), the same on the way into a paged cache (ttc_pages_append), and attention over that cache (ttc_attend_pages), which holds 16, 8 or
4 bits.  A case is one call (or the two that always follow each other), as a program that serves or trains a layer makes it: handles, workspaces
and result tensors are kept by the program, inputs are on the GPU.

`op` names the operator:
  rotate  queries and keys of a packed batch: norm of every head, weights, rotation by the token's position
  grad    its backward pass: gradients of queries, keys and both weights
  append  the same on the way of a step's tokens into the cache, values with them; the queries come back packed.  From a cache in 4 bits the step's
          keys and values are read back, which is how that cache's contents are seen as the values they stand for
  attend  the step's queries over the pages of their requests, causal, possibly within a window

Sizes are generic: heads of 64 to 256 elements, dense powers of two and odd ones, 1 to 8 queries for each key, single tokens to prompts of
thousands, contexts to 32,768.  Every tensor is row-major here: the library's column-major index 0 is torch's last.
"""
import math

import torch

own = False                 # True: the library's kernels; False: the plain form, elementary torch operations in 32 bits

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "f8": torch.float8_e4m3fn, "q4": torch.uint8}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
F8_MAX, EPS = 448.0, 1e-6


def _heads(name, op, tokens, q_heads, kv_heads, dim, dtype="bf16", rotated=None, paired=False, norm=True, base=10000.0, sequences=1):
    """paired: the two elements of a rotation are neighbours; otherwise they are half the rotated part apart."""
    return {"name": name, "op": op, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
            "rotated": dim if rotated is None else rotated, "paired": paired, "norm": norm, "base": base, "sequences": sequences}


def _append(name, requests, cached, fresh, page, q_heads=32, kv_heads=8, dim=128, dtype="bf16", cache="bf16", order="slots", rotated=None,
            paired=False, norm=True, base=500000.0):
    """cached, fresh: the longest; lengths are spread below them (fresh == 1: one token for every request)."""
    return {"name": name, "op": "append", "requests": requests, "cached": cached, "fresh": fresh, "page": page, "q_heads": q_heads,
            "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "cache": cache, "order": order, "rotated": dim if rotated is None else rotated,
            "paired": paired, "norm": norm, "base": base}


def _attend(name, requests, cached, fresh, page, q_heads=32, kv_heads=8, dim=128, dtype="bf16", cache="bf16", order="slots", window=0):
    return {"name": name, "op": "attend", "requests": requests, "cached": cached, "fresh": fresh, "page": page, "q_heads": q_heads,
            "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "cache": cache, "order": order, "window": window}


def listed():
    return [
        # a decoding step of 64 requests before another library's attention: latency is what counts
        _heads("rotate step", "rotate", 64, 32, 8, 128, base=500000.0, sequences=64),
        # the forward pass of a training micro-batch of packed documents
        _heads("rotate batch", "rotate", 16384, 32, 8, 128, sequences=11),
        # its backward pass
        _heads("grad batch", "grad", 8192, 32, 8, 128, sequences=5),
        # training in 32 bits: odd heads, a part of each rotated, neighbours paired
        _heads("grad odd", "grad", 1037, 6, 3, 80, "f32", rotated=40, paired=True, sequences=3),
        # a decoding step's queries, keys and values
        _append("append decode", 128, 6000, 1, 16),
        # packed prompts behind cached prefixes into an 8-bit cache that lies head by head
        _append("append prompts 8 bit", 16, 1000, 4000, 64, cache="f8", order="heads"),
        # a chunk of prompts into a cache in 4 bits, and out again
        _append("append prompts 4 bit", 8, 2000, 2600, 32, 28, 4, 64, dtype="f16", cache="q4", order="heads", norm=False),
        # one request that generates: the smallest call there is
        _attend("attend one", 1, 700, 1, 16, 8, 2, 64),
        # a decoding step of a batch with contexts of all lengths
        _attend("attend decode", 96, 8000, 1, 16),
        # long contexts in 4 bits
        _attend("attend decode 4 bit", 48, 32768, 1, 64, cache="q4", order="heads"),
        # prompts behind cached prefixes, four queries for each key: the largest case
        _attend("attend prompts", 6, 2048, 6000, 32, 20, 5),
        # a few drafted tokens for each request in 32 bits, odd heads, an 8-bit cache, a window
        _attend("attend drafts odd", 9, 3000, 7, 24, 10, 5, 80, dtype="f32", cache="f8", window=1000),
    ]


def draw(rng):
    def spread(lo, hi):
        return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))

    while True:
        op = rng.choice(["rotate", "grad", "append", "append", "attend", "attend", "attend"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        dim = rng.choice([64, 80, 96, 128, 128, 192, 256])
        kv_heads, group = rng.randint(1, 10), rng.choice([1, 2, 3, 4, 4, 5, 8])
        rotated = rng.choice([dim, dim, dim // 2, dim // 4])
        paired, norm, base = rng.random() < 0.3, rng.random() < 0.6, rng.choice([10000.0, 500000.0, 1000000.0])
        cache = rng.choice([dtype, dtype, "f8", "q4"])
        page, order = rng.choice([8, 16, 24, 32, 64, 128]), rng.choice(["slots", "heads"])
        fresh = 1 if rng.random() < 0.4 else spread(2, 6000)
        requests, cached = spread(1, 256), spread(1, 32768)
        if op in ("rotate", "grad"):
            tokens = spread(1, 32768)
            case = _heads("", op, tokens, kv_heads * group, kv_heads, dim, dtype, rotated, paired, norm, base, spread(1, min(tokens, 64)))
        elif op == "append":
            if cache == "q4" and rotated % 16:
                continue
            case = _append("", requests, cached, fresh, page, kv_heads * group, kv_heads, dim, dtype, cache, order, rotated, paired, norm, base)
        else:
            case = _attend("", requests, cached, fresh, page, kv_heads * group, kv_heads, dim, dtype, cache, order, rng.choice([0, 0, 0, spread(16, 4096)]))
        if op in ("append", "attend") and requests * (cached + fresh) * kv_heads * dim > 1 << 31:
            continue                                              # the cache itself, and its copy in 32 bits in the plain form
        if op == "attend" and requests * fresh * kv_heads * group * (cached + fresh) > 3 << 30:
            continue                                              # the plain form's scores
        w = work(case)
        if w["bytes"] <= 1.05e9 and w["flops"] <= 4.0e11 * (1 if dtype != "f32" else 0.25):
            del case["name"]
            return case


# ---- inputs ------------------------------------------------------------------------------------------

def _rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, dtype):
    x = torch.empty(shape, dtype=dtype if dtype != TYPES["f8"] else torch.bfloat16, device="cuda").normal_(generator=g)
    return x.to(dtype)


def _spread_lengths(n, most, one=False):
    """n lengths up to `most`, spread like the square of a uniform number: many short ones, a few long."""
    return [most if one or most <= 1 else int(1 + ((i + 0.5) / n) ** 2 * (most - 1)) for i in range(n)]


def _lengths(g, n, most, one=False):
    """The same; the seed says which request has which."""
    x = torch.tensor(_spread_lengths(n, most, one), dtype=torch.int32, device="cuda")
    return x[torch.randperm(n, generator=g, device="cuda")]


def _angles(case):
    """Radians for each position, one for each pair of elements."""
    half = case["rotated"] // 2
    return [case["base"] ** (-i / half) for i in range(half)]


def _starts(count):
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    return torch.cat([zero, count.cumsum(0).to(torch.int32)])


def _weights(g, case):
    return [1 + 0.1 * torch.randn(case["dim"], generator=g, device="cuda") if case["norm"] else None for _ in range(2)]


def _heads_inputs(case, seed):
    g, dtype, t, d = _rng(seed), TYPES[case["dtype"]], case["tokens"], case["dim"]
    hq, hk = case["q_heads"], case["kv_heads"]
    s = {"case": case, "tokens": t}
    if case["sequences"] == t:                                    # a step: every token somewhere in a request of its own
        s["positions"] = _lengths(g, t, 100000)
    else:
        ends = (torch.rand(case["sequences"], generator=g, device="cuda").cumsum(0) + 0.1)
        ends = (ends / ends[-1] * t).long()
        ends[-1] = t
        begin = torch.cat([torch.zeros_like(ends[:1]), ends[:-1]])
        i = torch.arange(t, device="cuda")
        s["positions"] = (i - begin[torch.searchsorted(ends, i, right=True)]).to(torch.int32)
    # queries, keys and values are parts of one fused projection
    qkv = _normal(g, (t, (hq + 2 * hk) * d), dtype)
    s["qkv"], s["q"], s["k"] = qkv, qkv[:, :hq * d], qkv[:, hq * d:(hq + hk) * d]
    s["q_weight"], s["k_weight"] = _weights(g, case)
    if case["op"] == "grad":
        s["dq_out"], s["dk_out"] = _normal(g, (t, hq * d), dtype), _normal(g, (t, hk * d), dtype)
    return s


def _blocks(length, page):
    return torch.div(length + (page - 1), page, rounding_mode="floor")


def _record(case):
    """Elements (bytes, in 4 bits: a step and a minimum in bf16, then the codes) of a vector of the cache."""
    return case["dim"] // 2 + 4 if case["cache"] == "q4" else case["dim"]


def _cache(g, case, pages):
    """A cache that has been in use."""
    page, heads, rec = case["page"], case["kv_heads"], _record(case)
    shape = (pages, page, heads, rec) if case["order"] == "slots" else (pages, heads, page, rec)
    if case["cache"] != "q4":
        return _normal(g, shape, TYPES[case["cache"]])
    x = torch.randint(0, 256, shape, dtype=torch.uint8, generator=g, device="cuda")
    step = (0.15 + 0.1 * torch.rand(shape[:3], generator=g, device="cuda")).to(torch.bfloat16)
    low = (-7.5 * step.float() + 0.2 * torch.randn(shape[:3], generator=g, device="cuda")).to(torch.bfloat16)
    x[..., :4] = torch.stack([step, low], -1).view(torch.uint8)
    return x


def _pages_inputs(case, seed):
    g, page, dtype = _rng(seed), case["page"], TYPES[case["dtype"]]
    requests, heads, d = case["requests"], case["kv_heads"], case["dim"]
    cached = _lengths(g, requests, case["cached"])
    fresh = _lengths(g, requests, case["fresh"], case["fresh"] <= 1)
    need = _blocks(cached + fresh, page)
    width = (case["cached"] + case["fresh"]) // page + 2
    pages = int(_blocks(cached, page).sum() + _blocks(fresh, page).sum()) + requests + 3                   # enough, however they are paired
    table = torch.full((requests, width), -1, dtype=torch.int32, device="cuda")
    inside = torch.arange(width, device="cuda")[None, :] < need[:, None]
    table[inside] = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)[: int(need.sum())]    # pages in no order
    owner = torch.repeat_interleave(torch.arange(requests, device="cuda"), fresh)
    starts = _starts(fresh)
    at = torch.arange(owner.numel(), device="cuda") - starts[owner] + cached[owner]
    s = {"case": case, "pages": pages, "table": table, "cached": cached, "fresh": fresh, "starts": starts, "tokens": owner.numel(),
         "positions": at.to(torch.int32), "slots": (table[owner, at // page] * page + at % page).to(torch.int32), "owner": owner}
    s["k_cache"], s["v_cache"] = _cache(g, case, pages), _cache(g, case, pages)
    for which in ("k_scale", "v_scale"):
        s[which] = torch.rand(heads, generator=g, device="cuda") * 0.02 + 0.005 if case["cache"] == "f8" else None
    if case["op"] == "append":
        # one fused projection; its values have bounded tails, as projections of normed inputs do
        qkv = torch.randn(s["tokens"], (case["q_heads"] + 2 * heads) * d, generator=g, device="cuda").clamp(-2, 2).to(dtype)
        s["qkv"], s["q"], s["k"], s["v"] = qkv, *qkv.split([case["q_heads"] * d, heads * d, heads * d], 1)
        s["q_weight"], s["k_weight"] = _weights(g, case)
    else:
        s["q"] = (2 * torch.randn(s["tokens"], case["q_heads"] * d, generator=g, device="cuda")).to(dtype)
        if s["k_scale"] is not None:                              # as much apart as without a scale
            s["k_scale"], s["v_scale"] = s["k_scale"] * 50, s["v_scale"] * 50
    return s


def _inputs(case, seed):
    return (_heads_inputs if case["op"] in ("rotate", "grad") else _pages_inputs)(case, seed)


def _library():
    import paper_1603_02297_amd as ttc
    return ttc


class _Handle:
    """A handle that is given back with its owner."""

    def __init__(self, create, destroy, *args):
        import weakref
        self.handle = create(*args)
        weakref.finalize(self, destroy, self.handle)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _results(s, case)
    return s


def _results(s, case):
    """What a program keeps beside its inputs: handles, workspaces and result tensors."""
    ttc = _library()
    code = {"f32": ttc.TTC_F32, "bf16": ttc.TTC_BF16, "f16": ttc.TTC_F16, "f8": ttc.TTC_F8, "q4": ttc.TTC_Q4}
    empty = lambda shape, t: torch.empty(shape, dtype=t, device="cuda")  # noqa: E731
    s["stream"] = torch.cuda.current_stream().cuda_stream
    dtype, hq, hk, d, t = TYPES[case["dtype"]], case["q_heads"], case["kv_heads"], case["dim"], s["tokens"]
    if case["op"] != "attend":
        s["heads"] = _Handle(ttc.ttc_heads_create, ttc.ttc_heads_destroy, code[case["dtype"]], hq, hk, d, case["rotated"], int(case["paired"]),
                             _angles(case), int(case["norm"]), EPS)
        s["q_out"] = empty((t, hq * d), dtype)
    if case["op"] == "rotate":
        s["k_out"] = empty((t, hk * d), dtype)
    if case["op"] == "grad":
        s["dq"], s["dk"] = empty((t, hq * d), dtype), empty((t, hk * d), dtype)
        s["dq_weight"], s["dk_weight"] = (empty(d, torch.float32) if case["norm"] else None for _ in range(2))
        s["workspace"] = empty(max(1, ttc.ttc_heads_workspace(s["heads"].handle, t)), torch.uint8)
    if case["op"] in ("append", "attend"):
        rec, page = _record(case), case["page"]
        strides = (rec, hk * rec, page * hk * rec) if case["order"] == "slots" else (page * rec, rec, page * hk * rec)
        s["handle"] = _Handle(ttc.ttc_pages_create, ttc.ttc_pages_destroy, code[case["dtype"]], code[case["cache"]], hk, d, page, s["pages"], strides)
    if case["op"] == "append" and case["cache"] == "q4":
        s["k_back"], s["v_back"] = empty((t, hk * d), dtype), empty((t, hk * d), dtype)
    if case["op"] == "attend":
        s["attend"] = _Handle(ttc.ttc_attend_create, ttc.ttc_attend_destroy, s["handle"].handle, hq, d ** -0.5, case["window"])
        s["out"] = empty((t, hq * d), dtype)
        s["workspace"] = empty(max(1, ttc.ttc_attend_workspace(s["attend"].handle, case["requests"], t, s["table"].shape[1])), torch.uint8)


# ---- the library's kernels ---------------------------------------------------------------------------

def _ptr(x):
    return 0 if x is None else x.data_ptr()


def _own_rotate(s, case):
    ld, d = s["qkv"].shape[1], case["dim"]
    _library().ttc_heads_rotate(s["heads"].handle, s["tokens"], _ptr(s["positions"]), _ptr(s["q"]), ld, _ptr(s["k"]), ld, _ptr(s["q_weight"]),
                                _ptr(s["k_weight"]), _ptr(s["q_out"]), case["q_heads"] * d, _ptr(s["k_out"]), case["kv_heads"] * d, s["stream"])
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_grad(s, case):
    ld, lq, lk = s["qkv"].shape[1], case["q_heads"] * case["dim"], case["kv_heads"] * case["dim"]
    _library().ttc_heads_rotate_grad(s["heads"].handle, s["tokens"], _ptr(s["positions"]), _ptr(s["dq_out"]), lq, _ptr(s["dk_out"]), lk, _ptr(s["q"]), ld,
                                     _ptr(s["k"]), ld, _ptr(s["q_weight"]), _ptr(s["k_weight"]), _ptr(s["dq"]), lq, _ptr(s["dk"]), lk,
                                     _ptr(s["dq_weight"]), _ptr(s["dk_weight"]), _ptr(s["workspace"]), s["stream"])
    return {k: s[k] for k in ("dq", "dk", "dq_weight", "dk_weight")}


def _own_append(s, case):
    ttc, ld, lk, t = _library(), s["qkv"].shape[1], case["kv_heads"] * case["dim"], s["tokens"]
    ttc.ttc_pages_append(s["handle"].handle, s["heads"].handle, t, _ptr(s["slots"]), _ptr(s["positions"]), _ptr(s["q"]), ld, _ptr(s["k"]), ld, _ptr(s["v"]), ld,
                         _ptr(s["q_weight"]), _ptr(s["k_weight"]), _ptr(s["q_out"]), s["q_out"].shape[1], _ptr(s["k_cache"]), _ptr(s["v_cache"]),
                         _ptr(s["k_scale"]), _ptr(s["v_scale"]), s["stream"])
    if case["cache"] != "q4":
        return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    ttc.ttc_pages_read(s["handle"].handle, t, _ptr(s["slots"]), _ptr(s["k_cache"]), _ptr(s["v_cache"]), 0, 0, _ptr(s["k_back"]), lk, _ptr(s["v_back"]), lk,
                       s["stream"])
    return {"q": s["q_out"], "k": s["k_back"], "v": s["v_back"]}


def _own_attend(s, case):
    lq = case["q_heads"] * case["dim"]
    _library().ttc_attend_pages(s["attend"].handle, case["requests"], s["tokens"], _ptr(s["q"]), lq, _ptr(s["starts"]), _ptr(s["cached"]), _ptr(s["table"]),
                                s["table"].shape[1], _ptr(s["k_cache"]), _ptr(s["v_cache"]), _ptr(s["k_scale"]), _ptr(s["v_scale"]), _ptr(s["out"]), lq, 0,
                                _ptr(s["workspace"]), s["stream"])
    return {"out": s["out"]}


# ---- the plain form ----------------------------------------------------------------------------------

def _cos_sin(s, case):
    """[tokens, 1, pairs]: angles of far positions in 64 bits."""
    angle = s["positions"].double()[:, None, None] * torch.tensor(_angles(case), dtype=torch.float64, device="cuda")
    return angle.cos().float(), angle.sin().float()


def _pairs(x, case):
    """The two elements of every rotation, and what is not rotated."""
    r = case["rotated"]
    if case["paired"]:
        return x[..., 0:r:2], x[..., 1:r:2], x[..., r:]
    return x[..., :r // 2], x[..., r // 2:r], x[..., r:]


def _joined(a, b, rest, case):
    both = torch.stack([a, b], -1).flatten(-2) if case["paired"] else torch.cat([a, b], -1)
    return torch.cat([both, rest], -1)


def _turn(x, cos, sin, case):
    a, b, rest = _pairs(x, case)
    return _joined(a * cos - b * sin, b * cos + a * sin, rest, case)


def _plain_heads(x, weight, cos, sin, case):
    """[tokens, heads*dim] of any type -> [tokens, heads, dim] in 32 bits."""
    x = x.float().reshape(x.shape[0], -1, case["dim"])
    if case["norm"]:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight
    return _turn(x, cos, sin, case)


def _plain_rotate(s, case):
    cos, sin = _cos_sin(s, case)
    return {w: _plain_heads(s[w], s[w + "_weight"], cos, sin, case).flatten(1).to(TYPES[case["dtype"]]) for w in ("q", "k")}


def _plain_grad_of(dy, x, weight, cos, sin, case):
    x, dy = (v.float().reshape(v.shape[0], -1, case["dim"]) for v in (x, dy))
    du = _turn(dy, cos, -sin, case)
    if not case["norm"]:
        return du, None
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    hat, g = x * r, du * weight
    return r * (g - hat * (g * hat).mean(-1, keepdim=True)), (du * hat).sum((0, 1))


def _plain_grad(s, case):
    cos, sin = _cos_sin(s, case)
    dq, dq_weight = _plain_grad_of(s["dq_out"], s["q"], s["q_weight"], cos, sin, case)
    dk, dk_weight = _plain_grad_of(s["dk_out"], s["k"], s["k_weight"], cos, sin, case)
    dtype = TYPES[case["dtype"]]
    return {"dq": dq.flatten(1).to(dtype), "dk": dk.flatten(1).to(dtype), "dq_weight": dq_weight, "dk_weight": dk_weight}


def _by_slot(case, cache):
    """A view of the cache as [page, slot in page, head, element]."""
    return cache if case["order"] == "slots" else cache.transpose(1, 2)


def _bf16_towards(x, up):
    """The nearest value of bf16 that is not below (not above) x."""
    bits = x.contiguous().view(torch.int32)
    away = (bits < 0) != up                                       # the magnitude grows
    return torch.where(away, bits + 0xffff, bits).bitwise_and(-0x10000).view(torch.float32)


def _to_records(x):
    """[..., dim] in 32 bits -> records of the 4-bit cache.  Values half way between two codes are common (inputs of 16 bits, steps of 8): in 64 bits,
    where these quotients are what they are."""
    low = _bf16_towards(x.amin(-1, keepdim=True), False)
    step = _bf16_towards(((x.amax(-1, keepdim=True).double() - low) / 15).float(), True)
    code = torch.where(step > 0, ((x.double() - low) / step).round().clamp(0, 15), 0).to(torch.uint8)
    head = torch.cat([step, low], -1).to(torch.bfloat16).view(torch.uint8)
    return torch.cat([head, code[..., 0::2] | code[..., 1::2] << 4], -1)


def _from_records(rec):
    """Records -> [..., dim] in 32 bits."""
    head = rec[..., :4].contiguous().view(torch.bfloat16).float()
    code = torch.stack([rec[..., 4:] & 15, rec[..., 4:] >> 4], -1).flatten(-2)
    return head[..., 1:] + code * head[..., :1]


def _plain_append(s, case):
    cos, sin = _cos_sin(s, case)
    dtype, slots = TYPES[case["dtype"]], s["slots"].long()
    at = slots // case["page"], slots % case["page"]
    k = _plain_heads(s["k"], s["k_weight"], cos, sin, case)
    v = s["v"].float().reshape(k.shape)

    def into(x, cache, scale):
        if case["cache"] == "q4":
            _by_slot(case, cache)[at] = _to_records(x)
        elif case["cache"] == "f8":
            _by_slot(case, cache.view(torch.uint8))[at] = (x / scale[None, :, None]).clamp(-F8_MAX, F8_MAX).to(cache.dtype).view(torch.uint8)
        else:
            _by_slot(case, cache)[at] = x.to(cache.dtype)

    into(k, s["k_cache"], s["k_scale"])
    into(v, s["v_cache"], s["v_scale"])
    q = _plain_heads(s["q"], s["q_weight"], cos, sin, case).flatten(1).to(dtype)
    if case["cache"] != "q4":
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    back = lambda cache: _from_records(_by_slot(case, cache)[at]).flatten(1).to(dtype)  # noqa: E731
    return {"q": q, "k": back(s["k_cache"]), "v": back(s["v_cache"])}


def _plain_attend(s, case):
    page, d, kv, group = case["page"], case["dim"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    requests, longest, most = case["requests"], case["cached"] + case["fresh"], case["fresh"]
    pos = torch.arange(longest, device="cuda")
    held = s["table"][:, pos // page].long().clamp(min=0)         # [request, position]: the page
    length = s["cached"].long() + s["fresh"]

    def context(cache, scale):
        """[request, head, position, dim] in 32 bits; positions past the end are 0."""
        bits = cache.view(torch.uint8) if case["cache"] == "f8" else cache
        x = _by_slot(case, bits)[held, (pos % page).expand_as(held)]
        x = _from_records(x) if case["cache"] == "q4" else x.view(cache.dtype).float()
        if scale is not None:
            x = x * scale[:, None]
        return torch.where((pos < length[:, None])[:, :, None, None], x, 0.0).transpose(1, 2).contiguous()

    i = torch.arange(most, device="cuda")
    row = (s["starts"][:-1, None] + i).clamp(max=s["tokens"] - 1).long()                          # [request, query]
    q = s["q"].float().reshape(-1, kv, group, d)[row].permute(0, 2, 3, 1, 4).reshape(requests, kv, group * most, d)
    k = context(s["k_cache"], s["k_scale"])
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * d ** -0.5
    del k
    mine = (s["cached"].long()[:, None] + i)[:, :, None]           # [request, query, 1]: the query's position
    seen = (pos <= mine) & (pos < length[:, None, None])
    if case["window"]:
        seen &= pos > mine - case["window"]
    scores = scores.view(requests, kv, group, most, longest).masked_fill_(~seen[:, None, None], -torch.inf)
    scores = torch.exp(scores - scores.amax(-1, keepdim=True))
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.view(requests, kv, group * most, longest), context(s["v_cache"], s["v_scale"])).view(requests, kv, group, most, d) / total
    out = out.permute(0, 3, 1, 2, 4).reshape(requests, most, -1)
    return {"out": out[i < s["fresh"][:, None]].to(TYPES[case["dtype"]])}


OWN = {"rotate": _own_rotate, "grad": _own_grad, "append": _own_append, "attend": _own_attend}
PLAIN = {"rotate": _plain_rotate, "grad": _plain_grad, "append": _plain_append, "attend": _plain_attend}


def run(state):
    case = state["case"]
    return (OWN if own else PLAIN)[case["op"]](state, case)


# ---- what a pass cannot do without -------------------------------------------------------------------

def _vector_bytes(case):
    return {"q4": case["dim"] / 2 + 4, "f8": case["dim"]}.get(case["cache"], case["dim"] * SIZE[case["dtype"]])


def work(case):
    d, hq, hk, el = case["dim"], case["q_heads"], case["kv_heads"], SIZE[case["dtype"]]
    if case["op"] in ("rotate", "grad"):
        values = case["tokens"] * (hq + hk) * d
        if case["op"] == "rotate":
            return {"bytes": values * 2 * el + case["tokens"] * 4, "flops": values * (8 if case["norm"] else 4)}
        return {"bytes": values * (3 if case["norm"] else 2) * el + case["tokens"] * 4, "flops": values * (18 if case["norm"] else 4)}
    cached, fresh = _spread_lengths(case["requests"], case["cached"]), _spread_lengths(case["requests"], case["fresh"], case["fresh"] <= 1)
    tokens = sum(fresh)
    if case["op"] == "append":
        back = 2 * hk * (_vector_bytes(case) + d * el) if case["cache"] == "q4" else 0
        return {"bytes": tokens * (2 * hq * d * el + 2 * hk * (d * el + _vector_bytes(case)) + back + 8), "flops": tokens * (hq + hk) * d * 8}
    # which prefix meets which prompt is the seed's: taken in order here
    pairs = keys = 0.0
    for c, f in zip(cached, fresh):
        w = case["window"] or c + f
        keys += min(c + f, w + f - 1)
        full = max(0, min(f, c + f - w))                          # queries that see a whole window
        pairs += full * w + (f - full) * c + (f - full) * (f - full + 1) / 2
    return {"bytes": tokens * 2 * hq * d * el + keys * 2 * hk * _vector_bytes(case), "flops": pairs * hq * 4 * d}


# ---- the definitions in 64 bits ----------------------------------------------------------------------

def _exact_turn(x, s, case, back=False):
    """Every pair as a complex number, times one of the unit circle."""
    r = case["rotated"]
    angle = s["positions"].double()[:, None, None] * torch.tensor(_angles(case), dtype=torch.float64, device="cuda")
    unit = torch.polar(torch.ones_like(angle), -angle if back else angle)
    if case["paired"]:
        z = torch.view_as_complex(x[..., :r].reshape(*x.shape[:-1], r // 2, 2).contiguous()) * unit
        turned = torch.view_as_real(z).reshape(*x.shape[:-1], r)
    else:
        z = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * unit
        turned = torch.cat([z.real, z.imag], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _exact_heads(s, which, case):
    x = s[which].double().reshape(s["tokens"], -1, case["dim"])
    if case["norm"]:
        x = x / ((x * x).sum(-1, keepdim=True) / case["dim"] + EPS).sqrt() * s[which + "_weight"].double()
    return _exact_turn(x, s, case)


def _exact_grad(s, which, case):
    x, dy = (v.double().reshape(s["tokens"], -1, case["dim"]) for v in (s[which], s["d" + which + "_out"]))
    du = _exact_turn(dy, s, case, back=True)
    if not case["norm"]:
        return du.flatten(1), None
    size = ((x * x).sum(-1, keepdim=True) / case["dim"] + EPS).sqrt()
    g = du * s[which + "_weight"].double()
    dx = g / size - x * (g * x).sum(-1, keepdim=True) / (case["dim"] * size ** 3)
    return dx.flatten(1), (du * x / size).sum(0).sum(0)


def _exact_bf16(x, towards):
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -126))) - 7)
    return towards(x / step) * step


def _exact_cached(x, case, scale):
    """What a cache of this type holds for x, as the values it stands for."""
    if case["cache"] == "f8":
        x = (x / scale.double()[:, None]).clamp(-F8_MAX, F8_MAX)
        step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
        return torch.round(x / step) * step
    if case["cache"] == "q4":
        low = _exact_bf16(x.amin(-1, keepdim=True), torch.floor)
        step = _exact_bf16((x.amax(-1, keepdim=True) - low) / 15, torch.ceil)
        return torch.where(step > 0, torch.round((x - low) / step), 0.0) * step + low
    return x


def _exact_context(s, case, which, r):
    """[positions, heads, dim] of one request."""
    cache, scale = s[which + "_cache"], s[which + "_scale"]
    pos = torch.arange(int(s["cached"][r] + s["fresh"][r]), device="cuda")
    bits = cache.view(torch.uint8) if case["cache"] == "f8" else cache
    x = _by_slot(case, bits)[s["table"][r, pos // case["page"]].long(), pos % case["page"]].contiguous()
    if case["cache"] == "q4":
        head = x[..., :4].contiguous().view(torch.bfloat16).double()
        low, high = (x[..., 4:] % 16).double(), torch.div(x[..., 4:], 16, rounding_mode="floor").double()
        code = torch.empty(*x.shape[:-1], case["dim"], dtype=torch.float64, device="cuda")
        code[..., 0::2], code[..., 1::2] = low, high
        return code * head[..., :1] + head[..., 1:]
    x = x.view(cache.dtype).double()
    return x if scale is None else x * scale.double()[:, None]


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "rotate":
        return {w: _exact_heads(s, w, case).flatten(1) for w in ("q", "k")}
    if case["op"] == "grad":
        (dq, dq_weight), (dk, dk_weight) = _exact_grad(s, "q", case), _exact_grad(s, "k", case)
        return {"dq": dq, "dk": dk, "dq_weight": dq_weight, "dk_weight": dk_weight}
    if case["op"] == "append":
        result = {"q": _exact_heads(s, "q", case).flatten(1)}
        slots = s["slots"].long()
        for which in ("k", "v"):
            x = _exact_heads(s, "k", case) if which == "k" else s["v"].double().reshape(s["tokens"], -1, case["dim"])
            x = _exact_cached(x, case, s[which + "_scale"])
            if case["cache"] == "q4":
                result[which] = x.flatten(1)
            else:
                wide = s[which + "_cache"].double()
                (wide if case["order"] == "slots" else wide.permute(0, 2, 1, 3))[slots // case["page"], slots % case["page"]] = x
                result[which + "_cache"] = wide
        return result
    if work(case)["flops"] > 6e11:
        return None
    d, group = case["dim"], case["q_heads"] // case["kv_heads"]
    out = torch.empty(s["tokens"], case["q_heads"], d, dtype=torch.float64, device="cuda")
    for r in range(case["requests"]):
        a, b, c = int(s["starts"][r]), int(s["starts"][r + 1]), int(s["cached"][r])
        k, v = _exact_context(s, case, "k", r), _exact_context(s, case, "v", r)
        q = s["q"][a:b].double().reshape(b - a, -1, d)
        key, query = torch.arange(c + b - a, device="cuda"), torch.arange(c, c + b - a, device="cuda")[:, None]
        hidden = key > query
        if case["window"]:
            hidden |= key + case["window"] <= query
        for h in range(case["q_heads"]):
            p = torch.softmax((q[:, h] @ k[:, h // group].T / math.sqrt(d)).masked_fill(hidden, -torch.inf), -1)
            out[a:b, h] = p @ v[:, h // group]
    return {"out": out.flatten(1)}
