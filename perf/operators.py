"""Performance cases of the moves whose index map is data: tokens sorted by expert and back (ttc_route_*), and the paged
cache of keys and values (ttc_pages_*).  A case is one call, or the two calls that always follow each other, as a program
that serves or trains a layer makes them: handles, workspaces and result tensors are kept by the program, inputs are on
the GPU.

`op` names the move:
  route   the ids that a router chose -> rows sorted by expert: the sort, then the tokens copied to their rows
  back    the experts' rows -> tokens, weighted, added up, and added to what the tokens hold (beta)
  grad    the backward pass of `back` (rows and weights) and of `route` (tokens)
  map     request lengths -> block tables, packed offsets, slots, positions
  write   keys and values of new tokens -> their slots of the cache
  read    slots of the cache -> packed keys and values

Sizes are generic: widths and head sizes of dense powers of two and odd ones, 8 to 256 experts, single tokens to prompts of
ten thousands.  Every tensor is row-major here: the library's column-major index 0 is torch's last.
"""
import torch

own = False                 # True: the library's kernels; False: the plain form, elementary torch operations in 32 bits

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "f8": torch.float8_e4m3fn}
F8_MAX = 448.0


def _route(name, op, tokens, topk, experts, width, dtype, ranks=1, align=1, ids="i64", beta=0.0, padded=0.0):
    return {"name": name, "op": op, "tokens": tokens, "topk": topk, "experts": experts, "width": width, "dtype": dtype,
            "ranks": ranks, "align": align, "ids": ids, "beta": beta, "padded": padded}


def _pages(name, op, requests, cached, fresh, page, heads=8, dim=128, dtype="bf16", cache="bf16", order="slots"):
    """cached, fresh: the longest; lengths are spread below them (fresh == 1: one token for every request)."""
    return {"name": name, "op": op, "requests": requests, "cached": cached, "fresh": fresh, "page": page, "heads": heads,
            "dim": dim, "dtype": dtype, "cache": cache, "order": order}


def listed():
    return [
        # a decoding step of 32 requests: two launches' latency is what counts
        _route("route decode", "route", 32, 8, 128, 2048, "bf16"),
        # a packed batch of prompts; segments padded to the rows of a matrix tile
        _route("route prompt", "route", 16384, 4, 64, 4096, "bf16", align=128),
        # one request that generates, the result added to the residual: the smallest call there is
        _route("back one token", "back", 1, 8, 64, 2048, "bf16", beta=1.0),
        # a large packed batch, some of it padding
        _route("back prompt", "back", 16384, 8, 128, 4096, "bf16", padded=0.03),
        # training in 32 bits on one of four ranks that hold the experts: three of four rows live elsewhere; odd width
        _route("grad ragged rank", "grad", 2050, 2, 8, 1001, "f32", ranks=4, align=16, ids="i32"),
        # a training step's micro-batch
        _route("grad batch", "grad", 8192, 8, 64, 2048, "bf16", align=64),
        # a decoding step: one token for each of 200 requests
        _pages("map decode", "map", 200, 6000, 1, 16),
        # ragged prompts behind a cached prefix
        _pages("map prompts", "map", 48, 3000, 5000, 32),
        # a decoding step's keys and values
        _pages("write decode", "write", 128, 2000, 1, 16),
        # prompts into an 8-bit cache that lies head by head, as a product over one head's slots reads it
        _pages("write prompts 8 bit", "write", 24, 1000, 2600, 64, cache="f8", order="heads"),
        # a few short contexts, odd head size
        _pages("read short", "read", 6, 300, 0, 16, heads=5, dim=80, dtype="f16", cache="f16", order="heads"),
        # the cached prefixes of a batch, out of an 8-bit cache
        _pages("read prefixes 8 bit", "read", 100, 2000, 0, 64, cache="f8"),
    ]


def draw(rng):
    def spread(lo, hi):
        return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))

    while True:
        op = rng.choice(["route", "back", "grad", "map", "write", "read"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if op in ("route", "back", "grad"):
            width = spread(64, 8192)
            if rng.random() < 0.6:
                width = -(-width // 64) * 64
            topk, experts, ranks = rng.randint(1, 8), spread(2, 256), rng.choice([1, 1, 2, 4])
            case = _route("", op, spread(1, 32768), min(topk, experts * ranks), experts, width, dtype, ranks, rng.choice([1, 1, 16, 64, 128]),
                          rng.choice(["i32", "i64"]), rng.choice([0.0, 1.0]) if op == "back" else 0.0, rng.choice([0.0, 0.0, 0.1]))
        else:
            fresh = 0 if op == "read" else 1 if rng.random() < 0.5 else spread(2, 4096)
            requests = spread(1, 2048 if op == "map" else 256)
            case = _pages("", op, requests, spread(1, 8192), fresh, rng.choice([8, 16, 24, 32, 64, 128]), rng.randint(1, 16),
                          rng.choice([64, 80, 96, 128, 192, 256]), dtype, rng.choice([dtype, dtype, "f8"]), rng.choice(["slots", "heads"]))
            if op != "map" and requests * (case["cached"] + fresh) * case["heads"] * case["dim"] > 1 << 30:
                continue                                          # the cache itself, of which a pass may touch little
        if work(case)["bytes"] <= 1.15e9:
            del case["name"]
            return case


# ---- inputs ------------------------------------------------------------------------------------------

def _rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, dtype):
    x = torch.empty(shape, dtype=dtype if dtype != TYPES["f8"] else torch.bfloat16, device="cuda").normal_(generator=g)
    return x.to(dtype)


def _lengths(g, n, most, one=False):
    """n lengths up to `most`, spread like the square of a uniform number: many short ones, a few long.  The seed says
    which request has which."""
    if one or most <= 1:
        return torch.full((n,), most, dtype=torch.int32, device="cuda")
    u = (torch.randperm(n, generator=g, device="cuda") + 0.5) / n
    return (1 + u * u * (most - 1)).to(torch.int32)


def _choices(case, g):
    """A router's choice: logits with a preference for some experts, their best topk and the softmax over those."""
    t, total = case["tokens"], case["experts"] * case["ranks"]
    logits = torch.randn(t, total, generator=g, device="cuda") + torch.randn(total, generator=g, device="cuda")
    best, ids = logits.topk(case["topk"], dim=1)
    if case["padded"]:
        ids = torch.where(torch.rand(t, 1, generator=g, device="cuda") < case["padded"], -1, ids)
    return ids.to(torch.int64 if case["ids"] == "i64" else torch.int32).contiguous(), best.softmax(1).contiguous()


def _capacity(case):
    """Rows of the sorted tensor that always suffice: ttc_route_rows."""
    n = case["tokens"] * case["topk"]
    return n + min(n, case["experts"]) * (case["align"] - 1)


def _first(case):
    return case["experts"] * (case["ranks"] // 2)                 # the rank in the middle


def _route_inputs(case, seed):
    g, dtype = _rng(seed), TYPES[case["dtype"]]
    s = {"case": case}
    s["ids"], s["weights"] = _choices(case, g)
    shape_t, shape_r = (case["tokens"], case["width"]), (_capacity(case), case["width"])
    if case["op"] == "route":
        s["x"] = _normal(g, shape_t, dtype)
    else:
        s["offsets"], s["counts"], s["position"], _ = _plain_sort(case, s["ids"])
        s["rows"] = _normal(g, shape_r, dtype)
    if case["op"] == "back":
        s["y"] = _normal(g, shape_t, dtype)
    if case["op"] == "grad":
        s["dy"] = _normal(g, shape_t, dtype)
        s["dinput"] = _normal(g, shape_r, dtype)                  # what the experts' backward pass leaves for their input rows
    return s


def _blocks(length, page):
    return torch.div(length + (page - 1), page, rounding_mode="floor")


def _pages_inputs(case, seed):
    g, page = _rng(seed), case["page"]
    cached = _lengths(g, case["requests"], case["cached"])
    fresh = _lengths(g, case["requests"], case["fresh"], case["fresh"] <= 1)
    have, need = _blocks(cached, page), _blocks(cached + fresh, page)
    width = (case["cached"] + case["fresh"]) // page + 2
    pages = int(_blocks(cached, page).sum() + _blocks(fresh, page).sum()) + case["requests"] + 3          # enough, however they are paired
    shuffled = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    # a full table first, in pages of a cache that has been in use: requests hold pages in no order
    table = torch.full((case["requests"], width), -1, dtype=torch.int32, device="cuda")
    inside = torch.arange(width, device="cuda")[None, :] < need[:, None]
    table[inside] = shuffled[: int(need.sum())]
    s = {"case": case, "pages": pages}
    if case["op"] == "map":
        taken = (torch.arange(width, device="cuda")[None, :] >= have[:, None]) & inside
        s["free"] = torch.cat([table[taken], shuffled[int(need.sum()):]]).contiguous()
        table[taken] = -1
        s["table"], s["cached"], s["fresh"] = table, cached, fresh
        s["tokens"] = int(fresh.sum()) + 5                        # a step's buffers are a little larger than the step
        return s
    begin, count = (cached, fresh) if case["op"] == "write" else (torch.zeros_like(cached), cached)
    owner = torch.repeat_interleave(torch.arange(case["requests"], device="cuda"), count)
    at = torch.arange(owner.numel(), device="cuda") - (count.cumsum(0) - count)[owner] + begin[owner]
    s["slots"] = (table[owner, at // page] * page + at % page).to(torch.int32)
    s["tokens"] = owner.numel()
    if s["tokens"] > 40:
        s["slots"][-2:] = -1                                      # padding at the end of a step's buffers
    cache_type, dtype, heads, dim = TYPES[case["cache"]], TYPES[case["dtype"]], case["heads"], case["dim"]
    # one page more than the library is told of: the plain form puts padding there
    shape = (pages + 1, page, heads, dim) if case["order"] == "slots" else (pages + 1, heads, page, dim)
    for which in ("k", "v"):
        s[which + "_cache"] = _normal(g, shape, cache_type)
        s[which + "_scale"] = torch.rand(heads, generator=g, device="cuda") * 0.02 + 0.005 if case["cache"] == "f8" else None
    if case["op"] == "write":
        # both are parts of one fused projection: a token's row holds queries, keys and values
        qkv = _normal(g, (s["tokens"], 4 * heads * dim), dtype)
        s["qkv"], s["k"], s["v"] = qkv, qkv[:, 2 * heads * dim:3 * heads * dim], qkv[:, 3 * heads * dim:]
    return s


def _library():
    import paper_1603_02297_amd as ttc
    return ttc


class _Handle:
    """A handle that is given back with its owner."""

    def __init__(self, create, destroy, *args, **kwargs):
        import weakref
        self.handle = create(*args, **kwargs)
        weakref.finalize(self, destroy, self.handle)


def prepare(case, seed):
    s = (_route_inputs if case["op"] in ("route", "back", "grad") else _pages_inputs)(case, seed)
    if own:
        _results(s, case)
    return s


def _results(s, case):
    """What a program keeps beside its inputs: the handle, workspaces and result tensors."""
    ttc = _library()
    code = {"f32": ttc.TTC_F32, "bf16": ttc.TTC_BF16, "f16": ttc.TTC_F16, "f8": ttc.TTC_F8}
    empty = lambda shape, t: torch.empty(shape, dtype=t, device="cuda")  # noqa: E731
    s["stream"] = torch.cuda.current_stream().cuda_stream
    if case["op"] in ("route", "back", "grad"):
        t, k, d, dtype = case["tokens"], case["topk"], case["width"], TYPES[case["dtype"]]
        create = lambda beta: _Handle(ttc.ttc_route_create, ttc.ttc_route_destroy, code[case["dtype"]], d, k, case["experts"], _first(case),  # noqa: E731
                                      case["align"], 8 if case["ids"] == "i64" else 4, 1.0, beta)
        s["route"] = create(case["beta"])
        if case["op"] == "route":
            s["offsets"], s["counts"] = empty(case["experts"] + 1, torch.int32), empty(case["experts"], torch.int32)
            s["position"], s["source"] = empty((t, k), torch.int32), empty(_capacity(case), torch.int32)
            s["workspace"] = empty(max(1, ttc.ttc_route_workspace(s["route"].handle, t)), torch.uint8)
            s["rows"] = torch.zeros((_capacity(case), d), dtype=dtype, device="cuda")
        if case["op"] == "grad":
            s["drows"] = torch.zeros((_capacity(case), d), dtype=dtype, device="cuda")
            s["dweights"], s["dx"] = empty((t, k), torch.float32), empty((t, d), dtype)
        return
    heads, dim = case["heads"], case["dim"]
    strides = (dim, heads * dim, case["page"] * heads * dim) if case["order"] == "slots" else (case["page"] * dim, dim, case["page"] * heads * dim)
    s["handle"] = _Handle(ttc.ttc_pages_create, ttc.ttc_pages_destroy, code[case["dtype"]], code[case["cache"]], heads, dim, case["page"], s["pages"], strides)
    if case["op"] == "map":
        s["starts"], s["page_starts"] = empty(case["requests"] + 1, torch.int32), empty(case["requests"] + 1, torch.int32)
        s["slots"], s["positions"], s["owner"] = (empty(s["tokens"], torch.int32) for _ in range(3))
    if case["op"] == "read":
        s["k"], s["v"] = (empty((s["tokens"], heads * dim), TYPES[case["dtype"]]) for _ in range(2))


# ---- the library's kernels ---------------------------------------------------------------------------

def _ptr(x):
    return 0 if x is None else x.data_ptr()


def _own_route(s, case):
    ttc, h, t, d = _library(), s["route"].handle, case["tokens"], case["width"]
    ttc.ttc_route_sort(h, t, _ptr(s["ids"]), case["topk"], _ptr(s["offsets"]), _ptr(s["counts"]), _ptr(s["position"]), _ptr(s["source"]),
                       _ptr(s["workspace"]), s["stream"])
    ttc.ttc_route_gather(h, t, _ptr(s["x"]), d, 0, _ptr(s["position"]), _ptr(s["offsets"]), _ptr(s["counts"]), _ptr(s["rows"]), d, s["stream"])
    return {k: s[k] for k in ("offsets", "counts", "position", "source", "rows")}


def _own_back(s, case):
    _library().ttc_route_combine(s["route"].handle, case["tokens"], _ptr(s["rows"]), case["width"], _ptr(s["weights"]), _ptr(s["position"]),
                                 _ptr(s["y"]), case["width"], s["stream"])
    return {"y": s["y"]}


def _own_grad(s, case):
    ttc, h, t, d = _library(), s["route"].handle, case["tokens"], case["width"]
    ttc.ttc_route_combine_grad(h, t, _ptr(s["dy"]), d, _ptr(s["rows"]), d, _ptr(s["weights"]), _ptr(s["position"]), _ptr(s["offsets"]),
                               _ptr(s["counts"]), _ptr(s["drows"]), d, _ptr(s["dweights"]), s["stream"])
    ttc.ttc_route_combine(h, t, _ptr(s["dinput"]), d, 0, _ptr(s["position"]), _ptr(s["dx"]), d, s["stream"])
    return {"drows": s["drows"], "dweights": s["dweights"], "dx": s["dx"]}


def _own_map(s, case):
    _library().ttc_pages_map(s["handle"].handle, case["requests"], 0, _ptr(s["cached"]), _ptr(s["fresh"]), _ptr(s["table"]), s["table"].shape[1],
                             _ptr(s["free"]), s["free"].numel(), s["tokens"], _ptr(s["starts"]), _ptr(s["page_starts"]), _ptr(s["slots"]),
                             _ptr(s["positions"]), _ptr(s["owner"]), s["stream"])
    return {k: s[k] for k in ("table", "starts", "page_starts", "slots", "positions", "owner")}


def _own_write(s, case):
    ld = s["qkv"].shape[1]
    _library().ttc_pages_write(s["handle"].handle, s["tokens"], _ptr(s["slots"]), _ptr(s["k"]), ld, _ptr(s["v"]), ld, _ptr(s["k_cache"]),
                               _ptr(s["v_cache"]), _ptr(s["k_scale"]), _ptr(s["v_scale"]), s["stream"])
    return {which: s[which][: s["pages"]] for which in ("k_cache", "v_cache")}


def _own_read(s, case):
    ld = case["heads"] * case["dim"]
    _library().ttc_pages_read(s["handle"].handle, s["tokens"], _ptr(s["slots"]), _ptr(s["k_cache"]), _ptr(s["v_cache"]), _ptr(s["k_scale"]),
                              _ptr(s["v_scale"]), _ptr(s["k"]), ld, _ptr(s["v"]), ld, s["stream"])
    return {"k": s["k"], "v": s["v"]}


# ---- the plain form ----------------------------------------------------------------------------------

def _plain_sort(case, ids):
    experts, n, device = case["experts"], ids.numel(), ids.device
    e = ids.reshape(-1).to(torch.int64) - _first(case)
    e = torch.where((e >= 0) & (e < experts), e, experts)         # the last bin: no expert of this rank
    order = torch.argsort(e, stable=True)
    every = torch.zeros(experts + 1, dtype=torch.int64, device=device).scatter_add_(0, e, torch.ones_like(e))
    counts = every[:experts]
    offsets = torch.cat([torch.zeros_like(every[:1]), (_blocks(counts, case["align"]) * case["align"]).cumsum(0)])
    sorted_e = e[order]
    rank = torch.arange(n, device=device) - (every.cumsum(0) - every)[sorted_e]
    rows = _capacity(case)
    at = torch.where(sorted_e < experts, offsets[sorted_e] + rank, rows)
    position = torch.empty(n, dtype=torch.int64, device=device).scatter_(0, order, torch.where(at < rows, at, -1))
    source = torch.full((rows + 1,), -1, dtype=torch.int64, device=device).scatter_(0, at, order)[:rows]   # the last entry: not here
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return i32(offsets), i32(counts), i32(position).view(ids.shape), i32(source)


def _plain_route(s, case):
    offsets, counts, position, source = _plain_sort(case, s["ids"])
    taken = s["x"].float()[torch.div(source.clamp(min=0), case["topk"], rounding_mode="floor")]
    rows = torch.where((source >= 0)[:, None], taken, 0.0).to(s["x"].dtype)
    return {"offsets": offsets, "counts": counts, "position": position, "source": source, "rows": rows}


def _plain_sum(rows, weights, position):
    at = position.long()[:, :, None]
    part = rows[at[:, :, 0].clamp(min=0)].float()                 # [token, k, width]
    if weights is not None:
        part = part * weights[:, :, None]
    return torch.where(at >= 0, part, 0.0).sum(1)


def _plain_back(s, case):
    total = _plain_sum(s["rows"], s["weights"], s["position"])
    if case["beta"]:
        total = total + case["beta"] * s["y"].float()
    s["y"].copy_(total)                                           # the program's tensor: the next call adds to it again
    return {"y": s["y"]}


def _plain_grad(s, case):
    dy, at = s["dy"].float()[:, None, :], s["position"].long()
    drows = torch.zeros((s["rows"].shape[0] + 1, case["width"]), dtype=torch.float32, device=dy.device)
    drows[torch.where(at >= 0, at, s["rows"].shape[0])] = dy * s["weights"][:, :, None]           # the last row: not here
    dweights = torch.where(at >= 0, (dy * s["rows"][at.clamp(min=0)].float()).sum(2), 0.0)
    dx = _plain_sum(s["dinput"], None, s["position"])
    return {"drows": drows[:-1].to(s["rows"].dtype), "dweights": dweights, "dx": dx.to(s["rows"].dtype)}


def _plain_map(s, case):
    page, table, tokens, device = case["page"], s["table"], s["tokens"], s["table"].device
    cached, fresh = s["cached"].long(), s["fresh"].long()
    have, need = _blocks(cached, page), _blocks(cached + fresh, page)
    zero = torch.zeros(1, dtype=torch.int64, device=device)
    starts, page_starts = torch.cat([zero, fresh.cumsum(0)]), torch.cat([zero, (need - have).cumsum(0)])
    block = torch.arange(table.shape[1], device=device)[None, :]
    new = (block >= have[:, None]) & (block < need[:, None])
    pick = (page_starts[:-1, None] + block - have[:, None]).clamp(0, s["free"].numel() - 1)
    table.copy_(torch.where(new, s["free"][pick], table))
    i = torch.arange(tokens, device=device)
    owner = torch.searchsorted(starts[1:], i, right=True)
    inside = owner < case["requests"]
    r = owner.clamp(max=case["requests"] - 1)
    at = cached[r] + i - starts[r]
    slots = table[r, (at // page).clamp(max=table.shape[1] - 1)] * page + at % page
    out = lambda x: torch.where(inside, x, -1).to(torch.int32)  # noqa: E731
    return {"table": table, "starts": starts.to(torch.int32), "page_starts": page_starts.to(torch.int32), "slots": out(slots),
            "positions": out(at), "owner": out(owner)}


def _by_slot(case, cache):
    """A view of the cache as [page, slot in page, head, dim]."""
    return cache if case["order"] == "slots" else cache.transpose(1, 2)


def _plain_write(s, case):
    slots = torch.where(s["slots"] >= 0, s["slots"], s["pages"] * case["page"]).long()

    def into(x, cache, scale):
        x = x.float().view(s["tokens"], case["heads"], case["dim"])
        if scale is not None:
            x = (x / scale[None, :, None]).clamp(-F8_MAX, F8_MAX).to(cache.dtype).view(torch.uint8)
            cache = cache.view(torch.uint8)
        _by_slot(case, cache)[slots // case["page"], slots % case["page"]] = x.to(cache.dtype)

    into(s["k"], s["k_cache"], s["k_scale"])
    into(s["v"], s["v_cache"], s["v_scale"])
    return {which: s[which][: s["pages"]] for which in ("k_cache", "v_cache")}


def _plain_read(s, case):
    slots = s["slots"].clamp(min=0).long()

    def out_of(cache, scale):
        bits = cache.view(torch.uint8) if case["cache"] == "f8" else cache
        x = _by_slot(case, bits)[slots // case["page"], slots % case["page"]].view(cache.dtype).float()
        if scale is not None:
            x = x * scale[None, :, None]
        x = torch.where((s["slots"] >= 0)[:, None, None], x, 0.0)
        return x.to(TYPES[case["dtype"]]).view(s["tokens"], -1)

    return {"k": out_of(s["k_cache"], s["k_scale"]), "v": out_of(s["v_cache"], s["v_scale"])}


OWN = {"route": _own_route, "back": _own_back, "grad": _own_grad, "map": _own_map, "write": _own_write, "read": _own_read}
PLAIN = {"route": _plain_route, "back": _plain_back, "grad": _plain_grad, "map": _plain_map, "write": _plain_write, "read": _plain_read}


def run(state):
    case = state["case"]
    return (OWN if own else PLAIN)[case["op"]](state, case)


# ---- what a pass cannot do without -------------------------------------------------------------------

def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2, "f8": 1}
    if case["op"] in ("route", "back", "grad"):
        t, k, d, el = case["tokens"], case["topk"], case["width"], size[case["dtype"]]
        live = t * k / case["ranks"] * (1 - case["padded"])       # rows that hold a token; padding rows are written, too
        pad = min(live, case["experts"]) * (case["align"] - 1) / 2
        if case["op"] == "route":
            return {"bytes": t * k * ((8 if case["ids"] == "i64" else 4) + 4) + _capacity(case) * 4 + t * d * el + (live + pad) * d * el, "flops": 0}
        if case["op"] == "back":
            return {"bytes": t * k * 8 + live * d * el + t * d * el * (2 if case["beta"] else 1), "flops": 2 * live * d}
        return {"bytes": t * k * 12 + t * d * el + live * d * el + (live + pad) * d * el + live * d * el + t * d * el, "flops": 4 * live * d}
    long, new = case["cached"] / 3, 1 if case["fresh"] == 1 else case["fresh"] / 3         # the mean of a squared uniform number
    if case["op"] == "map":
        held = 0 if case["fresh"] == 1 else 4 * new / case["page"]
        return {"bytes": case["requests"] * (8 + 8 + 8 + 12 * new + 2 * held), "flops": 0}
    tokens = case["requests"] * (new if case["op"] == "write" else long)
    one = 2 * case["heads"] * case["dim"] * (size[case["dtype"]] + size[case["cache"]])
    return {"bytes": tokens * (4 + one), "flops": 0}


# ---- the definitions in 64 bits ----------------------------------------------------------------------

def _exact_sort(case, ids):
    """Experts one after the other, each one's assignments in order."""
    flat, first = ids.reshape(-1), _first(case)
    position = torch.full((flat.numel(),), -1, dtype=torch.int64, device=flat.device)
    source = torch.full((_capacity(case),), -1, dtype=torch.int64, device=flat.device)
    offsets, counts = [0], []
    for e in range(case["experts"]):
        mine = torch.nonzero(flat == first + e).reshape(-1)
        rows = offsets[-1] + torch.arange(mine.numel(), device=flat.device)
        position[mine], source[rows] = rows, mine
        counts.append(mine.numel())
        offsets.append(offsets[-1] + (mine.numel() + case["align"] - 1) // case["align"] * case["align"])
    i32 = lambda x: torch.as_tensor(x, dtype=torch.int32, device=flat.device)  # noqa: E731
    return i32(offsets), i32(counts), i32(position).view(ids.shape), i32(source)


def exact(case, seed):
    op = case["op"]
    s = (_route_inputs if op in ("route", "back", "grad") else _pages_inputs)(case, seed)
    if op == "route":
        offsets, counts, position, source = _exact_sort(case, s["ids"])
        rows = torch.zeros((source.numel(), case["width"]), dtype=torch.float64, device="cuda")
        held = torch.nonzero(source >= 0).reshape(-1)
        rows[held] = s["x"][source[held].long() // case["topk"]].double()
        return {"offsets": offsets, "counts": counts, "position": position, "source": source, "rows": rows}
    if op in ("back", "grad"):
        token, k = torch.nonzero(s["position"] >= 0, as_tuple=True)
        at, w = s["position"][token, k].long(), s["weights"][token, k].double()
        shape = (case["tokens"], case["width"])
    if op == "back":
        y = case["beta"] * s["y"].double() if case["beta"] else torch.zeros(shape, dtype=torch.float64, device="cuda")
        return {"y": y.index_add_(0, token, s["rows"][at].double() * w[:, None])}
    if op == "grad":
        dy = s["dy"][token].double()
        drows = torch.zeros(s["rows"].shape, dtype=torch.float64, device="cuda")
        drows[at] = w[:, None] * dy
        dweights = torch.zeros(s["position"].shape, dtype=torch.float64, device="cuda")
        dweights[token, k] = (dy * s["rows"][at].double()).sum(1)
        dx = torch.zeros(shape, dtype=torch.float64, device="cuda").index_add_(0, token, s["dinput"][at].double())
        return {"drows": drows, "dweights": dweights, "dx": dx}
    if op == "map":
        page, table, free = case["page"], s["table"].cpu().numpy(), s["free"].tolist()
        starts, page_starts, slots, positions, owner = [0], [0], [], [], []
        for r, (c, f) in enumerate(zip(s["cached"].tolist(), s["fresh"].tolist())):
            for at in range(c, c + f):
                if at % page == 0:                                # the first token of a page takes the page
                    table[r, at // page] = free.pop(0)
                slots.append(int(table[r, at // page]) * page + at % page)
                positions.append(at)
                owner.append(r)
            starts.append(starts[-1] + f)
            page_starts.append(s["free"].numel() - len(free))
        spare = [-1] * (s["tokens"] - len(slots))
        i32 = lambda x: torch.as_tensor(x, dtype=torch.int32)  # noqa: E731
        return {"table": torch.from_numpy(table), "starts": i32(starts), "page_starts": i32(page_starts), "slots": i32(slots + spare),
                "positions": i32(positions + spare), "owner": i32(owner + spare)}
    held = torch.nonzero(s["slots"] >= 0).reshape(-1)
    at = s["slots"][held].long()
    result = {}
    for which in ("k", "v"):
        cache, scale = s[which + "_cache"], s[which + "_scale"]
        wide = cache[: s["pages"]].double()
        view = wide if case["order"] == "slots" else wide.permute(0, 2, 1, 3)
        by = torch.ones(case["heads"], dtype=torch.float64, device="cuda") if scale is None else scale.double()
        if op == "write":
            x = s[which].reshape(s["tokens"], case["heads"], case["dim"])[held].double() / by[:, None]
            if scale is not None:                                 # what the cache stands for is known to four bits: the nearest of its values
                x = x.clamp(-F8_MAX, F8_MAX)
                step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
                x = torch.round(x / step) * step
            view[at // case["page"], at % case["page"]] = x
            result[which + "_cache"] = wide
        else:
            out = torch.zeros((s["tokens"], case["heads"], case["dim"]), dtype=torch.float64, device="cuda")
            out[held] = view[at // case["page"], at % case["page"]] * by[:, None]
            result[which] = out.reshape(s["tokens"], -1)
    return result
