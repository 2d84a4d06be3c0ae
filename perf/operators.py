"""Operators of the paged K/V cache, as a serving or training program calls them.

Beside the latent cache stands a cache of whole keys and values in pages of 64
positions, shared between sequences through a page table: rotary positions, the
write of new tokens, the attention of one new token over the pages, and the
pages' own bookkeeping (sharing, copy on write, freeing, keeping a part).

``listed()`` names the cases, ``draw(rng)`` gives another of the same ranges,
``prepare`` makes a program's tensors, ``run`` is one pass through an operator
(plain torch, or the library's entry points where ``own`` is set), ``exact`` the
same in 64 bits from the definitions.

Layouts: keys [pages, kv heads, 64, width], values [pages, kv heads, width, 64];
table int32 [sequences, pages of a sequence], -1 where there is none; free list
int32 [1 + pages]: the count, then a stack whose last entry is taken first.
"""

import math

import torch

own = False

PAGE = 64
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _rope(dtype, batch, tokens, heads, width, turned, context, interleaved=False, backward=False, scaling="none",
          factor=1.0, fused=False):
    return {"op": "rope", "dtype": dtype, "batch": batch, "tokens": tokens, "heads": heads, "width": width,
            "turned": turned, "context": context, "interleaved": interleaved, "backward": backward,
            "scaling": scaling, "factor": factor, "fused": fused}


def _write(dtype, batch, tokens, kv_heads, width, turned, context, interleaved=False, ragged=False):
    return {"op": "write", "dtype": dtype, "batch": batch, "tokens": tokens, "kv_heads": kv_heads, "width": width,
            "turned": turned, "context": context, "interleaved": interleaved, "ragged": ragged}


def _decode(dtype, batch, context, heads, kv_heads, width, ragged=False, sink=0, window=0):
    return {"op": "decode", "dtype": dtype, "batch": batch, "context": context, "heads": heads, "kv_heads": kv_heads,
            "width": width, "ragged": ragged, "sink": sink, "window": window}


def _fork(parents, children, context, add, layers, kv_heads, width, dtype="bf16"):
    """layers 0: the tables alone."""
    return {"op": "fork", "dtype": dtype, "parents": parents, "children": children, "context": context, "add": add,
            "layers": layers, "kv_heads": kv_heads, "width": width}


def _gather(dtype, batch, context, kept, layers, kv_heads, width):
    return {"op": "gather", "dtype": dtype, "batch": batch, "context": context, "kept": kept, "layers": layers,
            "kv_heads": kv_heads, "width": width}


def listed():
    return [
        # The queries of one decode step of a batch, a slice of the fused projection's rows.
        {"name": "rope_step_b32", **_rope("bf16", 32, 1, 16, 128, 128, 4095, fused=True)},
        # The queries of a long prompt past the trained length, frequencies ramped by wavelength.
        {"name": "rope_prompt_b4_8k", **_rope("bf16", 4, 8192, 16, 128, 128, 0, scaling="yarn", factor=4.0)},
        # Training: the gradient of an interleaved embedding of part of the head, fp32, odd length.
        {"name": "rope_grad_f32_b3_1501", **_rope("f32", 3, 1501, 16, 96, 64, 0, interleaved=True, backward=True)},
        # The write of one new token of every sequence of a batch.
        {"name": "write_step_b32", **_write("bf16", 32, 1, 16, 128, 128, 4000, ragged=True)},
        # A batch of prompts of unequal length entering the cache.
        {"name": "write_prompt_b4_4001", **_write("bf16", 4, 4001, 16, 128, 128, 0, ragged=True)},
        # Few tokens of one sequence in fp32: latency counts.
        {"name": "decode_f32_b1_512", **_decode("f32", 1, 512, 16, 16, 128)},
        # A full batch's decode step with as many key heads as query heads.
        {"name": "decode_b32_4k", **_decode("bf16", 32, 4096, 16, 16, 128)},
        # One long sequence, 16 query heads on 2 key heads: the length has to be split.
        {"name": "decode_b1_32k", **_decode("bf16", 1, 32768, 16, 2, 128)},
        # Sequences of unequal length under a budget of first and last tokens, three query heads a key head.
        {"name": "decode_window_b24", **_decode("bf16", 24, 9001, 24, 8, 64, ragged=True, sink=4, window=1020)},
        # Sampled continuations of one prompt: old ones dropped, new ones share its pages and get room for an answer.
        {"name": "fork_tables_16", **_fork(1, 16, 2048, 200, 0, 16, 128)},
        # A beam step over all layers: children share their parent's pages and copy its open page.
        {"name": "fork_copy_8x4", **_fork(8, 4, 500, 1, 24, 16, 128)},
        # Eviction to a budget: a quarter of the tokens kept, scattered, moved into fresh pages.
        {"name": "gather_b8_4k_1k", **_gather("bf16", 8, 4096, 1024, 1, 16, 128)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("rope", "write", "decode", "decode", "fork", "gather"))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        width = rng.choice((32, 64, 96, 128, 128, 160, 256))
        if op == "rope":
            c = _rope(dtype, _log(rng, 1, 64), _log(rng, 1, 8192), _log(rng, 1, 32), width,
                      8 * rng.randint(1, width // 8), _log(rng, 1, 200000) - 1, rng.random() < 0.5, rng.random() < 0.4,
                      rng.choice(("none", "linear", "ntk", "yarn")), rng.choice((1.5, 2.0, 4.0, 8.0)),
                      rng.random() < 0.5)
        elif op == "write":
            c = _write(dtype, _log(rng, 1, 64), _log(rng, 1, 4096), _log(rng, 1, 16), width,
                       8 * rng.randint(0, width // 8), _log(rng, 1, 8192) - 1, rng.random() < 0.5, rng.random() < 0.5)
        elif op == "decode":
            kv_heads = _log(rng, 1, 16)
            budget = rng.random() < 0.25
            c = _decode(dtype, _log(rng, 1, 64), _log(rng, 1, 65536), kv_heads * rng.choice((1, 1, 2, 3, 4, 8, 20)),
                        kv_heads, width, rng.random() < 0.5, rng.choice((0, 4)) if budget else 0,
                        _log(rng, 16, 4096) if budget else 0)
        elif op == "fork":
            c = _fork(_log(rng, 1, 16), _log(rng, 1, 16), _log(rng, 1, 2000), rng.choice((1, 1, _log(rng, 1, 500))),
                      rng.choice((0, 1, 4, 24)), _log(rng, 1, 16), width, dtype)
        else:
            context = _log(rng, 2, 8192)
            c = _gather(dtype, _log(rng, 1, 16), context, rng.randint(1, context), rng.choice((1, 1, 4)),
                        _log(rng, 1, 16), width)
        if _cost(c) <= most and _pool_bytes(c) <= 3 << 30:
            return c


def _cost(c):
    return work(c)["bytes"]


# ---------------------------------------------------------------------------
# sizes
# ---------------------------------------------------------------------------

def _pages(n):
    return (n + PAGE - 1) // PAGE


def _new(c):
    """New tokens of each sequence: equal, or from all down to about half of them."""
    m, b = c["tokens"], c["batch"]
    return [m - (m // 2) * i // b if c["ragged"] else m for i in range(b)]


def _lens(c):
    """Tokens of each sequence attended by a decode: equal, or from all down to about a quarter."""
    n, b = c["context"], c["batch"]
    return [n - (3 * n // 4) * i // b if c["ragged"] else n for i in range(b)]


def _seen(c, n):
    return min(n, c["sink"] + c["window"]) if c["window"] else n


def _used_pages(c):
    """Pages of all sequences, and pages of the longest."""
    if c["op"] == "write":
        one = _pages(c["context"] + c["tokens"])
        return one * c["batch"], one
    if c["op"] == "decode":
        return sum(_pages(n) for n in _lens(c)), _pages(c["context"])
    if c["op"] == "fork":
        each = _pages(c["context"] + c["add"]) - c["context"] // PAGE
        return c["parents"] * (_pages(c["context"]) + c["children"] * each), _pages(c["context"] + c["add"])
    return c["batch"] * (_pages(c["context"]) + _pages(c["kept"])), _pages(c["context"])


def _pool_bytes(c):
    if c["op"] == "rope":
        return 2 * work(c)["bytes"]
    e = 4 if c["dtype"] == "f32" else 2
    return 2 * e * (_used_pages(c)[0] + 3) * max(1, c.get("layers", 1)) * c["kv_heads"] * c["width"] * PAGE


def work(c):
    e = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "rope":
        n = c["batch"] * c["tokens"] * c["heads"]
        return {"bytes": 2 * e * n * c["width"], "flops": 3 * n * c["turned"]}
    row = c["kv_heads"] * c["width"]
    if c["op"] == "write":
        n = sum(_new(c))
        return {"bytes": 4 * e * n * row, "flops": 3 * n * c["kv_heads"] * c["turned"]}
    if c["op"] == "decode":
        n = sum(_seen(c, x) for x in _lens(c))
        return {"bytes": 2 * e * n * row + 2 * e * c["batch"] * c["heads"] * c["width"],
                "flops": 4 * n * c["heads"] * c["width"]}
    if c["op"] == "fork":
        rows = c["parents"] * c["children"]
        words = rows * (3 * _pages(c["context"]) + 3 * _pages(c["add"]))
        copied = rows if c["context"] % PAGE else 0
        return {"bytes": 4 * words + 4 * e * copied * c["layers"] * row * PAGE, "flops": 0}
    return {"bytes": c["layers"] * 4 * e * c["batch"] * c["kept"] * row, "flops": 0}


def _frequencies(c):
    """Angle per position of every pair, and the factor on what is turned."""
    d, base, s, kind = c["turned"], 10000.0, c.get("factor", 1.0), c.get("scaling", "none")
    i = torch.arange(d // 2, dtype=torch.float64)
    if kind == "ntk" and d > 2:
        base *= s ** (d / (d - 2))
    f = base ** (-2.0 * i / d)
    if kind == "linear":
        return f / s, 1.0
    if kind == "yarn":
        original = 4096.0
        at = lambda turns: d * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        low, high = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), d - 1)
        keep = 1.0 - ((i - low) / max(high - low, 1e-3)).clamp(0.0, 1.0)
        return f / s * (1.0 - keep) + f * keep, 0.1 * math.log(s) + 1.0
    return f, 1.0


# ---------------------------------------------------------------------------
# a program's tensors
# ---------------------------------------------------------------------------

def prepare(c, seed):
    """Inputs from the seed: unit-variance projections, caches whose pages lie in
    any order of the pool, tables and lengths as the program keeps them."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    host = torch.Generator()
    host.manual_seed(int(seed))
    dt, b = DTYPES[c["dtype"]], c.get("batch", 0)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dt)

    def ints(x):
        return torch.as_tensor(x, dtype=torch.int32).cuda()

    s = {"case": c}
    if c.get("turned"):
        freq, s["magnitude"] = _frequencies(c)
        s["freq"] = freq.cuda()
    if c["op"] == "rope":
        h, m, d = c["heads"], c["tokens"], c["width"]
        # queries beside keys and values in the rows of one projection, or alone
        s["x"] = normal(b, m, 3 * h, d)[:, :, :h] if c["fused"] else normal(b, m, h, d)
        s["pos"] = ints(c["context"] + torch.randint(0, 64, (b,), generator=host))
        return s

    h, d, layers = c["kv_heads"], c["width"], c.get("layers", 1)
    used, per = _used_pages(c)
    total = used + 3                              # pages that no sequence holds
    order = torch.randperm(total, generator=host)
    lead = () if c["op"] in ("write", "decode") else (max(1, layers),)
    if layers:
        s["k_pages"], s["v_pages"] = normal(*lead, total, h, PAGE, d), normal(*lead, total, h, d, PAGE)
    if c["op"] == "write":
        s["table"] = ints(order[:used].view(b, per))
        fused = normal(b, c["tokens"], 3, h, d)
        s["k"], s["v"] = fused[:, :, 1], fused[:, :, 2]
        s["start"] = ints(torch.full((b,), c["context"]))
        s["new"] = ints(_new(c))
    elif c["op"] == "decode":
        table = torch.full((b, per), -1)
        at = 0
        for i, n in enumerate(_lens(c)):
            table[i, :_pages(n)] = order[at:at + _pages(n)]
            at += _pages(n)
        s["table"], s["length"] = ints(table), ints(_lens(c))
        s["q"] = normal(b, c["heads"], d)
    elif c["op"] == "fork":
        # parents in the first rows, then each parent's children, which hold what the last step gave them
        p, n, ctx, end = c["parents"], c["parents"] * c["children"], c["context"], c["context"] + c["add"]
        table, length, refs = torch.full((p + n, per), -1), torch.full((p + n,), end), torch.zeros(total, dtype=torch.long)
        table[:p, :_pages(ctx)] = order[:p * _pages(ctx)].view(p, -1)
        length[:p] = ctx
        shared, at = ctx // PAGE, p * _pages(ctx)
        src = torch.arange(n) // c["children"]
        table[p:, :shared] = table[src, :shared]
        table[p:, shared:_pages(end)] = order[at:at + n * (_pages(end) - shared)].view(n, -1)
        refs.index_add_(0, table[table >= 0], torch.ones_like(table[table >= 0]))
        free = torch.full((1 + total,), -1)
        free[0], free[1:4] = 3, order[used:]
        s.update(table=ints(table), length=ints(length), refs=ints(refs), free=ints(free), source=ints(src),
                 rows=ints(p + torch.arange(n)), add=ints(torch.full((n,), c["add"])), start=ints(torch.zeros(n)),
                 pairs=ints(torch.full((n, 2), -1)), result=ints(torch.zeros(4)))
    else:
        new = _pages(c["kept"])
        table = torch.full((2 * b, per), -1)
        table[:b] = order[:b * per].view(b, per)
        table[b:, :new] = order[b * per:used].view(b, new)
        s["table"] = ints(table)
        s["source"], s["rows"] = ints(torch.arange(b)), ints(b + torch.arange(b))
        score = torch.rand((b, c["context"]), generator=host)
        score[:, :4] = 2.0                        # the first and the most recent tokens stay
        score[:, -(c["kept"] // 4 + 1):] += 1.0
        s["keep"] = ints(score.topk(c["kept"], dim=1).indices.sort(dim=1).values)
        s["count"] = ints(torch.full((b,), c["kept"]))
    return s


# ---------------------------------------------------------------------------
# one pass, in plain torch
# ---------------------------------------------------------------------------

def _turn(x, angle, interleaved, magnitude):
    """x [..., heads, width] turned by angle [..., pairs], in 32 bits (angles in 64)."""
    half = angle.shape[-1]
    cos, sin = (magnitude * angle.cos()).float()[..., None, :], (magnitude * angle.sin()).float()[..., None, :]
    y = x.float()
    part = y[..., :2 * half]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else (part[..., :half], part[..., half:])
    a, b = a * cos - b * sin, b * cos + a * sin
    part = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((part, y[..., 2 * half:]), -1)


def _plain_rope(s):
    c, x = s["case"], s["x"]
    pos = s["pos"][:, None].double() + torch.arange(x.shape[1], device="cuda", dtype=torch.float64)
    angle = pos[..., None] * s["freq"]
    return _turn(x, -angle if c["backward"] else angle, c["interleaved"], s["magnitude"]).to(x.dtype)


def _plain_write(s):
    c, k, v = s["case"], s["k"], s["v"]
    m = torch.arange(k.shape[1], device="cuda")
    pos = s["start"][:, None].long() + m
    if c["turned"]:
        k = _turn(k, pos.double()[..., None] * s["freq"], c["interleaved"], s["magnitude"]).to(k.dtype)
    page = s["table"].long().gather(1, pos // PAGE)
    put = m < s["new"][:, None]
    s["k_pages"][page[put], :, (pos % PAGE)[put]] = k[put]
    s["v_pages"][page[put], :, :, (pos % PAGE)[put]] = v[put]


def _plain_decode(s):
    c, q, table = s["case"], s["q"], s["table"].long().clamp_min(0)
    b, h, d = q.shape
    g, n = c["kv_heads"], table.shape[1] * PAGE
    k = s["k_pages"][table].float().transpose(1, 2).reshape(b, g, n, d)
    v = s["v_pages"][table].float().permute(0, 2, 1, 4, 3).reshape(b, g, n, d)
    score = torch.matmul(q.float().view(b, g, h // g, d) / math.sqrt(d), k.transpose(2, 3).contiguous())
    at, length = torch.arange(n, device="cuda"), s["length"][:, None].long()
    seen = at < length
    if c["window"]:
        seen = seen & ((at < c["sink"]) | (at >= length - c["window"]))
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    p = (score - score.amax(-1, keepdim=True)).exp()
    return (torch.matmul(p, v) / p.sum(-1, keepdim=True)).view(b, h, d).to(q.dtype)


def _plain_fork(s):
    """Children dropped, forked from their parents, given room; open pages copied."""
    table, length, refs, free, rows = (s[x] for x in ("table", "length", "refs", "free", "rows"))
    rows, src, per = rows.long(), s["source"].long(), table.shape[1]
    at = torch.arange(per, device="cuda")
    # free: a page nobody holds goes back in the order in which it was met, the first on top
    held = at < ((length[rows] + PAGE - 1) // PAGE)[:, None]
    pages = table[rows][held].long()
    refs.index_add_(0, pages, torch.full_like(pages, -1, dtype=torch.int32))
    rank = torch.arange(pages.numel(), device="cuda")
    first = torch.full((refs.numel(),), pages.numel(), device="cuda").scatter_reduce(0, pages, rank, "amin")
    back = pages[(first[pages] == rank) & (refs[pages] == 0)].flip(0)
    free[1 + free[0].long() + torch.arange(back.numel(), device="cuda")] = back.int()
    free[0] += back.numel()
    # fork: the parent's row, one more holder of each of its pages
    table[rows], length[rows] = table[src], length[src]
    shared = table[rows][at < ((length[rows] + PAGE - 1) // PAGE)[:, None]].long()
    refs.index_add_(0, shared, torch.ones_like(shared, dtype=torch.int32))
    # reserve: a shared open page is replaced by a copy; then room for the new tokens
    old, add = length[rows].long(), s["add"].long()
    last = table[rows].long().gather(1, (old[:, None] - 1).clamp_min(0) // PAGE)[:, 0]
    same = (last[:, None] == last).tril(-1).sum(1)             # rows before this one with the same open page
    copy = (old % PAGE != 0) & (add > 0) & (refs[last] - same > 1)
    have = (old + PAGE - 1) // PAGE - copy.long()              # pages that stay
    need = (old + add + PAGE - 1) // PAGE - have
    before = need.cumsum(0) - need
    got = (at >= have[:, None]) & (at < (have + need)[:, None])
    place = free[0].long() - (before[:, None] + at - have[:, None])
    taken = free[place[got]]
    wide = table[rows]
    wide[got] = taken
    table[rows] = wide
    refs.index_add_(0, last[copy], torch.full_like(last[copy], -1, dtype=torch.int32))
    refs[taken.long()] = 1
    free[0] -= need.sum()
    s["start"].copy_(length[rows])
    length[rows] = (old + add).int()
    n = int(copy.sum())
    s["pairs"][:n, 0] = last[copy].int()
    s["pairs"][:n, 1] = table[rows].gather(1, have[:, None])[copy, 0]
    s["result"].copy_(torch.stack((need.new_tensor(0), need.new_tensor(n), need.sum(), free[0].long())))
    if s["case"]["layers"] and n:
        a, z = s["pairs"][:n].long().unbind(1)
        s["k_pages"][:, z] = s["k_pages"][:, a]
        s["v_pages"][:, z] = s["v_pages"][:, a]


def _plain_gather(s):
    table, keep = s["table"].long(), s["keep"].long()
    to = torch.arange(keep.shape[1], device="cuda").expand_as(keep)
    put = to < s["count"][:, None]
    a = table[s["source"].long()].gather(1, keep // PAGE)[put]
    z = table[s["rows"].long()].gather(1, to // PAGE)[put]
    s["k_pages"][:, z, :, (to % PAGE)[put]] = s["k_pages"][:, a, :, (keep % PAGE)[put]]
    s["v_pages"][:, z, :, :, (to % PAGE)[put]] = s["v_pages"][:, a, :, :, (keep % PAGE)[put]]


def _tables(s):
    return {x: s[x] for x in ("table", "length", "refs", "free", "start", "pairs", "result")}


def _pools(s):
    return {x: s[x] for x in ("k_pages", "v_pages") if x in s}


def run(s):
    c = s["case"]
    if own:
        return _own(s)
    if c["op"] == "rope":
        return _plain_rope(s)
    if c["op"] == "decode":
        return _plain_decode(s)
    {"write": _plain_write, "fork": _plain_fork, "gather": _plain_gather}[c["op"]](s)
    return {**_pools(s), **(_tables(s) if c["op"] == "fork" else {})}


def _own(s):
    from paper_2607_15456_amd import kv

    c = s["case"]
    if c["op"] == "rope":
        return kv.rope(s["x"], s["freq"], pos=s["pos"], interleaved=c["interleaved"], magnitude=s["magnitude"],
                       transpose=c["backward"])
    if c["op"] == "decode":
        return kv.decode_attn(s["q"], s["k_pages"], s["v_pages"], s["table"], s["length"], n_ctx=c["context"],
                              sink=c["sink"], window=c["window"], out_dtype=s["q"].dtype)
    if c["op"] == "write":
        kv.write(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["start"], n_new=s["new"],
                 freq=s.get("freq"), interleaved=c["interleaved"], magnitude=s.get("magnitude", 1.0))
        return _pools(s)
    if c["op"] == "gather":
        kv.gather(s["k_pages"], s["v_pages"], s["table"], s["source"], s["rows"], s["keep"], s["count"])
        return _pools(s)
    pages = kv.PageTable(s["table"], s["length"], s["refs"], s["free"])
    kv.free(pages, s["rows"], s["result"])
    kv.fork(pages, s["source"], s["rows"], s["result"])
    kv.reserve(pages, s["rows"], s["add"], s["start"], s["pairs"], s["result"])
    if c["layers"]:
        kv.copy_pages(s["k_pages"], s["v_pages"], s["pairs"], s["result"])
    return {**_pools(s), **_tables(s)}


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------

def _as_complex(x, pairs, interleaved):
    x = x.double()
    if interleaved:
        return torch.complex(x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2])
    return torch.complex(x[..., :pairs], x[..., pairs:2 * pairs])


def _rotated(x, pos, c, freq, magnitude, sign=1.0):
    """x [rows, heads, width] at positions pos [rows], as complex numbers times a unit phase."""
    n = freq.numel()
    z = _as_complex(x, n, c["interleaved"])
    z = z * torch.polar(torch.full_like(z.real, magnitude), (sign * pos[:, None] * freq)[:, None].expand_as(z.real))
    y = x.double().clone()
    if c["interleaved"]:
        y[..., 0:2 * n:2], y[..., 1:2 * n:2] = z.real, z.imag
    else:
        y[..., :n], y[..., n:2 * n] = z.real, z.imag
    return y


def _exact_fork(c, s):
    """One row after another on the host, as the definitions read."""
    table, length, refs = s["table"].tolist(), s["length"].tolist(), s["refs"].tolist()
    flat = s["free"].tolist()
    free, rows, source = flat[1:1 + flat[0]], s["rows"].tolist(), s["source"].tolist()
    tail = flat[1 + flat[0]:]
    back = []
    for r in rows:
        for i in range(_pages(length[r])):
            page, table[r][i] = table[r][i], -1
            refs[page] -= 1
            if refs[page] == 0:
                back.append(page)
        length[r] = 0
    free += back[::-1]
    tail = tail[len(back):]
    for r, p in zip(rows, source):
        table[r], length[r] = list(table[p]), length[p]
        for i in range(_pages(length[p])):
            refs[table[p][i]] += 1
    pairs, start, taken = [], [], 0

    def take():
        page = free.pop()
        tail.insert(0, page)
        refs[page] = 1
        return page

    for r in rows:
        n, end = length[r], length[r] + c["add"]
        if n % PAGE and c["add"] and refs[table[r][n // PAGE]] > 1:
            page = table[r][n // PAGE]
            refs[page] -= 1
            table[r][n // PAGE] = take()
            taken += 1
            pairs.append([page, table[r][n // PAGE]])
        for i in range(_pages(n), _pages(end)):
            table[r][i] = take()
            taken += 1
        start.append(n)
        length[r] = end
    moved = torch.tensor(pairs, device="cuda").view(-1, 2)
    out = {}
    for x in _pools(s):
        out[x] = s[x].double()
        out[x][:, moved[:, 1]] = out[x][:, moved[:, 0]]
    old = s["pairs"].tolist()
    values = {"table": table, "length": length, "refs": refs, "free": [len(free)] + free + tail, "start": start,
              "pairs": pairs + old[len(pairs):], "result": [0, len(pairs), taken, len(free)]}
    return {**out, **{x: torch.tensor(v, dtype=torch.int32, device="cuda") for x, v in values.items()}}


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "fork":
        return _exact_fork(c, s)
    if c["op"] == "rope":
        x = s["x"]
        out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for i in range(x.shape[0]):
            pos = s["pos"][i].item() + torch.arange(x.shape[1], device="cuda", dtype=torch.float64)
            out[i] = _rotated(x[i], pos, c, s["freq"], s["magnitude"], -1.0 if c["backward"] else 1.0)
        return out
    if c["op"] == "decode":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        group = c["heads"] // c["kv_heads"]
        for i, n in enumerate(_lens(c)):
            pages = s["table"][i, :_pages(n)].long()
            at = torch.arange(n, device="cuda")
            if c["window"]:
                at = at[(at < c["sink"]) | (at >= n - c["window"])]
            for g in range(c["kv_heads"]):
                k = s["k_pages"][pages, g].double().reshape(-1, c["width"])[at]
                v = s["v_pages"][pages, g].double().transpose(1, 2).reshape(-1, c["width"])[at]
                q = s["q"][i, g * group:(g + 1) * group].double() * c["width"] ** -0.5
                out[i, g * group:(g + 1) * group] = torch.softmax(q @ k.t().contiguous(), -1) @ v
        return out
    k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
    for i in range(c["batch"]):
        if c["op"] == "write":
            n = _new(c)[i]
            pos = torch.arange(c["context"], c["context"] + n, device="cuda")
            k, v, page = s["k"][i, :n], s["v"][i, :n].double(), s["table"][i].long()[pos // PAGE]
            k = _rotated(k, pos.double(), c, s["freq"], s["magnitude"]) if c["turned"] else k.double()
            k_pages[page, :, pos % PAGE], v_pages[page, :, :, pos % PAGE] = k, v
        else:
            keep = s["keep"][i].long()
            to = torch.arange(c["kept"], device="cuda")
            a, z = s["table"][i].long()[keep // PAGE], s["table"][c["batch"] + i].long()[to // PAGE]
            k_pages[:, z, :, to % PAGE] = k_pages[:, a, :, keep % PAGE]
            v_pages[:, z, :, :, to % PAGE] = v_pages[:, a, :, :, keep % PAGE]
    return {"k_pages": k_pages, "v_pages": v_pages}
