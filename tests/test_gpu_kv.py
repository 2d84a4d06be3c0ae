"""GPU parity of the paged K/V cache against its float64 oracle: rotary
positions, write, decode attention, tables, page copies and gathers, and all of
them as a serving program runs them.

Tolerances (eps = 2^-24 in fp32; a rounding to bf16 is off by at most 2^-8 of the
value): a turned feature is u cos - v sin with cos and sin off by at most 2^-23
each from the rounded angle (up to pi) and as much again from their evaluation,
then three roundings: 6e-7 (|u| + |v|) covers it.  Attention: a score is off by
at most (d + 2) eps sum |q k| scale; a weight by twice that, and by 2^-16 for the
two bf16 terms it is multiplied as and its exponential; the sums over the tokens
by their longest chains, (N/16 + 64) eps; each of them times sum p |v|.
"""

import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from paper_2607_15456_amd import kv, lla
from tests.helpers import f64, log

pytestmark = pytest.mark.gpu

DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
EPS = 2.0 ** -24


def normal(shape, seed, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV, dtype=F32).to(dtype)


def ints(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(DEV)


def half_step(dtype):
    return 2.0 ** -8 if dtype == BF else EPS


def near(got, ref, tol, what):
    got = f64(got)
    off = np.abs(got - ref)
    assert got.shape == ref.shape and np.all(np.isfinite(got)), what
    worst = float(np.max(off / tol))
    log(f"  {what}: {worst:.3f} of the bound")
    assert worst <= 1.0, (what, worst)


def rope_bound(x, freq_n, interleaved, magnitude, y, dtype):
    """Per element: 6e-7 (|u| + |v|) of its pair, and the rounding of the result."""
    b = np.zeros_like(x)
    n = freq_n
    a = np.abs(x)
    if interleaved:
        s = a[..., 0:2 * n:2] + a[..., 1:2 * n:2]
        b[..., 0:2 * n:2], b[..., 1:2 * n:2] = s, s
    else:
        s = a[..., :n] + a[..., n:2 * n]
        b[..., :n], b[..., n:2 * n] = s, s
    return 6e-7 * abs(magnitude) * b * (1 + half_step(dtype)) + half_step(dtype) * np.abs(y) + 1e-30


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,M,H,d,rot", [(1, 1, 1, 8, 8), (3, 1, 16, 128, 128), (2, 37, 3, 96, 64), (1, 700, 5, 128, 24),
                                         (2, 130, 4, 256, 256), (1, 65, 2, 512, 40), (40, 3, 7, 64, 56)])
def test_rope(dtype, interleaved, B, M, H, d, rot):
    freq, mag = kv.rope_frequencies(rot, scaling="yarn", factor=4.0, original=512)
    x = normal((B, M, H, d), 1, dtype)
    starts = np.arange(B) * 1237 + 5
    for transpose in (False, True):
        y = kv.rope(x, freq, pos=ints(starts), pos0=-1, interleaved=interleaved, magnitude=mag, transpose=transpose)
        pos = (starts[:, None] - 1 + np.arange(M))[..., None]
        ref = O.kv_rope(f64(x), np.broadcast_to(pos, (B, M, H)), f64(freq), interleaved, mag, transpose)
        near(y, ref, rope_bound(f64(x), rot // 2, interleaved, mag, ref, dtype), f"rope transpose={transpose}")
        assert torch.equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rope_views_positions_and_in_place(dtype):
    B, M, H, d, rot = 2, 19, 4, 64, 48
    freq, _ = kv.rope_frequencies(rot)
    fused = normal((B, M, 3 * H, d), 2, dtype)
    heads_first = normal((B, H, M, d), 3, dtype).transpose(1, 2)
    one_row = normal((1, M, 1, d), 4, dtype).expand(B, M, H, d)
    per_token = ints(np.random.default_rng(0).integers(-70, 300000, (B, M)))
    for x in (fused[:, :, H:2 * H], heads_first, one_row):
        pos = np.broadcast_to(per_token.cpu().numpy()[..., None] + 3, (B, M, H))
        ref = O.kv_rope(f64(x), pos, f64(freq))
        tol = rope_bound(f64(x), rot // 2, False, 1.0, ref, dtype)
        near(kv.rope(x, freq, pos=per_token, pos0=3), ref, tol, "positions of tokens")
        out = torch.zeros((B, H, M, d), dtype=dtype, device=DEV).transpose(1, 2)
        kv.rope(x, freq, pos=per_token, pos0=3, out=out)
        near(out, ref, tol, "into a transposed view")
    before = fused.clone()
    view = fused[:, :, H:2 * H]
    kv.rope(view, freq, pos0=7, out=view)
    ref = O.kv_rope(f64(before[:, :, H:2 * H]), np.broadcast_to(7 + np.arange(M)[:, None], (B, M, H)), f64(freq))
    near(view, ref, rope_bound(f64(before[:, :, H:2 * H]), rot // 2, False, 1.0, ref, dtype), "in place")
    assert torch.equal(fused[:, :, :H], before[:, :, :H]) and torch.equal(fused[:, :, 2 * H:], before[:, :, 2 * H:])
    with pytest.raises(lla.LLAError):  # rows that would share their place
        kv.rope(view, freq, out=torch.zeros((1, M, H, d), dtype=dtype, device=DEV).expand(B, M, H, d))
    with pytest.raises(lla.LLAError):  # rows that do not start on 16 bytes
        kv.rope(normal((1, 2, 2, 72), 0, dtype)[..., 1:65], freq)


def test_rope_gradient():
    """The transposed call is the formula's gradient and the limit of differences:
    of sum(g * rope(x)) in each direction e, which is linear in x."""
    freq, mag = kv.rope_frequencies(64, scaling="yarn", factor=2.0, original=128)
    x, g, e = (normal((2, 33, 3, 96), s, F32) for s in (5, 6, 7))
    args = dict(pos=ints([3, 900]), interleaved=True, magnitude=mag)
    grad = kv.rope(g, freq, transpose=True, **args)
    pos = np.broadcast_to((np.array([3, 900])[:, None] + np.arange(33))[..., None], (2, 33, 3))
    ref = O.kv_rope(f64(g), pos, f64(freq), True, mag, transpose=True)
    near(grad, ref, rope_bound(f64(g), 32, True, mag, ref, F32), "gradient")
    step = 0.5
    up, down = kv.rope(x + step * e, freq, **args), kv.rope(x - step * e, freq, **args)
    slope = np.sum(f64(g) * (f64(up) - f64(down))) / (2 * step)
    want = np.sum(f64(grad) * f64(e))
    # 2 * 19008 products of unit-size terms, each off by 1e-6 of them at most
    assert abs(slope - want) <= 1e-6 * np.sum(np.abs(f64(g))) * 6, (slope, want)


def test_rope_past_32_bit_offsets():
    """A row far behind 2^32 bytes of a buffer."""
    d, rows = 256, (1 << 23) + 5
    x = torch.zeros((1, rows, 2, d), dtype=BF, device=DEV)
    x[0, -3:] = normal((3, 2, d), 8, BF)
    freq, _ = kv.rope_frequencies(128)
    tail = x[:, -3:]
    ref = O.kv_rope(f64(tail), np.broadcast_to((rows - 3 + np.arange(3))[:, None], (1, 3, 2)), f64(freq))
    y = kv.rope(x, freq)
    near(y[:, -3:], ref, rope_bound(f64(tail), 64, False, 1.0, ref, BF), "far rows")
    assert not y[:, :1000].any()


# ---------------------------------------------------------------------------
# a program's cache
# ---------------------------------------------------------------------------

class Cache:
    """Pools full of NaN, a scattered table, and the sequences' tokens in 64 bits."""

    def __init__(self, dtype, lengths, Hkv, d, seed=0, spare=3, max_pages=None, n_pages=None):
        rng = np.random.default_rng(seed)
        per = [-(-n // 64) for n in lengths]
        used = sum(per) + spare
        P = n_pages or used
        self.max_pages = max_pages or max(1, *per)
        order = rng.permutation(P)[:used] if P < 1 << 20 else np.array([P - 1 - i for i in range(used)])
        table = np.full((len(lengths), self.max_pages), 1 << 30)  # never to be followed
        at = 0
        for i, n in enumerate(per):
            table[i, :n] = order[at:at + n]
            at += n
        self.lengths, self.host_table, self.d, self.Hkv, self.dtype = lengths, table, d, Hkv, dtype
        self.k, self.v = kv.alloc_pages(P, Hkv, d, dtype)
        if P < 1 << 16:
            self.k.fill_(float("nan"))
            self.v.fill_(float("nan"))
        self.table, self.length = ints(table), ints(lengths)
        for i, n in enumerate(lengths):  # tokens alone: the rest of a page stays NaN
            if not n:
                continue
            t = torch.arange(n, device=DEV)
            page = self.table[i].long()[t // 64]
            self.k[page, :, t % 64] = normal((n, Hkv, d), seed + 10 * i + 1, dtype)
            self.v[page, :, :, t % 64] = normal((n, Hkv, d), seed + 10 * i + 2, dtype)


def check_decode(c, H, *, rows=None, sink=0, window=0, n_ctx=None, out_dtype=F32, scale=None, q=None, seed=99):
    """Every (entry, head, feature) against the oracle's formula."""
    B = len(c.lengths) if rows is None else len(rows)
    d, group = c.d, H // c.Hkv
    q = normal((B, H, d), seed, c.dtype) if q is None else q
    lse = torch.empty((B, H), device=DEV)
    out = kv.decode_attn(q, c.k, c.v, c.table, c.length, rows=None if rows is None else ints(rows), sink=sink,
                         window=window, n_ctx=n_ctx or max(1, *c.lengths), out_dtype=out_dtype, scale=scale, lse=lse)
    torch.cuda.synchronize()
    assert out.dtype == out_dtype
    scale = d ** -0.5 if scale is None else scale
    got, got_lse, q64 = f64(out), f64(lse), f64(q)
    worst = 0.0
    for b in range(B):
        row = b if rows is None else rows[b]
        at = O.kv_seen(c.lengths[row], sink, window) if row >= 0 else []
        if not at:
            assert not got[b].any() and np.all(got_lse[b] == -np.inf), b
            continue
        at = torch.as_tensor(at, device=DEV)
        page = c.table[row].long()[at // 64]
        k, v = f64(c.k[page, :, at % 64]), f64(c.v[page, :, :, at % 64])  # [n, Hkv, d]
        n = len(at)
        for h in range(H):
            kh, vh = k[:, h // group], v[:, h // group]
            s = kh @ q64[b, h] * scale
            p = np.exp(s - s.max())
            ref, ref_lse = p @ vh / p.sum(), s.max() + np.log(p.sum())
            ds = (d + 2) * EPS * np.max(np.abs(kh) @ np.abs(q64[b, h])) * scale + EPS * np.max(np.abs(s))
            rel = 2 * ds + 2.0 ** -16 + (n / 16 + 64) * EPS
            tol = rel * (p / p.sum() @ np.abs(vh)) + half_step(out_dtype) * np.abs(ref) + 1e-30
            assert np.all(np.isfinite(got[b, h])), (b, h)
            worst = max(worst, float(np.max(np.abs(got[b, h] - ref) / tol)))
            # the sum's relative error, and the roundings of its logarithm
            assert abs(got_lse[b, h] - ref_lse) <= rel + 8 * EPS * (1 + abs(ref_lse)), (b, h, got_lse[b, h], ref_lse)
    log(f"  decode: {worst:.3f} of the bound")
    assert worst <= 1.0
    return out


# ---------------------------------------------------------------------------
# decode attention
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_decode_widths(dtype, d):
    check_decode(Cache(dtype, [1, 0, 63, 64, 65, 200], 2, d), 6)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (16, 16), (8, 1), (15, 5), (16, 1), (17, 1), (40, 2), (48, 3), (64, 1)])
def test_decode_groups(dtype, H, Hkv):
    check_decode(Cache(dtype, [130, 7, 449], Hkv, 64, seed=3), H, out_dtype=dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lengths", [[1], [2], [511], [513], [1025, 1], [4097], [5000, 64, 0, 2049], [9999],
                                     [40000], [100, 30000, 1]])
def test_decode_lengths(dtype, lengths):
    """From one token to lengths that are split over workgroups, alone and uneven."""
    check_decode(Cache(dtype, lengths, 2, 128, seed=4), 4)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("sink,window", [(0, 1), (4, 60), (0, 64), (64, 64), (1, 1000), (70, 130), (4, 1 << 30),
                                         ((1 << 31) - 1, 5), (0, 4999), (128, 4000)])
def test_decode_window(dtype, sink, window):
    """A budget of first and last tokens: pages between are not read (they hold NaN
    pages' numbers that may not be followed)."""
    lengths = [5000, 0, 1, 64, 65, 1023, 129]
    c = Cache(dtype, lengths, 1, 64, seed=5)
    for i, n in enumerate(lengths):  # positions outside the budget become NaN, whole pages unknown
        gone = sorted(set(range(n)) - set(O.kv_seen(n, sink, window)))
        kept = {t // 64 for t in O.kv_seen(n, sink, window)}
        for t in gone:
            if t // 64 in kept:
                c.k[c.host_table[i, t // 64], :, t % 64] = float("inf")
                c.v[c.host_table[i, t // 64], :, :, t % 64] = float("nan")
        for p in {t // 64 for t in gone} - kept:
            c.table[i, p] = -5
    check_decode(c, 2, sink=sink, window=window)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_decode_rows_and_bounds(dtype):
    """Rows in any order and more than once, padding, a bound above the lengths; a
    length, row or page out of range gives NaN to its entry alone."""
    c = Cache(dtype, [300, 0, 77, 1000], 2, 64, seed=6, max_pages=40)
    check_decode(c, 4, rows=[3, 0, 3, -1, 2, 1], n_ctx=2500)
    q = normal((4, 4, 64), 1, dtype)
    good = kv.decode_attn(q, c.k, c.v, c.table, c.length, n_ctx=1000)
    bad = kv.decode_attn(q, c.k, c.v, c.table, c.length, n_ctx=999)
    assert torch.isnan(bad[3]).all() and torch.equal(bad[:3], good[:3])
    bad = kv.decode_attn(q, c.k, c.v, c.table, c.length, rows=ints([0, 4, -2, 2]), n_ctx=1000)
    assert torch.isnan(bad[1:3]).all() and torch.isfinite(bad[0]).all() and torch.isfinite(bad[3]).all()
    for page in (-1, c.k.shape[0], 1 << 30):
        t = c.table.clone()
        t[0, 4] = page
        lse = torch.zeros((4, 4), device=DEV)
        bad = kv.decode_attn(q, c.k, c.v, t, c.length, n_ctx=1000, lse=lse)
        assert torch.isnan(bad[0]).all() and torch.equal(bad[1:], good[1:]) and torch.isnan(lse[0]).all()
    negative = c.length.clone()
    negative[2] = -3
    bad = kv.decode_attn(q, c.k, c.v, c.table, negative, n_ctx=1000)
    assert torch.isnan(bad[2]).all() and torch.equal(bad[3], good[3])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_decode_values_of_any_size(dtype):
    """Scores far apart and far from zero, -inf among them, and infinite values where attended."""
    c = Cache(dtype, [200, 3000], 1, 64, seed=7)
    q = normal((2, 2, 64), 8, dtype) * 30
    check_decode(c, 2, q=q, scale=1.0)
    check_decode(c, 2, q=torch.zeros_like(q))
    # a key of -inf weighs nothing, in a page of its own kind too
    q = q.abs() + 0.5
    full = kv.decode_attn(q, c.k, c.v, c.table, c.length, n_ctx=3000)
    lengths = ints([130, 3000])
    k = c.k.clone()
    pages = c.table[0].long()
    k[pages[:2]] = -float("inf")
    some = kv.decode_attn(q, k, c.v, c.table, lengths, n_ctx=3000)
    assert torch.isfinite(some).all() and torch.equal(some[1], full[1])
    k2, v2 = f64(c.k[pages[2:3]]), f64(c.v[pages[2:3]])  # two tokens are left
    ref = O.kv_decode_attn(f64(q)[:1], k2, v2, [[0]], [2])[0]
    ds = 66 * EPS * np.max(np.abs(k2[0, 0, :2]) @ np.abs(f64(q)[0].T)) / 8
    assert np.max(np.abs(f64(some[:1]) - ref)) <= (2 * ds + 2.0 ** -16 + 64 * EPS) * np.max(np.abs(v2[0, 0, :, :2]))
    v = c.v.clone()
    v[pages[1], :, 3, 10] = float("nan")
    hit = kv.decode_attn(q, c.k, v, c.table, c.length, n_ctx=3000)
    assert torch.isnan(hit[0, :, 3]).all() and torch.isfinite(hit[0, :, :3]).all() and torch.equal(hit[1], full[1])


def test_decode_past_32_bit_offsets():
    """Pages at the end of a pool of more than 2^32 elements."""
    c = Cache(BF, [150, 1000], 16, 256, seed=9, n_pages=(1 << 14) + 100)
    assert c.k.numel() > 1 << 32 and int(c.table[c.table < c.k.shape[0]].max()) > 1 << 13
    check_decode(c, 16)


def test_decode_is_repeatable_and_workspace_is_scratch():
    """The same bits every time, whatever the workspace holds, and on another stream."""
    c = Cache(BF, [30000, 500], 2, 128, seed=10)
    q = normal((2, 8, 128), 11, BF)
    need = kv.decode_workspace_bytes(BF, 2, 8, 2, 128, 30000)
    first = kv.decode_attn(q, c.k, c.v, c.table, c.length, n_ctx=30000)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for fill in (0, 255):
        ws = torch.full((max(need, 16),), fill, dtype=torch.uint8, device=DEV)
        assert torch.equal(kv.decode_attn(q, c.k, c.v, c.table, c.length, n_ctx=30000, workspace=ws), first)
        with torch.cuda.stream(side):
            other = kv.decode_attn(q, c.k, c.v, c.table, c.length, n_ctx=30000)
        side.synchronize()
        assert torch.equal(other, first)


def test_decode_join_of_two_halves():
    """Two calls over a sequence's halves, joined by their lse, are the whole."""
    c = Cache(F32, [2048], 1, 64, seed=12)
    q = normal((1, 4, 64), 13, F32)
    whole = f64(kv.decode_attn(q, c.k, c.v, c.table, c.length, n_ctx=2048))
    parts, weights = [], []
    for lo in (0, 16):
        lse = torch.empty((1, 4), device=DEV)
        t = c.table[:, lo:lo + 16].contiguous()
        parts.append(f64(kv.decode_attn(q, c.k, c.v, t, ints([1024]), n_ctx=1024, lse=lse)))
        weights.append(np.exp(f64(lse)))
    joined = (parts[0] * weights[0][..., None] + parts[1] * weights[1][..., None]) / (weights[0] + weights[1])[..., None]
    assert np.max(np.abs(joined - whole)) < 1e-5  # |v| < 5, fp32 sums of 2048


# ---------------------------------------------------------------------------
# write
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,M,Hkv,d,rot,inter", [(1, 1, 1, 32, 0, False), (5, 1, 16, 128, 128, False),
                                                 (3, 2, 2, 96, 64, True), (2, 64, 3, 64, 64, False),
                                                 (2, 193, 2, 160, 24, False), (1, 1000, 1, 256, 256, True),
                                                 (4, 65, 5, 224, 8, True), (33, 7, 4, 128, 128, True)])
def test_write(dtype, B, M, Hkv, d, rot, inter):
    """Into the middle of pages, uneven counts, rows in another order; every other
    slot of the pools keeps its bits."""
    rng = np.random.default_rng(B * M)
    starts = rng.integers(0, 200, B)
    starts[0] = 61
    counts = rng.integers(0, M + 1, B)
    counts[0] = M
    rows = rng.permutation(B + 1)[:B]
    lengths = [400 + M] * (B + 1)
    c = Cache(dtype, lengths, Hkv, d, seed=B + M)
    k0, v0 = c.k.clone(), c.v.clone()
    fused = normal((B, M, 3, Hkv, d), 20, dtype)
    k, v = fused[:, :, 1], fused[:, :, 2]
    freq, mag = kv.rope_frequencies(rot, scaling="yarn", factor=2.0, original=100) if rot else (None, 1.0)
    kv.write(k, v, c.k, c.v, c.table, ints(starts), rows=ints(rows), n_new=ints(counts), freq=freq, interleaved=inter,
             magnitude=mag)
    for b in range(B):
        t = torch.arange(starts[b], starts[b] + counts[b], device=DEV)
        if not len(t):
            continue
        page = c.table[int(rows[b])].long()[t // 64]
        got = c.k[page, :, t % 64]
        x = f64(k[b, :counts[b]])
        if rot:
            ref = O.kv_rope(x, np.broadcast_to(t.cpu().numpy()[:, None], x.shape[:2]), f64(freq), inter, mag)
            near(got, ref, rope_bound(x, rot // 2, inter, mag, ref, dtype), f"entry {b}")
        else:
            assert torch.equal(got, k[b, :counts[b]])
        assert torch.equal(c.v[page, :, :, t % 64], v[b, :counts[b]])
        c.k[page, :, t % 64], c.v[page, :, :, t % 64] = k0[page, :, t % 64], v0[page, :, :, t % 64]
    for now, before in ((c.k, k0), (c.v, v0)):
        bits = torch.int16 if dtype == BF else torch.int32
        assert torch.equal(now.view(bits), before.view(bits))


def test_write_passes_over_what_is_out_of_range():
    c = Cache(BF, [128] * 3, 2, 64, seed=21, max_pages=2)
    c.k.zero_()
    c.v.zero_()
    c.table[2, 0] = c.k.shape[0]
    k = torch.ones((5, 40, 2, 64), dtype=BF, device=DEV)
    # refused by reserve; a row too far; past the table's end; a page out of range, then the next page; negative row
    kv.write(k, k, c.k, c.v, c.table, ints([-1, 0, 100, 50, 0]), rows=ints([0, 3, 1, 2, -1]))
    want = torch.zeros_like(c.k)
    at = lambda r, t: (c.table[r].long()[t // 64], slice(None), t % 64)  # noqa: E731
    want[at(1, torch.arange(100, 128, device=DEV))] = 1
    want[at(2, torch.arange(64, 90, device=DEV))] = 1
    assert torch.equal(c.k, want) and torch.equal(c.v, want.transpose(2, 3))
    kv.write(k[:1], k[:1], c.k, c.v, c.table, ints([0]), n_new=ints([-7]))  # no tokens
    kv.write(k[:1, :5], k[:1, :5], c.k, c.v, c.table, ints([3]), n_new=ints([1 << 30]))  # at most M
    want[at(0, torch.arange(3, 8, device=DEV))] = 1
    assert torch.equal(c.k, want)


# ---------------------------------------------------------------------------
# tables, copies, gathers
# ---------------------------------------------------------------------------

def same_tables(pages, t, length_only=False):
    assert pages.length.tolist() == t.length
    assert pages.refs.tolist() == t.refs
    n = int(pages.free[0])
    assert n == len(t.free) and pages.free[1:1 + n].tolist() == t.free
    for r, n in enumerate(t.length):
        used = -(-n // 64)
        assert pages.table[r, :used].tolist() == t.table[r][:used], r


@pytest.mark.parametrize("n_seqs,max_pages,n_pages,most,seed", [(6, 5, 14, 130, 0), (40, 30, 400, 700, 1),
                                                                (300, 9, 1200, 200, 2), (1500, 4, 2500, 90, 3)])
def test_tables_against_rows_one_after_another(n_seqs, max_pages, n_pages, most, seed):
    rng = np.random.default_rng(seed)
    pages, t = kv.new_page_table(n_seqs, max_pages, n_pages), O.KvTables(n_seqs, max_pages, n_pages)
    seen = {}
    for step in range(60):
        kind = rng.choice(["reserve", "reserve", "fork", "free"])
        n = int(rng.integers(1, min(n_seqs, 1024) + 1)) if step % 3 else int(rng.integers(1, 4))
        rows = rng.permutation(n_seqs)[:n]
        if rng.random() < 0.1:
            rows[-1] = rng.choice([-1, n_seqs, rows[0]])
        result = torch.full((4,), -9, dtype=torch.int32, device=DEV)
        before = (pages.table.clone(), [x.clone() for x in pages[1:]])
        if kind == "reserve":
            add = rng.choice([0, 1, 1, 63, int(rng.integers(0, most))], n)
            if rng.random() < 0.05:
                add[0] = -1
            start, pairs = torch.full((n,), -9, dtype=torch.int32, device=DEV), torch.zeros((n, 2), dtype=torch.int32, device=DEV)
            kv.reserve(pages, ints(rows), ints(add), start, pairs, result)
            free = len(t.free)
            status, want_start, want_pairs = t.reserve(rows.tolist(), add.tolist())
            assert start.tolist() == want_start and pairs[:len(want_pairs)].tolist() == [list(p) for p in want_pairs]
            numbers = [len(want_pairs), free - len(t.free)]
        elif kind == "fork":
            empty = [r for r in range(n_seqs) if t.length[r] == 0]
            if empty and rng.random() < 0.8:
                rows = np.array(empty[:n])
            others = [r for r in range(n_seqs) if r not in set(rows.tolist())] or [0]
            src = rng.choice(others, len(rows))
            kv.fork(pages, ints(src), ints(rows), result)
            status, numbers = t.fork(src.tolist(), rows.tolist()), [0, 0]
        else:
            kv.free(pages, ints(rows), result)
            free = len(t.free)
            status = t.free_rows(rows.tolist())
            numbers = [0, len(t.free) - free]
        assert result.tolist() == [status, *numbers, len(t.free)], (step, kind)
        seen[kind, status] = seen.get((kind, status), 0) + 1
        if status:
            assert torch.equal(pages.table, before[0]) and all(torch.equal(a, b) for a, b in zip(pages[1:], before[1]))
        same_tables(pages, t)
    log(f"  {seen}")
    assert {("reserve", 0), ("free", 0), ("fork", 0)} <= set(seen)


def test_free_of_pages_shared_by_the_rows_freed():
    pages, t = kv.new_page_table(20, 40, 200), O.KvTables(20, 40, 200)
    r = ints([0] * 4)
    for rows, add in (([0], [2000]), ([1], [100])):
        start, pairs = ints([0]), ints([[0, 0]])
        kv.reserve(pages, ints(rows), ints(add), start, pairs, r)
        t.reserve(rows, add)
    dst = list(range(2, 18))
    kv.fork(pages, ints([0, 1] * 8), ints(dst), r)
    t.fork([0, 1] * 8, dst)
    n = len(dst)
    kv.reserve(pages, ints(dst), ints([7] * n), torch.zeros(n, dtype=torch.int32, device=DEV), ints([[0, 0]] * n), r)
    t.reserve(dst, [7] * n)
    for rows in ([5, 0, 9], [17, 3, 2, 4], [1, 16, 15, 14, 13, 12, 11, 10, 8, 7, 6]):
        kv.free(pages, ints(rows), r)
        t.free_rows(rows)
        same_tables(pages, t)
    assert int(pages.free[0]) == 200 and not pages.refs.any()


@pytest.mark.parametrize("shape,other", [((9, 2, 64, 32), (9, 2, 32, 64)), ((3, 9, 1, 64, 96), (3, 9, 5, 64, 8)),
                                         ((2, 9, 4, 64, 256), None)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_copy_pages(shape, other, dtype):
    a = normal(shape, 30, dtype)
    b = None if other is None else normal(other, 31, dtype)
    pairs = ints([[0, 3], [8, 1], [0, 7], [9, 2], [2, -1], [5, 6]])
    for count in (None, 4, 0, 99):
        x, y = a.clone(), None if b is None else b.clone()
        result = None if count is None else ints([0, count, 0, 0])
        kv.copy_pages(x, y, pairs, result)
        lead = len(shape) - 4
        for got, was in ((x, a), (y, b)):
            if got is None:
                continue
            want = was.clone()
            for s, z in pairs[:6 if count is None else min(count, 6)].tolist():
                if 0 <= s < 9 and 0 <= z < 9:
                    want.select(lead, z).copy_(was.select(lead, s))
            assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hkv,d,layers", [(1, 32, 1), (3, 128, 1), (2, 96, 3), (1, 256, 2)])
def test_gather(dtype, Hkv, d, layers):
    rng = np.random.default_rng(d)
    n_seqs, max_pages, P = 6, 6, 40
    k = normal((layers, P, Hkv, 64, d), 40, dtype)
    v = normal((layers, P, Hkv, d, 64), 41, dtype)
    order = rng.permutation(P)[:n_seqs * max_pages].reshape(n_seqs, max_pages)
    table = ints(order)
    most = 300
    src, dst, count = [4, 0, 4], [1, 5, 2], [300, 129, 0]
    keep = np.stack([np.sort(rng.permutation(384)[:most]), rng.permutation(384)[:most], np.arange(most)])
    keep[0, 17], keep[0, 18] = -1, 384  # no such position
    k0, v0 = k.clone(), v.clone()
    kk, vv = (k, v) if layers > 1 else (k[0], v[0])
    kv.gather(kk, vv, table, ints(src), ints(dst), ints(keep), ints(count))
    for j in range(3):
        for i in range(count[j]):
            t = int(keep[j, i])
            z = (slice(None), int(order[dst[j], i // 64]))
            if not 0 <= t < 384:
                assert torch.isnan(k[z][:, :, i % 64]).all() and torch.isnan(v[z][..., i % 64]).all()
                k0[z][:, :, i % 64], v0[z][..., i % 64] = 0, 0
                k[z][:, :, i % 64], v[z][..., i % 64] = 0, 0
            else:
                s = (slice(None), int(order[src[j], t // 64]))
                k0[z][:, :, i % 64], v0[z][..., i % 64] = k0[s][:, :, t % 64], v0[s][..., t % 64]
    assert torch.equal(k, k0) and torch.equal(v, v0)
    # rows and pages out of range: unreadable sources give NaN, unwritable destinations are left
    table[3, 0] = P
    kv.gather(kk, vv, table, ints([6, 0, 3, 0]), ints([1, -1, 5, 3]), ints([[0, 5]] * 4))
    z1, z5 = int(order[1, 0]), int(order[5, 0])
    for z in (z1, z5):
        assert torch.isnan(k[:, z, :, :2]).all() and torch.isnan(v[:, z, :, :, :2]).all()
        k[:, z, :, :2], v[:, z, :, :, :2] = k0[:, z, :, :2], v0[:, z, :, :, :2]
    assert torch.equal(k, k0) and torch.equal(v, v0)


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

class Server:
    """A small serving program over two layers, and its double in 64 bits."""

    def __init__(self, dtype, n_seqs=8, max_pages=8, n_pages=30, H=6, Hkv=2, d=64, layers=2):
        self.pages, self.host = kv.new_page_table(n_seqs, max_pages, n_pages), O.KvTables(n_seqs, max_pages, n_pages)
        self.k, self.v = kv.alloc_pages(n_pages, Hkv, d, dtype, layers=layers)
        self.k.fill_(float("nan"))
        self.v.fill_(float("nan"))
        self.freq, self.mag = kv.rope_frequencies(32, scaling="yarn", factor=4.0, original=64)
        self.tokens = {r: [[] for _ in range(layers)] for r in range(n_seqs)}  # (stored key, value) in 64 bits
        self.H, self.Hkv, self.d, self.layers, self.dtype = H, Hkv, d, layers, dtype

    def step(self, rows, add, M, x):
        """x: per layer the fused projection [B, M, H + 2 Hkv, d].  Device part only."""
        n = len(rows)
        self.rows, self.add = ints(rows), ints(add)
        self.start, self.pairs, self.result = ints([0] * n), ints([[0, 0]] * n), ints([0] * 4)
        return self.enqueue(M, x)

    def enqueue(self, M, x):
        H, Hkv, outs = self.H, self.Hkv, []
        kv.reserve(self.pages, self.rows, self.add, self.start, self.pairs, self.result)
        kv.copy_pages(self.k, self.v, self.pairs, self.result)
        for l in range(self.layers):
            q, k, v = x[l][:, :, :H], x[l][:, :, H:H + Hkv], x[l][:, :, H + Hkv:]
            kv.write(k, v, self.k[l], self.v[l], self.pages.table, self.start, rows=self.rows, n_new=self.add,
                     freq=self.freq, magnitude=self.mag)
            q = kv.rope(q, self.freq, pos=self.start, magnitude=self.mag)
            # the last new token's query attends the whole sequence
            last = torch.stack([q[i, max(0, a - 1)] for i, a in enumerate(self.add_host)]) if M > 1 else q[:, 0]
            outs.append(kv.decode_attn(last.contiguous(), self.k[l], self.v[l], self.pages.table, self.pages.length,
                                       rows=self.rows, n_ctx=64 * self.pages.table.shape[1]))
        return outs

    def check(self, rows, add, x, outs):
        status, start, _ = self.host.reserve(rows, add)
        assert self.result.tolist()[0] == status and self.start.tolist() == start
        same_tables(self.pages, self.host)
        freq = f64(self.freq)
        for l in range(self.layers):
            for i, r in enumerate(rows):
                for m in range(add[i] if status == 0 else 0):
                    key, value = f64(x[l][i, m, self.H:self.H + self.Hkv]), f64(x[l][i, m, self.H + self.Hkv:])
                    key = O.kv_rope(key, np.full(self.Hkv, start[i] + m), freq, magnitude=self.mag)
                    self.tokens[r][l].append((key, value))
            for i, r in enumerate(rows):
                toks = self.tokens[r][l]
                if status or not toks:
                    continue
                q = f64(x[l][i, max(0, add[i] - 1), :self.H])
                pos = start[i] + max(0, add[i] - 1)
                # a query of a row that got no token is turned to the next position
                q = O.kv_rope(q, np.full(self.H, pos), freq, magnitude=self.mag)
                k, v = np.stack([t[0] for t in toks]), np.stack([t[1] for t in toks])
                for h in range(self.H):
                    s = k[:, h // 3] @ q[h] / self.d ** 0.5
                    p = np.exp(s - s.max())
                    ref = p @ v[:, h // 3] / p.sum()
                    got = f64(outs[l][i, h])
                    # stored keys and queries are rounded once: scores off by 2 * 2^-8 (2^-24) of sum |q k|
                    u = half_step(self.dtype)
                    ds = 2 * (2 * u + 70 * EPS) * np.max(np.abs(k[:, h // 3]) @ np.abs(q[h])) / self.d ** 0.5
                    tol = (2 * ds + 2.0 ** -16 + 1e-5) * (p / p.sum() @ np.abs(v[:, h // 3]))
                    assert np.all(np.abs(got - ref) <= tol), (l, r, h, float(np.max(np.abs(got - ref) / tol)))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_serving_run(dtype):
    """Prompts, decode steps, a fork with copies on write, an eviction, a refused
    step, frees: outputs and tables as the double's at every step."""
    s = Server(dtype)
    rng = np.random.default_rng(50)
    seed = [100]

    def go(rows, add, M):
        seed[0] += 1
        x = [normal((len(rows), M, s.H + 2 * s.Hkv, s.d), seed[0] * 7 + l, dtype) for l in range(s.layers)]
        s.add_host = add
        outs = s.step(rows, add, M, x)
        s.check(rows, add, x, outs)
        return s.result.tolist()

    result = ints([0] * 4)
    go([0, 1, 2], [100, 1, 64], 100)
    for _ in range(3):
        go([2, 0, 1], [1, 1, 1], 1)
    kv.fork(s.pages, ints([0, 0, 2]), ints([3, 4, 5]), result)
    assert s.host.fork([0, 0, 2], [3, 4, 5]) == 0
    for a, b in ((0, 3), (0, 4), (2, 5)):
        s.tokens[b] = [list(t) for t in s.tokens[a]]
    assert go([0, 3, 4, 5, 2], [1] * 5, 1)[1] == 3       # copies: 0 and 3 leave the page to 4; 5 leaves it to 2
    go([0, 3, 4, 5, 2], [1, 0, 30, 2, 0], 30)
    # keep the first 2, the last 20 and some tokens of sequence 0, in the same row
    n = s.host.length[0]
    keep = [0, 1] + sorted(rng.permutation(np.arange(2, n - 20))[:30].tolist()) + list(range(n - 20, n))
    spare = ints([6])
    kv.fork(s.pages, ints([0]), spare, result)
    kv.free(s.pages, ints([0]), result)
    kv.reserve(s.pages, ints([0]), ints([len(keep)]), ints([0]), ints([[0, 0]]), result)
    kv.gather(s.k, s.v, s.pages.table, spare, ints([0]), ints([keep]))
    kv.free(s.pages, spare, result)
    s.host.fork([0], [6])
    s.host.free_rows([0])
    s.host.reserve([0], [len(keep)])
    s.host.free_rows([6])
    same_tables(s.pages, s.host)
    s.tokens[0] = [[t[i] for i in keep] for t in s.tokens[0]]
    # (from here its new tokens' positions go on from the kept count)
    go([0, 1], [1, 1], 1)
    bits = lambda: [x.view(torch.int16 if dtype == BF else torch.int32).clone() for x in (s.k, s.v)]  # noqa: E731
    before = bits()
    assert go([0, 1, 7], [1, 1, 10 ** 6], 1)[0] == kv.PAGES_BAD
    assert go([7, 1, 6], [512, 450, 512], 1)[0] == kv.PAGES_FULL
    assert all(torch.equal(a, b) for a, b in zip(before, bits()))  # a refused step writes nothing
    rows = list(range(8))
    kv.free(s.pages, ints(rows), result)
    s.host.free_rows(rows)
    same_tables(s.pages, s.host)
    assert int(s.pages.free[0]) == 30


def test_captured_decode_step():
    """One captured step (room, copies, write, turn, attention) replayed: every
    replay as the eager call, the program's own work between, two graphs sharing
    a workspace."""
    dtype, H, Hkv, d, n_ctx = BF, 8, 2, 128, 64 * 80

    def program():
        pages = kv.new_page_table(3, 80, 200)
        k, v = kv.alloc_pages(200, Hkv, d, dtype)
        freq, _ = kv.rope_frequencies(128)
        rows, result = ints([0, 1, 2]), ints([0] * 4)
        start, pairs = ints([0] * 3), ints([[0, 0]] * 3)
        kv.reserve(pages, rows, ints([4900, 63, 129]), start, pairs, result)
        x = normal((3, 4900, Hkv, d), 60, dtype)
        kv.write(x, x, k, v, pages.table, start, n_new=ints([4900, 63, 129]), freq=freq)
        one = ints([1, 1, 1])
        ws = torch.empty(max(16, kv.decode_workspace_bytes(dtype, 3, H, Hkv, d, n_ctx),
                             kv.decode_workspace_bytes(dtype, 3, H, Hkv, d, n_ctx, 4, 4000)), dtype=torch.uint8, device=DEV)
        qkv = torch.empty((3, 1, H + 2 * Hkv, d), dtype=dtype, device=DEV)
        outs = [torch.empty((3, H, d), device=DEV) for _ in range(2)]
        turned = torch.empty((3, 1, H, d), dtype=dtype, device=DEV)

        def step():
            kv.reserve(pages, rows, one, start, pairs, result)
            kv.copy_pages(k, v, pairs, result)
            kv.write(qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:], k, v, pages.table, start, freq=freq)
            kv.rope(qkv[:, :, :H], freq, pos=start, out=turned)
            kv.decode_attn(turned[:, 0], k, v, pages.table, pages.length, n_ctx=n_ctx, out=outs[0], workspace=ws)

        def windowed():
            kv.decode_attn(turned[:, 0], k, v, pages.table, pages.length, n_ctx=n_ctx, sink=4, window=4000,
                           out=outs[1], workspace=ws)
        return step, windowed, qkv, outs, pages

    eager, captured = program(), program()
    graphs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    for fn in captured[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            fn()
        graphs.append(g)
    assert captured[4].length.tolist() == [4900, 63, 129]  # capturing ran nothing
    for i in range(6):
        x = normal((3, 1, H + 2 * Hkv, d), 70 + i, dtype)
        for p in (eager, captured):
            p[2].copy_(x)
        for fn in eager[:2]:
            fn()
        for g in graphs:
            g.replay()
        if i % 2:
            torch.cuda.synchronize()
            kv.decode_attn(x[:, 0, :H].contiguous(), *kv.alloc_pages(4, Hkv, d, dtype), ints([[0]] * 3), ints([0] * 3), n_ctx=64)
        for a, b in zip(eager[3], captured[3]):
            assert torch.equal(a, b) and torch.isfinite(a).all(), i
        assert torch.equal(eager[4].table, captured[4].table) and eager[4].length.tolist() == [4901 + i, 64 + i, 130 + i]


def test_refusals_on_the_device():
    """What only device tensors can be refused for."""
    c = Cache(BF, [64], 2, 64)
    q = normal((1, 4, 64), 1, BF)
    args = (c.k, c.v, c.table, c.length)
    for bad in (lambda: kv.decode_attn(q.float(), *args, n_ctx=64),
                lambda: kv.decode_attn(q[..., :32].contiguous(), *args, n_ctx=64),
                lambda: kv.decode_attn(q.transpose(0, 1), *args, n_ctx=64),
                lambda: kv.decode_attn(q, c.k, c.v, c.table.long(), c.length, n_ctx=64),
                lambda: kv.decode_attn(q, c.k, c.v.transpose(2, 3), c.table, c.length, n_ctx=64),
                lambda: kv.decode_attn(q, *args, n_ctx=64, out=torch.empty((1, 4, 32), device=DEV)),
                lambda: kv.decode_attn(q, *args, n_ctx=64, lse=torch.empty((1, 4), device=DEV, dtype=BF)),
                lambda: kv.decode_attn(q, *args, n_ctx=64, rows=ints([0, 0])),
                lambda: kv.write(q[None], q[None], c.k, c.v, c.table, ints([0])),
                lambda: kv.write(q[:, None, :2].float(), q[:, None, :2], c.k, c.v, c.table, ints([0])),
                lambda: kv.write(normal((2, 1, 2, 64), 0, BF), normal((2, 1, 2, 64), 0, BF), c.k, c.v, c.table, ints([0, 0])),
                lambda: kv.rope(q[None], torch.ones(16, device=DEV)),
                lambda: kv.rope(q[None], torch.ones(40, device=DEV, dtype=torch.float64)),
                lambda: kv.rope(q[None], torch.ones(16, device=DEV, dtype=torch.float64), pos=ints([0, 1])),
                lambda: kv.rope(q[None].transpose(2, 3), torch.ones(2, device=DEV, dtype=torch.float64)),
                lambda: kv.gather(c.k, c.v, c.table, ints([0]), ints([0]), ints([0])),
                lambda: kv.copy_pages(c.k, c.v[:1], ints([[0, 0]]))):
        with pytest.raises((ValueError, TypeError, lla.LLAError)):
            bad()
    for bad in (dict(n_ctx=0), dict(n_ctx=65), dict(n_ctx=64, sink=2), dict(n_ctx=64, window=-1),
                dict(n_ctx=64, scale=0.0)):
        with pytest.raises(lla.LLAError):
            kv.decode_attn(q, *args, **bad)
    with pytest.raises(lla.LLAError):
        kv.decode_attn(normal((1, 3, 64), 0, BF), *args, n_ctx=64)


def test_free_of_more_entries_than_a_thread_holds():
    """More than 16384 (row, page) entries in one call, then shared ones among them."""
    n = 600
    pages, t = kv.new_page_table(n + 1, 40, 25000), O.KvTables(n + 1, 40, 25000)
    r, rows = ints([0] * 4), list(range(1, n + 1))
    start, pairs = torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros((n, 2), dtype=torch.int32, device=DEV)
    add = [64 * 30 + i % 64 for i in range(n)]
    kv.reserve(pages, ints(rows), ints(add), start, pairs, r)
    t.reserve(rows, add)
    same_tables(pages, t)
    kv.free(pages, ints(rows[::-1]), r)
    t.free_rows(rows[::-1])
    same_tables(pages, t)
    kv.reserve(pages, ints([0]), ints([2500]), start[:1], pairs[:1], r)
    t.reserve([0], [2500])
    kv.fork(pages, ints([0] * n), ints(rows), r)
    t.fork([0] * n, rows)
    kv.reserve(pages, ints(rows[:50]), ints([1] * 50), start[:50], pairs[:50], r)
    t.reserve(rows[:50], [1] * 50)
    same_tables(pages, t)
    everything = rows[7:] + [0] + rows[:7]
    kv.free(pages, ints(everything), r)
    t.free_rows(everything)
    same_tables(pages, t)
    assert int(pages.free[0]) == 25000


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,M,H,d,rot", [(1, 5, 300, 16, 8), (1, 33, 1, 512, 8), (70, 1, 3, 32, 16), (2, 100, 7, 40, 32),
                                         (1, 17, 2, 8, 8), (3, 40, 33, 256, 256)])
def test_rope_many_heads_or_tokens(dtype, B, M, H, d, rot):
    """Stretches that end inside a workgroup, in both orders of y's rows, more heads
    or parts than a workgroup has threads for, and positions of one row a token."""
    freq, _ = kv.rope_frequencies(rot)
    x = normal((B, M, H, d), 14, dtype)
    pos = np.broadcast_to((np.arange(M) + 9)[None, :, None], (B, M, H))
    ref = O.kv_rope(f64(x), pos, f64(freq))
    tol = rope_bound(f64(x), rot // 2, False, 1.0, ref, dtype)
    near(kv.rope(x, freq, pos0=9), ref, tol, "heads inside")
    out = torch.full((B, H, M, d), float("nan"), dtype=dtype, device=DEV).transpose(1, 2)
    near(kv.rope(x.transpose(1, 2).contiguous().transpose(1, 2), freq, pos0=9, out=out), ref, tol, "tokens inside")


def test_latent_pages_are_copied_too():
    """A sequence of the latent cache continues another: its pages copied, both
    attend the same."""
    H, P, d, r_k, r_v, n = 2, 5, 128, 18, 30, 180
    c_k, c_v = (normal((2, H, P, r, 64), 80 + r, BF) for r in (r_k, r_v))
    u_k, u_v = normal((H, d, r_k), 82, BF), normal((H, d, r_v), 83, BF)
    q = normal((1, H, d), 84, BF).expand(2, H, d).contiguous()
    before = c_k[1, :, 3:].clone()
    pairs = [[h * P + p, (H + h) * P + p] for h in range(H) for p in range(3)]  # page (b, h, p) is b H P + h P + p
    kv.copy_pages(c_k.view(2 * H * P, r_k, 64), c_v.view(2 * H * P, r_v, 64), ints(pairs))
    out = lla.decode_attn(q, c_k, c_v, u_k, u_v, n_ctx=n)
    assert torch.equal(out[0], out[1]) and torch.isfinite(out).all()
    assert torch.equal(c_k[1, :, :3], c_k[0, :, :3]) and torch.equal(c_k[1, :, 3:], before)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,Hkv,H,d,n", [(3, 50, 50, 32, 900), (24, 8, 24, 64, 1088), (2, 60, 120, 64, 700), (130, 1, 20, 32, 650)])
def test_decode_alone_on_a_compute_unit(dtype, B, Hkv, H, d, n):
    """No more workgroups than compute units, narrow heads, over eight steps each."""
    check_decode(Cache(dtype, [max(0, n - 37 * i % n) for i in range(B)], Hkv, d, seed=90), H)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [96, 160, 192, 224, 256])
def test_decode_wide_heads_in_two_tiles(dtype, d):
    """More than 16 query heads a key head at every size of a step, one to several
    wavefronts, in one slice and in several, with a budget that cuts into pages."""
    check_decode(Cache(dtype, [1, 77, 0, 230], 1, d, seed=91), 20)
    check_decode(Cache(dtype, [3001, 64], 2, d, seed=92), 66)
    check_decode(Cache(dtype, [1500], 1, d, seed=93), 17, sink=5, window=333)


def test_copy_of_a_pool_without_pages_is_refused():
    with pytest.raises(lla.LLAError) as e:
        kv.copy_pages(torch.empty((0, 2, 64, 32), device=DEV), None, ints([[0, 0]]))
    assert e.value.status == lla.LLA_ERR_INVALID_ARG


@pytest.mark.parametrize("dtype,d", [(BF, 32), (BF, 64), (F32, 32), (F32, 64)])
@pytest.mark.parametrize("B,Hkv", [(3, 2), (2, 200)])
def test_decode_narrow_heads_around_128_kb(dtype, d, B, Hkv):
    """Contexts of up to 128 KB of keys and values a head, which stay with one
    workgroup where each has a compute unit, and of a page more."""
    most = (128 << 10) // (2 * d * (2 if dtype == BF else 4))
    for n in (most // 2 + 7, most, most + 1):
        check_decode(Cache(dtype, [n] + [max(0, n - 65 * i) for i in range(1, B)], Hkv, d, seed=94), Hkv)
