"""GPU parity of packed batches and shared prompts over the paged K/V cache against
the float64 oracle: slot maps, packed writes, causal attention of packed tokens,
decode over a shared prompt, and a run of them as a serving program makes it.

Tolerances (eps = 2^-24; a rounding to bf16 is off by at most 2^-8 of the value).
With s_n the scores in natural units: a score is a sum of d products in any order,
times a constant of one rounding, its difference to the maximum one more: off by
e = (d + 4) eps scale max_n sum|q k|; the exponential adds 2^-21.  A weight and the
sum of weights are each off by that, sums over N tokens by their longest chains
(N / 16 + 64) eps, all relative to sum p |v|.  Weights rounded to bf16 add 2^-8 in the
numerator and, as they are summed as rounded, as much in the denominator; weights
of 16 bits (over a shared prompt, with results in bf16) 2^-16 in the numerator.
"""

import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from paper_2607_15456_amd import kv, lla
from tests.helpers import f64, log
from tests.test_gpu_kv import rope_bound

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
    assert got.shape == ref.shape and np.all(np.isfinite(got)), what
    worst = float(np.max(np.abs(got - ref) / tol))
    log(f"  {what}: {worst:.3f} of the bound")
    assert worst <= 1.0, (what, worst)


def bounds(q, k, v, seen, scale, dtype, out_dtype, rounded):
    """(out, lse, tolerance of out, of lse) of queries q [m, d] over keys [n, d] with
    the mask seen [m, n], in 64 bits."""
    s = q @ k.T * scale
    mag = np.abs(q) @ np.abs(k).T * scale
    s = np.where(seen, s, -np.inf)
    top = s.max(axis=1, keepdims=True)
    p = np.exp(s - top)
    total = p.sum(axis=1, keepdims=True)
    out, spread = p @ v / total, p @ np.abs(v) / total
    e = (q.shape[1] + 4) * EPS * np.max(np.where(seen, mag, 0.0), axis=1, keepdims=True)
    n = seen.sum(axis=1, keepdims=True)
    off = 2 * e + 2 * 2.0 ** -21 + 2 * (n / 16 + 64) * EPS + rounded
    tol = off * spread * (1 + half_step(out_dtype)) + half_step(out_dtype) * np.abs(out) + 1e-30
    lse = (top + np.log(total))[:, 0]
    return out, lse, tol, (off + 4 * EPS * np.abs(lse)[:, None] + 1e-6)[:, 0]


def pool(seed, pages, H_kv, d, dtype):
    return normal((pages, H_kv, 64, d), seed, dtype), normal((pages, H_kv, d, 64), seed + 1, dtype)


def pages_for(ends, rng, spare=3):
    """A table of scattered pages for sequences of these ends."""
    need = [-(-n // 64) for n in ends]
    order = rng.permutation(sum(need) + spare)
    table = np.full((len(ends), max(need + [1])), -1)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return table, len(order)


def places(table, row, n, k_pages, v_pages, g):
    at = np.arange(n)
    pages = np.asarray(table)[row, at // 64]
    return k_pages[pages, g, at % 64], v_pages[pages, g, :, at % 64]


def prefill_reference(q, k_pages, v_pages, table, offset, start, rows, scale, sink, window, dtype, out_dtype):
    """(out, lse, tolerances) of the tokens that are an entry's."""
    q, k_pages, v_pages = f64(q), f64(k_pages), f64(v_pages)
    group = q.shape[1] // k_pages.shape[1]
    out, tol = np.zeros(q.shape), np.ones(q.shape)
    lse, lse_tol = np.zeros(q.shape[:2]), np.ones(q.shape[:2])
    for b in range(len(start)):
        t0, t1 = offset[b], offset[b + 1]
        row = b if rows is None else rows[b]
        if t0 == t1:
            continue
        pos = start[b] + np.arange(t1 - t0)
        n = pos[-1] + 1
        at = np.arange(n)
        seen = at <= pos[:, None]
        if window:
            seen &= (at < sink) | (at > pos[:, None] - window)
        for h in range(q.shape[1]):
            k, v = places(table, row, n, k_pages, v_pages, h // group)
            out[t0:t1, h], lse[t0:t1, h], tol[t0:t1, h], lse_tol[t0:t1, h] = bounds(
                q[t0:t1, h], k, v, seen, scale, dtype, out_dtype, 2 * 2.0 ** -8 if dtype == BF and out_dtype == BF else 0.0)
    return out, lse, tol, lse_tol


# ---------------------------------------------------------------------------
# maps
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("B,most,total,seed", [(1, 1, 1, 0), (1, 700, 700, 1), (3, 5, 64, 2), (5, 40, 30, 3), (64, 1, 64, 4),
                                               (200, 9, 1000, 5), (1024, 3, 3000, 6), (1000, 64, 20000, 7)])
def test_slots(B, most, total, seed):
    """Equal to the lists, with empty entries, padding, refused rows, bad pages, more and
    less room than tokens."""
    rng = np.random.default_rng(seed)
    n_seqs, max_pages, n_pages = B + 2, 9 + most // 64, 4 * B + 7
    table = rng.integers(0, n_pages, (n_seqs, max_pages))
    table[rng.random(table.shape) < 0.05] = -1
    table[rng.random(table.shape) < 0.02] = n_pages
    start = rng.integers(0, 64 * max_pages - most + 8, B)
    new = rng.integers(0, most + 1, B)
    rows = rng.permutation(n_seqs)[:B]
    if B > 4:
        start[2], rows[3], new[4], rows[1] = -1, -1, -5, n_seqs + 3
    pos0 = rng.integers(0, 2 ** 31 - 3, B)
    for r, p in ((rows, None), (None, None), (rows, pos0)):
        pages = kv.PageTable(ints(table), ints(np.zeros(n_seqs)), ints(np.zeros(n_pages)), ints(np.zeros(n_pages + 1)))
        got = kv.slots(pages, ints(start), ints(new), total, rows=None if r is None else ints(r),
                       pos=None if p is None else ints(p))
        want = O.kv_slots(table.tolist(), start.tolist(), new.tolist(), total, n_pages,
                          None if r is None else r.tolist(), None if p is None else p.tolist())
        for x, y, name in zip(got, want, got._fields):
            assert x.tolist() == y, name
        again = kv.new_slots(B, total)
        for x in again:
            x.fill_(77)
        kv.slots(pages, ints(start), ints(new), total, rows=None if r is None else ints(r),
                 pos=None if p is None else ints(p), out=again)
        assert all(torch.equal(x, y) for x, y in zip(got, again))


def test_slots_of_lengths_past_32_bits():
    """Lengths whose sum passes 2^31 are cut to the room that there is."""
    pages = kv.new_page_table(3, 2, 4)
    big = 2 ** 31 - 1
    got = kv.slots(pages, ints([0, 0, 0]), ints([5, big, big]), 12)
    assert got.offset.tolist() == [0, 5, 12, 12] and got.entry.tolist() == [0] * 5 + [1] * 7
    assert got.pos.tolist() == list(range(5)) + list(range(7)) and got.slot.tolist() == [-1] * 12


@pytest.mark.parametrize("B,max_pages,seed", [(1, 1, 0), (2, 3, 1), (17, 5, 2), (64, 130, 3), (65, 130, 4), (300, 40, 5),
                                              (1024, 3, 6)])
@pytest.mark.parametrize("least", [1, 65, 300])
def test_shared_prefix(B, max_pages, seed, least):
    rng = np.random.default_rng(seed)
    n_seqs, n_pages = B + 1, 64
    table = rng.integers(0, n_pages, (n_seqs, max_pages))
    for b in range(1, n_seqs):  # neighbours share some leading pages, mostly
        n = rng.integers(0, max_pages + 1)
        table[b, :n] = table[b - 1, :n]
    table[rng.random(table.shape) < 0.01] = -1
    length = rng.integers(0, 64 * max_pages + 1, n_seqs)
    length[rng.random(n_seqs) < 0.3] = 64 * max_pages
    rows = np.arange(B)
    if B > 10:
        rows[4], rows[7], rows[9] = -1, n_seqs + 2, rows[8]
    pages = kv.PageTable(ints(table), ints(length), ints(np.zeros(n_pages)), ints(np.zeros(n_pages + 1)))
    for r in (rows, None):
        want = O.kv_shared_prefix(table.tolist(), length.tolist(), n_pages, None if r is None else r.tolist(), least)
        if r is None and n_seqs > 1024:
            continue
        lead, shared = kv.shared_prefix(pages, None if r is None else ints(r), least=least)
        assert lead.tolist() == want[0] and shared.tolist() == want[1]


# ---------------------------------------------------------------------------
# packed write
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("total,H,d,rot,interleaved", [(1, 1, 32, 0, False), (3, 5, 96, 48, True), (64, 2, 128, 128, False),
                                                       (130, 3, 256, 64, True), (777, 16, 64, 64, False), (65, 4, 160, 24, False)])
def test_write_slots(dtype, total, H, d, rot, interleaved):
    """Runs of neighbours that begin and end inside pages, scattered tokens, tokens without
    a slot; everything else in the pools stays as it was."""
    rng = np.random.default_rng(total)
    n_pages = 3 * total // 64 + 5
    slot = np.full(total, -1)
    free = rng.permutation(n_pages)
    t = page = 0
    while t < total:  # runs over a page's places, then a token or two anywhere
        n, first = int(rng.integers(1, 65)), int(rng.integers(0, 64))
        n = min(n, 64 - first, total - t)
        if page < n_pages - 1:
            slot[t:t + n] = free[page] * 64 + first + np.arange(n)
        page += 1
        t += n
    if total > 8:
        slot[5], slot[6], slot[total - 1] = -1, 64 * n_pages + 3, -(1 << 40)
        slot[1], slot[2] = slot[2], slot[1]
    pos = rng.integers(0, 100000, total)
    fused = normal((total, 3, H, d), 1, dtype)
    k, v = fused[:, 1], fused[:, 2]
    kp, vp = pool(2, n_pages, H, d, dtype)
    want_k, want_v = kp.clone(), vp.clone()
    freq = kv.rope_frequencies(rot)[0] if rot else None
    ok = [i for i in range(total) if 0 <= slot[i] < 64 * n_pages]
    for i in ok:
        want_k[slot[i] // 64, :, slot[i] % 64] = k[i]
        want_v[slot[i] // 64, :, :, slot[i] % 64] = v[i]
    kv.write_slots(k, v, kp, vp, torch.as_tensor(slot).to(DEV), pos=ints(pos) if rot else None, freq=freq,
                   interleaved=interleaved)
    assert torch.equal(vp, want_v)
    if rot:  # turned keys against the oracle; with these put in, all else has to be the same
        page, at = torch.as_tensor(slot[ok] // 64).to(DEV), torch.as_tensor(slot[ok] % 64).to(DEV)
        got = kp[page, :, at]
        ref = O.kv_rope(f64(k)[ok], np.broadcast_to(pos[ok][:, None], (len(ok), H)), f64(freq), interleaved)
        near(got, ref, rope_bound(f64(k)[ok], rot // 2, interleaved, 1.0, ref, dtype), "turned keys")
        assert torch.equal(got[..., rot:], k[ok][..., rot:])
        want_k[page, :, at] = got
    assert torch.equal(kp, want_k)


def test_write_slots_past_32_bit_offsets():
    """Pages behind 2^32 bytes of a pool."""
    H, d, n_pages = 16, 256, 9000
    kp = torch.zeros((n_pages, H, 64, d), dtype=BF, device=DEV)
    vp = torch.zeros((n_pages, H, d, 64), dtype=BF, device=DEV)
    assert kp.numel() * 2 > 1 << 32
    k, v = normal((70, H, d), 0, BF), normal((70, H, d), 1, BF)
    slot = 64 * (n_pages - 2) + 3 + torch.arange(70, device=DEV)
    kv.write_slots(k, v, kp, vp, slot)
    assert torch.equal(kp[-2:].transpose(1, 2).reshape(128, H, d)[3:73], k)
    assert torch.equal(vp[-2:].permute(0, 3, 1, 2).reshape(128, H, d)[3:73], v)
    assert not kp[:-2].any() and not vp[:-2].any()


# ---------------------------------------------------------------------------
# causal attention of packed tokens
# ---------------------------------------------------------------------------

def check_prefill(dtype, out_dtype, H, H_kv, d, new, start, sink=0, window=0, seed=0, rows=None, spare=0, fused=False,
                  n_ctx=None, scale=None):
    rng = np.random.default_rng(seed)
    ends = [s + n for s, n in zip(start, new)]
    n_seqs = len(new) if rows is None else max(rows) + 1
    by_row = [1] * n_seqs
    for b, e in enumerate(ends):
        by_row[b if rows is None else rows[b]] = e
    table, n_pages = pages_for(by_row, rng)
    kp, vp = pool(seed + 10, n_pages, H_kv, d, dtype)
    total = sum(new) + spare
    q = normal((total, 3 * H, d), seed + 20, dtype)[:, :H] if fused else normal((total, H, d), seed + 20, dtype)
    offset = np.concatenate(([0], np.cumsum(new)))
    out = torch.full((total, H, d), 7.0, dtype=out_dtype, device=DEV)
    lse = torch.full((total, H), 7.0, dtype=F32, device=DEV)
    n_ctx = table.shape[1] * 64 if n_ctx is None else n_ctx
    need = kv.prefill_workspace_bytes(dtype, len(new), total, H, H_kv, d, n_ctx, sink, window, out_dtype=out_dtype)
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV) if need else None  # NaN
    kv.prefill_attn(q, kp, vp, ints(table), ints(offset), ints(start), n_ctx=n_ctx,
                    rows=None if rows is None else ints(rows), sink=sink, window=window, out=out, lse=lse, workspace=ws,
                    scale=scale)
    s = d ** -0.5 if scale is None else scale
    ref, ref_lse, tol, lse_tol = prefill_reference(q, kp, vp, table, offset, start, rows, s, sink, window, dtype, out_dtype)
    n = sum(new)
    what = f"prefill {dtype} {out_dtype} H={H}/{H_kv} d={d} new={new[:6]} start={start[:6]} w={sink}+{window}"
    near(out[:n], ref[:n], tol[:n], what)
    near(lse[:n], ref_lse[:n], lse_tol[:n], what + " lse")
    assert (out[n:] == 7).all() and (lse[n:] == 7).all()
    without = kv.prefill_attn(q, kp, vp, ints(table), ints(offset), ints(start), n_ctx=n_ctx,
                              rows=None if rows is None else ints(rows), sink=sink, window=window, out_dtype=out_dtype,
                              scale=scale)
    assert torch.equal(without[:n], out[:n])


TYPES = [(BF, BF), (BF, F32), (F32, F32), (F32, BF)]


@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_prefill_widths(dtype, out_dtype, d):
    check_prefill(dtype, out_dtype, 3, 1, d, [70, 1, 200], [0, 300, 13], seed=d)
    check_prefill(dtype, out_dtype, 2, 2, d, [300], [65], seed=d + 1)


@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("H,H_kv", [(1, 1), (16, 16), (16, 2), (6, 2), (40, 2), (64, 1), (33, 1)])
def test_prefill_groups(dtype, out_dtype, H, H_kv):
    check_prefill(dtype, out_dtype, H, H_kv, 64, [5, 1, 37], [100, 0, 63], seed=H)


@pytest.mark.parametrize("dtype,out_dtype", TYPES[:3])
@pytest.mark.parametrize("new,start", [([1], [0]), ([1], [63]), ([1], [64]), ([2], [63]), ([64], [0]), ([65], [0]), ([33], [31]),
                                       ([257], [0]), ([129], [4000]), ([1] * 40, list(range(0, 4000, 100))),
                                       ([0, 3, 0, 0, 1, 0], [5, 60, 0, 9, 700, 1]), ([300, 1, 1, 64], [0, 5000, 1, 64]),
                                       ([1, 511, 2], [2000, 1, 3000])])
def test_prefill_lengths(dtype, out_dtype, new, start):
    check_prefill(dtype, out_dtype, 4, 2, 128, new, start, seed=sum(new), spare=3, fused=True)


@pytest.mark.parametrize("dtype,out_dtype", TYPES[:3])
@pytest.mark.parametrize("sink,window", [(0, 1), (0, 64), (4, 60), (70, 100), (4, 100000), (1, 31), (500, 3)])
def test_prefill_windows(dtype, out_dtype, sink, window):
    check_prefill(dtype, out_dtype, 4, 2, 64, [150, 1, 1, 280], [0, 400, 63, 700], sink, window, seed=window % 97)


def test_prefill_rows_and_far_bound():
    """Sequences in any order of the table; a bound far above the lengths, as a captured step has."""
    check_prefill(BF, BF, 8, 2, 128, [40, 3, 1], [100, 900, 64], rows=[4, 1, 6], spare=9, n_ctx=None)
    rng = np.random.default_rng(0)
    table, n_pages = pages_for([1000, 64], rng)
    wide = np.full((2, 2000), -1)
    wide[:, :table.shape[1]] = table
    kp, vp = pool(1, n_pages, 2, 128, BF)
    q = normal((130, 4, 128), 2, BF)
    args = (q, kp, vp)
    near_, far = (kv.prefill_attn(*args, ints(t), ints([0, 129, 130]), ints([871, 63]), n_ctx=n) for t, n in
                  ((table, 1000), (wide, 128000)))
    ref = prefill_reference(q, kp, vp, table, [0, 129, 130], [871, 63], None, 128 ** -0.5, 0, 0, BF, F32)
    near(near_, ref[0], ref[2], "near bound")
    near(far, ref[0], ref[2], "far bound")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("long", [False, True])
def test_prefill_padding_and_bad_indices(dtype, long):
    """Zeros for padding, NaN where an index is out of range, and no harm to the others."""
    new = [300 if long else 2] * 7
    rng = np.random.default_rng(3)
    start = [70, 70, -1, 70, 70, 70, 70]
    n = new[0]
    table, n_pages = pages_for([70 + n] * 6, rng)
    table[4, 1] = n_pages  # of places 64 .. 127
    table[5, 1] = -1
    rows = [0, -1, 2, 6, 4, 5, 1]
    kp, vp = pool(4, n_pages, 2, 64, dtype)
    q = normal((sum(new), 4, 64), 5, dtype)
    offset = np.concatenate(([0], np.cumsum(new)))
    lse = torch.zeros((sum(new), 4), device=DEV)
    out = kv.prefill_attn(q, kp, vp, ints(table), ints(offset), ints(start), n_ctx=64 * table.shape[1], rows=ints(rows), lse=lse)
    at = lambda b: slice(offset[b], offset[b + 1])  # noqa: E731
    for b in (1, 2):
        assert (out[at(b)] == 0).all() and (lse[at(b)] == -np.inf).all()
    for b in (3, 4, 5):
        assert out[at(b)].isnan().all() and lse[at(b)].isnan().all(), b
    fine = [0, 6]
    good = np.where(np.isin(np.arange(7), fine), start, 0)
    ref = prefill_reference(q, kp, vp, np.where((table < 0) | (table >= n_pages), 0, table), offset, good,
                            [r if b in fine else 0 for b, r in enumerate(rows)], 64 ** -0.5, 0, 0, dtype, F32)
    for b in fine:
        near(out[at(b)], ref[0][at(b)], ref[2][at(b)], f"entry {b}")
    # tokens before a bad page, and before the bound, are whole
    start2 = ints([0])
    table2 = table[4:5].copy()
    out = kv.prefill_attn(q[:130], kp, vp, ints(table2), ints([0, 130]), start2, n_ctx=64 * table.shape[1]) if long else None
    if long:
        ref = prefill_reference(q[:64], kp, vp, table2, [0, 64], [0], None, 64 ** -0.5, 0, 0, dtype, F32)
        near(out[:64], ref[0], ref[2], "before a bad page")
        assert out[64:].isnan().all()
        out = kv.prefill_attn(q[:64], kp, vp, ints(table[:1]), ints([0, 64]), ints([0]), n_ctx=33)
        ref = prefill_reference(q[:33], kp, vp, table[:1], [0, 33], [0], None, 64 ** -0.5, 0, 0, dtype, F32)
        near(out[:33], ref[0], ref[2], "before the bound")
        assert out[33:].isnan().all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("offsets", [[0, 300, 0, 300, 0, 300], [300, 0, 300, 0], [-5, 400, -(1 << 31), (1 << 31) - 1, 3], [7] * 6])
def test_prefill_offsets_that_decrease_do_no_harm(dtype, offsets):
    """Which tokens are done is not defined; nothing but the results and the workspace is written, and a call after it is whole."""
    B, total = len(offsets) - 1, 300
    table, n_pages = pages_for([1200] * B, np.random.default_rng(0))
    kp, vp = pool(1, n_pages, 2, 64, dtype)
    q = normal((total, 4, 64), 2, dtype)
    need = kv.prefill_workspace_bytes(dtype, B, total, 4, 2, 64, 1216)
    ws = torch.full((need + 65536,), 90, dtype=torch.uint8, device=DEV)
    out = torch.full((total + 64, 4, 64), 7.0, device=DEV)
    before = kp.clone(), vp.clone()
    kv.prefill_attn(q, kp, vp, ints(table), ints(offsets), ints([800] * B), n_ctx=1216, out=out[:total], workspace=ws[:need])
    assert (ws[need:] == 90).all() and (out[total:] == 7).all()
    assert torch.equal(kp, before[0]) and torch.equal(vp, before[1])
    kv.prefill_attn(q, kp, vp, ints(table[:1]), ints([0, total]), ints([900]), n_ctx=1216, out=out[:total], workspace=ws[:need])
    ref = prefill_reference(q, kp, vp, table[:1], [0, total], [900], None, 1 / 8, 0, 0, dtype, F32)
    near(out[:total], ref[0], ref[2], "after it")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("starts", [[0, 100000, 0], [1 << 30, 5, (1 << 31) - 1], [700, 1 << 24, 1 << 26]])
def test_prefill_places_far_past_the_bound(dtype, starts):
    """NaN, and nothing else of the batch is harmed: the order of the tiles goes by places within the bound."""
    new, n_ctx = [300, 280, 310], 200
    table, n_pages = pages_for([700] * 3, np.random.default_rng(0))
    kp, vp = pool(1, n_pages, 2, 64, dtype)
    q = normal((sum(new), 4, 64), 2, dtype)
    offset = np.concatenate(([0], np.cumsum(new)))
    out = kv.prefill_attn(q, kp, vp, ints(table), ints(offset), ints(starts), n_ctx=n_ctx)
    for b in range(3):
        fine = max(0, min(new[b], n_ctx - starts[b]))
        assert out[offset[b] + fine:offset[b + 1]].isnan().all()
        if fine:
            rows = slice(offset[b], offset[b] + fine)
            ref = prefill_reference(q[rows], kp, vp, table[b:b + 1], [0, fine], [starts[b]], None, 1 / 8, 0, 0, dtype, F32)
            near(out[rows], ref[0], ref[2], f"entry {b}")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n,start", [(2, 70), (40, 50), (300, 100)])
def test_prefill_masked_places_may_hold_anything(dtype, bad, n, start):
    """A token does not see what later places hold, nor places outside its window; those that attend a bad value
    are not finite in its feature alone."""
    rng = np.random.default_rng(n)
    end = start + n
    table, n_pages = pages_for([end], rng)
    q = normal((n, 4, 64), 1, dtype)
    for sink, window in ((0, 0), (3, 40)):
        kp, vp = pool(2, n_pages, 2, 64, dtype)
        clean = kv.prefill_attn(q, kp, vp, ints(table), ints([0, n]), ints([start]), n_ctx=end, sink=sink, window=window)
        page = table[0, (end - 1) // 64]
        if end % 64:
            kp[page, :, end % 64:], vp[page, :, :, end % 64:] = bad, bad
        got = kv.prefill_attn(q, kp, vp, ints(table), ints([0, n]), ints([start]), n_ctx=end, sink=sink, window=window)
        assert torch.equal(got, clean), "slots behind the last token"
        i = n // 2                                  # a token whose value is bad in one feature of key head 1
        at = start + i
        vp[table[0, at // 64], 1, 9, at % 64] = bad
        got = f64(kv.prefill_attn(q, kp, vp, ints(table), ints([0, n]), ints([start]), n_ctx=end, sink=sink, window=window))
        sees = np.zeros(n, dtype=bool)
        sees[i:] = True
        if window:
            sees[i + window:] = False
        want = f64(clean)
        assert np.all(~np.isfinite(got[sees][:, 2:, 9]))
        keep = np.ones(got.shape, dtype=bool)
        keep[sees, 2:, 9] = False
        assert np.array_equal(got[keep], want[keep])
        vp[table[0, at // 64], 1, 9, at % 64] = 1.0
        clean = f64(kv.prefill_attn(q, kp, vp, ints(table), ints([0, n]), ints([start]), n_ctx=end, sink=sink, window=window))
        kp[table[0, at // 64], 1, at % 64, 5] = float("nan")
        got = f64(kv.prefill_attn(q, kp, vp, ints(table), ints([0, n]), ints([start]), n_ctx=end, sink=sink, window=window))
        assert np.isnan(got[sees][:, 2:]).all() and np.array_equal(got[~sees], clean[~sees])
        assert np.array_equal(got[:, :2], clean[:, :2])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_prefill_scores_past_2_31(dtype):
    """Finite scores of any size give finite results: the largest key takes all."""
    table, n_pages = pages_for([200], np.random.default_rng(0))
    kp, vp = pool(0, n_pages, 1, 64, dtype)
    kp[:] = 0
    for n in range(200):
        kp[table[0, n // 64], 0, n % 64, 0] = 2.0 ** 16 * (n % 50 + 1)
    q = torch.zeros((200, 1, 64), dtype=dtype, device=DEV)
    q[:, 0, 0] = 2.0 ** 20
    out = f64(kv.prefill_attn(q, kp, vp, ints(table), ints([0, 200]), ints([0]), n_ctx=200))
    _, v = places(table, 0, 200, f64(kp), f64(vp), 0)
    for p in range(200):
        top = max(n % 50 for n in range(p + 1))
        want = np.mean([v[n] for n in range(p + 1) if n % 50 == top], axis=0)
        assert np.allclose(out[p, 0], want, rtol=1e-5, atol=1e-6), p


def test_prefill_past_32_bit_offsets():
    """Pages behind 2^32 bytes of a pool."""
    H, d, n_pages = 16, 256, 9000
    kp, vp = pool(0, 12, H, d, BF)
    big_k = torch.zeros((n_pages, H, 64, d), dtype=BF, device=DEV)
    big_v = torch.zeros((n_pages, H, d, 64), dtype=BF, device=DEV)
    big_k[-12:], big_v[-12:] = kp, vp
    table = np.arange(12)[None]
    for n in (1, 300):
        q = normal((n, H, d), n, BF)
        args = dict(n_ctx=768, out_dtype=BF)
        a = kv.prefill_attn(q, kp, vp, ints(table), ints([0, n]), ints([768 - n]), **args)
        b = kv.prefill_attn(q, big_k, big_v, ints(table + n_pages - 12), ints([0, n]), ints([768 - n]), **args)
        assert torch.equal(a, b)


# ---------------------------------------------------------------------------
# decode over a shared prompt
# ---------------------------------------------------------------------------

def check_shared(dtype, out_dtype, H, H_kv, d, groups, seed=0, rows=None, scale=None):
    """groups: (shared places, own lengths of its members)."""
    rng = np.random.default_rng(seed)
    lead, shared, ends = [], [], []
    for prefix, mine in groups:
        lead += [len(ends)] * len(mine)
        shared += [prefix] * len(mine)
        ends += [prefix + n for n in mine]
    B = len(ends)
    table, n_pages = pages_for(ends, rng)
    kp, vp = pool(seed + 1, n_pages, H_kv, d, dtype)
    # what entries hold below `shared` is not read: it stays their own
    q = normal((B, H, d), seed + 2, dtype)
    lse = torch.zeros((B, H), device=DEV)
    order = np.arange(B) if rows is None else np.asarray(rows)
    big, length = np.full((max(order) + 1, table.shape[1]), -1), np.zeros(max(order) + 1, dtype=int)
    big[order], length[order] = table, ends
    args = dict(n_ctx=table.shape[1] * 64, rows=None if rows is None else ints(rows), scale=scale)
    need = kv.shared_workspace_bytes(dtype, B, H, H_kv, d, args["n_ctx"])
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)  # NaN
    out = kv.decode_attn_shared(q, kp, vp, ints(big), ints(length), ints(lead), ints(shared), out_dtype=out_dtype, lse=lse,
                                workspace=ws, **args)
    qn, kn, vn = f64(q), f64(kp), f64(vp)
    ref, tol = np.zeros(q.shape), np.ones(q.shape)
    ref_lse, lse_tol = np.zeros((B, H)), np.ones((B, H))
    s = d ** -0.5 if scale is None else scale
    for b in range(B):
        if ends[b] == 0:
            continue
        for g in range(H_kv):
            k, v = places(table, b, ends[b], kn, vn, g)
            first = places(table, lead[b], shared[b], kn, vn, g)
            k[:shared[b]], v[:shared[b]] = first
            hs = slice(g * H // H_kv, (g + 1) * H // H_kv)
            ref[b, hs], ref_lse[b, hs], tol[b, hs], lse_tol[b, hs] = bounds(
                qn[b, hs], k, v, np.ones((H // H_kv, ends[b]), dtype=bool), s, dtype, out_dtype,
                2.0 ** -16 if dtype == BF and out_dtype == BF else 0.0)
    what = f"shared {dtype} {out_dtype} H={H}/{H_kv} d={d} {[(p, m[:3], len(m)) for p, m in groups][:4]}"
    some = np.array(ends) > 0
    near(out[torch.as_tensor(some)], ref[some], tol[some], what)
    near(lse[torch.as_tensor(some)], ref_lse[some], lse_tol[some], what + " lse")
    assert (out[torch.as_tensor(~some)] == 0).all() and (lse[torch.as_tensor(~some)] == -np.inf).all()


@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_shared_widths(dtype, out_dtype, d):
    check_shared(dtype, out_dtype, 6, 2, d, [(200, [5, 70, 1]), (0, [300]), (64, [0, 64])], seed=d)
    check_shared(dtype, out_dtype, 8, 1, d, [(900, [3] * 20)], seed=d)


@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("H,H_kv", [(1, 1), (16, 16), (16, 2), (40, 2), (64, 1), (33, 1), (300, 1)])
def test_shared_groups_of_heads(dtype, out_dtype, H, H_kv):
    check_shared(dtype, out_dtype, H, H_kv, 64, [(130, [5, 0, 80]), (64, [1] * 9), (1, [1, 63])], seed=H)


@pytest.mark.parametrize("dtype,out_dtype", TYPES[:3])
@pytest.mark.parametrize("groups", [[(1, [0])], [(0, [1])], [(64, [0] * 3)], [(5000, [1, 100])], [(65, [1] * 70)],
                                    [(63, [1]), (63, [2]), (64, [3]), (65, [4])], [(0, [0]), (10, [3, 0, 200]), (0, [7])],
                                    [(300, [i % 5 for i in range(100)]), (700, [2] * 33)], [(64 * i + 3, [1] * (i % 4 + 1)) for i in range(40)]])
def test_shared_lengths(dtype, out_dtype, groups):
    check_shared(dtype, out_dtype, 4, 2, 128, groups, seed=len(groups))


def test_shared_rows_and_large_batches():
    check_shared(BF, F32, 4, 2, 64, [(100, [5, 6, 7]), (0, [64])], rows=[6, 0, 3, 2])
    check_shared(BF, F32, 2, 1, 32, [(130, [i % 3 for i in range(1000)]), (64, [1] * 24)], seed=5)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_shared_padding_and_bad_indices(dtype):
    rng = np.random.default_rng(1)
    table, n_pages = pages_for([200] * 9, rng)
    kp, vp = pool(1, n_pages, 2, 64, dtype)
    q = normal((12, 4, 64), 2, dtype)
    length = [200] * 8 + [0]
    rows = [0, 1, -1, 8, 2, 9, 3, 4, 5, 6, 7, 0]
    lead = [0, 0, 0, 0, 0, 5, 12, -1, 8, 9, 2, 11]
    shared = [100, 100, 0, 0, 201, 0, 100, 100, -1, 200, 50, 0]
    lse = torch.zeros((12, 4), device=DEV)
    out = kv.decode_attn_shared(q, kp, vp, ints(table), ints(length), ints(lead), ints(shared), n_ctx=256, rows=ints(rows), lse=lse)
    for b in (2, 3):
        assert (out[b] == 0).all() and (lse[b] == -np.inf).all()
    for b in (4, 5, 6, 7, 8, 10):
        assert out[b].isnan().all() and lse[b].isnan().all(), b
    plain = kv.decode_attn(q, kp, vp, ints(table), ints(length), n_ctx=256, rows=ints(rows))
    qn, kn, vn = f64(q), f64(kp), f64(vp)
    for b in (0, 1, 9, 11):
        for h in range(4):
            k, v = places(table, rows[b], 200, kn, vn, h // 2)
            k[:shared[b]], v[:shared[b]] = places(table, rows[lead[b]], shared[b], kn, vn, h // 2)
            ref, _, tol, _ = bounds(qn[b, h:h + 1], k, v, np.ones((1, 200), dtype=bool), 1 / 8, dtype, F32, 0.0)
            near(out[b, h:h + 1], ref, tol, f"entry {b}")
            if b in (0, 11):
                near(plain[b, h:h + 1], ref, tol, f"decode of {b}")
    # bad pages: of the prompt for its readers, of an entry's own for it
    table2 = table.copy()
    table2[0, 0] = -1
    again = lambda t: kv.decode_attn_shared(q, kp, vp, ints(t), ints(length), ints(lead), ints(shared), n_ctx=256,  # noqa: E731
                                            rows=ints(rows))
    out = again(table2)
    assert out[0].isnan().all() and out[1].isnan().all() and out[11].isnan().all() and out[9].isfinite().all()
    table2 = table.copy()
    table2[1, 3] = n_pages
    out = again(table2)
    assert out[1].isnan().all() and out[0].isfinite().all() and out[9].isfinite().all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_shared_slots_not_attended_may_hold_anything(dtype):
    """Behind the lengths, and an entry's own places below what it shares."""
    table, n_pages = pages_for([130, 140, 77], np.random.default_rng(2))
    kp, vp = pool(3, n_pages, 1, 64, dtype)
    q = normal((3, 5, 64), 4, dtype)
    args = (ints(table), ints([130, 140, 77]), ints([0, 0, 2]), ints([100, 100, 0]))
    clean = kv.decode_attn_shared(q, kp, vp, *args, n_ctx=192)
    for row, a, z in ((0, 130, 192), (1, 0, 100), (1, 140, 192), (2, 77, 128)):
        for n in range(a, z):
            kp[table[row, n // 64], :, n % 64] = float("nan")
            vp[table[row, n // 64], :, :, n % 64] = float("inf")
    assert torch.equal(kv.decode_attn_shared(q, kp, vp, *args, n_ctx=192), clean)


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

class Server:
    """One layer of a small model's cache, and what its steps call."""

    def __init__(self, dtype, n_seqs=8, max_pages=12, n_pages=60, H=6, H_kv=2, d=64):
        self.dtype, self.H, self.H_kv, self.d = dtype, H, H_kv, d
        self.pages = kv.new_page_table(n_seqs, max_pages, n_pages)
        self.kp, self.vp = kv.alloc_pages(n_pages, H_kv, d, dtype, layers=1)
        self.kp.fill_(float("nan")), self.vp.fill_(float("nan"))
        self.freq, _ = kv.rope_frequencies(d)
        self.n_ctx = 64 * max_pages

    def step(self, rows, add, x, total, shared=False):
        """x [total, H + 2 H_kv, d]: queries, keys and values of packed tokens."""
        n, H, G = rows.numel(), self.H, self.H_kv
        start, pairs = torch.empty_like(rows), torch.empty((n, 2), dtype=torch.int32, device=DEV)
        result = torch.empty(4, dtype=torch.int32, device=DEV)
        kv.reserve(self.pages, rows, add, start, pairs, result)
        kv.copy_pages(self.kp, self.vp, pairs, result)
        at = kv.slots(self.pages, start, add, total, rows=rows)
        q = kv.rope(x[None, :, :H], self.freq, pos=at.pos[None])[0]
        kv.write_slots(x[:, H:H + G], x[:, H + G:], self.kp[0], self.vp[0], at.slot, pos=at.pos, freq=self.freq)
        if shared:
            lead, common = kv.shared_prefix(self.pages, rows)
            return kv.decode_attn_shared(q, self.kp[0], self.vp[0], self.pages.table, self.pages.length, lead, common,
                                         n_ctx=self.n_ctx, rows=rows, out_dtype=self.dtype)
        out = torch.zeros((total, H, self.d), dtype=self.dtype, device=DEV)
        return kv.prefill_attn(q, self.kp[0], self.vp[0], self.pages.table, at.offset, start, n_ctx=self.n_ctx, rows=rows,
                               out=out)


def history_attention(server, history, x, lens):
    """Attention of packed tokens from the projections alone, in 64 bits, and its tolerance.
    history: per entry, all projections of its sequence, these tokens' last."""
    H, G, d = server.H, server.H_kv, server.d
    out, tol = [], []
    freq = f64(server.freq)
    for past, n in zip(history, lens):
        if n == 0:
            continue
        end = len(past)
        pos = np.arange(end)
        # queries and keys as the cache holds them: turned, rounded once
        turn = lambda y, p: f64(torch.as_tensor(O.kv_rope(y, np.broadcast_to(p[:, None], y.shape[:2]), freq)).to(server.dtype))  # noqa: E731
        q, k, v = turn(past[end - n:, :H], pos[end - n:]), turn(past[:, H:H + G], pos), past[:, H + G:]
        o, t = np.zeros((n, H, d)), np.zeros((n, H, d))
        seen = pos <= pos[end - n:, None]
        for h in range(H):
            g = h * G // H
            # a turned value may round to its other neighbour: one step more of q and k in each score
            o[:, h], _, t[:, h], _ = bounds(q[:, h], k[:, g], v[:, g], seen, d ** -0.5, server.dtype, server.dtype,
                                            2 * 2.0 ** -8 if server.dtype == BF else 0.0)
            mag = np.max(np.abs(q[:, h]) @ np.abs(k[:, g]).T, axis=1, keepdims=True) * d ** -0.5
            flips = 2.0 ** -7 if server.dtype == BF else 2.0 ** -20
            t[:, h] += 2 * 2 * flips * mag * np.max(np.abs(v[:, g]))
        out.append(o)
        tol.append(t)
    return np.concatenate(out), np.concatenate(tol)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_serving_run(dtype):
    """Prompts of unequal length, a piece of another beside single tokens, children that
    share a prompt, their tokens read with the prompt once: every step against the projections."""
    s = Server(dtype)
    past = {}

    def step(rows, add, total, seed, shared=False):
        x = normal((total, s.H + 2 * s.H_kv, s.d), seed, dtype)
        got = s.step(ints(rows), ints(add), x, total, shared)
        t = 0
        for r, n in zip(rows, add):
            if r >= 0:
                past[r] = np.concatenate((past.get(r, np.zeros((0, s.H + 2 * s.H_kv, s.d))), f64(x[t:t + n])))
            t += n
        live = [(r, n) for r, n in zip(rows, add) if r >= 0]
        ref, tol = history_attention(s, [past[r] for r, _ in live], x, [n for _, n in live])
        near(got[:len(ref)], ref, tol, f"step {rows} {add}")
        return got

    step([0, 3], [130, 65], 200, 1)
    step([3, 0, 5], [1, 1, 300], 302, 2)
    got = step([5, 0, -1], [40, 1, 0], 50, 3)
    assert (got[41:] == 0).all()
    result = torch.empty(4, dtype=torch.int32, device=DEV)
    kv.fork(s.pages, ints([0, 0, 5]), ints([1, 2, 6]), result)
    past[1], past[2], past[6] = past[0].copy(), past[0].copy(), past[5].copy()
    assert result[0].item() == kv.PAGES_OK
    for i in range(3):
        step([0, 1, 2, 5, 6], [1] * 5, 5, 10 + i, shared=True)
    lead, common = kv.shared_prefix(s.pages, ints([0, 1, 2, 5, 6]))
    assert lead.tolist() == [0, 0, 0, 3, 3] and common.tolist() == [128, 128, 128, 320, 320]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shared", [False, True])
def test_captured_steps(dtype, shared):
    """A step captured once and replayed, with the program's own work between, equals the
    eager one; padding rows serve fewer sequences, and more than one graph of one pool lives."""
    a, b = Server(dtype), Server(dtype)
    warm = [normal((500, a.H + 2 * a.H_kv, a.d), 30 + i, dtype) for i in range(2)]
    result = torch.empty(4, dtype=torch.int32, device=DEV)
    for s in (a, b):
        s.step(ints([0, 2]), ints([200, 300]), warm[0], 500)
        kv.fork(s.pages, ints([0, 0, 2]), ints([1, 4, 3]), result)
    rows, add, total = ints([0, 1, 4, 2, 3, -1]), ints([1] * 5 + [0]), 6
    x = torch.zeros((total, a.H + 2 * a.H_kv, a.d), dtype=dtype, device=DEV)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):  # (loads kernels; the lengths grow by one in both)
        xs = normal(tuple(x.shape), 99, dtype)
        x.copy_(xs)
        a.step(rows, add, x, total, shared)
    torch.cuda.current_stream().wait_stream(side)
    b.step(rows, add, xs, total, shared)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = a.step(rows, add, x, total, shared)
    for i in range(6):
        xs = normal(tuple(x.shape), 50 + i, dtype)
        r = [0, 1, 4, 2, 3, -1] if i % 2 == 0 else [0, 1, -1, 2, 3, -1]
        n = [1, 1, 1, 1, 1, 0] if i % 2 == 0 else [1, 1, 0, 1, 1, 0]
        if shared and i % 2:
            n = [1, 1, 1, 1, 1, 0]  # a decode step's entry b is packed token b, padding too
        rows.copy_(ints(r)), add.copy_(ints(n)), x.copy_(xs)
        graph.replay()
        want = b.step(ints(r), ints(n), xs, total, shared)
        torch.cuda.synchronize()
        used = sum(n) if not shared else total
        assert torch.equal(out[:used], want[:used]), i
        assert torch.equal(a.pages.length, b.pages.length)
        (xs.float() @ xs.float().transpose(1, 2)).sum().item()  # the program's own work


def test_captured_calls_share_a_workspace():
    """Two graphs with one workspace, replayed in turn with the program's own work between: nothing is kept in it."""
    table, n_pages = pages_for([3000, 2500, 700], np.random.default_rng(4))
    kp, vp = pool(1, n_pages, 2, 128, BF)
    t, off, start = ints(table), ints([0, 129, 130, 160]), ints([2871, 2499, 670])
    length, lead, shared = ints([3000, 2500, 700]), ints([0, 0, 0]), ints([640, 640, 640])
    need = max(kv.prefill_workspace_bytes(BF, 3, 160, 8, 2, 128, 3008), kv.shared_workspace_bytes(BF, 3, 8, 2, 128, 3008))
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    q, one = normal((160, 8, 128), 2, BF), normal((3, 8, 128), 3, BF)
    calls = [lambda **kw: kv.prefill_attn(q, kp, vp, t, off, start, n_ctx=3008, **kw),
             lambda **kw: kv.decode_attn_shared(one, kp, vp, t, length, lead, shared, n_ctx=3008, **kw)]
    outs = [torch.empty((160, 8, 128), device=DEV), torch.empty((3, 8, 128), device=DEV)]
    graphs, side = [], torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for call, out in zip(calls, outs):
        with torch.cuda.stream(side):
            call(out=out, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call(out=out, workspace=ws)
        graphs.append(g)
    for i in range(4):
        q.copy_(normal((160, 8, 128), 20 + i, BF)), one.copy_(normal((3, 8, 128), 30 + i, BF))
        for g in graphs if i % 2 else graphs[::-1]:
            g.replay()
        want = [call() for call in calls]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want)), i
        (kp[0].float() @ vp[0].float()).sum().item()


def test_other_streams_and_two_at_once():
    """Calls on side streams with workspaces of their own do not disturb each other."""
    dtype = BF
    table, n_pages = pages_for([3000, 2500], np.random.default_rng(0))
    kp, vp = pool(1, n_pages, 2, 128, dtype)
    q = normal((130, 8, 128), 2, dtype)
    args = (kp, vp, ints(table), ints([0, 129, 130]), ints([2871, 2499]))
    want = kv.prefill_attn(q, *args, n_ctx=3000)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for s in streams * 4:
        with torch.cuda.stream(s):
            got.append(kv.prefill_attn(q, *args, n_ctx=3000))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)


def test_results_do_not_vary():
    """No order of atomics shows: the same call gives the same bits."""
    table, n_pages = pages_for([5000, 200], np.random.default_rng(0))
    kp, vp = pool(1, n_pages, 2, 64, BF)
    q = normal((300, 8, 64), 2, BF)
    lead, shared = ints([0] * 40), ints([4990] * 40)
    for i in range(5):
        a = kv.prefill_attn(q, kp, vp, ints(table), ints([0, 200, 300]), ints([4800, 100]), n_ctx=5000)
        b = kv.decode_attn_shared(q[:40], kp, vp, ints(table[:1].repeat(40, 0)), ints([5000] * 40), lead, shared, n_ctx=5000)
        if i == 0:
            first = a, b
        assert torch.equal(a, first[0]) and torch.equal(b, first[1])


def test_calls_with_gradients_are_refused():
    kp, vp = pool(0, 3, 1, 32, F32)
    q = normal((1, 1, 32), 0, F32).requires_grad_()
    t, one = ints([[0]]), ints([1])
    for call in (lambda: kv.prefill_attn(q, kp, vp, t, ints([0, 1]), ints([0]), n_ctx=1),
                 lambda: kv.decode_attn_shared(q, kp, vp, t, one, ints([0]), ints([0]), n_ctx=1),
                 lambda: kv.write_slots(q, q, kp, vp, torch.zeros(1, dtype=torch.int64, device=DEV))):
        with pytest.raises(ValueError):
            call()
        with torch.no_grad():
            call()


def test_wrong_arguments_are_refused():
    kp, vp = pool(0, 3, 2, 32, BF)
    q = normal((5, 4, 32), 0, BF)
    t, off, st = ints([[0, 1]]), ints([0, 5]), ints([0])
    ok = dict(n_ctx=100)
    kv.prefill_attn(q, kp, vp, t, off, st, **ok)
    for args, kw in (((q[0], kp, vp, t, off, st), ok), ((q.float(), kp, vp, t, off, st), ok),
                     ((q[..., :16], kp, vp, t, off, st), ok), ((q, kp, vp, t, off[:1], st), ok),
                     ((q, kp, vp, t, off.long(), st), ok), ((q, kp, vp, t, off.cpu(), st), ok),
                     ((q, kp, vp, t, ints([0, 1, 5]), ints([0, 0])), ok), ((q, kp, vp, t, off, st), dict(n_ctx=129)),
                     ((q, kp, vp, t, off, st), dict(n_ctx=0)), ((q, kp, vp, t, off, st), dict(n_ctx=100, sink=1)),
                     ((q[:, :3], kp, vp, t, off, st), ok), ((q, kp, vp, t, off, st), dict(n_ctx=100, scale=-1.0)),
                     ((q, kp, vp, t, off, st), dict(n_ctx=100, out=torch.zeros(4, 4, 32, device=DEV))),
                     ((q, kp, vp, t, off, st), dict(n_ctx=100, lse=torch.zeros(5, 3, device=DEV))),
                     ((q.transpose(0, 1).contiguous().transpose(0, 1), kp, vp, t, off, st), ok),
                     ((q, kp, vp, t, off, st), dict(n_ctx=(1 << 32) + 1))):
        with pytest.raises((ValueError, TypeError, lla.LLAError)):
            kv.prefill_attn(*args, **kw)
    need = kv.prefill_workspace_bytes(BF, 1, 5, 4, 2, 32, 4096)
    assert need
    with pytest.raises(lla.LLAError) as e:
        kv.prefill_attn(q, kp, vp, ints(np.zeros((1, 64))), off, st, n_ctx=4096,
                        workspace=torch.zeros(need - 16, dtype=torch.uint8, device=DEV))
    assert e.value.status == lla.LLA_ERR_WORKSPACE
