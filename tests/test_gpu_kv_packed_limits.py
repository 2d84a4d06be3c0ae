"""GPU parity of packed batches over the paged K/V cache at the limits of what their
headers allow: sums of lengths that do not fit 32 bits, batches of hundreds of entries,
more tiles than a launch has workgroups, weights with all of their bits.

Tolerances are those of tests/test_gpu_kv_packed.py.
"""

import numpy as np
import pytest
import torch

from paper_2607_15456_amd import kv
from tests import test_gpu_kv_packed as packed
from tests.helpers import f64
from tests.test_gpu_kv_packed import BF, DEV, F32, bounds, ints, near, normal, pages_for, places, pool, prefill_reference

pytestmark = pytest.mark.gpu


def pages_for_all(ends):
    """A table of pages for sequences of these ends, in any order."""
    return pages_for(ends, np.random.default_rng(len(ends)))


@pytest.mark.parametrize("B,total,least", [(1024, 1 << 22, 1 << 22), (512, 1 << 23, 1 << 23), (1024, (1 << 24) - 1, 1 << 30),
                                           (1000, 1 << 20, 900), (1024, 5000, (1 << 31) - 9)])
def test_slots_whose_lengths_add_up_past_32_bits(B, total, least):
    """offset[b] = min(total, the sum of the lengths before b), in which every sum of a part of the entries
    may be past the largest that is counted."""
    rng = np.random.default_rng(B)
    new = np.minimum(least + rng.integers(0, 7, B), 2 ** 31 - 1)
    start = rng.integers(0, 100, B)
    table = torch.arange(B, dtype=torch.int32, device=DEV)[:, None].repeat(1, 2)
    pages = kv.PageTable(table, ints(np.zeros(B)), ints(np.zeros(B)), ints(np.zeros(B + 1)))
    got = kv.slots(pages, ints(start), ints(new), total)
    offset = np.minimum(np.concatenate(([0], np.cumsum(new.astype(np.int64)))), total)
    assert got.offset.tolist() == offset.tolist()
    t = torch.arange(total, device=DEV)
    at = torch.as_tensor(offset).to(DEV)
    entry = torch.searchsorted(at[1:], t, right=True)
    some = entry < B
    entry = entry.clamp_max(B - 1)
    place = ints(start).long()[entry] + t - at[entry]
    assert torch.equal(got.entry.long(), torch.where(some, entry, -1))
    assert torch.equal(got.pos.long(), torch.where(some, place, -1))
    assert torch.equal(got.slot, torch.where(some & (place < 128), 64 * entry + place % 64, -1))


# ---------------------------------------------------------------------------
# more tiles than a launch has workgroups
# ---------------------------------------------------------------------------

def same_bits(x, y):
    return torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


@pytest.mark.parametrize("dtype,out_dtype,H,n,copies", [(BF, BF, 64, 257, 256), (BF, F32, 64, 257, 256), (BF, F32, 128, 3, 256),
                                                        (F32, F32, 128, 17, 128)])
def test_prefill_of_more_tiles_than_workgroups(dtype, out_dtype, H, n, copies):
    """A workgroup that takes a second tile leaves nothing of the first one in it, values that are not finite among
    them: four entries, one with such values, and copies of them that have to have the same bits."""
    d, starts = 32, [0, 5, 64, 100]
    table, n_pages = pages_for_all([s + n for s in starts])
    kp, vp = pool(1, n_pages, H, d, dtype)
    clean = vp.clone()
    vp[table[2, (64 + n // 2) // 64], :, 7, (64 + n // 2) % 64] = float("nan")  # of entry 2's token n // 2
    q = normal((4 * n, H, d), 3, dtype)
    t, st = ints(np.tile(table, (copies, 1))), ints(starts * copies)
    offset = ints(np.arange(4 * copies + 1) * n)
    assert 4 * copies * -(-n // (256 if dtype == BF else 16)) * H > 1 << 16
    out = kv.prefill_attn(q.repeat(copies, 1, 1), kp, vp, t, offset, st, n_ctx=64 * table.shape[1], out_dtype=out_dtype)
    one = out[:4 * n].clone()
    for i in range(copies):
        assert same_bits(out[4 * n * i:4 * n * (i + 1)], one), i
    bad = torch.zeros_like(one, dtype=torch.bool)
    bad[2 * n + n // 2:3 * n, :, 7] = True
    assert torch.equal(one.isfinite(), ~bad)
    heads = [0, 1, H - 1]
    ref = prefill_reference(q[:, heads].contiguous(), kp[:, heads], clean[:, heads], table, np.arange(5) * n, starts, None, d ** -0.5,
                            0, 0, dtype, out_dtype)
    ok = (~bad)[:, heads].cpu().numpy()
    got = one[:, heads].cpu()
    near(got[torch.as_tensor(ok)], ref[0][ok], ref[2][ok], f"{dtype} {out_dtype} {n}")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_shared_decode_of_more_tiles_than_workgroups(dtype):
    H, d, B = 128, 32, 1024
    table, n_pages = pages_for_all([70, 90, 130, 65])
    kp, vp = pool(1, n_pages, H, d, dtype)
    q = normal((4, H, d), 3, dtype)
    rows, length = ints(list(range(4)) * (B // 4)), ints([70, 90, 130, 65])
    lead, shared = ints([4 * (b // 4) for b in range(B)]), ints([50] * B)
    assert B * H > 1 << 16
    out = kv.decode_attn_shared(q.repeat(B // 4, 1, 1), kp, vp, ints(table), length, lead, shared, n_ctx=192, rows=rows)
    assert same_bits(out, out[:4].repeat(B // 4, 1, 1))
    kn, vn, qn = f64(kp), f64(vp), f64(q)
    for b, end in enumerate([70, 90, 130, 65]):
        for h in (0, H - 1):
            k, v = places(table, b, end, kn, vn, h)
            k[:50], v[:50] = places(table, 0, 50, kn, vn, h)
            ref, _, tol, _ = bounds(qn[b, h:h + 1], k, v, np.ones((1, end), dtype=bool), d ** -0.5, dtype, F32, 0.0)
            near(out[b, h:h + 1], ref, tol, f"entry {b} head {h}")


# ---------------------------------------------------------------------------
# batches of hundreds of entries
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("B,n_ctx,kind", [(65, 256, "mixed"), (130, 256, "tied"), (1024, 256, "mixed"), (1024, 192, "tied"),
                                          (300, 1000, "mixed"), (70, 1000, "tied")])
def test_prefill_of_many_entries(dtype, out_dtype, B, n_ctx, kind):
    """Empty entries, single tokens, few and many tokens at places that spread, or that are all the same, so
    that the order of the tiles goes by the entries' numbers alone.  Up to 256 places no tile is cut."""
    rng = np.random.default_rng(B + n_ctx)
    H, H_kv, d = 2, 2, 32
    if kind == "tied":
        new, start = np.full(B, 40), np.full(B, n_ctx - 40)
        new[5], new[B - 2] = 1, 0
    else:
        new = rng.choice([0, 1, 3, 16, 17, 30, 60], B)
        new[rng.integers(0, B, 3)] = 190
        start = rng.integers(0, n_ctx - new + 1)
    assert kind != "tied" or (new * H // H_kv > 16).sum() > 64
    seqs = 5  # whose pages all entries read
    table, n_pages = pages_for_all([n_ctx] * seqs)
    rows = rng.integers(0, seqs, B)
    kp, vp = pool(7, n_pages, H_kv, d, dtype)
    total = int(new.sum())
    q = normal((total + 3, H, d), 8, dtype)
    offset = np.concatenate(([0], np.cumsum(new)))
    out = torch.full((total + 3, H, d), 7.0, dtype=out_dtype, device=DEV)
    lse = torch.full((total + 3, H), 7.0, dtype=F32, device=DEV)
    kv.prefill_attn(q, kp, vp, ints(table), ints(offset), ints(start), n_ctx=n_ctx, rows=ints(rows), out=out, lse=lse)
    ref, ref_lse, tol, lse_tol = prefill_reference(q, kp, vp, table, offset, start, rows, d ** -0.5, 0, 0, dtype, out_dtype)
    near(out[:total], ref[:total], tol[:total], f"{B} entries, {kind}")
    near(lse[:total], ref_lse[:total], lse_tol[:total], f"{B} entries, {kind}, lse")
    assert (out[total:] == 7).all() and (lse[total:] == 7).all()


# ---------------------------------------------------------------------------
# weights keep all of their bits
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_results_in_bf16_are_those_in_fp32_rounded_once(dtype, d):
    """Whatever kind of tile an entry is of, and whatever else is in its batch: nothing but the results' rounding
    goes by the results' type."""
    ends = [700, 300, 64, 1500]
    table, n_pages = pages_for_all(ends)
    kp, vp = pool(d, n_pages, 2, d, dtype)
    t = ints(table)
    for new in ([300, 1, 5, 40], [1, 1, 64, 1], [0, 0, 0, 900]):
        q, start = normal((sum(new), 8, d), 5, dtype), [e - n for e, n in zip(ends, new)]
        offset = ints(np.concatenate(([0], np.cumsum(new))))
        for sink, window in ((0, 0), (3, 130)):
            one, two = (kv.prefill_attn(q, kp, vp, t, offset, ints(start), n_ctx=1536, sink=sink, window=window, out_dtype=o)
                        for o in (F32, BF))
            assert one.isfinite().all() and torch.equal(one.to(BF), two), (new, sink)
    q = normal((300, 8, d), 6, dtype)
    for B in (3, 130, 300):  # answers to one prompt
        args = (q[:B], kp, vp, t, ints([1500] * 4), ints([0] * B), ints([640] * B))
        one, two = (kv.decode_attn_shared(*args, n_ctx=1536, rows=ints([3] * B), out_dtype=o) for o in (F32, BF))
        assert one.isfinite().all() and torch.equal(one.to(BF), two), B


@pytest.mark.parametrize("out_dtype", [BF, F32])
def test_a_token_does_not_depend_on_its_batch(out_dtype):
    """The same entry alone, with more room, and among others: each time within what sums in 32 bits allow, which no
    rounding of weights to fewer bits is."""
    d, H = 128, 4
    table, n_pages = pages_for_all([900, 1000, 800])
    kp, vp = pool(3, n_pages, 1, d, BF)
    q = normal((700, H, d), 4, BF)
    t = ints(table)
    ref, _, tol, _ = prefill_reference(q[:6], kp, vp, table[:1], [0, 6], [890], None, d ** -0.5, 0, 0, BF, F32)
    calls = [(6, [0, 6], [890]), (700, [0, 6], [890]), (306, [0, 6, 306], [890, 700]), (6, [0, 6, 6, 6], [890, 0, 0])]
    for total, offset, start in calls:
        out = kv.prefill_attn(q[:total], kp, vp, t, ints(offset), ints(start), n_ctx=1024, out_dtype=out_dtype)[:6]
        near(out, ref, tol if out_dtype == F32 else tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref), f"{total} {offset}")


# ---------------------------------------------------------------------------
# shared prompts under a bound far above the lengths, from which on their tiles are large ones
# ---------------------------------------------------------------------------

def far_bound(monkeypatch, entries, H, d):
    """Tables that are wide enough for a bound at which the entries' products with all of it are past 3 * 2^30."""
    pages = -(-(3 << 30) // (entries * H * d * 64)) + 1

    def wide(ends, rng, spare=3):
        table, n = pages_for(ends, rng, spare)
        return np.concatenate((table, np.full((len(ends), max(0, pages - table.shape[1])), -1)), axis=1), n

    monkeypatch.setattr(packed, "pages_for", wide)


@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_shared_widths_under_a_far_bound(monkeypatch, out_dtype, d):
    far_bound(monkeypatch, 6, 6, d)
    packed.check_shared(BF, out_dtype, 6, 2, d, [(200, [5, 70, 1]), (0, [300]), (64, [0, 64])], seed=d)
    far_bound(monkeypatch, 40, 8, d)
    packed.check_shared(BF, out_dtype, 8, 1, d, [(900, [3] * 40)], seed=d)


@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("H,H_kv,groups", [(4, 2, [(300, [i % 5 for i in range(100)]), (700, [2] * 33)]), (300, 1, [(130, [5, 0, 80])]),
                                           (40, 2, [(130, [5, 0, 80]), (64, [1] * 9), (1, [1, 63])]), (4, 2, [(5000, [1, 100])]),
                                           (2, 2, [(64 * i + 3, [1] * (i % 40 + 1)) for i in range(12)]), (64, 1, [(65, [1] * 70)])])
def test_shared_runs_under_a_far_bound(monkeypatch, out_dtype, H, H_kv, groups):
    """Runs of few and of many rows side by side, cut inside, of more heads than a tile has rows."""
    far_bound(monkeypatch, sum(len(m) for _, m in groups), H, 64)
    packed.check_shared(BF, out_dtype, H, H_kv, 64, groups, seed=len(groups))


def test_shared_bad_indices_under_a_far_bound(monkeypatch):
    """NaN for those whose prompt cannot be read, in runs of few rows and of many, and no harm to the others."""
    far_bound(monkeypatch, 120, 4, 64)
    table, n_pages = packed.pages_for([200] * 8, np.random.default_rng(1))
    kp, vp = pool(1, n_pages, 2, 64, BF)
    B = 120
    q = normal((B, 4, 64), 2, BF)
    rows, lead, shared = np.arange(B) % 7, np.repeat([0, 0, 40, B, 80, -1], 20), np.full(B, 100)
    shared[45], rows[50], rows[51] = 201, -1, 8
    bad_table = table.copy()
    bad_table[rows[80], 1] = n_pages
    out = kv.decode_attn_shared(q, kp, vp, ints(bad_table), ints([200] * 8), ints(lead), ints(shared), n_ctx=64 * table.shape[1],
                                rows=ints(rows))
    nan = (lead < 0) | (lead == B) | (lead == 80) | (shared > 200) | (rows == 8) | (rows == rows[80])
    nan[50] = False
    assert (out[50] == 0).all()
    assert np.array_equal(out.isnan().all(2).all(1).cpu().numpy(), nan) and np.array_equal(out.isnan().any(2).any(1).cpu().numpy(), nan)
    kn, vn, qn = f64(kp), f64(vp), f64(q)
    for b in np.flatnonzero(~nan)[::7]:
        if b == 50:
            continue
        for h in range(4):
            k, v = places(table, rows[b], 200, kn, vn, h // 2)
            k[:100], v[:100] = places(table, rows[lead[b]], 100, kn, vn, h // 2)
            ref, _, tol, _ = bounds(qn[b, h:h + 1], k, v, np.ones((1, 200), dtype=bool), 1 / 8, BF, F32, 0.0)
            near(out[b, h:h + 1], ref, tol, f"entry {b} head {h}")


# ---------------------------------------------------------------------------
# entries with room for more tokens, from 1024 rows of which on those of more than 32 rows take large tiles
# ---------------------------------------------------------------------------

ROOM = 2100


@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_prefill_widths_with_room(out_dtype, d):
    packed.check_prefill(BF, out_dtype, 3, 1, d, [70, 1, 200], [0, 300, 13], seed=d, spare=ROOM)
    packed.check_prefill(BF, out_dtype, 2, 2, d, [300], [65], seed=d + 1, spare=ROOM)
    packed.check_prefill(BF, out_dtype, 2, 1, d, [3, 10, 16, 17, 9], [400, 0, 65, 130, 250], seed=d, spare=ROOM)


@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("H,H_kv", [(1, 1), (16, 16), (16, 2), (6, 2), (40, 2), (64, 1), (33, 1)])
def test_prefill_groups_with_room(out_dtype, H, H_kv):
    packed.check_prefill(BF, out_dtype, H, H_kv, 64, [5, 1, 37], [100, 0, 63], seed=H, spare=ROOM)
    packed.check_prefill(BF, out_dtype, H, H_kv, 64, [5], [100], seed=H, spare=ROOM)


@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("new,start", [([1], [0]), ([1], [64]), ([64], [0]), ([33], [31]), ([129], [4000]), ([0, 3, 0, 17, 1, 0], [5, 60, 0, 9, 700, 1]),
                                       ([300, 1, 1, 64], [0, 5000, 1, 64]), ([16, 17, 15, 32, 33], [0, 1, 2, 3, 4])])
def test_prefill_lengths_with_room(out_dtype, new, start):
    packed.check_prefill(BF, out_dtype, 4, 2, 128, new, start, seed=sum(new), spare=ROOM, fused=True)
    packed.check_prefill(BF, out_dtype, 4, 2, 96, new, start, seed=sum(new), spare=ROOM)


@pytest.mark.parametrize("sink,window", [(0, 1), (0, 64), (4, 60), (70, 100), (4, 100000), (1, 31), (500, 3)])
def test_prefill_windows_with_room(sink, window):
    packed.check_prefill(BF, BF, 4, 2, 64, [150, 1, 1, 280], [0, 400, 63, 700], sink, window, seed=window % 97, spare=ROOM)
    packed.check_prefill(BF, F32, 4, 2, 64, [14, 16, 1, 180], [0, 400, 63, 700], sink, window, seed=window % 97, spare=ROOM)


@pytest.mark.parametrize("offsets", [[0, 1500, 0, 1500, 0, 1500], [1500, 0, 1500, 0], [-5, 1600, -(1 << 31), (1 << 31) - 1, 3], [7] * 6])
def test_prefill_offsets_that_decrease_with_room(offsets):
    """Which tokens are done is not defined; nothing but the results and the workspace is written, and a call after it is whole."""
    B, total = len(offsets) - 1, 1500
    table, n_pages = pages_for_all([2500] * B)
    kp, vp = pool(1, n_pages, 2, 64, BF)
    q = normal((total, 4, 64), 2, BF)
    n_ctx = 64 * table.shape[1]
    need = kv.prefill_workspace_bytes(BF, B, total, 4, 2, 64, n_ctx)
    ws = torch.full((need + 65536,), 90, dtype=torch.uint8, device=DEV)
    out = torch.full((total + 64, 4, 64), 7.0, device=DEV)
    kv.prefill_attn(q, kp, vp, ints(table), ints(offsets), ints([800] * B), n_ctx=n_ctx, out=out[:total], workspace=ws[:need])
    assert (ws[need:] == 90).all() and (out[total:] == 7).all()
    kv.prefill_attn(q, kp, vp, ints(table[:1]), ints([0, total]), ints([900]), n_ctx=n_ctx, out=out[:total], workspace=ws[:need])
    ref = prefill_reference(q[:, [0, 3]].contiguous(), kp, vp, table[:1], [0, total], [900], None, 1 / 8, 0, 0, BF, F32)
    near(out[:total][:, [0, 3]], ref[0], ref[2], "after it")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("far", [False, True])
def test_an_empty_entry_shares_nothing(monkeypatch, dtype, far):
    """Places shared beyond a length of 0 are places shared beyond the length: NaN; with none shared, zeros."""
    if far:
        far_bound(monkeypatch, 40, 4, 64)
    table, n_pages = packed.pages_for([200, 100], np.random.default_rng(0))
    kp, vp = pool(1, n_pages, 2, 64, dtype)
    q, lse = normal((40, 4, 64), 2, dtype), torch.zeros((40, 4), device=DEV)
    rows, shared, lead = np.zeros(40, dtype=int), np.full(40, 90), np.zeros(40, dtype=int)
    rows[5], rows[6], shared[6], rows[7], shared[7], rows[8] = 1, 1, 0, 1, -3, -1
    out = kv.decode_attn_shared(q, kp, vp, ints(table), ints([200, 0]), ints(lead), ints(shared), n_ctx=64 * table.shape[1],
                                rows=ints(rows), lse=lse)
    for b in range(40):
        if b in (5, 7):
            assert out[b].isnan().all() and lse[b].isnan().all(), b
        elif b in (6, 8):
            assert (out[b] == 0).all() and (lse[b] == -np.inf).all(), b
        else:
            assert out[b].isfinite().all() and lse[b].isfinite().all(), b


# ---------------------------------------------------------------------------
# two graphs of one pool
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
def test_two_captured_steps_of_one_pool(dtype):
    """A packed step and a step over shared prompts, each captured once, replayed in turn with the program's own work
    between; both equal the eager ones of another pool.  The side stream waits for what the tensors hold."""
    a, b = packed.Server(dtype), packed.Server(dtype)
    width = a.H + 2 * a.H_kv
    result = torch.empty(4, dtype=torch.int32, device=DEV)
    first = normal((500, width, a.d), 30, dtype)
    for s in (a, b):
        s.step(ints([0, 2]), ints([200, 300]), first, 500)
        kv.fork(s.pages, ints([0, 0, 2]), ints([1, 4, 3]), result)
    rows, add = [ints([0, 1, 4, 2, 3, -1]), ints([2, 0, -1])], [ints([1] * 5 + [0]), ints([3, 7, 0])]
    totals, shared = (6, 12), (True, False)
    x = [torch.zeros((n, width, a.d), dtype=dtype, device=DEV) for n in totals]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for i in range(2):  # (loads kernels; the lengths grow alike in both)
        with torch.cuda.stream(side):
            a.step(rows[i], add[i], x[i], totals[i], shared[i])
        torch.cuda.current_stream().wait_stream(side)
        b.step(rows[i], add[i], x[i], totals[i], shared[i])
        side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    for i in range(2):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(a.step(rows[i], add[i], x[i], totals[i], shared[i]))
        graphs.append(g)
    for turn in range(8):
        i = turn % 2 if turn < 6 else 1
        xs = normal(tuple(x[i].shape), 50 + turn, dtype)
        if i:
            add[1].copy_(ints([turn, 9 - turn, 0]))
        x[i].copy_(xs)
        graphs[i].replay()
        want = b.step(rows[i], add[i], xs, totals[i], shared[i])
        torch.cuda.synchronize()
        used = totals[i] if shared[i] else int(add[i].clamp_min(0).sum())
        assert outs[i][:used].isfinite().all() and torch.equal(outs[i][:used], want[:used]), turn
        assert torch.equal(a.pages.length, b.pages.length) and torch.equal(a.pages.table, b.pages.table)
        (xs.float() @ xs.float().transpose(1, 2)).sum().item()  # the program's own work
