"""Calls of the paged K/V cache that its header and binding allow and that come up
in use beside the plain ones: against the definitions in 64 bits (EPS = 2^-24)."""

import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from paper_2607_15456_amd import kv, lla
from tests.helpers import f64, log
from tests.test_gpu_kv import BF, DEV, EPS, F32, Cache, check_decode, half_step, ints, near, normal, rope_bound, same_tables

pytestmark = pytest.mark.gpu


def rope_abi(x, freq, pos, pos_tokens, pos0):
    """lla_rope_positions itself on a dense x."""
    B, M, H, d = x.shape
    y, strides = torch.empty_like(x), (M * H * d, H * d, d)
    kv._call("lla_rope_positions", x.device, lla._dt(x), B, M, H, d, 2 * freq.numel(), 0, 0, x.data_ptr(), *strides,
             None if pos is None else pos.data_ptr(), pos_tokens, pos0, freq.data_ptr(), 1.0, y.data_ptr(), *strides)
    return y


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rope_without_positions_counts_tokens(dtype):
    """pos NULL: token m is at pos0 + m, whatever pos_tokens says."""
    freq, _ = kv.rope_frequencies(64)
    x = normal((2, 37, 3, 64), 1, dtype)
    want = kv.rope(x, freq, pos0=11)
    for pos_tokens in (0, 1, -1):
        assert torch.equal(rope_abi(x, freq, None, pos_tokens, 11), want), pos_tokens


def two_token_weights(dtype, B, H):
    """Entries of two tokens: the first's score is 0 and its values 0, the second's
    score is a product that 32 bits hold, its values 1.  Results are w / (1 + w)."""
    c = Cache(dtype, [2] * B, 1, 64, seed=1)
    q, b = torch.zeros((B, H, 64), dtype=dtype, device=DEV), normal((B,), 2, F32).abs().clamp(0.1, 2.0).to(dtype)
    q[:, :, 0] = normal((B, H), 3, F32).abs().clamp(0.1, 2.0).to(dtype)
    page = c.table[:, 0].long()
    c.k[page, 0, :2] = 0
    c.k[page, 0, 1, 0] = -b
    c.v[page, 0, :, 0] = 0
    c.v[page, 0, :, 1] = 1
    return c, q, np.exp(-f64(q[:, :, 0]) * f64(b)[:, None])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_decode_weights_keep_32_bits(dtype):
    """Scores of at most 4: off by 8 EPS (two roundings), so the weight by 10 with its
    exponential; sum and product take 4 roundings, the sum's share of the weight's
    error is half of it at most, the division 1: 20 EPS in all, held to 32 (2^-19).
    A weight cut to two bf16 is off by up to 256."""
    c, q, w = two_token_weights(dtype, 60, 40)
    lse = torch.empty((60, 40), device=DEV)
    out = f64(kv.decode_attn(q, c.k, c.v, c.table, c.length, n_ctx=2, scale=1.0, lse=lse))
    off = np.abs(out / (w / (1 + w))[..., None] - 1) / EPS
    log(f"  {off.max():.1f} EPS")
    assert off.max() <= 32
    assert np.max(np.abs(f64(lse) - np.log1p(w))) <= 32 * EPS


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lengths", [[40], [3000, 100]])
def test_decode_of_far_scores(dtype, lengths):
    """Finite scores of up to 200 * 2^40, of which the greatest stands alone: its
    values are the result, and it is the lse."""
    c = Cache(dtype, lengths, 1, 64, seed=2)
    q = torch.zeros((len(lengths), 2, 64), dtype=dtype, device=DEV)
    q[:, 0, 0], q[:, 1, 0] = 2.0 ** 20, 2.0 ** 15
    want = []
    for i, n in enumerate(lengths):
        t = torch.arange(n, device=DEV)
        page = c.table[i].long()[t // 64]
        level = (t * 37 % 101 + 1).float()
        level[n // 3] = 200
        c.k[page, 0, t % 64] = 0
        c.k[page, 0, t % 64, 0] = (level * 2.0 ** 20).to(dtype)
        want.append(f64(c.v[page[n // 3], 0, :, n // 3 % 64]))
    lse = torch.empty((len(lengths), 2), device=DEV)
    out = f64(kv.decode_attn(q, c.k, c.v, c.table, c.length, n_ctx=max(lengths), scale=1.0, lse=lse))
    for h, top in ((0, 200 * 2.0 ** 40), (1, 200 * 2.0 ** 35)):
        assert np.array_equal(out[:, h], np.stack(want)), h
        # the factor log2(e), the score, the lse: a rounding each, and ln 2's
        assert np.all(np.abs(f64(lse)[:, h] - top) <= 5 * EPS * top)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [1, 300, 9000])
def test_decode_of_infinite_and_large_values(dtype, n):
    """An attended value that is not finite makes its feature's result not finite and
    no other; values of 2^100 are averaged as any others."""
    c = Cache(dtype, [n], 1, 64, seed=3)
    q = normal((1, 3, 64), 4, dtype)
    plain = kv.decode_attn(q, c.k, c.v, c.table, c.length, n_ctx=n)
    v = c.v.clone()
    page, t = int(c.table[0, (n - 1) // 64]), (n - 1) % 64
    v[page, 0, 3, t], v[page, 0, 5, t], v[page, 0, 9, t] = float("inf"), -float("inf"), float("nan")
    out = kv.decode_attn(q, c.k, v, c.table, c.length, n_ctx=n)
    bad = torch.zeros(64, dtype=torch.bool, device=DEV)
    bad[[3, 5, 9]] = True
    assert not torch.isfinite(out[..., bad]).any() and torch.equal(out[..., ~bad], plain[..., ~bad])
    c.v *= 2.0 ** 100  # (a power of two: the same roundings)
    assert torch.equal(kv.decode_attn(q, c.k, c.v, c.table, c.length, n_ctx=n), plain * 2.0 ** 100)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_decode_workspace_of_the_largest_call_serves_all(dtype):
    """A program's one workspace, for its most entries and longest context, in every
    call below: the same bits as with one of its own."""
    c = Cache(dtype, [2112, 2048, 1088, 1024, 300, 77, 5000, 700], 4, 128, seed=6)
    q = normal((8, 8, 128), 7, dtype)
    ws = torch.empty(kv.decode_workspace_bytes(dtype, 8, 8, 4, 128, 5000), dtype=torch.uint8, device=DEV)
    for B, n in ((1, 1024), (1, 1088), (1, 2048), (1, 2112), (2, 5000), (3, 2112), (7, 4097), (8, 5000), (8, 64), (5, 257)):
        args = (q[:B], c.k, c.v, c.table, c.length.clamp(max=n))
        assert torch.equal(kv.decode_attn(*args, n_ctx=n, workspace=ws), kv.decode_attn(*args, n_ctx=n)), (B, n)


@pytest.mark.parametrize("dtype,most", [(BF, 131072), (F32, 131072), (BF, 20000)])
def test_decode_splits_an_entry_under_a_far_bound(dtype, most):
    """A bound far above the lengths (a step captured once for a sequence's whole
    life) does not leave an entry to one workgroup a head: the partials of eight
    slices and more are laid into the workspace."""
    n, H, d = 4096, 16, 128
    c = Cache(dtype, [n, 70, 0], H, d, seed=5, max_pages=-(-most // 64))
    q = normal((3, H, d), 99, dtype)
    ws = torch.full((kv.decode_workspace_bytes(dtype, 3, H, H, d, most),), 0xa5, dtype=torch.uint8, device=DEV)
    for b in (1, 3):
        ws.fill_(0xa5)
        out = kv.decode_attn(q[:b], c.k, c.v, c.table, c.length, n_ctx=most, workspace=ws)
        assert int((ws.view(torch.int32) != -0x5a5a5a5b).sum()) >= (8 if b == 1 else 4) * H * (d + 1), b
        assert torch.isfinite(out).all()
    check_decode(c, H, n_ctx=most)


def test_rope_takes_gradients():
    """Backward of rope is the transposed call, through views, shared rows and a
    second derivative, and against differences."""
    freq, mag = kv.rope_frequencies(32, scaling="yarn", factor=2.0, original=128)
    fused, g = normal((2, 9, 6, 64), 5, F32).requires_grad_(), normal((2, 9, 2, 64), 6, F32)
    args = dict(pos=ints([3, 900]), magnitude=mag, interleaved=True)
    pos = np.broadcast_to((np.array([3, 900])[:, None] + np.arange(9))[..., None], (2, 9, 2))
    y = kv.rope(fused[:, :, 2:4], freq, **args)
    assert y.requires_grad
    (y * g).sum().backward()
    ref = O.kv_rope(f64(g), pos, f64(freq), True, mag, transpose=True)
    tol = rope_bound(f64(g), 16, True, mag, ref, F32)
    near(fused.grad[:, :, 2:4], ref, tol, "gradient of a slice")
    assert not fused.grad[:, :, :2].any() and not fused.grad[:, :, 4:].any()
    # one row that every head and token shares: gradients add up
    row = normal((2, 1, 1, 64), 7, F32).requires_grad_()
    got, = torch.autograd.grad(kv.rope(row.expand(2, 9, 2, 64), freq, **args), row, g)
    near(got, ref.sum((1, 2), keepdims=True), tol.sum((1, 2), keepdims=True) + 18 * EPS * np.abs(ref).sum((1, 2), keepdims=True),
         "a shared row")
    # a gradient without strides of its own, the transposed call's gradient, and a derivative of the gradient
    x = normal((2, 9, 2, 64), 8, F32).requires_grad_()
    got, = torch.autograd.grad(kv.rope(x, freq, **args).sum(), x)
    one = O.kv_rope(np.ones((2, 9, 2, 64)), pos, f64(freq), True, mag, transpose=True)
    near(got, one, rope_bound(np.ones(one.shape), 16, True, mag, one, F32), "gradient of a sum")
    got, = torch.autograd.grad(kv.rope(x, freq, transpose=True, **args), x, g)
    back = O.kv_rope(f64(g), pos, f64(freq), True, mag)
    near(got, back, rope_bound(f64(g), 16, True, mag, back, F32), "gradient of the transposed")
    gg = g.clone().requires_grad_()
    first, = torch.autograd.grad(kv.rope(x, freq, **args), x, gg, create_graph=True)
    second, = torch.autograd.grad(first, gg, g)
    near(second, back, rope_bound(f64(g), 16, True, mag, back, F32), "derivative of the gradient")
    # differences: rope is linear
    e = normal((2, 9, 2, 64), 9, F32)
    with torch.no_grad():
        slope = np.sum(f64(g) * (f64(kv.rope(x + e, freq, **args)) - f64(kv.rope(x - e, freq, **args)))) / 2
    assert abs(slope - np.sum(ref * f64(e))) <= 1e-6 * np.sum(np.abs(f64(g))) * 6


def test_rope_gradient_keeps_its_positions():
    """Positions that a step overwrites before the backward pass (reserve writes its
    start without torch's knowledge) are the forward's in the gradient."""
    freq, _ = kv.rope_frequencies(64)
    x, g, pos = normal((2, 3, 2, 64), 5, BF).requires_grad_(), normal((2, 3, 2, 64), 6, BF), ints([5, 70])
    y = kv.rope(x, freq, pos=pos)
    pages, result, pairs = kv.new_page_table(2, 4, 8), ints([0] * 4), ints([[0, 0]] * 2)
    kv.reserve(pages, ints([0, 1]), ints([1, 1]), pos, pairs, result)
    got, = torch.autograd.grad(y, x, g)
    assert pos.tolist() == [0, 0] and torch.equal(got, kv.rope(g, freq, pos=ints([5, 70]), transpose=True))


def test_rope_in_place_does_not_lose_gradients():
    freq, _ = kv.rope_frequencies(64)
    x = normal((1, 4, 2, 64), 5, F32)
    leaf = x.clone().requires_grad_()
    for a, out in ((leaf, torch.empty_like(x)), (leaf * 1, None), (x, leaf)):
        with pytest.raises(ValueError):
            kv.rope(a, freq, out=a if out is None else out)
    with pytest.raises(ValueError):
        kv.rope(x, freq.clone().requires_grad_())
    with torch.no_grad():
        want = kv.rope(leaf, freq)
        assert torch.equal(kv.rope(leaf, freq, out=torch.empty_like(x)), want) and not want.requires_grad
        kv.rope(leaf, freq, out=leaf)
    assert torch.equal(leaf, want)
    assert not kv.rope(x, freq).requires_grad


def test_rows_of_a_padded_batch():
    """Rows of -1 pass through every call of a step: no room taken, start -1, nothing
    written, zeros; several of them, and a batch of nothing else."""
    pages, t = kv.new_page_table(5, 6, 20), O.KvTables(5, 6, 20)
    result = ints([0] * 4)

    def reserve(rows, add, n):
        start, pairs = ints([-9] * n), ints([[-9, -9]] * n)
        kv.reserve(pages, ints(rows), ints(add), start, pairs, result)
        status, want, want_pairs = t.reserve(rows, add)
        assert start.tolist() == want and pairs[:len(want_pairs)].tolist() == [list(p) for p in want_pairs]
        assert result[0] == status and result[3] == len(t.free)
        same_tables(pages, t)
        return status

    assert reserve([-1, 2, -1, 0], [1, 70, -5, 3], 4) == O.OK
    assert reserve([-1, -1], [1, 1], 2) == O.OK
    kv.fork(pages, ints([0, -1, 2, 77]), ints([1, -1, 4, -1]), result)
    assert t.fork([0, -1, 2, 77], [1, -1, 4, -1]) == O.OK == int(result[0])
    same_tables(pages, t)
    assert reserve([-1, 4, 2, 0, -1, 1], [1] * 6, 6) == O.OK
    assert reserve([-1, 2, -1, 2], [1] * 4, 4) == O.BAD
    assert reserve([-2, 2], [1] * 2, 2) == O.BAD
    kv.fork(pages, ints([-1]), ints([3]), result)  # a source is a sequence
    assert t.fork([-1], [3]) == O.BAD == int(result[0])
    kv.free(pages, ints([-1, 1, -1, 0]), result)
    assert t.free_rows([-1, 1, -1, 0]) == O.OK == int(result[0])
    same_tables(pages, t)
    kv.free(pages, ints([-1] * 3), result)
    assert t.free_rows([-1] * 3) == O.OK and result.tolist() == [0, 0, 0, len(t.free)]
    same_tables(pages, t)


def test_captured_step_with_padding():
    """One captured step of four entries replayed with fewer and other live
    sequences: as the eager step of these alone."""
    dtype, H, Hkv, d, n_ctx = BF, 4, 2, 64, 64 * 6

    def program(n):
        pages = kv.new_page_table(6, 6, 40)
        k, v = (x.zero_() for x in kv.alloc_pages(40, Hkv, d, dtype))
        freq, _ = kv.rope_frequencies(d)
        rows, add, start, pairs, result = ints([-1] * n), ints([1] * n), ints([0] * n), ints([[0, 0]] * n), ints([0] * 4)
        x = torch.zeros((n, 1, H + 2 * Hkv, d), dtype=dtype, device=DEV)
        out = torch.zeros((n, H, d), device=DEV)

        def step():
            kv.reserve(pages, rows, add, start, pairs, result)
            kv.copy_pages(k, v, pairs, result)
            kv.write(x[:, :, H:H + Hkv], x[:, :, H + Hkv:], k, v, pages.table, start, rows=rows, freq=freq)
            q = kv.rope(x[:, :, :H], freq, pos=start)
            kv.decode_attn(q[:, 0].contiguous(), k, v, pages.table, pages.length, rows=rows, n_ctx=n_ctx, out=out)
        return step, rows, x, out, pages, (k, v), result

    captured, eager = program(4), {n: program(n) for n in (1, 2, 3, 4)}
    whole = eager[4]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    captured[0]()  # (with padding alone: nothing changes)
    torch.cuda.synchronize()
    assert not captured[4].length.any() and int(captured[4].free[0]) == 40
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        captured[0]()
    for i, rows in enumerate(([0, 1, 2, 3], [1, -1, 3, -1], [-1, -1, -1, 5], [4, 3, -1, 0], [-1] * 4, [5, 4, 2, 1])):
        x = normal((4, 1, H + 2 * Hkv, d), 40 + i, dtype)
        captured[1].copy_(ints(rows))
        captured[2].copy_(x)
        g.replay()
        live = [j for j in range(4) if rows[j] >= 0]
        if i % 2:
            torch.cuda.synchronize()
        if live:  # the same step without padding, over the same tables and pools
            p = eager[len(live)]
            for mine, its in zip((*p[4], *p[5]), (*whole[4], *whole[5])):
                mine.copy_(its)
            p[1].copy_(ints([rows[j] for j in live]))
            p[2].copy_(x[live])
            p[0]()
            if p is not whole:
                for mine, its in zip((*whole[4], *whole[5]), (*p[4], *p[5])):
                    mine.copy_(its)
            assert torch.equal(captured[3][live], p[3]), i
        assert captured[6][0] == 0 and not captured[3][[j for j in range(4) if j not in live]].any(), i
        for mine, its in zip((*captured[4], *captured[5]), (*whole[4], *whole[5])):
            assert torch.equal(mine, its), i


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,inter", [(1, False), (3, True), (70, False)])
def test_write_turns_to_given_positions(dtype, M, inter):
    """pos: a token's place in the cache is start + m, its key's angle pos + m; the same as
    rope to these positions and a write that does not turn."""
    c, d, Hkv, B = Cache(dtype, [200] * 3, 2, 64, seed=7), 64, 2, 3
    fused = normal((B, M, 3, Hkv, d), 20, dtype)
    k, v = fused[:, :, 1], fused[:, :, 2]
    freq, mag = kv.rope_frequencies(48, scaling="yarn", factor=2.0, original=100)
    start, pos = [61, 0, -1], [5000, -3, 7]
    k0, v0 = c.k.clone(), c.v.clone()
    kv.write(k, v, c.k, c.v, c.table, ints(start), pos=ints(pos), freq=freq, interleaved=inter, magnitude=mag)
    for b in (0, 1):
        t = torch.arange(start[b], start[b] + M, device=DEV)
        page = c.table[b].long()[t // 64]
        at = np.broadcast_to((pos[b] + np.arange(M))[:, None], (M, Hkv))
        ref = O.kv_rope(f64(k[b]), at, f64(freq), inter, mag)
        near(c.k[page, :, t % 64], ref, rope_bound(f64(k[b]), 24, inter, mag, ref, dtype), f"entry {b}")
        assert torch.equal(c.v[page, :, :, t % 64], v[b])
        c.k[page, :, t % 64], c.v[page, :, :, t % 64] = k0[page, :, t % 64], v0[page, :, :, t % 64]
    bits = torch.int16 if dtype == BF else torch.int32
    assert torch.equal(c.k.view(bits), k0.view(bits)) and torch.equal(c.v.view(bits), v0.view(bits))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("fused", [True, False])
def test_steps_after_an_eviction(dtype, fused):
    """After gather keeps a part of a sequence, its next tokens are written behind the
    kept ones and turned to their true positions (in the write, or by rope before it):
    attention is the softmax over the kept and the new tokens at the positions they
    were generated at."""
    H, Hkv, d, n = 4, 2, 64, 400
    pages = kv.new_page_table(2, 8, 20)
    k, v = kv.alloc_pages(20, Hkv, d, dtype)
    k.fill_(float("nan"))
    v.fill_(float("nan"))
    freq, mag = kv.rope_frequencies(d, scaling="yarn", factor=4.0, original=64)
    start, pairs, result = ints([0]), ints([[0, 0]]), ints([0] * 4)
    row, other, keys, values = ints([0]), ints([1]), [], []

    def put(x, pos):
        kv.reserve(pages, row, ints([x.shape[1]]), start, pairs, result)
        key, val = x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
        if fused:
            kv.write(key, val, k, v, pages.table, start, rows=row, pos=ints([pos]), freq=freq, magnitude=mag)
        else:
            kv.write(kv.rope(key, freq, pos=ints([pos]), magnitude=mag), val, k, v, pages.table, start, rows=row)
        at = np.broadcast_to((pos + np.arange(x.shape[1]))[:, None], (x.shape[1], Hkv))
        keys.extend(O.kv_rope(f64(key[0]), at, f64(freq), magnitude=mag))
        values.extend(f64(val[0]))

    put(normal((1, n, H + 2 * Hkv, d), 30, dtype), 0)
    keep = [0, 1] + list(range(100, 300, 7)) + list(range(n - 20, n))
    kv.fork(pages, row, other, result)
    kv.free(pages, row, result)
    kv.reserve(pages, row, ints([len(keep)]), start, pairs, result)
    kv.gather(k, v, pages.table, other, row, ints([keep]))
    kv.free(pages, other, result)
    keys[:], values[:] = [keys[i] for i in keep], [values[i] for i in keep]
    for step in range(3):
        pos = n + step
        x = normal((1, 1, H + 2 * Hkv, d), 31 + step, dtype)
        put(x, pos)
        assert int(pages.length[0]) == len(keep) + step + 1 and int(start) == len(keep) + step
        q = kv.rope(x[:, :, :H], freq, pos=ints([pos]), magnitude=mag)
        out = f64(kv.decode_attn(q[:, 0].contiguous(), k, v, pages.table, pages.length, rows=row, n_ctx=512))
        q64 = O.kv_rope(f64(x[0, 0, :H]), np.full(H, pos), f64(freq), magnitude=mag)
        for h in range(H):
            kh, vh = np.stack(keys)[:, h // 2], np.stack(values)[:, h // 2]
            s = kh @ q64[h] / 8
            p = np.exp(s - s.max()) / np.exp(s - s.max()).sum()
            # stored keys and queries are rounded once: scores off by 2 * 2^-8 (2^-24) of sum |q k|
            ds = 2 * (2 * half_step(dtype) + 70 * EPS) * np.max(np.abs(kh) @ np.abs(q64[h])) / 8
            assert np.all(np.abs(out[0, h] - p @ vh) <= (2 * ds + 1e-5) * (p @ np.abs(vh))), (step, h)


def test_positions_past_32_bits_are_refused():
    """A whole number that the library's int would cut is refused, not cut."""
    freq, _ = kv.rope_frequencies(64)
    c = Cache(BF, [64], 1, 64)
    x, q = normal((1, 2, 1, 64), 1, BF), normal((1, 1, 64), 2, BF)
    for pos0 in (1 << 31, -(1 << 31) - 1, 1 << 32):
        with pytest.raises(ValueError):
            kv.rope(x, freq, pos0=pos0)
    near(kv.rope(x, freq, pos0=(1 << 31) - 2), ref := O.kv_rope(f64(x), (1 << 31) - 2 + np.arange(2)[None, :, None], f64(freq)),
         rope_bound(f64(x), 32, False, 1.0, ref, BF), "the last position")
    for bad in (dict(n_ctx=(1 << 32) + 64), dict(n_ctx=64, window=(1 << 32) + 5), dict(n_ctx=64, window=1, sink=1 << 32)):
        with pytest.raises(ValueError):
            kv.decode_attn(q, c.k, c.v, c.table, c.length, **bad)
