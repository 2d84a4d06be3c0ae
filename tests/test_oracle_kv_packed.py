"""Pins of the oracle of packed batches and shared prompts (CPU)."""

import math

import numpy as np

from oracle import kv_oracle as O


def test_slots_by_hand():
    table = [[7, 2, -1], [4, 0, 1]]
    offset, entry, pos, slot = O.kv_slots(table, [63, 126, -1], [2, 3, 1], 8, 8, rows=[0, 1, -1])
    assert offset == [0, 2, 5, 6]
    assert entry == [0, 0, 1, 1, 1, 2, -1, -1]
    assert pos == [63, 64, 126, 127, 128, -1, -1, -1]
    assert slot == [7 * 64 + 63, 2 * 64, 62, 63, 64, -1, -1, -1]
    assert O.kv_slots(table, [0], [5], 3, 8)[0] == [0, 3]
    assert O.kv_slots(table, [126], [3], 3, 8)[3] == [2 * 64 + 62, 2 * 64 + 63, -1]  # the third page is none
    assert O.kv_slots(table, [3], [1], 1, 8, pos0=[900])[2:] == ([900], [7 * 64 + 3])


def test_shared_prefix_by_hand():
    table = [[5, 6, 7], [5, 6, 8], [5, 6, 9], [1, 6, 7], [1, 2, 3]]
    assert O.kv_shared_prefix(table, [192, 150, 100, 192, 30], 10) == ([0, 0, 0, 3, 3], [100, 100, 100, 30, 30])
    assert O.kv_shared_prefix(table, [192, 150, 100, 192, 30], 10, least=31) == ([0, 0, 0, 3, 4], [100, 100, 100, 0, 0])
    assert O.kv_shared_prefix(table, [192] * 5, 10, rows=[0, 0, -1, 1]) == ([0, 0, 2, 3], [192, 192, 0, 0])


def test_prefill_is_a_decode_at_every_token():
    rng = np.random.default_rng(0)
    k, v = rng.normal(size=(6, 2, 64, 8)), rng.normal(size=(6, 2, 8, 64))
    table = [[3, 1, 5], [0, 2, -1]]
    q = rng.normal(size=(7, 4, 8))
    for sink, window in ((0, 0), (2, 5)):
        out, lse = O.kv_prefill_attn(q, k, v, table, [0, 4, 5], [61, 100], sink=sink, window=window)
        for t, (b, n) in enumerate([(0, 62), (0, 63), (0, 64), (0, 65), (1, 101)]):
            lengths = [0, 0]
            lengths[b] = n
            ref, ref_lse = O.kv_decode_attn(q[t][None], k, v, table, lengths, rows=[b], sink=sink, window=window)
            assert np.allclose(out[t], ref[0], rtol=1e-12, atol=1e-14) and np.allclose(lse[t], ref_lse[0], rtol=1e-12)
        assert np.isnan(out[5:]).all()


def test_prefill_brute_force():
    rng = np.random.default_rng(1)
    k, v, q = rng.normal(size=(2, 1, 64, 4)), rng.normal(size=(2, 1, 4, 64)), rng.normal(size=(2, 1, 4))
    out, lse = O.kv_prefill_attn(q, k, v, [[1, 0]], [0, 2], [63], scale=0.7)
    for t, p in enumerate((63, 64)):
        w = [math.exp(0.7 * sum(q[t, 0, i] * k[1 - n // 64, 0, n % 64, i] for i in range(4))) for n in range(p + 1)]
        for i in range(4):
            want = sum(w[n] * v[1 - n // 64, 0, i, n % 64] for n in range(p + 1)) / sum(w)
            assert abs(out[t, 0, i] - want) < 1e-12
        assert abs(lse[t, 0] - math.log(sum(w))) < 1e-12
