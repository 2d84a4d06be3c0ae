"""The paged K/V cache's oracle against pure Python and closed forms (CPU)."""

import cmath
import math
import random

import numpy as np
import pytest

from oracle import kv_oracle as O


def test_rope_is_complex_multiplication():
    rng = np.random.default_rng(0)
    x, freq = rng.standard_normal(14), [1.0, 0.3, 0.02]
    for inter in (False, True):
        for pos, mag in ((0, 1.0), (7, 1.0), (-3, 1.25), (100000, 0.5)):
            y = O.kv_rope(x, pos, freq, inter, mag)
            for i, f in enumerate(freq):
                a, b = (2 * i, 2 * i + 1) if inter else (i, i + 3)
                z = complex(x[a], x[b]) * cmath.exp(1j * pos * f) * mag
                assert abs(complex(y[a], y[b]) - z) < 1e-12
            assert np.array_equal(y[6:], x[6:])
    # the transposed rotation is the adjoint: <g, R x> = <R^T g, x>
    g = rng.standard_normal(14)
    for inter in (False, True):
        lhs = g[:6] @ O.kv_rope(x, 11, freq, inter, 1.5)[:6]
        rhs = O.kv_rope(g, 11, freq, inter, 1.5, transpose=True)[:6] @ x[:6]
        assert abs(lhs - rhs) < 1e-12


def test_frequencies():
    plain, one = O.kv_rope_frequencies(64)
    assert one == 1.0 and plain[0] == 1.0 and plain[31] == pytest.approx(10000 ** (-62 / 64), rel=1e-15)
    assert np.allclose(O.kv_rope_frequencies(64, scaling="linear", factor=4.0)[0] * 4, plain, rtol=1e-15)
    ntk = O.kv_rope_frequencies(64, scaling="ntk", factor=4.0)[0]  # first pair kept, last interpolated
    assert ntk[0] == 1.0 and ntk[31] == pytest.approx(plain[31] / 4, rel=1e-14)
    yarn, mag = O.kv_rope_frequencies(128, scaling="yarn", factor=8.0, original=4096)
    plain = O.kv_rope_frequencies(128)[0]
    turns = 4096 * plain / (2 * math.pi)
    assert np.array_equal(yarn[turns > 40], plain[turns > 40]) and (turns > 40).any()
    assert np.allclose(yarn[turns < 0.9] * 8, plain[turns < 0.9], rtol=1e-15) and (turns < 0.9).any()
    assert np.all(np.diff(yarn) < 0) and mag == pytest.approx(1 + 0.1 * math.log(8))


def test_decode_against_loops():
    rng = np.random.default_rng(1)
    P, Hkv, H, d, S = 5, 2, 4, 6, 3
    k, v = rng.standard_normal((P, Hkv, 64, d)), rng.standard_normal((P, Hkv, d, 64))
    table, length = [[3, 1], [0, -1], [-1, -1]], [70, 9, 0]
    q = rng.standard_normal((4, H, d))
    rows = [1, 0, 2, -1]
    for sink, window in ((0, 0), (2, 5), (0, 66), (3, 100)):
        out, lse = O.kv_decode_attn(q, k, v, table, length, rows, sink=sink, window=window)
        for b, row in enumerate(rows):
            for h in range(H):
                w, z = [0.0] * d, 0.0
                for t in range(length[row] if row >= 0 else 0):
                    if window and not (t < sink or t >= length[row] - window):
                        continue
                    p, s = table[row][t // 64], t % 64
                    e = math.exp(sum(q[b, h, i] * k[p, h // 2, s, i] for i in range(d)) / math.sqrt(d))
                    z += e
                    for i in range(d):
                        w[i] += e * v[p, h // 2, i, s]
                if z == 0:
                    assert not out[b, h].any() and lse[b, h] == -math.inf
                else:
                    assert np.allclose(out[b, h], np.array(w) / z, atol=1e-12) and abs(lse[b, h] - math.log(z)) < 1e-12
    assert O.kv_seen(10, 2, 3) == [0, 1, 7, 8, 9] and O.kv_seen(4, 2, 3) == [0, 1, 2, 3] and O.kv_seen(0, 2, 3) == []


def test_tables_conserve_pages():
    """Whatever happens, refs count the entries and every page is free or held."""
    rnd = random.Random(2)
    t = O.KvTables(6, 5, 14)
    seen = set()
    for _ in range(3000):
        kind = rnd.choice(("reserve", "reserve", "fork", "free"))
        rows = rnd.sample(range(6), rnd.randint(1, 3))
        if kind == "reserve":
            status, start, pairs = t.reserve(rows, [rnd.choice((0, 1, 1, 30, 64, 130)) for _ in rows])
            seen.add((kind, status, bool(pairs)))
            for old, new in pairs:
                assert t.refs[old] >= 1 and t.refs[new] == 1
        elif kind == "fork":
            seen.add((kind, t.fork([rnd.randrange(6) for _ in rows], rows)))
        else:
            seen.add((kind, t.free_rows(rows)))
        held = [p for r in range(6) for p in t.table[r][:-(-t.length[r] // 64)]]
        assert [held.count(p) for p in range(14)] == t.refs
        assert sorted(t.free + sorted(set(held))) == list(range(14))
    assert seen >= {("reserve", 0, True), ("reserve", 0, False), ("reserve", 1, False), ("reserve", 2, False),
                    ("fork", 0), ("fork", 2), ("free", 0)}


def test_copy_on_write_by_turns():
    t = O.KvTables(3, 2, 8)
    t.reserve([0], [70])
    t.fork([0, 0], [1, 2])
    status, start, pairs = t.reserve([0, 1, 2], [1, 1, 1])
    # the first two take copies of the open page, the last holder keeps it
    assert status == 0 and start == [70] * 3 and pairs == [(1, 2), (1, 3)]
    assert [r[:2] for r in t.table] == [[0, 2], [0, 3], [0, 1]] and t.refs[:4] == [3, 1, 1, 1]
    t.free_rows([2, 1, 0])
    assert t.free[-4:] == [2, 3, 1, 0]  # met first: page 0 in row 2, then 1, 3, 2
