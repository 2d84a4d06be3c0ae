"""The paged K/V cache's oracle in calls beside the plain ones (CPU)."""

import random

from oracle import kv_oracle as O


def test_padding_changes_nothing():
    """Any call with rows of -1 between its own is the call without them."""
    rnd = random.Random(3)
    a, b = O.KvTables(6, 5, 14), O.KvTables(6, 5, 14)
    seen = set()
    for _ in range(2000):
        kind = rnd.choice(("reserve", "reserve", "fork", "free"))
        rows = rnd.sample(range(6), rnd.randint(0, 3))
        more = [rnd.choice((0, 1, 30, 130)) if kind == "reserve" else rnd.randrange(6) for _ in rows]
        padded = list(zip(rows, more))
        for _ in range(rnd.randint(0, 3)):
            padded.insert(rnd.randint(0, len(padded)), (-1, rnd.choice((-5, -1, 0, 3, 10 ** 6))))
        wide, beside = [p[0] for p in padded], [p[1] for p in padded]
        if kind == "reserve":
            (status, start, pairs), (want, want_start, want_pairs) = a.reserve(wide, beside), b.reserve(rows, more)
            assert [s for s, r in zip(start, wide) if r != -1] == want_start and pairs == want_pairs
            assert all(s == -1 for s, r in zip(start, wide) if r == -1)
        elif kind == "fork":
            status, want = a.fork(beside, wide), b.fork(more, rows)
        else:
            status, want = a.free_rows(wide), b.free_rows(rows)
        seen.add((kind, status))
        assert status == want and (a.table, a.length, a.refs, a.free) == (b.table, b.length, b.refs, b.free)
    assert {("reserve", 0), ("reserve", 2), ("fork", 0), ("fork", 2), ("free", 0)} <= seen
