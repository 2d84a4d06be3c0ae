"""GPU parity of packed batches over the paged K/V cache at the limits of what their
headers allow: sums of lengths that do not fit 32 bits, batches of hundreds of entries,
more tiles than a launch has workgroups, weights with all of their bits.

Tolerances are those of tests/test_gpu_kv_packed.py.
"""

import numpy as np
import pytest
import torch

from paper_2607_15456_amd import kv
from tests.test_gpu_kv_packed import DEV, ints

pytestmark = pytest.mark.gpu


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
