"""Workspaces of packed batches and shared prompts where the kind of tiles changes (no GPU needed)."""

import pytest
import torch

from paper_2607_15456_amd import kv


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,H_kv,d", [(16, 16, 128), (16, 2, 64), (40, 2, 256), (300, 1, 32)])
def test_a_workspace_serves_calls_of_the_other_kind_of_tiles(dtype, H, H_kv, d):
    """Sizes on both sides of where a batch gets other tiles: what the larger one needs is enough."""
    for B in (1, 2, 16, 100, 1024):
        sizes = [kv.shared_workspace_bytes(dtype, B, H, H_kv, d, n) for n in (64, 4096, 20000, 100000, 1 << 20, 1 << 26)]
        assert sizes == sorted(sizes), B
    for n in (64, 5000, 100000, 1 << 24):
        sizes = [kv.shared_workspace_bytes(dtype, B, H, H_kv, d, n) for B in range(1, 1025, 31)]
        assert sizes == sorted(sizes), n


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,H_kv,d", [(16, 16, 128), (16, 2, 64), (11, 1, 96), (40, 2, 256), (300, 1, 32), (2048, 1, 32), (1024, 512, 32)])
def test_a_prefill_workspace_serves_calls_of_the_other_kinds_of_tiles(dtype, H, H_kv, d):
    """Few and many rows, of one entry and of several, down to the smallest bound."""
    for n in (64, 300, 5000, 100000):
        need = lambda B, total: kv.prefill_workspace_bytes(dtype, B, total, H, H_kv, d, n)  # noqa: E731, B023
        totals = sorted({1, 2, 30, 31, 32, 33, 63, 64, 65, 90, 100, 127, 128, 129, 500, 513, 1023, 1024, 1025, 3000})
        for B in (1, 2, 3, 40, 1024):
            sizes = [need(B, t) for t in totals]
            assert sizes == sorted(sizes), (n, B)
        for t in totals:
            sizes = [need(B, t) for B in (1, 2, 3, 5, 17, 64, 300, 1024)]
            assert sizes == sorted(sizes), (n, t)
