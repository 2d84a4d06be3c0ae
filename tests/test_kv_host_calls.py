"""Host-side checks of calls of the paged K/V cache beside the plain ones (no GPU needed)."""

import pytest
import torch

from paper_2607_15456_amd import kv, lla


def test_numbers_past_32_bits_are_refused():
    """Not cut to the library's int: a window of 2^32 + 5 is not one of 5."""
    for bad in (dict(n_ctx=(1 << 32) + 64), dict(n_ctx=64, window=(1 << 32) + 5), dict(n_ctx=64, window=1, sink=1 << 32),
                dict(n_ctx=64 - (1 << 32)), dict(n_ctx=1 << 31)):
        with pytest.raises(ValueError):
            kv.decode_workspace_bytes(torch.bfloat16, 1, 1, 1, 64, **bad)
    for bad in (dict(n_ctx=-1), dict(n_ctx=64, window=-1), dict(n_ctx=64, window=1, sink=-(1 << 31))):
        with pytest.raises(lla.LLAError):
            kv.decode_workspace_bytes(torch.bfloat16, 1, 1, 1, 64, **bad)
    assert kv.decode_workspace_bytes(torch.bfloat16, 1, 1, 1, 64, 64, 5, (1 << 31) - 1) == 0
