"""Host-side checks of calls of the paged K/V cache beside the plain ones (no GPU needed)."""

import pytest
import torch

from paper_2607_15456_amd import kv, lla
from tests.test_kv_host import CALLS, P


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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,H_kv,d", [(16, 16, 128), (16, 2, 128), (24, 8, 64), (64, 1, 96), (8, 8, 32), (40, 2, 256)])
@pytest.mark.parametrize("sink,window", [(0, 0), (4, 3000)])
def test_a_workspace_serves_smaller_calls(dtype, H, H_kv, d, sink, window):
    """What the largest batch and context of a program need is enough for all below."""
    sizes = [1, 2, 3, 5, 8, 15, 16, 17, 31, 33, 64, 200, 513]
    bounds = [1, 64, 129, 257, 500, 513, 1024, 1025, 1088, 2048, 2112, 3000, 4097, 8192, 16384, 20000, 32768, 40000, 131072]
    need = {(B, n): kv.decode_workspace_bytes(dtype, B, H, H_kv, d, n, sink, window) for B in sizes for n in bounds}
    assert any(need.values()) and not any(need[B, 64] for B in sizes)
    for i, B in enumerate(sizes):
        for j, n in enumerate(bounds):
            if i:
                assert need[sizes[i - 1], n] <= need[B, n], (B, n)
            if j:
                assert need[B, bounds[j - 1]] <= need[B, n], (B, n)


def test_write_at_refusals():
    """lla_kv_write_at is lla_kv_write with positions of its own: the same refusals, and theirs."""
    good, changes = CALLS["lla_kv_write"]
    place = list(good).index("start") + 1
    fn = kv.lib().lla_kv_write_at
    for arg, value in changes:
        args = list({**good, arg: value}.values())
        assert fn(*args[:place], None, *args[place:]) == lla.LLA_ERR_INVALID_ARG, (arg, value)
        assert fn(*args[:place], P, *args[place:]) == lla.LLA_ERR_INVALID_ARG, (arg, value)
    args = list(good.values())
    assert fn(*args[:place], P + 2, *args[place:]) == lla.LLA_ERR_INVALID_ARG


def test_no_kernel_is_built_that_nothing_launches():
    """Eight pairs a thread are for bf16 rows alone."""
    built = open(lla.LIB_PATH, "rb").read()
    for kernel in (b"rotary_kernel", b"write_few_kernel", b"write_page_kernel"):
        assert kernel + b"IfLi4" in built and kernel + b"ItLi8" in built and kernel + b"IfLi8" not in built, kernel
