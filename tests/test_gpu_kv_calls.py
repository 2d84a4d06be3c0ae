"""Calls of the paged K/V cache that its header and binding allow and that come up
in use beside the plain ones: against the definitions in 64 bits (EPS = 2^-24)."""

import numpy as np
import pytest
import torch

from paper_2607_15456_amd import kv, lla
from tests.helpers import f64, log
from tests.test_gpu_kv import BF, DEV, EPS, F32, Cache, normal

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
