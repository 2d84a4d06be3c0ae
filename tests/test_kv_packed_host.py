"""Host-side checks of packed batches and shared prompts over the paged K/V cache (no GPU
needed): every refusal, and the workspaces; no call here reaches a kernel."""

import math

import pytest
import torch

from paper_2607_15456_amd import kv, lla

P = 1 << 20  # an aligned address that no call gets to use

# name: the arguments of a call that is accepted but for its null stream's work
# (never made), then the single changes that have to be refused
CALLS = {
    "lla_kv_slots": (
        dict(B=2, total=9, n_seqs=2, max_pages=8, n_pages=16, table=P, rows=None, start=P, pos0=None, n_new=P, offset=P,
             entry=P, pos=P, slot=P, stream=None),
        [("B", 0), ("B", 1025), ("total", 0), ("total", 1 << 24), ("n_seqs", 0), ("max_pages", 0), ("max_pages", (1 << 20) + 1),
         ("n_pages", 0), ("table", None), ("rows", P + 2), ("start", None), ("pos0", P + 1), ("n_new", None), ("offset", None),
         ("entry", P + 2), ("pos", None), ("slot", None), ("slot", P + 4)]),
    "lla_kv_write_slots": (
        dict(dtype=1, total=9, H_kv=4, d_head=64, d_rot=64, interleaved=0, k=P, k_t=768, v=P, v_t=256, freq=P, magnitude=1.0,
             n_pages=16, slot=P, pos=P, k_pages=P, v_pages=P, stream=None),
        [("dtype", 2), ("total", 0), ("total", -1), ("H_kv", 0), ("H_kv", 65536), ("d_head", 40), ("d_head", 288), ("d_rot", 72),
         ("d_rot", 4), ("d_rot", 0), ("k", None), ("k", P + 8), ("k_t", 4), ("k_t", -8), ("v", None), ("v_t", 2), ("freq", None),
         ("freq", P + 4), ("magnitude", math.nan), ("n_pages", 0), ("n_pages", (1 << 30) + 1), ("slot", None), ("slot", P + 4),
         ("pos", None), ("pos", P + 2), ("k_pages", None), ("v_pages", P + 8)]),
    "lla_kv_prefill_attn": (
        dict(dtype=1, out_dtype=1, B=2, total=9, H=8, H_kv=4, d_head=64, n_seqs=2, max_pages=8, n_pages=16, n_ctx=64, sink=0,
             window=0, table=P, rows=None, offset=P, start=P, q=P, q_t=512, k_pages=P, v_pages=P, scale=0.125, out=P, lse=None,
             workspace=P, ws_bytes=1 << 32, stream=None),
        [("dtype", 2), ("out_dtype", -1), ("B", 0), ("B", 1025), ("total", 0), ("total", 1 << 24), ("H", 0), ("H", 6), ("H_kv", 0),
         ("H_kv", 3), ("d_head", 48), ("d_head", 512), ("n_seqs", 0), ("max_pages", 0), ("n_pages", 0), ("n_ctx", 0), ("n_ctx", 513),
         ("sink", -1), ("sink", 1), ("window", -1), ("table", None), ("rows", P + 2), ("offset", None), ("offset", P + 2),
         ("start", None), ("q", None), ("q", P + 8), ("q_t", 4), ("q_t", -8), ("k_pages", None), ("v_pages", P + 4), ("scale", 0.0),
         ("scale", -1.0), ("scale", math.nan), ("scale", 3e38), ("out", None), ("lse", P + 1)]),
    "lla_pages_shared": (
        dict(B=2, least=1, rows=None, n_seqs=2, max_pages=8, n_pages=16, table=P, length=P, lead=P, shared=P, stream=None),
        [("B", 0), ("B", 1025), ("least", 0), ("rows", P + 2), ("n_seqs", 0), ("max_pages", 0), ("n_pages", 0), ("table", None),
         ("length", None), ("lead", P + 2), ("shared", None)]),
    "lla_kv_decode_attn_shared": (
        dict(dtype=0, out_dtype=0, B=2, H=8, H_kv=4, d_head=64, n_seqs=2, max_pages=8, n_pages=16, n_ctx=64, table=P, length=P,
             rows=None, lead=P, shared=P, q=P, k_pages=P, v_pages=P, scale=0.125, out=P, lse=None, workspace=P, ws_bytes=1 << 32,
             stream=None),
        [("dtype", -1), ("out_dtype", 2), ("B", 0), ("B", 1025), ("H", 0), ("H", 6), ("H_kv", 0), ("d_head", 16), ("n_seqs", 0),
         ("max_pages", 0), ("n_pages", 0), ("n_ctx", 0), ("n_ctx", 513), ("table", None), ("length", None), ("rows", P + 1),
         ("lead", None), ("lead", P + 2), ("shared", None), ("q", P + 8), ("k_pages", None), ("v_pages", None), ("scale", 0.0),
         ("scale", math.inf), ("out", None), ("out", P + 8), ("lse", P + 2)]),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_refusals(name):
    good, changes = CALLS[name]
    fn = getattr(kv.lib(), name)
    for arg, value in changes:
        assert fn(*{**good, arg: value}.values()) == lla.LLA_ERR_INVALID_ARG, (arg, value)


@pytest.mark.parametrize("name", ["lla_kv_prefill_attn", "lla_kv_decode_attn_shared"])
def test_workspace_refusals(name):
    good = {**CALLS[name][0], "n_ctx": 8192, "max_pages": 128}
    fn = getattr(kv.lib(), name)
    for ws, size in ((None, 0), (P, 1024), (P + 8, 1 << 32), (None, 1 << 32), (P, 0)):
        assert fn(*{**good, "workspace": ws, "ws_bytes": size}.values()) == lla.LLA_ERR_WORKSPACE, (ws, size)


def test_more_work_than_a_launch_takes_is_refused():
    fn = kv.lib().lla_kv_write_slots
    good = CALLS["lla_kv_write_slots"][0]
    assert fn(*{**good, "total": 1 << 24, "H_kv": 64}.values()) == lla.LLA_ERR_INVALID_ARG
    fn = kv.lib().lla_kv_prefill_attn
    good = CALLS["lla_kv_prefill_attn"][0]
    for H in (256, 128):
        assert fn(*{**good, "total": 1 << 23, "H": H, "H_kv": H}.values()) == lla.LLA_ERR_INVALID_ARG
    fn = kv.lib().lla_kv_decode_attn_shared
    good = CALLS["lla_kv_decode_attn_shared"][0]
    assert fn(*{**good, "B": 1024, "H": 1 << 14}.values()) == lla.LLA_ERR_INVALID_ARG


SIZES = [1, 2, 3, 7, 8, 16, 31, 64, 200, 513, 1024]
BOUNDS = [1, 64, 65, 256, 257, 500, 1024, 3000, 4097, 8192, 20000, 32768, 131072]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,H_kv,d", [(16, 16, 128), (16, 2, 128), (24, 8, 64), (64, 1, 96), (40, 2, 256), (300, 1, 32)])
def test_a_workspace_serves_smaller_calls(dtype, H, H_kv, d):
    """What the largest batch, tokens and bound of a program need is enough for all below."""
    totals = [1, 5, 33, 256, 700, 4096, 30000]
    for sink, window in ((0, 0), (4, 3000)):
        for out in (torch.bfloat16, torch.float32):
            need = {(B, m, n): kv.prefill_workspace_bytes(dtype, B, m, H, H_kv, d, n, sink, window, out_dtype=out)
                    for B in SIZES for m in totals for n in BOUNDS}
            assert any(need.values())
            for (B, m, n), x in need.items():
                for smaller in ((SIZES[SIZES.index(B) - 1], m, n), (B, totals[totals.index(m) - 1], n),
                                (B, m, BOUNDS[BOUNDS.index(n) - 1])):
                    if smaller <= (B, m, n):
                        assert need[smaller] <= x, (smaller, (B, m, n))
    need = {(B, n): kv.shared_workspace_bytes(dtype, B, H, H_kv, d, n) for B in SIZES for n in BOUNDS}
    for (B, n), x in need.items():
        assert need[SIZES[max(0, SIZES.index(B) - 1)], n] <= x and need[B, BOUNDS[max(0, BOUNDS.index(n) - 1)]] <= x


def test_workspace_queries_refuse():
    for bad in (dict(B=0), dict(B=1025), dict(total=0), dict(n_ctx=0), dict(H=3, H_kv=2), dict(d=100), dict(window=-1), dict(sink=3),
                dict(total=1 << 24), dict(n_ctx=(1 << 26) + 1)):
        with pytest.raises(lla.LLAError):
            kv.prefill_workspace_bytes(**{**dict(dtype=torch.float32, B=1, total=5, H=4, H_kv=4, d=64, n_ctx=100), **bad})
    for bad in (dict(B=0), dict(B=1025), dict(n_ctx=0), dict(H=3, H_kv=2), dict(d=100)):
        with pytest.raises(lla.LLAError):
            kv.shared_workspace_bytes(**{**dict(dtype=torch.float32, B=1, H=4, H_kv=4, d=64, n_ctx=100), **bad})
    for bad in (dict(n_ctx=(1 << 32) + 64), dict(total=1 << 31)):
        with pytest.raises(ValueError):
            kv.prefill_workspace_bytes(**{**dict(dtype=torch.float32, B=1, total=5, H=4, H_kv=4, d=64, n_ctx=100), **bad})
    with pytest.raises(ValueError):
        kv.shared_workspace_bytes(torch.float32, 1, 4, 4, 64, 1 << 32)


def test_binding_refuses_before_the_library():
    """Shapes, types and devices that the C ABI cannot see (CPU tensors here)."""
    k, v = kv.alloc_pages(3, 2, 32, device="cpu")
    q = torch.zeros(1, 2, 32, dtype=torch.bfloat16)
    ints = torch.zeros(1, dtype=torch.int32)
    t = kv.new_page_table(2, 2, 3, device="cpu")
    for call in (lambda: kv.slots(t, ints, ints, 1), lambda: kv.shared_prefix(t, ints),
                 lambda: kv.write_slots(q, q, k, v, torch.zeros(1, dtype=torch.int64)),
                 lambda: kv.prefill_attn(q, k, v, t.table, torch.zeros(2, dtype=torch.int32), ints, n_ctx=1),
                 lambda: kv.decode_attn_shared(q, k, v, t.table, t.length, ints, ints, n_ctx=1)):
        with pytest.raises(ValueError):
            call()
