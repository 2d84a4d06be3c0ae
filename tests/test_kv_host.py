"""Host-side checks of the paged K/V cache's C ABI (no GPU needed): names, host
functions, and every refusal; no call here reaches a kernel."""

import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from paper_2607_15456_amd import kv, lla

HEADER = os.path.join(os.path.dirname(lla.LIB_PATH), "..", "include", "lla_kv.h")


def test_header_binding_and_library_agree():
    src = open(HEADER).read()
    names = set(re.findall(r"^(?:int|lla_status)\s+(lla_\w+)\(", src, re.M))
    assert names == set(kv._SIGS)
    for name in names:
        decl = re.search(r"^(?:int|lla_status)\s+" + name + r"\(([^)]*)\)", src, re.M).group(1)
        given = [] if decl.strip() == "void" else decl.split(",")
        assert len(given) == len(kv._SIGS[name]), name
        for text, want in zip(given, kv._SIGS[name]):
            kind = (ctypes.c_void_p if "*" in text else ctypes.c_int64 if "int64_t" in text else
                    ctypes.c_size_t if "size_t" in text else ctypes.c_double if "double" in text else
                    ctypes.c_float if "float" in text else ctypes.c_int)
            assert want is kind or (kind is ctypes.c_void_p and hasattr(want, "contents")), (name, text)
        assert hasattr(lla.lib(), name)
    assert kv.lib().lla_kv_abi_version() == kv.ABI_VERSION
    assert f"LLA_KV_MAX_ROWS {kv.MAX_ROWS} " in src


@pytest.mark.parametrize("d_rot", [8, 24, 64, 128, 256])
@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
def test_frequencies(d_rot, scaling):
    for base, factor, original in ((10000.0, 1.0, 4096), (500000.0, 8.0, 2048), (1.5, 2.5, 64)):
        f, m = kv.rope_frequencies(d_rot, base=base, scaling=scaling, factor=factor, original=original, device="cpu")
        ref, mag = O.kv_rope_frequencies(d_rot, base, scaling, factor, original)
        # pow and log of two libraries: a few steps of 2^-53
        assert f.dtype == torch.float64 and np.allclose(f.numpy(), ref, rtol=2e-14, atol=0) and abs(m - mag) < 1e-14


def test_frequencies_refused():
    for d_rot, kw in ((0, {}), (12, {}), (264, {}), (64, {"base": 1.0}), (64, {"base": math.inf}),
                      (64, {"scaling": "linear", "factor": 0.5}), (64, {"scaling": "ntk", "factor": math.nan}),
                      (64, {"scaling": "ntk", "factor": 1e308}),
                      (64, {"scaling": "yarn", "factor": 2.0, "original": 0.0}),
                      (64, {"scaling": "yarn", "factor": 2.0, "beta_fast": 1.0, "beta_slow": 1.0})):
        with pytest.raises(lla.LLAError) as e:
            kv.rope_frequencies(d_rot, device="cpu", **kw)
        assert e.value.status == lla.LLA_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        kv.rope_frequencies(64, scaling="cubic", device="cpu")


def test_new_page_table():
    t = kv.new_page_table(3, 4, 5, device="cpu")
    assert t.free.tolist() == [5, 4, 3, 2, 1, 0] and t.refs.tolist() == [0] * 5 and t.length.tolist() == [0] * 3
    assert t.table.shape == (3, 4) and (t.table == -1).all()
    k, v = kv.alloc_pages(5, 2, 32, device="cpu", layers=3)
    assert k.shape == (3, 5, 2, 64, 32) and v.shape == (3, 5, 2, 32, 64)


P = 1 << 20  # an aligned address that no call gets to use

# name: the arguments of a call that is accepted but for its null stream's work
# (never made), then the single changes that have to be refused
CALLS = {
    "lla_rope_positions": (
        dict(dtype=1, B=2, M=3, H=4, d_head=128, d_rot=64, interleaved=0, transpose=0, x=P, x_b=1536, x_m=512, x_h=128,
             pos=P, pos_tokens=0, pos0=0, freq=P, magnitude=1.0, y=P, y_b=1536, y_m=512, y_h=128, stream=None),
        [("dtype", 2), ("B", 0), ("M", 0), ("H", 0), ("H", 1 << 30), ("H", 65536), ("d_head", 4), ("d_head", 132), ("d_head", 520),
         ("d_rot", 0), ("d_rot", 12), ("d_rot", 136), ("x", None), ("x", P + 8), ("x_b", -8), ("x_m", 4), ("x_h", 12),
         ("pos", P + 2), ("freq", None), ("freq", P + 4), ("magnitude", math.nan), ("y", None), ("y", P + 2),
         ("y_b", 0), ("y_m", 64), ("y_h", 0), ("y_b", 1024), ("y_b", 128), ("y_m", 384), ("y_h", 256), ("x_b", 1544)]),
    "lla_kv_write": (
        dict(dtype=0, B=2, M=3, H_kv=4, d_head=64, d_rot=64, interleaved=1, k=P, k_b=768, k_m=256, v=P, v_b=768, v_m=256,
             freq=P, magnitude=1.0, n_seqs=2, max_pages=8, n_pages=16, table=P, rows=None, start=P, n_new=None, k_pages=P,
             v_pages=P, stream=None),
        [("dtype", -1), ("B", 0), ("B", 1 << 30), ("M", 0), ("H_kv", 0), ("H_kv", 65536), ("d_head", 16), ("d_head", 288),
         ("d_head", 40), ("d_rot", 72), ("d_rot", 4), ("d_rot", 0), ("k", None), ("k", P + 4), ("k_b", -4), ("k_m", 2),
         ("v", None), ("v_b", 3), ("v_m", 1), ("freq", None), ("magnitude", math.inf), ("n_seqs", 0), ("max_pages", 0),
         ("max_pages", (1 << 20) + 1), ("n_pages", 0), ("n_pages", (1 << 30) + 1), ("table", None), ("rows", P + 1),
         ("start", None), ("n_new", P + 3), ("k_pages", None), ("v_pages", P + 8)]),
    "lla_kv_decode_attn": (
        dict(dtype=1, out_dtype=1, B=2, H=8, H_kv=4, d_head=64, n_seqs=2, max_pages=8, n_pages=16, n_ctx=64, sink=0,
             window=0, table=P, length=P, rows=None, q=P, k_pages=P, v_pages=P, scale=0.125, out=P, lse=None,
             workspace=P, ws_bytes=1 << 30, stream=None),
        [("dtype", 2), ("out_dtype", 2), ("B", 0), ("B", 1 << 24), ("H", 0), ("H", 6), ("H", 1 << 19), ("H_kv", 0), ("H_kv", 3),
         ("d_head", 0), ("d_head", 48), ("d_head", 512), ("n_seqs", 0), ("max_pages", 0), ("n_pages", 0), ("n_ctx", 0),
         ("n_ctx", 513), ("sink", -1), ("sink", 1), ("window", -1), ("table", None), ("length", None), ("length", P + 2),
         ("rows", P + 2), ("q", P + 8), ("k_pages", None), ("v_pages", None), ("scale", 0.0), ("scale", -1.0),
         ("scale", math.inf), ("out", None), ("lse", P + 1)]),
    "lla_pages_reserve": (
        dict(n=2, rows=P, add=P, n_seqs=2, max_pages=8, n_pages=16, table=P, length=P, refs=P, free_pages=P, start=P,
             pairs=P, result=P, stream=None),
        [("n", 0), ("n", 1025), ("rows", None), ("add", None), ("n_seqs", 0), ("max_pages", 0), ("n_pages", 0),
         ("table", None), ("length", None), ("refs", P + 2), ("free_pages", None), ("start", None), ("pairs", None),
         ("result", None)]),
    "lla_pages_fork": (
        dict(n=2, src=P, dst=P, n_seqs=2, max_pages=8, n_pages=16, table=P, length=P, refs=P, free_pages=P, result=P,
             stream=None),
        [("n", 0), ("n", 1025), ("src", None), ("dst", None), ("n_seqs", -1), ("max_pages", 0), ("n_pages", 0),
         ("table", None), ("length", P + 1), ("refs", None), ("free_pages", None), ("result", None)]),
    "lla_pages_free": (
        dict(n=2, rows=P, n_seqs=2, max_pages=8, n_pages=16, table=P, length=P, refs=P, free_pages=P, result=P,
             stream=None),
        [("n", 0), ("n", 1025), ("rows", None), ("n_seqs", 0), ("max_pages", 0), ("n_pages", 0), ("table", None),
         ("length", None), ("refs", None), ("free_pages", None), ("result", P + 2)]),
    "lla_pages_copy": (
        dict(layers=2, n_pages=16, a=P, a_bytes=4096, b=P, b_bytes=4096, pairs=P, n_pairs=3, count=None, stream=None),
        [("layers", 0), ("layers", 65536), ("n_pages", 0), ("a", None), ("a", P + 8), ("a_bytes", 0), ("a_bytes", 24), ("a_bytes", 1 << 43),
         ("b", None), ("b", P + 4), ("b_bytes", 0), ("b_bytes", 8), ("pairs", None), ("n_pairs", 0),
         ("n_pairs", (1 << 20) + 1), ("count", P + 2)]),
    "lla_kv_gather": (
        dict(dtype=1, B=2, max_keep=100, layers=1, H_kv=2, d_head=64, n_seqs=4, max_pages=8, n_pages=16, table=P, src=P,
             dst=P, keep=P, n_keep=None, k_pages=P, v_pages=P, stream=None),
        [("dtype", 3), ("B", 0), ("max_keep", 0), ("max_keep", 513), ("layers", 0), ("layers", 32768), ("H_kv", 0),
         ("H_kv", 65536), ("d_head", 16), ("n_seqs", 0), ("max_pages", 0), ("n_pages", 0), ("table", None), ("src", None),
         ("dst", P + 2), ("keep", None), ("n_keep", P + 1), ("k_pages", None), ("v_pages", P + 8)]),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_refusals(name):
    good, changes = CALLS[name]
    fn = getattr(kv.lib(), name)
    decl = re.search(r"lla_status\s+" + name + r"\(([^)]*)\)", open(HEADER).read()).group(1)
    assert [re.split(r"[\s*]+", a.strip())[-1] for a in decl.split(",")] == list(good)
    for arg, value in changes:
        assert value != good[arg], arg
        assert fn(*{**good, arg: value}.values()) == lla.LLA_ERR_INVALID_ARG, (name, arg, value)


def test_copy_refuses_more_pieces_than_a_grid_holds():
    good = {**CALLS["lla_pages_copy"][0], "a_bytes": 1 << 40}  # 2^27 pieces of 8 KB a pair
    assert kv.lib().lla_pages_copy(*{**good, "n_pairs": 16}.values()) == lla.LLA_ERR_INVALID_ARG


def test_workspace_refused():
    good = CALLS["lla_kv_decode_attn"][0]
    fn = kv.lib().lla_kv_decode_attn
    assert fn(*{**good, "workspace": None}.values()) == lla.LLA_ERR_WORKSPACE       # bytes without a buffer
    assert fn(*{**good, "ws_bytes": 0}.values()) == lla.LLA_ERR_WORKSPACE           # a buffer without bytes
    assert fn(*{**good, "workspace": P + 8}.values()) == lla.LLA_ERR_WORKSPACE
    long = {**good, "B": 1, "n_ctx": 32768, "max_pages": 512, "H": 4}
    need = kv.decode_workspace_bytes(torch.bfloat16, 1, 4, 4, 64, 32768)
    assert need > 0
    assert fn(*{**long, "ws_bytes": need - 1}.values()) == lla.LLA_ERR_WORKSPACE
    assert fn(*{**long, "workspace": None, "ws_bytes": 0}.values()) == lla.LLA_ERR_WORKSPACE
    for bad in (dict(B=0), dict(n_ctx=0), dict(H=3, H_kv=2), dict(d=100), dict(window=-1), dict(sink=3)):
        args = {**dict(dtype=torch.float32, B=1, H=4, H_kv=4, d=64, n_ctx=100), **bad}
        with pytest.raises(lla.LLAError):
            kv.decode_workspace_bytes(**args)


def test_binding_refuses_before_the_library():
    """Shapes, types and devices that the C ABI cannot see (CPU tensors here)."""
    k, v = kv.alloc_pages(3, 2, 32, device="cpu")
    q = torch.zeros(1, 2, 32, dtype=torch.bfloat16)
    ints = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        kv.decode_attn(q, k, v, ints.view(1, 1), ints, n_ctx=1)
    with pytest.raises(ValueError):
        kv.rope(torch.zeros(1, 1, 2, 32), torch.zeros(16, dtype=torch.float64))
    with pytest.raises(ValueError):
        kv.write(q[None], q[None], k, v, ints.view(1, 1), ints)
    t = kv.new_page_table(2, 2, 3, device="cpu")
    for change in (dict(table=t.table[0]), dict(table=t.table.long()), dict(table=t.table.t()), dict(length=t.length[:1]),
                   dict(free=t.free[1:]), dict(refs=t.refs.view(1, 3)), dict(refs=t.refs[::2])):
        with pytest.raises(ValueError):
            kv.PageTable(**{**t._asdict(), **change})
    for call in (lambda: kv.free(t, ints, torch.zeros(4, dtype=torch.int32)),
                 lambda: kv.fork(t, ints, ints, torch.zeros(4, dtype=torch.int32)),
                 lambda: kv.copy_pages(k, v, torch.zeros(1, 2, dtype=torch.int32)),
                 lambda: kv.gather(k, v, t.table, ints, ints, ints.view(1, 1))):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("name,changes", [
    ("lla_rope_positions", dict(B=1, M=1 << 24, H=1, d_head=8, d_rot=8, x_m=8, y_m=8)),
    ("lla_kv_write", dict(B=1 << 21, M=4, H_kv=4)),
    ("lla_kv_write", dict(B=1 << 22, M=1, H_kv=4)),
    ("lla_kv_decode_attn", dict(B=1 << 21, H=8, H_kv=8)),
    ("lla_pages_copy", dict(n_pairs=1 << 20, a_bytes=1 << 16, b_bytes=1 << 16)),
    ("lla_kv_gather", dict(B=1 << 24, max_keep=1)),
])
def test_refuses_more_threads_than_a_launch_takes(name, changes):
    """256 threads a workgroup: 2^24 workgroups along a dimension are 2^32 threads."""
    assert getattr(kv.lib(), name)(*{**CALLS[name][0], **changes}.values()) == lla.LLA_ERR_INVALID_ARG


def test_scale_that_overflows_in_base_two_is_refused():
    """Scores are taken in powers of two: an infinite factor would make NaN of zeros."""
    good = CALLS["lla_kv_decode_attn"][0]
    assert kv.lib().lla_kv_decode_attn(*{**good, "scale": 3e38}.values()) == lla.LLA_ERR_INVALID_ARG
