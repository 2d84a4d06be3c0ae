"""Binding of the paged K/V cache (include/lla_kv.h; argument marshalling only).

The full-memory path beside the latent cache of ``lla``: keys and values of
every token in pages of 64 positions that sequences share through a page table.
A decode step of a batch, every call enqueued and none waiting for the host::

    kv.reserve(pages, rows, add, start, pairs, result)     # room; copy on write
    kv.copy_pages(k_pages, v_pages, pairs, result)         # all layers
    ... per layer:
    q = kv.rope(q, freq, pos=start)
    kv.write(k, v, k_pages[l], v_pages[l], pages.table, start, rows=rows, freq=freq)
    o = kv.decode_attn(q[:, 0], k_pages[l], v_pages[l], pages.table, pages.length, rows=rows, n_ctx=n)

rope is differentiable; no gradient passes through the cache.

Rows of -1 are padding in every call: a step captured for a fixed number of rows
serves fewer sequences.

Pools: keys [n_pages, H_kv, 64, d], values [n_pages, H_kv, d, 64], with a leading
layer dimension for the calls that take all layers at once.
"""

from __future__ import annotations

import ctypes
import math
from contextlib import nullcontext
from typing import NamedTuple

import torch

from . import lla
from .lla import PAGE, _c_f, _c_i64, _c_int, _c_sz, _c_vp, _check, _dt, _need, _out_code, _ptr

ABI_VERSION = 2  # LLA_KV_ABI_VERSION of include/lla_kv.h this binding follows
MAX_ROWS = 1024
PAGES_OK, PAGES_FULL, PAGES_BAD = range(3)  # result[0] of the table calls
SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}

_c_d, _I64, _VP = ctypes.c_double, [_c_i64], [_c_vp]

_SIGS = {
    "lla_kv_abi_version": [],
    "lla_rope_frequencies": [_c_int, _c_d, _c_int, _c_d, _c_d, _c_d, _c_d, _c_vp, ctypes.POINTER(_c_d)],
    "lla_rope_positions": [_c_int] * 8 + _VP + _I64 * 3 + _VP + [_c_int] * 2 + _VP + [_c_f] + _VP + _I64 * 3 + _VP,
    "lla_kv_write": [_c_int] * 7 + (_VP + _I64 * 2) * 2 + _VP + [_c_f] + [_c_int] * 3 + _VP * 7,
    "lla_kv_write_at": [_c_int] * 7 + (_VP + _I64 * 2) * 2 + _VP + [_c_f] + [_c_int] * 3 + _VP * 8,
    "lla_kv_decode_workspace_bytes": [_c_int] * 8 + [ctypes.POINTER(_c_sz)],
    "lla_kv_decode_attn": [_c_int] * 12 + _VP * 6 + [_c_f] + _VP * 3 + [_c_sz] + _VP,
    "lla_pages_reserve": [_c_int] + _VP * 2 + [_c_int] * 3 + _VP * 8,
    "lla_pages_fork": [_c_int] + _VP * 2 + [_c_int] * 3 + _VP * 6,
    "lla_pages_free": [_c_int] + _VP + [_c_int] * 3 + _VP * 6,
    "lla_pages_copy": [_c_int] * 2 + (_VP + _I64) * 2 + _VP + [_c_int] + _VP * 2,
    "lla_kv_gather": [_c_int] * 9 + _VP * 8,
}

_lib = None


def lib() -> ctypes.CDLL:
    """liblla.so with the entry points of lla_kv.h."""
    global _lib
    if _lib is None:
        h = lla.lib()
        for name, args in _SIGS.items():
            fn = getattr(h, name)
            fn.restype, fn.argtypes = _c_int, args
        if h.lla_kv_abi_version() != ABI_VERSION:
            raise RuntimeError(f"{lla.LIB_PATH} has K/V ABI version {h.lla_kv_abi_version()}, this binding "
                               f"needs {ABI_VERSION}; rebuild it")
        _lib = h
    return _lib


# The current device's number and a device's current stream handle; torch's own
# short ways to them where it has these (its public ones build objects).
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda i: torch.cuda.current_stream(i).cuda_stream)


def _call(name, dev, *args):
    """An entry point on dev's current stream, with dev the current device."""
    fn, index = getattr(_lib or lib(), name), dev.index
    if _device() == index:
        status = fn(*args, _stream(index))
    else:
        with torch.cuda.device(dev):
            status = fn(*args, _stream(index))
    if status:
        _check(status)


def _ints(t, name, shape, dev):
    if t.dtype is not torch.int32 or t.shape != shape or t.device != dev or not t.is_contiguous() or not t.is_cuda:
        _need(t, name, torch.int32, dev)
        raise ValueError(f"{name} must have shape {list(shape)}")


def _whole(x, names):
    """x: numbers joined by or, that the library takes in 32 bits (ctypes would cut them)."""
    if x >> 31 not in (0, -1):
        raise ValueError(f"{names} must fit 32 bits")


def _rows_of(t, name, dev, dtype):
    """Strides of t [B, M, heads, width] whose rows are dense (of a dimension of
    one entry, which torch leaves as it happens to be, 0)."""
    if t.device != dev or not t.is_cuda:
        raise ValueError(f"{name} must be a tensor on {dev}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.dim() != 4:
        raise ValueError(f"{name} must be [B, M, heads, width]")
    (B, M, H, d), (b, m, h, one) = t.shape, t.stride()
    if one != 1 and d != 1:
        raise ValueError(f"{name} must have dense rows")
    return b if B > 1 else 0, m if M > 1 else 0, h if H > 1 else 0


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------

def rope_frequencies(d_rot: int, *, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                     original: float = 4096.0, beta_fast: float = 32.0, beta_slow: float = 1.0, device="cuda"):
    """(float64 device tensor [d_rot / 2] of angles per position, magnitude) for
    rope and write.  scaling: "none", "linear", "ntk" or "yarn" (with the trained
    length ``original`` and its two turn counts)."""
    if scaling not in SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(SCALINGS)}")
    freq, mag = torch.empty(max(d_rot // 2, 1), dtype=torch.float64), _c_d()
    _check(lib().lla_rope_frequencies(d_rot, base, SCALINGS[scaling], factor, original, beta_fast, beta_slow,
                                      freq.data_ptr(), ctypes.byref(mag)))
    return freq.to(device), mag.value


def _freq(freq, width, dev):
    """Features that freq turns."""
    rot = 2 * freq.numel()
    if freq.dtype is not torch.float64 or freq.device != dev or freq.dim() != 1 or rot > width or not freq.is_contiguous():
        _need(freq, "freq", torch.float64, dev)
        raise ValueError("freq must be [d_rot / 2] with d_rot at most the rows' width")
    return rot


def rope(x, freq, *, pos=None, pos0: int = 0, interleaved: bool = False, magnitude: float = 1.0,
         transpose: bool = False, out=None):
    """Rows x [B, M, H, d] (any strides, dense rows) turned to their positions:
    pos0 + m, plus pos[b] (int32 [B]), or pos0 + pos[b, m] (int32 [B, M]).  The
    first 2 * len(freq) features turn in pairs, half-split or ``interleaved``, and
    are multiplied by ``magnitude``; the rest is copied.  ``transpose`` takes the
    gradient of the result to the gradient of x; autograd calls it where x
    requires one.  ``out`` may be x (in place)."""
    if torch.is_grad_enabled() and (x.requires_grad or freq.requires_grad or out is not None and out.requires_grad):
        if out is not None or freq.requires_grad:
            raise ValueError("no gradient passes through out or freq; leave out away, or call under torch.no_grad()")
        return _Rope.apply(x, freq, pos, pos0, interleaved, magnitude, transpose)
    dev, dtype = x.device, x.dtype
    xs = _rows_of(x, "x", dev, dtype)
    shape = x.shape
    B, M, H, d = shape
    _whole(pos0, "pos0")
    rot, at, per_token = _freq(freq, d, dev), None, 0
    if pos is not None:
        per_token = int(pos.dim() == 2)
        _ints(pos, "pos", (B, M) if per_token else (B,), dev)
        at = pos.data_ptr()
    if out is None:
        out, ys = torch.empty(shape, dtype=dtype, device=dev), (M * H * d, H * d, d)
    else:
        if out.shape != shape:
            raise ValueError("out must have x's shape")
        ys = _rows_of(out, "out", dev, dtype)
    _call("lla_rope_positions", dev, _dt(x), B, M, H, d, rot, int(interleaved), int(transpose), x.data_ptr(), *xs, at,
          per_token, pos0, freq.data_ptr(), magnitude, out.data_ptr(), *ys)
    return out


class _Rope(torch.autograd.Function):
    """rope with the transposed call as its gradient.  Positions are kept as they
    are at the call: reserve writes them without torch's knowledge."""

    @staticmethod
    def forward(ctx, x, freq, pos, pos0, interleaved, magnitude, transpose):
        ctx.save_for_backward(freq)
        ctx.pos = None if pos is None else pos.clone()
        ctx.args = dict(pos0=pos0, interleaved=interleaved, magnitude=magnitude)
        ctx.transpose = transpose
        return rope(x, freq, pos=pos, transpose=transpose, **ctx.args)

    @staticmethod
    def backward(ctx, grad):
        freq, = ctx.saved_tensors
        return rope(grad.contiguous(), freq, pos=ctx.pos, transpose=not ctx.transpose, **ctx.args), *[None] * 6


# ---------------------------------------------------------------------------
# Pools and tables
# ---------------------------------------------------------------------------

class _Pages(NamedTuple):
    table: torch.Tensor    # [n_seqs, max_pages]
    length: torch.Tensor   # [n_seqs] tokens
    refs: torch.Tensor     # [n_pages] holders
    free: torch.Tensor     # [1 + n_pages] count, then a stack


class PageTable(_Pages):
    """Which pages the sequences hold: int32 device tensors table [n_seqs, max_pages],
    length [n_seqs], refs [n_pages] and free [1 + n_pages]; one for all layers."""
    __slots__ = ()

    def __new__(cls, table, length, refs, free):
        for t, name, shape in ((table, "table", table.shape), (length, "length", table.shape[:1]),
                               (refs, "refs", refs.shape), (free, "free", (1 + refs.numel(),))):
            if t.dtype != torch.int32 or t.shape != shape or t.device != table.device or not t.is_contiguous():
                raise ValueError(f"{name} must be a dense int32 tensor of shape {list(shape)} on {table.device}")
        if table.dim() != 2 or refs.dim() != 1:
            raise ValueError("table must be [n_seqs, max_pages] and refs [n_pages]")
        return super().__new__(cls, table, length, refs, free)


def new_page_table(n_seqs: int, max_pages: int, n_pages: int, device="cuda") -> PageTable:
    """Empty sequences and a pool of free pages (page 0 is taken first)."""
    free = torch.arange(n_pages, -1, -1, dtype=torch.int32, device=device)
    free[0] = n_pages
    free[1:] = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device)
    zeros = lambda n: torch.zeros(n, dtype=torch.int32, device=device)  # noqa: E731
    return PageTable(torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device=device), zeros(n_seqs),
                     zeros(n_pages), free)


def alloc_pages(n_pages: int, H_kv: int, d: int, dtype=torch.bfloat16, device="cuda", layers: int | None = None):
    """Key and value pools of one layer, or of ``layers`` in one piece."""
    lead = (n_pages, H_kv) if layers is None else (layers, n_pages, H_kv)
    return (torch.empty((*lead, PAGE, d), dtype=dtype, device=device),
            torch.empty((*lead, d, PAGE), dtype=dtype, device=device))


def _pools(k_pages, v_pages, layered=False):
    """(layers, n_pages, H_kv, d) of a pair of pools."""
    shape, layers = k_pages.shape, 1
    if len(shape) == 4:
        P, H, page, d = shape
        other = (P, H, d, PAGE)
    elif layered and len(shape) == 5:
        layers, P, H, page, d = shape
        other = (layers, P, H, d, PAGE)
    else:
        raise ValueError("k_pages must be [n_pages, H_kv, 64, d]" + (", or with a layer dimension" if layered else ""))
    if page != PAGE or v_pages.shape != other:
        raise ValueError("k_pages must be [n_pages, H_kv, 64, d] and v_pages [n_pages, H_kv, d, 64]")
    if (not k_pages.is_cuda or v_pages.dtype is not k_pages.dtype or v_pages.device != k_pages.device
            or not k_pages.is_contiguous() or not v_pages.is_contiguous()):
        _need(k_pages, "k_pages")
        _need(v_pages, "v_pages", k_pages.dtype, k_pages.device)
    return layers, P, H, d


def _page_table(p, dev):
    """(n_seqs, max_pages, n_pages) of a page table on dev."""
    if p.table.device != dev or not p.table.is_cuda:
        raise ValueError(f"the page table is on {p.table.device}, expected {dev}")
    return (*p.table.shape, p.refs.numel())


def reserve(pages: PageTable, rows, add, start, pairs, result):
    """Room for add[i] new tokens of sequence rows[i]; start[i] gets its length
    before (-1 where the call is refused, and of padding), pairs the pages to copy (copy on write)
    and result (status, number of pairs, pages taken, pages left).  All int32:
    rows, add, start [n], pairs [n, 2], result [4]."""
    dev, n = rows.device, rows.numel()
    sizes = _page_table(pages, dev)
    for t, name, shape in ((rows, "rows", (n,)), (add, "add", (n,)), (start, "start", (n,)), (pairs, "pairs", (n, 2)),
                           (result, "result", (4,))):
        _ints(t, name, shape, dev)
    _call("lla_pages_reserve", dev, n, _ptr(rows), _ptr(add), *sizes, *map(_ptr, pages), _ptr(start), _ptr(pairs),
          _ptr(result))


def fork(pages: PageTable, src, dst, result):
    """The empty sequences dst[i] become src[i], sharing its pages (int32 [n])."""
    dev, n = dst.device, dst.numel()
    sizes = _page_table(pages, dev)
    for t, name, shape in ((src, "src", (n,)), (dst, "dst", (n,)), (result, "result", (4,))):
        _ints(t, name, shape, dev)
    _call("lla_pages_fork", dev, n, _ptr(src), _ptr(dst), *sizes, *map(_ptr, pages), _ptr(result))


def free(pages: PageTable, rows, result):
    """Empty the sequences rows (int32 [n]); pages without a holder become free."""
    dev, n = rows.device, rows.numel()
    sizes = _page_table(pages, dev)
    for t, name, shape in ((rows, "rows", (n,)), (result, "result", (4,))):
        _ints(t, name, shape, dev)
    _call("lla_pages_free", dev, n, _ptr(rows), *sizes, *map(_ptr, pages), _ptr(result))


def copy_pages(a, b, pairs, result=None):
    """Copy pages pairs[i, 0] -> pairs[i, 1] of the pools a and b (b may be None): the
    first dimension numbers the pages, of five dimensions the second (layers
    first); with the result of reserve, only the pairs that it gave.  A latent
    cache is a pool too, seen as [B * H * n_max / 64, r, 64]."""
    dev, pools = a.device, []
    lead = a.shape[:2] if a.dim() == 5 else (1, a.shape[0])
    for t, name in ((a, "a"), (b, "b")):
        if t is None:
            pools += [None, 0]
            continue
        _need(t, name, None, dev)
        if (t.shape[:2] if t.dim() == 5 else (1, t.shape[0])) != lead:
            raise ValueError("a and b must have the same layers and pages")
        pools += [_ptr(t), t.numel() // max(lead[0] * lead[1], 1) * t.element_size()]
    _ints(pairs, "pairs", (pairs.shape[0], 2), dev)
    if result is not None:
        _ints(result, "result", (4,), dev)
    _call("lla_pages_copy", dev, *lead, *pools, _ptr(pairs), pairs.shape[0], None if result is None else _ptr(result) + 4)


def gather(k_pages, v_pages, table, src, dst, keep, n_keep=None):
    """Position i of sequence dst[j] becomes position keep[j, i] of sequence src[j],
    for i < n_keep[j] (all of keep's columns without n_keep); int32 tensors.  Keys
    stay turned to their old positions, so a length is no position any more: the
    caller counts all tokens, and gives the count to rope and write as ``pos``."""
    dev = k_pages.device
    layers, P, H, d = _pools(k_pages, v_pages, layered=True)
    n_seqs, max_pages = table.shape
    B, most = keep.shape
    for t, name, shape in ((table, "table", (n_seqs, max_pages)), (src, "src", (B,)), (dst, "dst", (B,)),
                           (keep, "keep", (B, most))):
        _ints(t, name, shape, dev)
    if n_keep is not None:
        _ints(n_keep, "n_keep", (B,), dev)
    _call("lla_kv_gather", dev, _dt(k_pages), B, most, layers, H, d, n_seqs, max_pages, P, _ptr(table), _ptr(src),
          _ptr(dst), _ptr(keep), _ptr(n_keep), _ptr(k_pages), _ptr(v_pages))


# ---------------------------------------------------------------------------
# Write and attention
# ---------------------------------------------------------------------------

def write(k, v, k_pages, v_pages, table, start, *, rows=None, n_new=None, pos=None, freq=None,
          interleaved: bool = False, magnitude: float = 1.0):
    """Write new tokens k, v [B, M, H_kv, d] (heads and rows dense, B and M of any
    strides) at positions start[b] + m of sequences rows[b] (None: b), m < n_new[b]
    (None: M), into one layer's pools; with freq, keys are turned to their
    positions as by rope, or to pos[b] + m (int32 [B]) where places in the cache
    are not positions, as after gather."""
    dev = k_pages.device
    _, P, H, d = _pools(k_pages, v_pages)
    ks, vs = _rows_of(k, "k", dev, k_pages.dtype), _rows_of(v, "v", dev, k_pages.dtype)
    B, M = k.shape[:2]
    if k.shape != (B, M, H, d) or v.shape != k.shape:
        raise ValueError("k and v must be [B, M, H_kv, d] with the pools' heads")
    if H > 1 and (ks[2] != d or vs[2] != d):
        raise ValueError("the heads of k and v must be dense")
    rot = 0 if freq is None else _freq(freq, d, dev)
    n_seqs, max_pages = table.shape
    for t, name, shape in ((table, "table", (n_seqs, max_pages)), (start, "start", (B,))):
        _ints(t, name, shape, dev)
    for t, name in ((rows, "rows"), (n_new, "n_new"), (pos, "pos")):
        if t is not None:
            _ints(t, name, (B,), dev)
    if rows is None and B > n_seqs:
        raise ValueError("more entries than sequences")
    _call("lla_kv_write_at", dev, _dt(k_pages), B, M, H, d, rot, int(interleaved), _ptr(k), *ks[:2], _ptr(v), *vs[:2],
          _ptr(freq), float(magnitude), n_seqs, max_pages, P, _ptr(table), _ptr(rows), _ptr(start), _ptr(pos),
          _ptr(n_new), _ptr(k_pages), _ptr(v_pages))


def decode_workspace_bytes(dtype: torch.dtype, B: int, H: int, H_kv: int, d: int, n_ctx: int, sink: int = 0,
                           window: int = 0) -> int:
    """Workspace of decode_attn on the current device for up to B entries and bounds up
    to n_ctx (0: none of these splits a context over workgroups)."""
    out = _c_sz()
    _whole(n_ctx | sink | window, "n_ctx, sink and window")
    _check(lib().lla_kv_decode_workspace_bytes(_out_code(dtype), B, H, H_kv, d, n_ctx, sink, window, ctypes.byref(out)))
    return out.value


def decode_attn(q, k_pages, v_pages, table, length, *, n_ctx: int, rows=None, scale: float | None = None,
                sink: int = 0, window: int = 0, out=None, out_dtype=torch.float32, lse=None, workspace=None):
    """Attention of q [B, H, d] over the pages of sequences rows[b] (None: b) with
    length[row] <= n_ctx tokens each: all of them, or with ``window`` the first
    ``sink`` and the last ``window``.  H is a multiple of the pools' heads.  An
    empty sequence or row -1 gives zeros.  lse: float32 [B, H] or None; workspace:
    uint8 of decode_workspace_bytes(...) (allocated here if None).  Returns out
    [B, H, d]."""
    dev = q.device
    _, P, Hkv, d = _pools(k_pages, v_pages)
    B, H, width = q.shape
    _need(q, "q", k_pages.dtype, dev)
    if width != d or k_pages.device != dev or v_pages.device != dev:
        raise ValueError("q must be [B, H, d] with the pools' width, on their device")
    n_seqs, max_pages = table.shape
    _whole(n_ctx | sink | window, "n_ctx, sink and window")
    for t, name, shape in ((table, "table", (n_seqs, max_pages)), (length, "length", (n_seqs,))):
        _ints(t, name, shape, dev)
    if rows is not None:
        _ints(rows, "rows", (B,), dev)
    if out is None:
        out = torch.empty((B, H, d), dtype=out_dtype, device=dev)
    else:
        _need(out, "out", None, dev)
        if out.shape != q.shape:
            raise ValueError("out must have q's shape")
    if lse is not None:
        _need(lse, "lse", torch.float32, dev)
        if lse.shape != (B, H):
            raise ValueError("lse must be [B, H]")
    if rows is None and B > n_seqs:
        raise ValueError("more entries than sequences")
    if workspace is None:
        with torch.cuda.device(dev) if _device() != dev.index else nullcontext():
            need = decode_workspace_bytes(q.dtype, B, H, Hkv, d, n_ctx, sink, window)
        workspace = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    else:
        _need(workspace, "workspace", None, dev)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _call("lla_kv_decode_attn", dev, _dt(q), _out_code(out.dtype), B, H, Hkv, d, n_seqs, max_pages, P, n_ctx, sink,
          window, _ptr(table), _ptr(length), _ptr(rows), _ptr(q), _ptr(k_pages), _ptr(v_pages),
          float(1.0 / math.sqrt(d) if scale is None else scale), _ptr(out), _ptr(lse), _ptr(workspace), ws_bytes)
    return out
