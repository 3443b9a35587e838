"""Operators over the tokens of long videos, on torch tensors: rotary positions, attention over selected key blocks, quantised
cache entries (the C ABI's section of the same name in include/lightcache.h, which has the definitions).

Tensors are [B, T, heads, head_dim] views of any strides with channels next to each other (rows of packed q,k,v, say). Calls
enqueue on torch's current stream of the tensors' device and take outputs and workspaces from torch's allocator on it, so
they order with torch's own work and may be captured into a graph. No gradients are recorded (the map of :func:`rope` has its
transpose: ``inverse=True``). Formats of entries are the C ABI's: "mxfp8" and "mxfp4" groups hold what such groups commonly do (e4m3 and
e2m1 codes, scale bytes of exponent + 127), "mxint8" codes count ones, where the published format of that name counts 2^-6. What a call refuses raises :class:`binding.LcError`, or ``ValueError`` where it never gets there.
"""
from __future__ import annotations

import functools
from typing import Optional, Sequence

import torch

from . import binding as lcb

LAYOUTS = {"half": lcb.LC_ROPE_HALF, "interleaved": lcb.LC_ROPE_INTERLEAVED}
SCALINGS = {"none": lcb.LC_ROPE_UNSCALED, "linear": lcb.LC_ROPE_LINEAR, "base": lcb.LC_ROPE_BASE, "parts": lcb.LC_ROPE_PARTS}
FORMATS = {"mxint8": lcb.LC_ENTRY_INT8, "mxfp8": lcb.LC_ENTRY_FP8, "mxfp4": lcb.LC_ENTRY_FP4}
_DTYPES = {torch.float32: lcb.LC_F32, torch.bfloat16: lcb.LC_BF16}


def _named(table, what, key):
    if key not in table:
        raise ValueError(f"{what} must be one of {', '.join(table)}")
    return table[key]


def _dtype(name, dtype):
    if dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32 or bfloat16, not {dtype}")
    return _DTYPES[dtype]


def _launch(device, call, *args):
    """call(*args, stream) on torch's current stream of that GPU."""
    i = device.index
    if i == torch.cuda.current_device():
        call(*args, torch._C._cuda_getCurrentRawStream(i))
    else:
        with torch.cuda.device(i):
            call(*args, torch._C._cuda_getCurrentRawStream(i))


def _on(device, *tensors):
    """The tensors that are given are on that GPU."""
    if device.type != "cuda":
        raise ValueError("tensors must be on a GPU (there is no CPU fallback)")
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"tensors on {device} and on {t.device}")


def _strides(name, shape, stride):
    """Strides of [B, T, heads, head_dim]; those of axes of length one are what a dense tensor would have."""
    if len(shape) != 4:
        raise ValueError(f"{name} must be [B, T, heads, head_dim], not of shape {tuple(shape)}")
    B, T, H, d = shape
    if d > 1 and stride[3] != 1:
        raise ValueError(f"{name}: the channels of a head must lie next to each other")
    head = stride[2] if H > 1 else d
    token = stride[1] if T > 1 else max(d, head * H)
    return lcb.lc_strides(stride[0] if B > 1 else max(token * T, head * H), token, head)


def _lens(name, t, B):
    if t is None:
        return None
    if t.dtype != torch.int32 or t.shape != (B,) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor of shape ({B},)")
    return t.data_ptr()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _out(out, shape, dtype, device, name="out"):
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if out.shape != shape or out.dtype != dtype:
        raise ValueError(f"{name} must be {dtype} of shape {tuple(shape)}")
    return out


# Descriptors depend on shapes, strides, types and options alone: those of the last few hundred kinds of call are kept, so that a
# repeated call does not pay for making one. A position, an offset or a length that moves from call to call is one of those options: such
# calls make theirs each time (us of the host, repeated and moving: rope 6.2 and 8.3, block_select 6.1 and 8.5, block_attention 14.2 and 17.8).
_kept = functools.lru_cache(maxsize=512)


# ---- rotary positions -------------------------------------------------------------------------------------------------
def make_rope(head_dim: int, axes: Optional[Sequence[int]] = None, base: float = 10000.0, layout: str = "half", scaling: str = "none",
              factor: float = 1.0, orig_len: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0) -> lcb.lc_rope_table:
    """The table :func:`rope` takes, made once for a model. ``axes``: the channels that each position axis turns, those of the
    first axis first (default: one axis, the whole head)."""
    dims = [head_dim] if axes is None else list(axes)
    if not 1 <= len(dims) <= 3:
        raise ValueError("there are one to three axes")
    lcb.fits("head_dim orig_len axes", head_dim, orig_len, max(dims))
    return lcb.lc_rope_make(lcb.lc_rope_config(head_dim=head_dim, axes=len(dims), axis_dim=(lcb.C.c_int32 * 3)(*dims),
                                               layout=_named(LAYOUTS, "layout", layout), scaling=_named(SCALINGS, "scaling", scaling),
                                               orig_len=orig_len, base=base, factor=factor, beta_fast=beta_fast, beta_slow=beta_slow))


def rope(x, table: lcb.lc_rope_table, pos=None, grid: Optional[Sequence[int]] = None, start=0, inverse: bool = False, out=None):
    """x [B, T, heads, head_dim] turned by its tokens' positions; ``out`` may be x. Positions: ``pos`` (int32, [T, axes], [B, T, axes], or
    without the last axis where there is one), else the cells of ``grid`` in row-major order, else running numbers;
    ``start`` (a number or one an axis) is added to the latter two."""
    if x.dim() == 4 and x.shape[3] != table.head_dim:
        raise ValueError(f"heads of {x.shape[3]} channels, the table is for {table.head_dim}")
    out = _out(out, x.shape, x.dtype, x.device)
    n = table.axes
    starts = (start,) * n if isinstance(start, int) else tuple(start)
    pos_batch = 0
    if pos is not None:
        B, T = x.shape[:2]
        if grid is not None or any(starts):
            raise ValueError("pos holds the positions: no grid and no start beside it")
        if n == 1 and tuple(pos.shape) in ((T,), (B, T)) and tuple(pos.shape) != (T, 1):
            pos = pos.unsqueeze(-1)
        if pos.dtype != torch.int32 or not pos.is_contiguous() or tuple(pos.shape) not in ((T, n), (B, T, n)):
            raise ValueError(f"pos must be contiguous int32 of shape {(T, n)} or {(B, T, n)}")
        pos_batch = T * n if pos.dim() == 3 else 0
    a = _rope_args(x.shape, x.stride(), out.stride(), x.dtype, n, None if grid is None else tuple(grid), starts, bool(inverse), pos_batch)
    _on(x.device, out, pos)
    if x.numel() == 0:
        return out
    _launch(x.device, lcb.lc_op_rope, table, a, x.data_ptr(), _ptr(pos), out.data_ptr())
    return out


@_kept
def _rope_args(shape, x_stride, y_stride, dtype, n, grid, starts, inverse, pos_batch):
    if len(starts) != n or (grid is not None and len(grid) != n):
        raise ValueError(f"grid and start have one value for each of the {n} axes")
    xs = _strides("x", shape, x_stride)
    lcb.fits("T grid start", max(shape), max(grid or (0,), key=abs), max(starts, key=abs) >> 32)
    ys = xs if y_stride == x_stride else _strides("out", shape, y_stride)
    return lcb.lc_rope_args(B=shape[0], T=shape[1], heads=shape[2], dtype=_dtype("x", dtype), x=xs, y=ys,
                            inverse=int(inverse), grid=(lcb.C.c_int32 * 3)(*(grid or ())), start=(lcb.C.c_int64 * 3)(*starts),
                            pos_batch=pos_batch)


# ---- attention over selected blocks -----------------------------------------------------------------------------------
def block_means(k, block: int = 64, k_len=None, first: int = 0, count: Optional[int] = None, out=None):
    """Means of the key blocks [first, first + count) of k [B, Tk, kv_heads, head_dim], in float64 [B, kv_heads, head_dim, blocks];
    ``out``: the tensor of an earlier call, whose other blocks stay."""
    a, nk = _means_args(k.shape, k.stride(), k.dtype, block)
    B, Tk, Hkv, d = k.shape
    count = nk - first if count is None else count
    lcb.fits("first count", first, count)
    if out is None and (first, count) != (0, nk):
        raise ValueError("some blocks of a tensor: give the tensor")
    _on(k.device, k_len, out)
    out = _out(out, (B, Hkv, d, nk), torch.float64, k.device)
    if not out.is_contiguous():
        raise ValueError("out must be contiguous")
    _launch(k.device, lcb.lc_op_block_means, a, k.data_ptr(), _lens("k_len", k_len, B), out.data_ptr(), first, count)
    return out


@_kept
def _means_args(shape, stride, dtype, block):
    s = _strides("k", shape, stride)
    B, Tk, Hkv, d = shape
    lcb.fits("Tk block", max(shape), block)
    a = lcb.lc_sparse_args(B=B, Tq=1, Tk=Tk, heads=Hkv, kv_heads=Hkv, head_dim=d, dtype=_dtype("k", dtype), block=block, q_block=1, keep=1,
                           window=-1, k=s)
    return a, lcb.lc_sparse_blocks(a)


def block_select(q, means, Tk: int, keep: int, block: int = 64, q_block: int = 128, sink: int = 0, window: int = -1, q_pos0: int = 0,
                 q_len=None, k_len=None, out=None):
    """The lists of the groups of q_block queries of q [B, Tq, heads, head_dim]: int32 [B, heads, groups, keep], ascending, -1 behind
    their ends. ``means``: :func:`block_means` of the Tk keys."""
    a, shape = _select_args(q.shape, q.stride(), q.dtype, means.shape, Tk, keep, block, q_block, sink, window, q_pos0)
    B = q.shape[0]
    if means.dtype != torch.float64 or not means.is_contiguous():
        raise ValueError("means must be what block_means made")
    _on(q.device, means, q_len, k_len, out)
    out = _out(out, shape, torch.int32, q.device)
    if not out.is_contiguous():
        raise ValueError("out must be contiguous")
    _launch(q.device, lcb.lc_op_block_select, a, q.data_ptr(), means.data_ptr(), _lens("q_len", q_len, B), _lens("k_len", k_len, B),
            out.data_ptr())
    return out


@_kept
def _select_args(shape, stride, dtype, m_shape, Tk, keep, block, q_block, sink, window, q_pos0):
    s = _strides("q", shape, stride)
    B, Tq, H, d = shape
    if len(m_shape) != 4 or m_shape[0] != B or m_shape[2] != d:
        raise ValueError("means must be what block_means made for these sizes")
    lcb.fits("Tq Tk keep block q_block sink window q_pos0", max(shape), Tk, keep, block, q_block, sink, window, q_pos0 >> 32)
    a = lcb.lc_sparse_args(B=B, Tq=Tq, Tk=Tk, heads=H, kv_heads=m_shape[1], head_dim=d, dtype=_dtype("q", dtype), block=block,
                           q_block=q_block, keep=keep, sink=sink, window=window, q_pos0=q_pos0, q=s)
    if m_shape[3] != lcb.lc_sparse_blocks(a):
        raise ValueError(f"means of {m_shape[3]} blocks, {Tk} keys have {lcb.lc_sparse_blocks(a)}")
    return a, (B, H, lcb.lc_sparse_groups(a), max(keep, 0))


def block_attention(q, k, v, index, block: int = 64, q_block: int = 128, q_len=None, k_len=None, q_prescaled: bool = False, out=None):
    """Attention of q [B, Tq, heads, head_dim] over the keys and values [B, Tk, kv_heads, head_dim] of the blocks that ``index`` (int32
    [B, heads, groups, keep], of :func:`block_select` or of the caller's own) lists for each group of q_block queries."""
    _on(q.device, k, v, index, q_len, k_len, out)
    out = _out(out, q.shape, q.dtype, q.device)
    a, groups, need = _attention_args(q.shape, q.stride(), q.dtype, k.shape, k.stride(), v.shape, v.stride(), out.stride(), index.shape,
                                      block, q_block, bool(q_prescaled))
    B, H = q.shape[0], q.shape[2]
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("k and v must be of q's type")
    if index.dtype != torch.int32 or not index.is_contiguous() or index.shape[:3] != (B, H, groups):
        raise ValueError(f"index must be contiguous int32 of shape {(B, H, groups)} x keep")
    ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None  # (its own: captured calls share none)
    _launch(q.device, lcb.lc_op_block_attention, a, q.data_ptr(), k.data_ptr(), v.data_ptr(), index.data_ptr(), _lens("q_len", q_len, B),
            _lens("k_len", k_len, B), out.data_ptr(), _ptr(ws), need)
    return out


@_kept
def _attention_args(q_shape, q_stride, dtype, k_shape, k_stride, v_shape, v_stride, out_stride, index_shape, block, q_block, q_prescaled):
    sq, sk = _strides("q", q_shape, q_stride), _strides("k", k_shape, k_stride)
    sv = sk if (v_shape, v_stride) == (k_shape, k_stride) else _strides("v", v_shape, v_stride)
    B, Tq, H, d = q_shape
    if k_shape != v_shape or k_shape[0] != B or k_shape[3] != d:
        raise ValueError("k and v must be [B, Tk, kv_heads, head_dim] of q's batch and head_dim")
    lcb.fits("Tq Tk keep block q_block", max(q_shape), max(k_shape), max(index_shape), block, q_block)
    a = lcb.lc_sparse_args(B=B, Tq=Tq, Tk=k_shape[1], heads=H, kv_heads=k_shape[2], head_dim=d, dtype=_dtype("q", dtype), block=block,
                           q_block=q_block, keep=index_shape[3] if len(index_shape) == 4 else 0, window=-1, q_prescaled=int(q_prescaled),
                           q=sq, k=sk, v=sv, out=_strides("out", q_shape, out_stride))
    return a, lcb.lc_sparse_groups(a), lcb.lc_block_attention_workspace(a)


# ---- quantised cache entries ------------------------------------------------------------------------------------------
def entry_bytes(rows: int, cols: int, fmt: str) -> int:
    """Bytes of an entry of rows x cols values."""
    lcb.fits("rows cols", rows >> 32, cols)
    return lcb.lc_entry_packed_bytes(lcb.lc_entry_args(format=_named(FORMATS, "fmt", fmt), rows=rows, cols=cols))


def entry_pack(x, fmt: str, base=None, out=None, entry=None):
    """Writes x [rows, cols] into an entry (uint8; ``entry``, or a new one, which is returned). With ``out`` [rows, cols] also
    out = base + what the entry stands for (base None: zeros), in the same pass."""
    a, need = _entry_args(fmt, x.shape, x.stride(), x.dtype, *_rest(base, out))
    _on(x.device, base, out, entry)
    entry = _out(entry, (need,), torch.uint8, x.device, "entry")
    if not entry.is_contiguous():
        raise ValueError("entry must be contiguous")
    _launch(x.device, lcb.lc_op_entry_pack, a, x.data_ptr(), entry.data_ptr(), _ptr(base), _ptr(out))
    return entry


def entry_unpack(entry, rows: int, cols: int, fmt: str, base=None, out=None, dtype=torch.float32):
    """out [rows, cols] = base + the values of an entry (base None: zeros)."""
    _on(entry.device, base, out)
    if out is None:
        out = torch.empty(rows, cols, dtype=dtype if base is None else base.dtype, device=entry.device)
    a, need = _entry_args(fmt, (rows, cols), None, None, *_rest(base, out))
    if entry.dtype != torch.uint8 or entry.dim() != 1 or not entry.is_contiguous() or entry.numel() < need:
        raise ValueError(f"entry must be contiguous uint8 of {need} bytes")
    _launch(entry.device, lcb.lc_op_entry_unpack, a, entry.data_ptr(), _ptr(base), out.data_ptr())
    return out


def _rest(base, out):
    """What a descriptor says of base and out."""
    if out is None:
        if base is not None:
            raise ValueError("base without out")
        return None, None, None
    if base is not None and (base.shape != out.shape or base.dtype != out.dtype or
                             (base.stride() != out.stride() and _row_stride("base", base.shape, base.stride()) != _row_stride("out", out.shape, out.stride()))):
        raise ValueError("base must have the shape, type and row stride of out")
    return out.shape, out.stride(), out.dtype


def _row_stride(name, shape, stride):
    if len(shape) != 2:
        raise ValueError(f"{name} must be [rows, cols], not of shape {tuple(shape)}")
    if shape[1] > 1 and stride[1] != 1:
        raise ValueError(f"{name}: the values of a row must lie next to each other")
    return stride[0] if shape[0] > 1 else max(shape[1], stride[0])


@_kept
def _entry_args(fmt, shape, x_stride, x_dtype, y_shape, y_stride, y_dtype):
    a = lcb.lc_entry_args(format=_named(FORMATS, "fmt", fmt))
    if x_stride is not None:
        a.x_ld, a.x_dtype = _row_stride("x", shape, x_stride), _dtype("x", x_dtype)
    a.rows, a.cols = shape
    lcb.fits("cols", shape[1])
    if y_shape is not None:
        if tuple(y_shape) != tuple(shape):
            raise ValueError(f"out must be of shape {tuple(shape)}")
        a.y_ld, a.y_dtype = _row_stride("out", y_shape, y_stride), _dtype("out", y_dtype)
    return a, lcb.lc_entry_packed_bytes(a)
