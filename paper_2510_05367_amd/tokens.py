"""Operators over the tokens of long videos, on torch tensors: rotary positions, attention over selected key blocks, quantised
cache entries (the C ABI's section of the same name in include/lightcache.h, which has the definitions).

Tensors are [B, T, heads, head_dim] views of any strides with channels next to each other (rows of packed q,k,v, say). Calls
enqueue on torch's current stream of the tensors' device and take outputs and workspaces from torch's allocator on it, so
they order with torch's own work and may be captured into a graph. No gradients are recorded (the map of :func:`rope` has its
transpose: ``inverse=True``). What a call refuses raises :class:`binding.LcError`, or ``ValueError`` where it never gets there.
"""
from __future__ import annotations

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


def _dtype(name, t):
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    return _DTYPES[t.dtype]


def _on(device, **tensors):
    """The tensors that are given are on that GPU."""
    if device.type != "cuda":
        raise ValueError("tensors must be on a GPU (there is no CPU fallback)")
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError(f"{name} is on {t.device}, not on {device}")


def _strides(name, t):
    """Strides of [B, T, heads, head_dim]; those of axes of length one are what a dense tensor would have."""
    if t.dim() != 4:
        raise ValueError(f"{name} must be [B, T, heads, head_dim], not of shape {tuple(t.shape)}")
    if t.shape[3] > 1 and t.stride(3) != 1:
        raise ValueError(f"{name}: the channels of a head must lie next to each other")
    B, T, H, d = t.shape
    head = t.stride(2) if H > 1 else d
    token = t.stride(1) if T > 1 else max(d, head * H)
    return lcb.lc_strides(t.stride(0) if B > 1 else max(token * T, head * H), token, head)


def _lens(name, t, B):
    if t is None:
        return None
    if t.dtype != torch.int32 or tuple(t.shape) != (B,) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor of shape ({B},)")
    return t.data_ptr()


def _out(out, shape, dtype, device, name="out"):
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if tuple(out.shape) != tuple(shape) or out.dtype != dtype:
        raise ValueError(f"{name} must be {dtype} of shape {tuple(shape)}")
    return out


def _stream(device):
    return torch.cuda.current_stream(device).cuda_stream


# ---- rotary positions -------------------------------------------------------------------------------------------------
def make_rope(head_dim: int, axes: Optional[Sequence[int]] = None, base: float = 10000.0, layout: str = "half", scaling: str = "none",
              factor: float = 1.0, orig_len: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0) -> lcb.lc_rope_table:
    """The table :func:`rope` takes, made once for a model. ``axes``: the channels that each position axis turns, those of the
    first axis first (default: one axis, the whole head)."""
    dims = [head_dim] if axes is None else list(axes)
    if not 1 <= len(dims) <= 3:
        raise ValueError("there are one to three axes")
    return lcb.lc_rope_make(lcb.lc_rope_config(head_dim=head_dim, axes=len(dims), axis_dim=(lcb.C.c_int32 * 3)(*dims),
                                               layout=_named(LAYOUTS, "layout", layout), scaling=_named(SCALINGS, "scaling", scaling),
                                               orig_len=orig_len, base=base, factor=factor, beta_fast=beta_fast, beta_slow=beta_slow))


def rope(x, table: lcb.lc_rope_table, pos=None, grid: Optional[Sequence[int]] = None, start=0, inverse: bool = False, out=None):
    """x [B, T, heads, head_dim] turned by its tokens' positions; ``out`` may be x. Positions: ``pos`` (int32, [T, axes], [B, T, axes], or
    without the last axis where there is one), else the cells of ``grid`` in row-major order, else running numbers;
    ``start`` (a number or one an axis) is added to the latter two."""
    if x.dim() != 4:
        raise ValueError(f"x must be [B, T, heads, head_dim], not of shape {tuple(x.shape)}")
    B, T, H, d = x.shape
    if d != table.head_dim:
        raise ValueError(f"heads of {d} channels, the table is for {table.head_dim}")
    out = _out(out, x.shape, x.dtype, x.device)
    _on(x.device, out=out, pos=pos)
    n = table.axes
    starts = [start] * n if isinstance(start, int) else list(start)
    if len(starts) != n or (grid is not None and len(grid) != n):
        raise ValueError(f"grid and start have one value for each of the {n} axes")
    a = lcb.lc_rope_args(B=B, T=T, heads=H, dtype=_dtype("x", x), x=_strides("x", x), y=_strides("out", out), inverse=int(bool(inverse)),
                         grid=(lcb.C.c_int32 * 3)(*(grid or [])), start=(lcb.C.c_int64 * 3)(*starts), pos_batch=0)
    if pos is not None:
        if grid is not None or any(starts):
            raise ValueError("pos holds the positions: no grid and no start beside it")
        if n == 1 and pos.shape[-1:] != (1,) or pos.dim() == 1:
            pos = pos.unsqueeze(-1)
        if pos.dtype != torch.int32 or not pos.is_contiguous() or tuple(pos.shape) not in ((T, n), (B, T, n)):
            raise ValueError(f"pos must be contiguous int32 of shape {(T, n)} or {(B, T, n)}")
        a.pos_batch = T * n if pos.dim() == 3 else 0
    if x.numel() == 0:
        return out
    with torch.cuda.device(x.device):
        lcb.lc_op_rope(table, a, x.data_ptr(), None if pos is None else pos.data_ptr(), out.data_ptr(), _stream(x.device))
    return out


# ---- attention over selected blocks -----------------------------------------------------------------------------------
def block_means(k, block: int = 64, k_len=None, first: int = 0, count: Optional[int] = None, out=None):
    """Means of the key blocks [first, first + count) of k [B, Tk, kv_heads, head_dim], in float64 [B, kv_heads, head_dim, blocks];
    ``out``: the tensor of an earlier call, whose other blocks stay."""
    s = _strides("k", k)
    B, Tk, Hkv, d = k.shape
    a = lcb.lc_sparse_args(B=B, Tq=1, Tk=Tk, heads=Hkv, kv_heads=Hkv, head_dim=d, dtype=_dtype("k", k), block=block, q_block=1, keep=1,
                           window=-1, k=s)
    nk = lcb.lc_sparse_blocks(a)
    count = nk - first if count is None else count
    if out is None and (first, count) != (0, nk):
        raise ValueError("some blocks of a tensor: give the tensor")
    out = _out(out, (B, Hkv, d, nk), torch.float64, k.device)
    if not out.is_contiguous():
        raise ValueError("out must be contiguous")
    _on(k.device, k_len=k_len, out=out)
    with torch.cuda.device(k.device):
        lcb.lc_op_block_means(a, k.data_ptr(), _lens("k_len", k_len, B), out.data_ptr(), first, count, _stream(k.device))
    return out


def block_select(q, means, Tk: int, keep: int, block: int = 64, q_block: int = 128, sink: int = 0, window: int = -1, q_pos0: int = 0,
                 q_len=None, k_len=None, out=None):
    """The lists of the groups of q_block queries of q [B, Tq, heads, head_dim]: int32 [B, heads, groups, keep], ascending, -1 behind
    their ends. ``means``: :func:`block_means` of the Tk keys."""
    s = _strides("q", q)
    B, Tq, H, d = q.shape
    if means.dim() != 4 or means.dtype != torch.float64 or not means.is_contiguous() or means.shape[0] != B or means.shape[2] != d:
        raise ValueError("means must be what block_means made for these sizes")
    a = lcb.lc_sparse_args(B=B, Tq=Tq, Tk=Tk, heads=H, kv_heads=means.shape[1], head_dim=d, dtype=_dtype("q", q), block=block,
                           q_block=q_block, keep=keep, sink=sink, window=window, q_pos0=q_pos0, q=s)
    if means.shape[3] != lcb.lc_sparse_blocks(a):
        raise ValueError(f"means of {means.shape[3]} blocks, {Tk} keys have {lcb.lc_sparse_blocks(a)}")
    out = _out(out, (B, H, lcb.lc_sparse_groups(a), max(keep, 0)), torch.int32, q.device)
    if not out.is_contiguous():
        raise ValueError("out must be contiguous")
    _on(q.device, means=means, q_len=q_len, k_len=k_len, out=out)
    with torch.cuda.device(q.device):
        lcb.lc_op_block_select(a, q.data_ptr(), means.data_ptr(), _lens("q_len", q_len, B), _lens("k_len", k_len, B), out.data_ptr(),
                               _stream(q.device))
    return out


def block_attention(q, k, v, index, block: int = 64, q_block: int = 128, q_len=None, k_len=None, q_prescaled: bool = False, out=None):
    """Attention of q [B, Tq, heads, head_dim] over the keys and values [B, Tk, kv_heads, head_dim] of the blocks that ``index`` (int32
    [B, heads, groups, keep], of :func:`block_select` or of the caller's own) lists for each group of q_block queries."""
    sq, sk, sv = _strides("q", q), _strides("k", k), _strides("v", v)
    B, Tq, H, d = q.shape
    Tk, Hkv = k.shape[1], k.shape[2]
    if k.shape != v.shape or k.shape[0] != B or k.shape[3] != d or k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("k and v must be [B, Tk, kv_heads, head_dim] of q's type, batch and head_dim")
    out = _out(out, q.shape, q.dtype, q.device)
    a = lcb.lc_sparse_args(B=B, Tq=Tq, Tk=Tk, heads=H, kv_heads=Hkv, head_dim=d, dtype=_dtype("q", q), block=block, q_block=q_block,
                           keep=index.shape[-1] if index.dim() == 4 else 0, window=-1, q_prescaled=int(bool(q_prescaled)), q=sq, k=sk, v=sv,
                           out=_strides("out", out))
    if index.dtype != torch.int32 or not index.is_contiguous() or tuple(index.shape[:3]) != (B, H, lcb.lc_sparse_groups(a)):
        raise ValueError(f"index must be contiguous int32 of shape {(B, H, lcb.lc_sparse_groups(a))} x keep")
    _on(q.device, k=k, v=v, index=index, q_len=q_len, k_len=k_len, out=out)
    need = lcb.lc_block_attention_workspace(a)
    with torch.cuda.device(q.device):
        ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
        lcb.lc_op_block_attention(a, q.data_ptr(), k.data_ptr(), v.data_ptr(), index.data_ptr(), _lens("q_len", q_len, B),
                                  _lens("k_len", k_len, B), out.data_ptr(), ws.data_ptr() if need else None, need, _stream(q.device))
    return out


# ---- quantised cache entries ------------------------------------------------------------------------------------------
def _rows(name, t):
    if t.dim() != 2:
        raise ValueError(f"{name} must be [rows, cols], not of shape {tuple(t.shape)}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the values of a row must lie next to each other")
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], t.stride(0))


def entry_bytes(rows: int, cols: int, fmt: str) -> int:
    """Bytes of an entry of rows x cols values."""
    return lcb.lc_entry_packed_bytes(lcb.lc_entry_args(format=_named(FORMATS, "fmt", fmt), rows=rows, cols=cols))


def entry_pack(x, fmt: str, base=None, out=None, entry=None):
    """Writes x [rows, cols] into an entry (uint8; ``entry``, or a new one, which is returned). With ``out`` [rows, cols] also
    out = base + what the entry stands for (base None: zeros), in the same pass."""
    ld = _rows("x", x)
    rows, cols = x.shape
    a = lcb.lc_entry_args(format=_named(FORMATS, "fmt", fmt), rows=rows, cols=cols, x_dtype=_dtype("x", x), x_ld=ld)
    _rest(a, base, out)
    need = lcb.lc_entry_packed_bytes(a)
    entry = _out(entry, (need,), torch.uint8, x.device, "entry")
    _on(x.device, base=base, out=out, entry=entry)
    if not entry.is_contiguous():
        raise ValueError("entry must be contiguous")
    with torch.cuda.device(x.device):
        lcb.lc_op_entry_pack(a, x.data_ptr(), entry.data_ptr(), None if base is None else base.data_ptr(),
                             None if out is None else out.data_ptr(), _stream(x.device))
    return entry


def entry_unpack(entry, rows: int, cols: int, fmt: str, base=None, out=None, dtype=torch.float32):
    """out [rows, cols] = base + the values of an entry (base None: zeros)."""
    if out is None:
        out = torch.empty(rows, cols, dtype=dtype if base is None else base.dtype, device=entry.device)
    if tuple(out.shape) != (rows, cols):
        raise ValueError(f"out must be of shape {(rows, cols)}")
    a = lcb.lc_entry_args(format=_named(FORMATS, "fmt", fmt), rows=rows, cols=cols)
    _rest(a, base, out)
    if entry.dtype != torch.uint8 or entry.dim() != 1 or not entry.is_contiguous() or entry.numel() < lcb.lc_entry_packed_bytes(a):
        raise ValueError(f"entry must be contiguous uint8 of {lcb.lc_entry_packed_bytes(a)} bytes")
    _on(entry.device, base=base, out=out)
    with torch.cuda.device(entry.device):
        lcb.lc_op_entry_unpack(a, entry.data_ptr(), None if base is None else base.data_ptr(), out.data_ptr(), _stream(entry.device))
    return out


def _rest(a, base, out):
    """base and out of an entry call: of one shape, type and row stride."""
    if out is None:
        if base is not None:
            raise ValueError("base without out")
        return
    a.y_dtype, a.y_ld = _dtype("out", out), _rows("out", out)
    if tuple(out.shape) != (a.rows, a.cols):
        raise ValueError(f"out must be of shape {(a.rows, a.cols)}")
    if base is not None and (base.shape != out.shape or base.dtype != out.dtype or _rows("base", base) != a.y_ld):
        raise ValueError("base must have the shape, type and row stride of out")
