"""What the operators over the tokens of long videos refuse, and their host-only helpers: no call here reaches a GPU (each is
refused before anything is launched; the pointers are never followed)."""
import ctypes

import pytest
import torch

from paper_2510_05367_amd import binding as lcb
from paper_2510_05367_amd import tokens

P = 1 << 20  # an aligned address that nobody reads


def refused(status, words, call):
    with pytest.raises(lcb.LcError) as e:
        call()
    assert e.value.status == status, e.value
    assert words in str(e.value) and words in lcb.lc_last_error()


def rope_config(**kw):
    c = dict(head_dim=64, axes=1, dims=(64, 0, 0), layout=0, scaling=0, orig_len=0, base=1e4, factor=1.0, beta_fast=32.0, beta_slow=1.0)
    c.update(kw)
    dims = c.pop("dims")
    return lcb.lc_rope_config(axis_dim=(ctypes.c_int32 * 3)(*dims), **c)


def test_struct_layouts():
    assert ctypes.sizeof(lcb.lc_strides) == 24 and ctypes.sizeof(lcb.lc_rope_config) == 64
    assert ctypes.sizeof(lcb.lc_rope_table) == 32 + 8 + 8 * lcb.LC_ROPE_MAX_PAIRS
    assert ctypes.sizeof(lcb.lc_rope_args) == 16 + 48 + 16 + 24 + 8
    assert ctypes.sizeof(lcb.lc_sparse_args) == 48 + 16 + 96 and ctypes.sizeof(lcb.lc_entry_args) == 40


@pytest.mark.parametrize("kw,status,words", [
    (dict(head_dim=0), 2, "head_dim"), (dict(head_dim=130), 2, "head_dim"), (dict(axes=0), 2, "axes"), (dict(axes=4), 2, "axes"),
    (dict(dims=(63, 0, 0)), 2, "axis_dim"), (dict(dims=(0, 0, 0)), 2, "axis_dim"), (dict(dims=(66, 0, 0)), 2, "axis_dim"),
    (dict(axes=2, dims=(40, 40, 0)), 2, "more channels"), (dict(layout=2), 1, "layout"), (dict(scaling=4), 1, "scaling"),
    (dict(base=1.0), 2, "base"), (dict(base=float("nan")), 2, "base"), (dict(scaling=1, factor=0.0), 2, "factor"),
    (dict(scaling=2, factor=float("inf")), 2, "factor"), (dict(scaling=3, factor=2.0), 2, "orig_len"),
    (dict(scaling=3, factor=2.0, orig_len=64, beta_fast=1.0), 2, "beta_fast")])
def test_rope_tables(kw, status, words):
    refused(status, words, lambda: lcb.lc_rope_make(rope_config(**kw)))


def test_rope_table_values_and_python_checks():
    t = tokens.make_rope(64, axes=(16, 24, 24), scaling="linear", factor=2.0)
    two_pi = 6.283185307179586
    assert t.rot_dim == 64 and t.amplitude == 1.0 and t.turns[0] == pytest.approx(0.5 / two_pi) and t.turns[8] == t.turns[20] == t.turns[0]
    assert t.turns[1] == pytest.approx(0.5 * 1e4 ** (-2 / 16) / two_pi) and t.turns[9] == pytest.approx(0.5 * 1e4 ** (-2 / 24) / two_pi)
    assert tokens.make_rope(64, scaling="parts", factor=0.5, orig_len=64).amplitude == 1.0
    for bad in (lambda: tokens.make_rope(64, axes=()), lambda: tokens.make_rope(64, layout="quarter"), lambda: tokens.make_rope(64, scaling="x")):
        with pytest.raises(ValueError):
            bad()


def rope_args(**kw):
    a = dict(B=1, T=4, heads=2, dtype=lcb.LC_F32, x=lcb.lc_strides(512, 128, 64), y=lcb.lc_strides(512, 128, 64))
    a.update(kw)
    return lcb.lc_rope_args(**a)


@pytest.mark.parametrize("kw,status,words", [
    (dict(B=0), 2, "positive"), (dict(T=-1), 2, "positive"), (dict(heads=0), 2, "positive"), (dict(dtype=2), 1, "dtype"),
    (dict(inverse=2), 1, "inverse"), (dict(B=65536), 2, "B must"), (dict(heads=(1 << 20) + 1), 2, "heads"), (dict(T=(1 << 27) + 1), 2, "tokens"),
    (dict(start=(ctypes.c_int64 * 3)((1 << 40) + 1, 0, 0)), 2, "start")])
def test_rope_calls(kw, status, words):
    refused(status, words, lambda: lcb.lc_op_rope(tokens.make_rope(64), rope_args(**kw), P, None, 2 * P, None))


def test_rope_pointers_tables_and_grids():
    t = tokens.make_rope(64)
    for x, y in ((None, P), (P, None)):
        refused(1, "NULL", lambda: lcb.lc_op_rope(t, rope_args(), x, None, y, None))
    refused(1, "lc_rope_make", lambda: lcb.lc_op_rope(lcb.lc_rope_table(), rope_args(), P, None, 2 * P, None))
    refused(2, "same strides", lambda: lcb.lc_op_rope(t, rope_args(y=lcb.lc_strides(512, 64, 256)), P, None, P, None))
    refused(2, "grid", lambda: lcb.lc_op_rope(tokens.make_rope(64, axes=(32, 32)), rope_args(), P, None, 2 * P, None))
    for y in (lcb.lc_strides(0, 128, 64), lcb.lc_strides(512, 0, 64), lcb.lc_strides(512, 128, 0)):
        refused(2, "overlap", lambda: lcb.lc_op_rope(t, rope_args(B=2, y=y), P, None, 2 * P, None))
    t.axis_dim[0] = 32
    refused(1, "lc_rope_make", lambda: lcb.lc_op_rope(t, rope_args(), P, None, 2 * P, None))


def sparse_args(**kw):
    s = lcb.lc_strides(1000 * 128, 128, 64)
    a = dict(B=2, Tq=1000, Tk=1000, heads=2, kv_heads=2, head_dim=64, dtype=lcb.LC_BF16, block=64, q_block=128, keep=4, sink=0, window=-1,
             q_pos0=0, q_prescaled=0, q=s, k=s, v=s, out=s)
    a.update(kw)
    return lcb.lc_sparse_args(**a)


BAD_SPARSE = [(dict(B=0), 2, "positive"), (dict(Tq=0), 2, "positive"), (dict(Tk=0), 2, "positive"), (dict(heads=3), 2, "multiple of kv_heads"),
              (dict(kv_heads=0), 2, "positive"), (dict(head_dim=24), 2, "head_dim"), (dict(dtype=7), 1, "dtype"), (dict(block=0), 2, "block"),
              (dict(block=96), 2, "block"), (dict(block=-64), 2, "block"), (dict(q_block=0), 2, "q_block"), (dict(q_block=129), 2, "q_block"),
              (dict(keep=0), 2, "keep"), (dict(keep=65537), 2, "keep"), (dict(Tk=64 * 8192 + 1), 2, "8192"),
              (dict(Tk=(1 << 30) + 1), 2, "2^30"), (dict(block=1 << 21), 2, "2^20"), (dict(B=(1 << 31) - 1, heads=(1 << 31) - 1, kv_heads=1), 2, "2^24")]
means_call = lambda a: lcb.lc_op_block_means(a, P, None, P, 0, 1, None)  # noqa: E731
select_call = lambda a: lcb.lc_op_block_select(a, P, P, None, None, P, None)  # noqa: E731
attend_call = lambda a: lcb.lc_op_block_attention(a, P, P, P, P, None, None, P, P, 1 << 40, None)  # noqa: E731


@pytest.mark.parametrize("call", [means_call, select_call, attend_call])
@pytest.mark.parametrize("kw,status,words", BAD_SPARSE)
def test_sparse_descriptors(call, kw, status, words):
    refused(status, words, lambda: call(sparse_args(**kw)))
    assert lcb.lc_block_attention_workspace(sparse_args(**kw)) == 0


@pytest.mark.parametrize("call,names", [(means_call, "k"), (select_call, "q"), (attend_call, "qkv")])
def test_sparse_alignment(call, names):
    for n in list(names) + (["out"] if names == "qkv" else []):
        for bad in (lcb.lc_strides(1000 * 128 + 4, 128, 64), lcb.lc_strides(1000 * 128, 132, 64), lcb.lc_strides(1000 * 128, 128, 68)):
            refused(2, "16-byte aligned", lambda: call(sparse_args(**{n: bad})))


def test_sparse_pointers_ranges_and_workspaces():
    a = sparse_args()
    refused(1, "NULL", lambda: lcb.lc_op_block_means(a, None, None, P, 0, 1, None))
    refused(1, "NULL", lambda: lcb.lc_op_block_means(a, P, None, None, 0, 1, None))
    refused(2, "aligned", lambda: lcb.lc_op_block_means(a, P + 2, None, P, 0, 1, None))
    for first, count in ((-1, 1), (0, -1), (0, 17), (16, 1), (2147483647, 2147483647)):
        refused(1, "range", lambda: lcb.lc_op_block_means(a, P, None, P, first, count, None))
    lcb.lc_op_block_means(a, P, None, P, 3, 0, None)  # nothing to do
    refused(1, "NULL", lambda: lcb.lc_op_block_select(a, P, None, None, None, P, None))
    refused(1, "NULL", lambda: lcb.lc_op_block_select(a, P, P, None, None, None, None))
    refused(1, "sink", lambda: select_call(sparse_args(sink=-1)))
    refused(2, "q_pos0", lambda: select_call(sparse_args(q_pos0=(1 << 40) + 1)))
    refused(1, "index is NULL", lambda: lcb.lc_op_block_attention(a, P, P, P, None, None, None, P, P, 1 << 40, None))
    refused(1, "out is NULL", lambda: lcb.lc_op_block_attention(a, P, P, P, P, None, None, None, P, 1 << 40, None))
    refused(1, "q_prescaled", lambda: attend_call(sparse_args(q_prescaled=2)))
    refused(2, "overlap", lambda: attend_call(sparse_args(k=lcb.lc_strides(1000 * 128, 56, 64))))
    refused(2, "2^30", lambda: attend_call(sparse_args(v=lcb.lc_strides(0, 1 << 24, 64))))
    refused(2, "2^30", lambda: attend_call(sparse_args(k=lcb.lc_strides(0, -128, 64))))
    refused(2, "overlap", lambda: attend_call(sparse_args(out=lcb.lc_strides(0, 128, 64))))
    few = sparse_args(Tq=1, keep=16)
    need = lcb.lc_block_attention_workspace(few)
    assert need > 0 and need % (2 * 2 * 1 * 66 * 4) == 0
    for ws, n in ((None, need), (P, need - 1)):
        refused(4, "workspace", lambda: lcb.lc_op_block_attention(few, P, P, P, P, None, None, P, ws, n, None))
    refused(1, "workspace", lambda: lcb.lc_op_block_attention(few, P, P, P, P, None, None, P, P + 4, need, None))
    assert lcb.lc_block_attention_workspace(sparse_args(B=64, q_block=1)) == 0
    assert lcb.lc_sparse_groups(a) == 8 and lcb.lc_sparse_blocks(a) == 16 and lcb.lib().lc_sparse_groups(None) == 0


def entry_args(**kw):
    a = dict(format=lcb.LC_ENTRY_INT8, cols=100, rows=10, x_dtype=lcb.LC_F32, y_dtype=lcb.LC_F32, x_ld=100, y_ld=100)
    a.update(kw)
    return lcb.lc_entry_args(**a)


def test_entries():
    pack = lambda a, x=P, e=P, b=P, y=P: lcb.lc_op_entry_pack(a, x, e, b, y, None)  # noqa: E731
    unpack = lambda a, e=P, b=P, y=P: lcb.lc_op_entry_unpack(a, e, b, y, None)  # noqa: E731
    for call in (pack, unpack):
        for f in (-1, 3):
            refused(1, "format", lambda: call(entry_args(format=f)))
        for kw in (dict(rows=0), dict(cols=0), dict(rows=-1), dict(rows=1 << 40), dict(rows=(1 << 27) - 15)):
            refused(2, "rows and cols", lambda: call(entry_args(**kw)))
        refused(1, "entry is NULL", lambda: call(entry_args(), e=None))
        refused(1, "16-byte", lambda: call(entry_args(), e=P + 8))
        refused(1, "y_dtype", lambda: call(entry_args(y_dtype=2)))
        refused(2, "y_ld", lambda: call(entry_args(y_ld=99)))
    refused(1, "x is NULL", lambda: pack(entry_args(), x=None))
    refused(1, "x_dtype", lambda: pack(entry_args(x_dtype=-1)))
    refused(2, "x_ld", lambda: pack(entry_args(x_ld=99)))
    refused(1, "base without y", lambda: pack(entry_args(), y=None))
    refused(1, "y is NULL", lambda: unpack(entry_args(), y=None))
    # 10 rows of 128 codes and four scale bytes
    assert lcb.lc_entry_packed_bytes(entry_args()) == 1280 + 40
    assert lcb.lc_entry_packed_bytes(entry_args(format=lcb.LC_ENTRY_FP4)) == 640 + 40
    assert tokens.entry_bytes(8192, 1024, "mxint8") == 8192 * 1024 + 8192 * 32
    assert lcb.lc_entry_packed_bytes(entry_args(format=7)) == 0 and lcb.lc_entry_packed_bytes(entry_args(rows=0)) == 0


def test_entries_written_over_their_values_keep_rows_in_place():
    """A thread's values go where other threads still read, unless rows and types are the same."""
    for kw in (dict(y_ld=104), dict(x_ld=104), dict(y_dtype=lcb.LC_BF16), dict(x_dtype=lcb.LC_BF16)):
        refused(2, "in place", lambda: lcb.lc_op_entry_pack(entry_args(**kw), P, P, None, P, None))


def test_tensors_that_are_refused_before_the_library():
    """There is no CPU fallback, and shapes and types are told apart by name."""
    x = torch.zeros(1, 4, 2, 64)
    t = tokens.make_rope(64)
    i = torch.zeros(1, 2, 1, 3, dtype=torch.int32)
    for bad in (lambda: tokens.rope(x, t), lambda: tokens.block_means(x), lambda: tokens.block_attention(x, x, x, i),
                lambda: tokens.entry_pack(x[0, 0], "mxint8"), lambda: tokens.rope(x[..., :32], t), lambda: tokens.rope(x[0], t),
                lambda: tokens.rope(x.half(), t), lambda: tokens.rope(x.transpose(2, 3).reshape(1, 4, 64, 2).transpose(2, 3), t),
                lambda: tokens.rope(x, t, pos=torch.zeros(4)), lambda: tokens.rope(x, t, grid=(1, 2)), lambda: tokens.block_means(x, count=0),
                lambda: tokens.block_attention(x, x[:, :, :1], x, i), lambda: tokens.block_attention(x, x, x, i[:, :1]),
                lambda: tokens.block_attention(x, x, x, i.long()), lambda: tokens.entry_pack(x, "mxint8"),
                lambda: tokens.entry_pack(x[0, 0], "int8"), lambda: tokens.entry_pack(x[0, 0], "mxint8", base=x[0, 0]),
                lambda: tokens.entry_unpack(torch.zeros(8, dtype=torch.uint8), 1, 64, "mxint8")):
        with pytest.raises(ValueError):
            bad()
