"""The operators over the tokens of long videos against their float64 oracle, at the sizes, layouts and masks where they can go
wrong. Bounds are derived: a rounding to a type t is off by at most finfo(t).eps / 2 of the value (bf16 2^-8, float 2^-24).

  rotary     a turn is rounded to float (at most half of one, off by 2^-26: 2^-23.3 in the angle), sine and cosine are good to 2^-22.5
             (float) or 2^-17.5 (the hardware's, bf16), and amplitude, products and sum round three times: below
             (|u| + |v|) A 2^-21 or 2^-17, and the rounding of the result.
  attention  probabilities are rounded to the operands' type before they meet V, alike in numerator and denominator: an output is
             off by at most r (sum w |v| + |o|), r the type's half step; scores of exact products summed in float are off by (d + 2)
             2^-24 sum |q k|, which weighs twice; the exponent's argument, the exponential and sums over n keys add (n + 64) 2^-24; then
             the rounding of the result.
  means      sums in 64 bits; selections and entries are exact."""
import math

import numpy as np
import pytest
import torch

from oracle import tokens_oracle as tko
from paper_2510_05367_amd import binding as lcb
from paper_2510_05367_amd import tokens

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
BF, F32 = torch.bfloat16, torch.float32
NAN = float("nan")


def gpu(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda", dtype)


def f64(t):
    return t.double().cpu().numpy()


def ints(a):
    return None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")


def close(got, ref, bound):
    got = f64(got)
    assert got.shape == ref.shape
    off = np.abs(got - ref) - bound
    assert np.all(off <= 0), f"off by {np.max(np.abs(got - ref)):.3e}, beyond the bound by {np.max(off):.3e} at {np.unravel_index(np.argmax(off), off.shape)}"


# ---- rotary positions ------------------------------------------------------------------------------------------------
def check_rope(x, y, pos, axes, layout, inverse, **scaling):
    xs = f64(x)
    ref = tko.rope(xs, pos, axes, layout, inverse, **scaling)
    size = np.zeros_like(xs)
    for u, v, _, _ in tko.rope_pairs(axes, layout):
        size[..., u] = size[..., v] = np.abs(xs[..., u]) + np.abs(xs[..., v])
    amp = 0.1 * math.log(scaling.get("factor", 1.0)) + 1.0
    close(y, ref, amp * size * (2.0 ** -21 if x.dtype == F32 else 2.0 ** -17) + HALF_STEP[x.dtype] * np.abs(ref))
    rot = sum(axes)
    assert torch.equal(x[..., rot:], y[..., rot:])


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("B,T,H,d,axes", [(1, 1, 1, 2, (2,)), (1, 1, 16, 64, (64,)), (2, 37, 3, 64, (16, 24, 24)), (3, 5, 2, 40, (40,)), (1, 67, 5, 128, (96,)),
                                          (2, 9, 7, 30, (4, 6)), (1, 130, 1, 128, (128,)), (2, 4100, 2, 16, (8,)), (1, 3, 300, 8, (2, 2, 2))])
def test_rope(dtype, layout, B, T, H, d, axes):
    rng = np.random.default_rng(T * d)
    x = gpu(rng.normal(size=(B, T, H, d)), dtype)
    t = tokens.make_rope(d, axes=axes, layout=layout)
    grid = (-(-T // 12), 4, 3)[3 - len(axes):] if len(axes) > 1 else None
    tt = np.arange(T)
    cells = {1: [tt], 2: [tt // 3, tt % 3], 3: [tt // 12, tt // 3 % 4, tt % 3]}[len(axes)]
    start = tuple(range(5, 5 + len(axes)))
    pos = np.stack([c + s for c, s in zip(cells, start)], axis=-1)
    full = np.broadcast_to(pos, (B, T, len(axes)))
    for inverse in (False, True):
        y = tokens.rope(x, t, grid=grid, start=start, inverse=inverse)
        check_rope(x, y, full, axes, layout, inverse)
        assert torch.equal(y, tokens.rope(x, t, pos=ints(pos.tolist()), inverse=inverse))
        z = x.clone()
        assert tokens.rope(z, t, grid=grid, start=start, inverse=inverse, out=z) is z and torch.equal(y, z)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("scaling,kw", [("linear", dict(factor=4.0)), ("base", dict(factor=8.0)), ("parts", dict(factor=32.0, orig_len=4096))])
def test_rope_far_positions_and_scalings(dtype, scaling, kw):
    rng = np.random.default_rng(3)
    x = gpu(rng.normal(size=(2, 6, 2, 64)), dtype)
    pos = np.array([[0, 1, 4095, 1000003, 2 ** 31 - 1, -7], [5, 4, 3, 2, 1, 2 ** 30]])[..., None]
    t = tokens.make_rope(64, axes=(48,), scaling=scaling, layout="interleaved", **kw)
    y = tokens.rope(x, t, pos=ints(pos.tolist()))
    check_rope(x, y, pos, (48,), "interleaved", False, scaling=scaling, **kw)
    far = 2 ** 40 - 8  # an angle of 10^12 radians, formed in 64 bits on both sides: off by 2^-53 of itself, 2^-13
    y = tokens.rope(x, tokens.make_rope(64), start=far)
    ref = tko.rope(f64(x), np.broadcast_to((far + np.arange(6))[None, :, None], (2, 6, 1)), (64,), "half")
    close(y, ref, 2.0 ** -9 * np.abs(f64(x)).max() * 2 + HALF_STEP[dtype] * np.abs(ref))


@pytest.mark.parametrize("dtype", [F32, BF])
def test_rope_layouts_of_memory(dtype):
    """Packed q,k,v rows, heads in front of tokens, a batch of stride zero, rows that are not aligned: the values of a dense
    tensor, and nothing beside the output is written."""
    rng = np.random.default_rng(4)
    t = tokens.make_rope(40, axes=(32,))
    dense = gpu(rng.normal(size=(2, 21, 6, 40)), dtype)
    y = tokens.rope(dense, t)
    packed = torch.full((2, 21, 9, 40), 7.0, dtype=dtype, device="cuda")
    packed[:, :, :6] = dense
    assert torch.equal(y, tokens.rope(packed[:, :, :6], t))
    tokens.rope(packed[:, :, :6], t, out=packed[:, :, :6])
    assert torch.equal(packed[:, :, :6], y) and torch.all(packed[:, :, 6:] == 7.0)
    assert torch.equal(y, tokens.rope(dense.transpose(1, 2).contiguous().transpose(1, 2), t))
    odd = torch.full((2, 21, 6, 43), 7.0, dtype=dtype, device="cuda")
    odd[..., 1:41] = dense
    tokens.rope(odd[..., 1:41], t, out=odd[..., 1:41])
    assert torch.equal(odd[..., 1:41], y) and torch.all(odd[..., 0] == 7.0) and torch.all(odd[..., 41:] == 7.0)
    same = dense[:1].expand(3, -1, -1, -1)
    assert torch.equal(tokens.rope(same, t), y[:1].expand(3, -1, -1, -1))
    assert tokens.rope(dense[:, :0], t).shape == (2, 0, 6, 40)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_transpose(layout):
    """inverse is the transpose: <rope(x), g> = <x, rope^T(g)>, the gradient, also of scaled amplitudes; and it agrees with differences."""
    rng = np.random.default_rng(5)
    kw = dict(axes=(24, 16), layout=layout, scaling="parts", factor=16.0, orig_len=512)
    t = tokens.make_rope(48, **kw)
    x, g = gpu(rng.normal(size=(1, 30, 3, 48)), F32), gpu(rng.normal(size=(1, 30, 3, 48)), F32)
    dx = tokens.rope(g, t, grid=(5, 6), inverse=True)
    lhs, rhs = (tokens.rope(x, t, grid=(5, 6)).double() * g.double()).sum().item(), (x.double() * dx.double()).sum().item()
    # 4320 products, each off by the bound of an element: |x| |g| 2 A 2^-21, summed as a worst case
    assert abs(lhs - rhs) <= 4320 * 2 * 1.3 * 2.0 ** -21 * 4 * 2
    pos = np.stack([np.arange(30) // 6, np.arange(30) % 6], -1)[None]
    f = lambda v: (tko.rope(v, pos, (24, 16), layout, scaling="parts", factor=16.0, orig_len=512) * f64(g)).sum()  # noqa: E731
    for i in [(0, 0, 0, 0), (0, 29, 2, 39), (0, 17, 1, 13), (0, 3, 0, 47)]:
        e = np.zeros(x.shape)
        e[i] = 0.5  # (linear: a difference of any size is the derivative)
        assert abs((f(f64(x) + e) - f(f64(x) - e)) - f64(dx)[i]) <= 2.0 ** -18


# ---- selection -------------------------------------------------------------------------------------------------------
def clusters(rng, B, T, H, d, run=50):
    shared = np.repeat(rng.normal(size=(B, -(-T // run), H, d)), run, axis=1)[:, :T]
    return 0.8 * shared + 0.6 * rng.normal(size=(B, T, H, d))


SELECT = [  # B, Tq, Tk, H, Hkv, d, block, q_block, keep, q_len, k_len
    (1, 1, 1, 1, 1, 8, 64, 1, 1, None, None),
    (1, 1, 4096, 4, 4, 64, 64, 128, 16, None, None),
    (2, 300, 300, 4, 2, 40, 64, 100, 3, [300, 129], [300, 129]),
    (3, 130, 1000, 2, 1, 128, 128, 64, 5, [0, 1, 130], [1000, 0, 65]),
    (2, 65, 700, 3, 3, 16, 64, 7, 20, None, [700, -3]),
    (1, 520, 2100, 8, 8, 32, 64, 1, 4, None, None),
    (2, 1000, 1000, 32, 8, 64, 64, 32, 6, None, None),
    (1, 2500, 9000, 16, 4, 64, 64, 32, 40, None, [8999]),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,Tq,Tk,H,Hkv,d,block,q_block,keep,q_len,k_len", SELECT)
def test_means_and_selection(dtype, B, Tq, Tk, H, Hkv, d, block, q_block, keep, q_len, k_len):
    rng = np.random.default_rng(Tk + d)
    k, q = gpu(clusters(rng, B, Tk, Hkv, d), dtype), gpu(clusters(rng, B, Tq, H, d), dtype)
    kf, qf = f64(k), f64(q)
    for b in range(B):  # what does not exist is not read
        if k_len is not None:
            k[b, max(k_len[b], 0):] = NAN
        if q_len is not None:
            q[b, q_len[b]:] = NAN
    means = tokens.block_means(k, block=block, k_len=ints(k_len))
    ref = tko.block_means(kf, block, k_len)
    assert means.dtype == torch.float64
    assert np.all(np.abs(means.cpu().numpy() - ref) <= 2.0 ** -53 * (block + 2) * 8.0)  # |k| < 8
    for sink, window, pos0 in ((0, -1, 0), (1, 0, Tk - Tq), (0, 1, 0), (3, 2, Tk - Tq), (0, 0, -200)):
        kw = dict(block=block, q_block=q_block, sink=sink, window=window, q_pos0=pos0)
        got = tokens.block_select(q, means, Tk, keep, q_len=ints(q_len), k_len=ints(k_len), **kw)
        want = tko.block_select(qf, ref, Tk, keep, q_len=q_len, k_len=k_len, **kw)
        assert np.array_equal(got.cpu().numpy(), want), (sink, window, pos0)


def test_selection_ties_nan_and_long_lists():
    """Equal scores go to the lower index, a score that is no number ranks last, and lists longer than the keys end in -1."""
    d, nk = 8, 200
    k = torch.zeros(1, nk * 64, 1, d, device="cuda")
    score = np.array([(j * 7) % 5 for j in range(nk)], dtype=np.float64)
    k[0, :, 0, 0] = torch.from_numpy(np.repeat(score, 64)).float().cuda()
    k[0, 64 * 3:64 * 4, 0, 0] = NAN
    q = torch.zeros(1, 3, 1, d, device="cuda")
    q[0, 0, 0, 0], q[0, 1, 0, 0], q[0, 2, 0, 0] = 1.0, -1.0, 0.0
    means = tokens.block_means(k)
    ref = tko.block_means(f64(k), 64)
    for keep in (1, 3, 39, 40, 41, 80, 199, 200, 201, 300):
        got = tokens.block_select(q, means, nk * 64, keep, q_block=1)
        assert np.array_equal(got.cpu().numpy(), tko.block_select(f64(q), ref, nk * 64, keep, 64, 1)), keep
    got = tokens.block_select(q, means, nk * 64, 10, q_block=1, sink=50)
    assert got[0, 0].tolist() == [list(range(10))] * 3
    many = torch.zeros(1, 8192 * 64, 1, d, device="cuda")
    many[0, ::64 * 1000, 0, 0] = 64.0
    got = tokens.block_select(q[:, :1], tokens.block_means(many), 8192 * 64, 9, q_block=1)
    assert got[0, 0, 0].tolist() == list(range(0, 8192, 1000))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("nk", [40, 100, 300, 500])
def test_selection_by_few_and_many_groups(dtype, nk):
    """Eight, four, two groups or one a workgroup, and more or fewer blocks than are held in registers, list alike; a block whose mean is
    no number changes no other's place."""
    rng = np.random.default_rng(nk)
    H, d, keep = 32, 16, 7
    k, q = gpu(clusters(rng, 1, nk * 64, 4, d), dtype), gpu(rng.normal(size=(1, 64, H, d)), dtype)
    k[0, 17 * 64 + 5, 1, 3], k[0, -1, 2, 0] = NAN, float("inf")
    means = tokens.block_means(k)
    got = tokens.block_select(q, means, nk * 64, keep, q_block=1, sink=1)
    want = tko.block_select(f64(q), tko.block_means(f64(k), 64), nk * 64, keep, 64, 1, sink=1)
    assert np.array_equal(got.cpu().numpy(), want)
    for n in (4, 16, 32, 33):
        assert torch.equal(tokens.block_select(q[:, :n], means, nk * 64, keep, q_block=1, sink=1), got[:, :, :n]), n


def test_means_of_a_growing_cache():
    rng = np.random.default_rng(9)
    k = gpu(rng.normal(size=(2, 1000, 3, 32)), BF)
    whole = tokens.block_means(k)
    some = tokens.block_means(k, k_len=ints([400, 400]))
    kept = some.clone()
    tokens.block_means(k, k_len=ints([600, 500]), first=6, count=4, out=some)
    assert torch.equal(some[..., :6], kept[..., :6]) and torch.equal(some[..., 10:], kept[..., 10:])
    assert torch.equal(some[0, ..., 6:9], whole[0, ..., 6:9]) and torch.all(some[1, ..., 8:10] == 0)
    assert np.allclose(some[1, :, :, 7].cpu().numpy(), f64(k)[1, 448:500].mean(0), rtol=0, atol=1e-14)


# ---- attention over the lists ----------------------------------------------------------------------------------------
def attention_bound(q, out, weight, dot, keys):
    d, r = q.shape[3], HALF_STEP[q.dtype]
    score = 2 * (d + 2) * 2.0 ** -24 * dot
    return (r + score + (keys + 64) * 2.0 ** -24 + 2.0 ** -20) * (weight + np.abs(out)) + r * np.abs(out)


def random_lists(rng, B, H, nq, keep, nk):
    out = np.full((B, H, nq, keep), -1, dtype=np.int32)
    for i in np.ndindex(B, H, nq):
        n = int(rng.integers(0, min(keep, nk) + 1)) if rng.random() < 0.3 else min(keep, nk)
        out[i][:n] = np.sort(rng.permutation(nk)[:n])
    return out


ATTEND = [  # B, Tq, Tk, H, Hkv, d, block, q_block, keep, q_len, k_len
    (1, 1, 1, 1, 1, 8, 64, 1, 1, None, None),
    (2, 1, 3000, 8, 2, 64, 64, 128, 33, None, [3000, 2999]),
    (1, 1, 5000, 2, 2, 128, 128, 1, 30, None, None),
    (2, 5, 130, 4, 4, 40, 64, 7, 3, None, [130, 66]),
    (3, 300, 300, 2, 2, 64, 64, 128, 4, [300, 129, 0], [300, 129, 0]),
    (2, 200, 460, 4, 1, 32, 64, 64, 5, None, [33, 460]),
    (1, 130, 700, 2, 2, 16, 192, 33, 3, None, None),
    (2, 257, 257, 3, 3, 128, 64, 100, 3, [257, 1], None),
    (1, 70, 640, 3, 1, 40, 128, 32, 5, None, None),
    (1, 64, 200, 1, 1, 8, 64, 128, 9, None, [65]),
    (1, 700, 1500, 8, 4, 64, 64, 1, 3, None, None),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,Tq,Tk,H,Hkv,d,block,q_block,keep,q_len,k_len", ATTEND)
def test_attention(dtype, B, Tq, Tk, H, Hkv, d, block, q_block, keep, q_len, k_len):
    rng = np.random.default_rng(Tq + Tk + d)
    q, k, v = (gpu(rng.normal(size=s), dtype) for s in ((B, Tq, H, d), (B, Tk, Hkv, d), (B, Tk, Hkv, d)))
    index = random_lists(rng, B, H, -(-Tq // q_block), keep, -(-Tk // block))
    kw = dict(block=block, q_block=q_block)
    ref, weight, dot = tko.block_attention(f64(q), f64(k), f64(v), index, q_len=q_len, k_len=k_len, **kw)
    for b in range(B):  # nothing that does not exist is read, and rows behind a sequence stay
        if k_len is not None:
            k[b, k_len[b]:], v[b, k_len[b]:] = NAN, float("inf")
        if q_len is not None:
            q[b, q_len[b]:] = NAN
    out = torch.full_like(q, 77.0)
    tokens.block_attention(q, k, v, ints(index.tolist()), q_len=ints(q_len), k_len=ints(k_len), out=out, **kw)
    for b, n in enumerate(q_len or []):
        assert torch.all(out[b, n:] == 77.0)
        out[b, n:] = 0
    close(out, ref, attention_bound(q, ref, weight, dot, keep * block))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Tq,q_block", [(3, 128), (60, 60), (128, 128)])
def test_attention_memory_layouts(dtype, Tq, q_block):
    """Packed rows, heads in front of tokens, shared batches: bit for bit what dense tensors give, and nothing else is written."""
    rng = np.random.default_rng(11)
    B, Tk, H, d = 2, 500, 3, 64
    qkv = gpu(rng.normal(size=(B, Tk, 3, H, d)), dtype)
    q, k, v = qkv[:, :Tq, 0], qkv[:, :, 1], qkv[:, :, 2]
    index = ints(random_lists(rng, B, H, 1, 5, 8).tolist())
    a = tokens.block_attention(q, k, v, index, q_block=q_block)
    b = tokens.block_attention(*(t.contiguous() for t in (q, k, v)), index, q_block=q_block)
    ht = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
    wide = torch.full((B, Tq, H + 2, d), 77.0, dtype=dtype, device="cuda")
    tokens.block_attention(ht(q), ht(k), ht(v), index, q_block=q_block, out=wide[:, :, 1:H + 1])
    assert torch.equal(a, b) and torch.equal(a, wide[:, :, 1:H + 1])
    assert torch.all(wide[:, :, 0] == 77.0) and torch.all(wide[:, :, H + 1] == 77.0)
    shared = tokens.block_attention(q, k[:1].expand(B, -1, -1, -1), v[:1].expand(B, -1, -1, -1), index, q_block=q_block)
    assert torch.equal(shared, tokens.block_attention(q, k[:1].repeat(B, 1, 1, 1), v[:1].repeat(B, 1, 1, 1), index, q_block=q_block))
    pre = (q.float() * (math.log2(math.e) / 8)).to(dtype)
    ref, weight, dot = tko.block_attention(f64(pre), f64(k), f64(v), index.cpu().numpy(), 64, q_block, scale=math.log(2.0))
    close(tokens.block_attention(pre, k, v, index, q_block=q_block, q_prescaled=True), ref, attention_bound(q, ref, weight, dot, 320))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Tq", [2, 50, 100])
def test_attention_of_one_key(dtype, Tq):
    """The stride of an axis of one token says nothing (zero, here); the one value is the result, infinities too."""
    rng = np.random.default_rng(17)
    q, k, v = (gpu(rng.normal(size=(1, n, 2, 64)), dtype) for n in (Tq, 1, 1))
    v[0, 0, 1, 5], v[0, 0, 0, 63] = float("inf"), -float("inf")
    out, one, row = torch.full_like(q, 77.0), lcb.lc_strides(0, 0, 64), lcb.lc_strides(0, 128, 64)
    a = lcb.lc_sparse_args(B=1, Tq=Tq, Tk=1, heads=2, kv_heads=2, head_dim=64, dtype=lcb.LC_BF16 if dtype == BF else lcb.LC_F32, block=64,
                           q_block=128, keep=1, window=-1, q=row, k=one, v=one, out=row)
    assert lcb.lc_block_attention_workspace(a) == 0
    index = ints([[[[0]], [[0]]]])
    lcb.lc_op_block_attention(a, q.data_ptr(), k.data_ptr(), v.data_ptr(), index.data_ptr(), None, None, out.data_ptr(), None, 0,
                              torch.cuda.current_stream().cuda_stream)
    # The one probability p (1, or next to it: its exponent is what a fused product leaves of a rounded one) is the denominator too,
    # so a result is fl(fl(p v) fl(1 / p)): three roundings, less than (1 + 2^-24)^3 - 1 < 2^-22 of v in float, and nothing
    # once it is rounded to bf16, where v lies.
    want, some = v.expand(1, Tq, 2, 64), torch.isfinite(v).expand(1, Tq, 2, 64)
    assert torch.equal(out[~some], want[~some])
    assert torch.all((out[some].double() - want[some].double()).abs() <= (0.0 if dtype == BF else 2.0 ** -22) * want[some].double().abs())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Tq", [2, 50, 100])
def test_lists_of_any_origin(dtype, Tq):
    """A list ends at its first entry that is no block with a key, or that does not ascend; blocks behind k_len have none."""
    rng = np.random.default_rng(12)
    q, k, v = gpu(rng.normal(size=(1, Tq, 1, 64)), dtype), gpu(rng.normal(size=(1, 1000, 1, 64)), dtype), gpu(rng.normal(size=(1, 1000, 1, 64)), dtype)
    for entries in ([1, 3, 3, 5], [4, 2, 5], [-1, 0, 1], [0, 1, 2147483647, 3], [2, -2147483648, 5], [7, 16, 3], [14, 15, 16], [9, 10, 11, 12]):
        index = np.array(entries, dtype=np.int32).reshape(1, 1, 1, -1)
        for k_len in (None, [11 * 64 + 1]):
            ref, weight, dot = tko.block_attention(f64(q), f64(k), f64(v), index, 64, 128, k_len=k_len)
            out = tokens.block_attention(q, k, v, ints(index.tolist()), k_len=ints(k_len))
            close(out, ref, attention_bound(q, ref, weight, dot, 256))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Tq,q_block", [(1, 1), (20, 32), (64, 64), (128, 128)])
@pytest.mark.parametrize("spread", [0.0, 8.0, 60.0])
def test_attention_far_scores(dtype, Tq, q_block, spread):
    """Scores from none to hundreds, rising along the list so that maxima keep rising, and values of one sign."""
    rng = np.random.default_rng(13)
    q, k = rng.normal(size=(1, Tq, 2, 32)), 0.1 * rng.normal(size=(1, 2000, 2, 32))
    q[..., 0] = 4.0
    k[..., 0] = spread * np.linspace(-1, 1, 2000)[None, :, None]
    q, k, v = gpu(q, dtype), gpu(k, dtype), gpu(rng.normal(size=(1, 2000, 2, 32)) + 2.0, dtype)
    index = random_lists(rng, 1, 2, 1, 32, 32)
    ref, weight, dot = tko.block_attention(f64(q), f64(k), f64(v), index, 64, q_block)
    close(tokens.block_attention(q, k, v, ints(index.tolist()), q_block=q_block), ref, attention_bound(q, ref, weight, dot, 2048))
    pre = (q.float() * (math.log2(math.e) / math.sqrt(32))).to(dtype)
    ref, weight, dot = tko.block_attention(f64(pre), f64(k), f64(v), index, 64, q_block, scale=math.log(2.0))
    close(tokens.block_attention(pre, k, v, ints(index.tolist()), q_block=q_block, q_prescaled=True), ref, attention_bound(q, ref, weight, dot, 2048))


def test_offsets_beyond_32_bits():
    """A cache of 2^31 elements (4 GiB) with the last blocks listed, and another batch element behind it."""
    T, H, d, block = 1 << 20, 16, 128, 128
    rng = np.random.default_rng(14)
    k = torch.empty(1, T + 640, H, d, dtype=BF, device="cuda")
    k[:, :640] = gpu(rng.normal(size=(1, 640, H, d)), BF)
    k[:, -1280:] = gpu(rng.normal(size=(1, 1280, H, d)), BF)
    q = gpu(rng.normal(size=(1, 40, H, d)), BF)
    kk, vv = k[:, 640:], k[:, :T]  # (views of one tensor)
    index = torch.tensor([8187, 8190, 8191], dtype=torch.int32, device="cuda").expand(1, H, 1, 3).contiguous()
    got = tokens.block_attention(q, kk, vv, index, block=block, q_block=64)
    near = torch.tensor([3, 6, 7], dtype=torch.int32, device="cuda").expand(1, H, 1, 3).contiguous()
    t0 = 8184 * block
    assert torch.equal(got, tokens.block_attention(q, kk[:, t0:].contiguous(), vv[:, t0:].contiguous(), near, block=block, q_block=64))
    two = torch.cat([q, q.flip(1)])
    halves = k[0, :T].view(2, T // 2, H, d)  # the second batch element starts beyond 2^30 elements, its last keys beyond 2^31 bytes
    last = torch.tensor([8190], dtype=torch.int32, device="cuda").expand(2, H, 1, 1).contiguous()
    a = tokens.block_attention(two, halves, halves, last, block=64, q_block=64)
    b = tokens.block_attention(two[1:], halves[1:, -128:].contiguous(), halves[1:, -128:].contiguous(), torch.zeros_like(last[1:]), block=64, q_block=64)
    assert torch.equal(a[1:], b)
    means = tokens.block_means(k[:, 640:], block=block)
    assert torch.equal(means[..., 8184:], tokens.block_means(kk[:, t0:].contiguous(), block=block))
    t = tokens.make_rope(d)
    assert torch.equal(tokens.rope(kk, t, start=5)[:, -9:], tokens.rope(kk[:, -9:].contiguous(), t, start=5 + T - 9))


# ---- entries ---------------------------------------------------------------------------------------------------------
def entry_input(rng, rows, cols, dtype):
    x = rng.normal(size=(rows, cols)) * np.exp2(rng.integers(-20, 20, size=(rows, 1)))
    x[rng.random((rows, cols)) < 0.05] = 0.0
    flat = x.reshape(-1)
    for i, s in enumerate([127.0, 448.0, 6.0, 0.25, 2.5, 5.0, 127.5, 3.5, -0.0]):  # tops of scales and ties
        flat[(i * 37) % flat.size] = s
    return gpu(x, dtype)


@pytest.mark.parametrize("fmt", ["mxint8", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 31), (2, 33), (7, 100), (33, 64), (5, 1000), (130, 77)])
def test_entries(fmt, dtype, rows, cols):
    rng = np.random.default_rng(rows * cols)
    x = entry_input(rng, rows, cols, dtype)
    ref, exps = tko.entry(f64(x), fmt)
    y = torch.full((rows, cols + 5), 7.0, device="cuda")
    entry = tokens.entry_pack(x, fmt, out=y[:, 2:cols + 2])
    assert entry.numel() == tokens.entry_bytes(rows, cols, fmt)
    assert np.array_equal(entry[entry.numel() - exps.size:].cpu().numpy().reshape(exps.shape), exps + 127)
    assert np.array_equal(f64(y[:, 2:cols + 2]), ref)
    assert torch.all(y[:, :2] == 7.0) and torch.all(y[:, cols + 2:] == 7.0)
    back = tokens.entry_unpack(entry, rows, cols, fmt)
    assert np.array_equal(f64(back), ref)
    base = gpu(rng.normal(size=(rows, cols)), F32)
    want = base + back
    assert torch.equal(tokens.entry_unpack(entry, rows, cols, fmt, base=base), want)
    again = base.clone()
    assert torch.equal(tokens.entry_pack(x, fmt, base=again, out=again), entry) and torch.equal(again, want)
    small = tokens.entry_unpack(entry, rows, cols, fmt, base=base.to(BF))
    assert small.dtype == BF and torch.equal(small, (base.to(BF).float() + back).to(BF))
    wide = torch.full((rows, cols + 3), NAN, dtype=dtype, device="cuda")  # rows of another stride and alignment
    wide[:, 1:cols + 1] = x
    assert torch.equal(tokens.entry_pack(wide[:, 1:cols + 1], fmt), entry)
    # what an entry stands for is kept as it is, at this scale and at the next smaller ones that still hold it
    assert torch.equal(tokens.entry_unpack(tokens.entry_pack(back, fmt), rows, cols, fmt), back)


@pytest.mark.parametrize("fmt", ["mxint8", "mxfp8", "mxfp4"])
def test_entries_of_extremes(fmt):
    """The largest and smallest numbers, denormal scales, infinities and NaNs: those mark their own group and no other."""
    x = np.zeros((1, 32 * 8), dtype=np.float32)
    x[0, 0:32] = np.finfo(np.float32).max * np.linspace(-1, 1, 32)
    x[0, 32:64] = np.float32(1e-45) * np.arange(32)
    x[0, 64:96] = np.float32(1.2e-38) * np.linspace(-1, 1, 32)
    x[0, 96:128] = np.float32(2.0 ** -121) * np.arange(32)
    x[0, 128:160] = 1.0
    x[0, 130] = np.inf
    x[0, 191] = np.nan
    x[0, 200] = -np.inf
    x[0, 224:256] = 3.0
    ref, exps = tko.entry(x, fmt)
    t = torch.from_numpy(x).cuda()
    y = torch.empty_like(t)
    entry = tokens.entry_pack(t, fmt, out=y)
    assert np.array_equal(entry[-8:].cpu().numpy(), exps[0] + 127) and list(exps[0, 4:]) == [128, 128, 128, exps[0, 7]]
    for got in (y, tokens.entry_unpack(entry, 1, 256, fmt)):
        assert np.array_equal(f64(got), ref.astype(np.float32), equal_nan=True)


# ---- together, as a step uses them -----------------------------------------------------------------------------------
def chain(qkv, table, entry, base, out):
    tokens.rope(qkv[:, :, :2].flatten(2, 3), table, grid=(3, 10, 20), out=qkv[:, :, :2].flatten(2, 3))
    q, k, v = qkv.unbind(2)
    index = tokens.block_select(q, tokens.block_means(k), k.shape[1], 4, q_block=64, sink=1, window=0)
    y = tokens.block_attention(q, k, v, index, q_block=64)
    tokens.entry_pack(y.flatten(2).flatten(0, 1), "mxint8", base=base, out=out, entry=entry)
    return index, y


@pytest.mark.parametrize("dtype", [BF, F32])
def test_together(dtype):
    rng = np.random.default_rng(15)
    B, T, H, d = 2, 600, 4, 64
    raw = gpu(clusters(rng, B, T, 3 * H, d).reshape(B, T, 3, H, d), dtype)
    table = tokens.make_rope(d, axes=(16, 24, 24))
    base = gpu(rng.normal(size=(B * T, H * d)), F32)
    entry = torch.empty(tokens.entry_bytes(B * T, H * d, "mxint8"), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(base)
    qkv = raw.clone()
    index, y = chain(qkv, table, entry, base, out)
    tt = np.arange(T)
    pos = np.broadcast_to(np.stack([tt // 200, tt // 20 % 10, tt % 20], -1), (B, T, 3))
    check_rope(raw[:, :, :2].flatten(2, 3), qkv[:, :, :2].flatten(2, 3), pos, (16, 24, 24), "half", False)
    assert torch.equal(qkv[:, :, 2], raw[:, :, 2])
    q, k, v = (f64(t) for t in qkv.unbind(2))  # each operator on what the one before left
    want = tko.block_select(q, tko.block_means(k, 64), T, 4, 64, 64, sink=1, window=0)
    assert np.array_equal(index.cpu().numpy(), want)
    ref, weight, dot = tko.block_attention(q, k, v, want, 64, 64)
    close(y, ref, attention_bound(y, ref, weight, dot, 256))
    values = tokens.entry_unpack(entry, B * T, H * d, "mxint8")
    rows = y.flatten(2).flatten(0, 1)
    got, _ = tko.entry(f64(rows[:50]), "mxint8")
    assert np.array_equal(f64(values[:50]), got) and torch.equal(out, base + values)


def test_captured_and_on_another_stream():
    """Two graphs of the chain, replayed in turn with eager calls between them, each checked against the eager result."""
    rng = np.random.default_rng(16)
    B, T, H, d = 1, 600, 4, 64
    table = tokens.make_rope(d, axes=(16, 24, 24))
    raws = [gpu(clusters(rng, B, T, 3 * H, d).reshape(B, T, 3, H, d), BF) for _ in range(3)]
    base = gpu(rng.normal(size=(B * T, H * d)), F32)

    def bufs():
        return (torch.empty(tokens.entry_bytes(B * T, H * d, "mxint8"), dtype=torch.uint8, device="cuda"), base, torch.empty_like(base))

    def few(qkv):  # one query against the rows: several workgroups share a list
        q, k, v = qkv.unbind(2)
        return tokens.block_attention(q[:, :1], k, v, torch.arange(10, dtype=torch.int32, device="cuda").expand(B, H, 1, 10).contiguous())

    want = []
    for r in raws:
        b, qkv = bufs(), r.clone()
        index, y = chain(qkv, table, *b)
        want.append((index.clone(), y.clone(), b[0].clone(), b[2].clone(), few(qkv)))
    graphs = []
    for _ in range(2):
        src, b = raws[0].clone(), bufs()
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            qkv = src.clone()
            index, y = chain(qkv, table, *b)
            last = few(qkv)
        graphs.append((g, src, index, y, b, last))
    for n in range(6):
        g, src, index, y, b, last = graphs[n % 2]
        src.copy_(raws[n % 3])
        g.replay()
        chain(raws[(n + 1) % 3].clone(), table, *bufs())
        torch.cuda.synchronize()
        for got, ref in zip((index, y, b[0], b[2], last), want[n % 3]):
            assert torch.equal(got, ref), n
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b, qkv = bufs(), raws[1].clone()
        index, y = chain(qkv, table, *b)
        last = few(qkv)
    side.synchronize()
    for got, ref in zip((index, y, b[0], b[2], last), want[1]):
        assert torch.equal(got, ref)


def test_results_do_not_depend_on_the_neighbours():
    """A query's output is the same bits whatever group tile, batch or launch it is in, as long as its list is the same."""
    rng = np.random.default_rng(17)
    q, k, v = (gpu(rng.normal(size=(2, n, 8, 64)), BF) for n in (512, 2048, 2048))
    q[0, :256] *= 30.0
    lists = ints(np.broadcast_to(np.arange(0, 32, 2, dtype=np.int32), (2, 8, 4, 16)).tolist())
    whole = tokens.block_attention(q, k, v, lists)
    perm = torch.randperm(512, device="cuda")
    assert torch.equal(tokens.block_attention(q[:, perm], k, v, lists), whole[:, perm])
    assert all(torch.equal(whole, tokens.block_attention(q, k, v, lists)) for _ in range(3))
