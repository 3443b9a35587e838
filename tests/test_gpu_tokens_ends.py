"""The operators of long videos where sequences, lists, number ranges and launches end, against their float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import tokens_oracle as tko
from paper_2510_05367_amd import tokens
from tests.test_gpu_tokens import BF, F32, NAN, clusters, f64, gpu, ints

pytestmark = pytest.mark.gpu


# ---- rotary positions ------------------------------------------------------------------------------------------------
def test_rope_of_2_to_24_tokens():
    """As many tokens as a launch has workgroups of one: 635 units each (a pair and 126 channels that are copied, of five heads)."""
    rng = np.random.default_rng(20)
    T, H, d, ends = 1 << 24, 5, 128, 9
    t = tokens.make_rope(d, axes=(2,))
    row = gpu(rng.normal(size=(1, 1, H, d)), BF)
    y = torch.zeros(1, T, H, d, dtype=BF, device="cuda")  # 21 GB
    tokens.rope(row.expand(1, T, H, d), t, start=3, out=y)
    for at in (0, T // 2 - 5, T - ends):
        assert torch.equal(y[:, at:at + ends], tokens.rope(row.expand(1, ends, H, d).contiguous(), t, start=3 + at)), at
    assert torch.equal(y[0, :, :, 2:].amax(0), row[0, 0, :, 2:]) and torch.equal(y[0, :, :, 2:].amin(0), row[0, 0, :, 2:])
    del y
    torch.cuda.empty_cache()


# ---- selection -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, F32])
def test_forced_blocks_are_those_of_queries_that_exist(dtype):
    """Keys reach beyond the queries: a short sequence's lists are those of the call that is not padded."""
    rng = np.random.default_rng(21)
    B, Tq, Tk, H, d, keep = 4, 300, 1000, 4, 32, 3
    k, q = gpu(clusters(rng, B, Tk, 2, d), dtype), gpu(clusters(rng, B, Tq, H, d), dtype)
    q_len = [1, 129, 300, 64]
    means, ref = tokens.block_means(k), tko.block_means(f64(k), 64)
    for q_block, window, pos0 in ((128, 0, 0), (100, 1, 40), (128, 2, 500), (7, 0, 63), (128, 0, -100)):
        kw = dict(q_block=q_block, window=window, q_pos0=pos0)
        got = tokens.block_select(q, means, Tk, keep, q_len=ints(q_len), **kw)
        assert np.array_equal(got.cpu().numpy(), tko.block_select(f64(q), ref, Tk, keep, 64, q_len=q_len, **kw)), kw
        for b, n in enumerate(q_len):
            alone = tokens.block_select(q[b:b + 1, :n], means[b:b + 1].contiguous(), Tk, keep, **kw)
            assert torch.equal(alone[0], got[b, :, :alone.shape[2]]), (kw, b)


def test_windows_of_any_width():
    """Positions may lie as far from the keys as a window is wide."""
    rng = np.random.default_rng(22)
    Tk, block = 64 * 12, 64
    k, q = gpu(rng.normal(size=(1, Tk, 2, 16)), F32), gpu(rng.normal(size=(1, 5, 2, 16)), F32)
    means, ref = tokens.block_means(k), tko.block_means(f64(k), block)
    most = 2 ** 31 - 1
    for at, window in ((70000, 69995), (70000, 69990), (-70000, 70003), (2 ** 31, most), (-(2 ** 31), most), (0, most), (2 ** 34 - 2, most), (7, 65536)):
        for keep in (2, 9):
            got = tokens.block_select(q, means, Tk, keep, q_block=2, window=window, q_pos0=at * block)
            assert np.array_equal(got.cpu().numpy(), tko.block_select(f64(q), ref, Tk, keep, block, 2, 0, window, at * block)), (at, window, keep)


# ---- attention over the lists ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, F32])
def test_first_key_of_a_cache_with_heads_in_front(dtype):
    """One key of a long cache whose heads lie in front of its tokens: its rows are a whole head apart."""
    rng = np.random.default_rng(24)
    B, H, T, d = 2, 16, 16384, 64
    k, v = (torch.full((B, H, T, d), NAN, dtype=dtype, device="cuda") for _ in range(2))
    k[:, :, :2], v[:, :, :2] = gpu(rng.normal(size=(B, H, 2, d)), dtype), gpu(rng.normal(size=(B, H, 2, d)), dtype)
    index = torch.zeros(B, H, 1, 1, dtype=torch.int32, device="cuda")
    for Tq in (1, 40):
        q = gpu(rng.normal(size=(B, Tq, H, d)), dtype)
        for n in (1, 2):
            kn, vn = (t[:, :, :n].transpose(1, 2) for t in (k, v))
            got = tokens.block_attention(q, kn, vn, index)
            assert torch.equal(got, tokens.block_attention(q, kn.contiguous(), vn.contiguous(), index)), (Tq, n)
            means = tokens.block_means(kn)
            assert torch.equal(means, tokens.block_means(kn.contiguous()))
            assert torch.equal(tokens.block_select(q, means, n, 1), index)


# ---- entries ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["mxint8", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_finite_entries_stay_finite_and_as_they_are(fmt, dtype):
    """Values at the top of the range, beside others of every size: what they are held as is finite, and is packed to itself."""
    rng = np.random.default_rng(23)
    big = float(torch.finfo(dtype).max)
    x = np.exp2(rng.uniform(100, 128, size=(64, 96))) * rng.choice([-1.0, 1.0], size=(64, 96))
    x = np.clip(x, -big, big)
    x[::2, ::32], x[1::4, 5::32] = big, -big * (1 - 2.0 ** -6)
    t = torch.from_numpy(x).to("cuda", dtype)
    ref, exps = tko.entry(f64(t), fmt)
    y = torch.empty(64, 96, device="cuda")
    entry = tokens.entry_pack(t, fmt, out=y)
    assert np.array_equal(entry[-64 * 3:].cpu().numpy().reshape(64, 3), exps + 127)
    assert bool(torch.isfinite(y).all()) and np.array_equal(f64(y), ref) and torch.equal(tokens.entry_unpack(entry, 64, 96, fmt), y)
    small = tokens.entry_unpack(entry, 64, 96, fmt, dtype=BF)
    assert np.array_equal(f64(small), ref)  # (codes have at most 7 bits: bf16 holds them too)
    for again in (y, small):
        assert torch.equal(tokens.entry_unpack(tokens.entry_pack(again, fmt), 64, 96, fmt), y)
