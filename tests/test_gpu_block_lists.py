"""Attention over listed blocks where lists are long and heads share keys: lists of more entries than are read at a time, lists that
end there, several heads of a key head placed together, calls that are shared out in different ways. Bounds are those of
test_gpu_tokens.py."""
import numpy as np
import pytest
import torch

from oracle import tokens_oracle as tko
from paper_2510_05367_amd import binding as lcb
from paper_2510_05367_amd import tokens
from tests.test_gpu_tokens import BF, F32, attention_bound, clusters, close, f64, gpu, ints, random_lists

pytestmark = pytest.mark.gpu

LONG = [  # B, Tq, Tk, H, Hkv, d, block, q_block, keep, k_len: entries are read 64 at a time
    (1, 1, 64 * 210, 2, 2, 64, 64, 1, 200, None),
    (1, 3, 64 * 300, 4, 2, 40, 64, 128, 257, [64 * 290 + 7]),
    (1, 40, 64 * 140, 2, 1, 64, 64, 64, 130, None),
    (2, 130, 64 * 80, 2, 2, 64, 64, 128, 65, [64 * 80, 64 * 66 - 1]),
    (1, 128, 128 * 75, 1, 1, 128, 128, 128, 70, None),
    (1, 33, 64 * 129, 1, 1, 16, 64, 33, 129, None),
    (4, 600, 64 * 70, 8, 4, 32, 64, 32, 66, None),
]


def case(rng, B, Tq, Tk, H, Hkv, d, dtype):
    return tuple(gpu(rng.normal(size=s), dtype) for s in ((B, Tq, H, d), (B, Tk, Hkv, d), (B, Tk, Hkv, d)))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,Tq,Tk,H,Hkv,d,block,q_block,keep,k_len", LONG)
def test_long_lists(dtype, B, Tq, Tk, H, Hkv, d, block, q_block, keep, k_len):
    rng = np.random.default_rng(Tk + d)
    q, k, v = case(rng, B, Tq, Tk, H, Hkv, d, dtype)
    index = random_lists(rng, B, H, -(-Tq // q_block), keep, -(-Tk // block))
    index[0, 0, 0] = np.sort(rng.permutation(-(-Tk // block))[:keep])
    kw = dict(block=block, q_block=q_block)
    ref, weight, dot = tko.block_attention(f64(q), f64(k), f64(v), index, k_len=k_len, **kw)
    for b in range(B):
        if k_len is not None:
            k[b, k_len[b]:], v[b, k_len[b]:] = float("nan"), float("inf")
    out = tokens.block_attention(q, k, v, ints(index.tolist()), k_len=ints(k_len), **kw)
    close(out, ref, attention_bound(q, ref, weight, dot, keep * block))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Tq", [2, 60, 128])
def test_lists_that_end_where_entries_are_read(dtype, Tq):
    """The first entry that ends a list is the last, the first or the second of those that are read together."""
    rng = np.random.default_rng(31)
    nk = 200
    q, k, v = case(rng, 1, Tq, nk * 64, 1, 1, 64, dtype)
    for at in (63, 64, 65, 127, 128, 129):
        for bad in (-1, nk, 2 ** 31 - 1, None, 0):  # None: the entry before it once more
            entries = np.arange(140)
            entries[at] = entries[at - 1] if bad is None else bad
            index = entries.astype(np.int32).reshape(1, 1, 1, -1)
            assert len(tko.listed_blocks(entries.tolist(), 64, nk * 64)) == at
            short = np.arange(at, dtype=np.int32).reshape(1, 1, 1, -1)
            ref, weight, dot = tko.block_attention(f64(q), f64(k), f64(v), short, 64, 128)
            out = tokens.block_attention(q, k, v, ints(index.tolist()))
            close(out, ref, attention_bound(q, ref, weight, dot, at * 64))


PLACED = [  # B * kv_heads a multiple of eight: the heads of a key head are placed together
    (2, 260, 64 * 30, 16, 4, 64, 128, 12), (4, 70, 500, 6, 2, 32, 32, 4), (1, 100, 700, 24, 8, 16, 7, 5), (8, 5, 300, 4, 1, 64, 2, 3), (1, 1, 4000, 32, 8, 128, 1, 40),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,Tq,Tk,H,Hkv,d,q_block,keep", PLACED)
def test_heads_that_share_keys_are_placed_together(dtype, B, Tq, Tk, H, Hkv, d, q_block, keep):
    rng = np.random.default_rng(Tk + H)
    q, k, v = case(rng, B, Tq, Tk, H, Hkv, d, dtype)
    assert B * Hkv % 8 == 0 and H > Hkv
    index = random_lists(rng, B, H, -(-Tq // q_block), keep, -(-Tk // 64))
    ref, weight, dot = tko.block_attention(f64(q), f64(k), f64(v), index, 64, q_block)
    out = tokens.block_attention(q, k, v, ints(index.tolist()), q_block=q_block)
    close(out, ref, attention_bound(q, ref, weight, dot, keep * 64))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_batches_that_are_shared_out_differently(dtype):
    """The same queries in batches of 1, 16 and 64: lists are cut, or tiles shared, or neither. Sums are then taken in another order; within
    a launch copies have the same bits."""
    rng = np.random.default_rng(33)
    q, k, v = case(rng, 1, 64, 1500, 8, 2, 64, dtype)
    index = random_lists(rng, 1, 8, 1, 16, 24)
    ref, weight, dot = tko.block_attention(f64(q), f64(k), f64(v), index, 64, 64)
    needs = []
    for B in (1, 16, 64):
        more = [t.expand(B, -1, -1, -1) for t in (q, k, v)]
        out = tokens.block_attention(*more, ints(index.tolist()).expand(B, -1, -1, -1).contiguous(), q_block=64)
        close(out[:1], ref, attention_bound(q, ref, weight, dot, 16 * 64))
        assert all(torch.equal(out[0], o) for o in out)
        a = lcb.lc_sparse_args(B=B, Tq=64, Tk=1500, heads=8, kv_heads=2, head_dim=64, dtype=lcb.LC_BF16 if dtype == BF else lcb.LC_F32, block=64, q_block=64,
                               keep=16, window=-1, q=lcb.lc_strides(32768, 512, 64), k=lcb.lc_strides(0, 128, 64), v=lcb.lc_strides(0, 128, 64),
                               out=lcb.lc_strides(32768, 512, 64))
        needs.append(lcb.lc_block_attention_workspace(a))
    assert needs[0] > 0 and needs[2] == 0


def test_captured_where_a_workgroup_takes_much_lds():
    """Selection over 8192 blocks and attention with heads of 128 ask for more LDS than a kernel has by itself: captured, and replayed with eager
    calls between, they give the eager bits."""
    rng = np.random.default_rng(34)
    nk, d, H = 8192, 128, 2
    k = gpu(rng.normal(size=(1, nk * 64, 1, d)), BF)
    qs = [gpu(clusters(rng, 1, 100, H, d), BF) for _ in range(3)]
    means = tokens.block_means(k)

    def both(q):
        index = tokens.block_select(q, means, nk * 64, 70, q_block=25, sink=1)
        return index, tokens.block_attention(q, k, k, index, q_block=25), tokens.block_attention(q.float(), k.float(), k.float(), index, q_block=25)

    src = qs[0].clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = both(src)
    for n in range(5):
        src.copy_(qs[n % 3])
        graph.replay()
        want = both(qs[n % 3])
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), n
    assert np.array_equal(want[0].cpu().numpy(), tko.block_select(f64(qs[1]), means.cpu().numpy(), nk * 64, 70, 64, 25, sink=1))
