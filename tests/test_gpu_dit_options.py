"""The transformer stack with rotary positions, attention over selected blocks and quantised entries, against its oracle with the
definitions of those operators in it; and the invariants of the method with them."""
import numpy as np
import pytest
import torch

from oracle import dit_oracle as dito
from oracle import tokens_oracle as tko
from paper_2510_05367_amd import binding as lcb
from paper_2510_05367_amd import synth, tokens
from tests.gpu_util import check, host

pytestmark = pytest.mark.gpu

F32 = synth.DitConfig("dit_f32", B=2, T=330, D=128, heads=2, head_dim=64, L=4, cache_a=1, cache_b=3, dtype="f32")
BF16 = synth.DitConfig("dit_bf16", B=1, T=200, D=320, heads=8, head_dim=40, L=3, cache_a=1, cache_b=2, dtype="bf16")
BF16_W = synth.DitConfig("dit_bf16_w", B=2, T=288, D=256, heads=4, head_dim=64, L=5, cache_a=0, cache_b=3, dtype="bf16", mlp_ratio=2)


class Oracle(dito.DitOracle):
    def __init__(self, cfg, weights, entry=None, sparse=None, axes=None, grid=None):
        super().__init__(cfg, weights)
        self.entry, self.sparse, self.axes, self.grid = entry, sparse, axes, grid

    def attn_branch(self, x, i, m):
        c, w, D = self.cfg, self.w, self.cfg.D
        h = dito.layer_norm(x, c.ln_eps) * (1.0 + m[1]) + m[0]
        q, k, v = np.split((h @ w[f"blk{i}.wqkv"].T + w[f"blk{i}.bqkv"]).reshape(1, c.T, 3 * c.heads, c.head_dim), 3, axis=2)
        if self.axes:
            t = np.arange(c.T)
            g = self.grid or (c.T,)
            pos = np.stack([t // int(np.prod(g[a + 1:])) % (g[a] if a else c.T) for a in range(len(g))], -1)[None]
            q, k = tko.rope(q, pos, self.axes), tko.rope(k, pos, self.axes)
        s = dict(block=64, q_block=128, keep=-(-c.T // 64), sink=0, window=-1)
        s.update(self.sparse or {})
        lists = tko.block_select(q, tko.block_means(k, s["block"]), c.T, s["keep"], s["block"], s["q_block"], s["sink"], s["window"])
        o = tko.block_attention(q, k, v, lists, s["block"], s["q_block"])[0].reshape(c.T, D)
        return m[2] * (o @ w[f"blk{i}.wo"].T + w[f"blk{i}.bo"])

    def _deep(self, xa, mod):
        delta = super()._deep(xa, mod)
        return tko.entry(delta.reshape(-1, self.cfg.D), self.entry)[0].reshape(delta.shape) if self.entry else delta


OPTIONS = [  # (with lists that the score chooses, float only: a rounding could choose another block)
    (F32, dict(sparse=dict(keep=3, q_block=64))),
    (F32, dict(sparse=dict(keep=2, block=128, q_block=100, sink=1), axes=(16, 24, 24), grid=(6, 5, 11))),
    (F32, dict(axes=(64,))),
    (BF16, dict(axes=(8, 16, 16), grid=(2, 10, 10))),
    (BF16, dict(sparse=dict(keep=9), axes=(40,))),
    (BF16_W, dict(sparse=dict(keep=1, q_block=64, window=0), axes=(32, 32), grid=(16, 18))),
]


def make(cfg, entry=None, sparse=None, axes=None, grid=None, **kw):
    w = synth.make_dit_weights(cfg, 0, sharp=8.0)
    dit = lcb.Dit(cfg, w, host_slots=1, dev_slots=2, **kw)
    rope = tokens.make_rope(cfg.head_dim, axes=axes) if axes else None
    dit.set_options(lcb.make_dit_options(entry=entry, rope=rope, grid=grid, **(sparse or {})))
    torch.cuda.set_stream(dit.compute)
    return dit, w


@pytest.mark.parametrize("B,T,D,heads,opt", [(2, 1, 256, 4, dict(sparse=dict(keep=2, sink=1), axes=(64,))), (1, 33, 320, 8, dict(sparse=dict(keep=1, q_block=1))),
                                             (2, 65, 256, 4, dict(sparse=dict(keep=5, q_block=20), axes=(16, 24, 24), grid=(1, 7, 10)))])
def test_few_tokens_in_a_workspace_of_nan(B, T, D, heads, opt):
    """Every block is listed; what lies behind the tokens in the workspace is whatever was there."""
    cfg = BF16_W.with_(B=B, T=T, D=D, heads=heads, head_dim=D // heads, L=2, cache_a=1, cache_b=2)
    dit, w = make(cfg, entry="mxint8", **opt)
    try:
        x, mod = synth.make_dit_hidden(cfg, 1), synth.make_dit_modulation(cfg, 2)
        out, again = dit.empty(*x.shape), dit.empty(*x.shape)
        xd, md = dit.to_device(x), dit.to_device(mod)
        dit.arena.fill_(255)
        torch.cuda.synchronize()
        dit.full_step(xd, md, out, 0)
        dit.cached_step(xd, md, again, 0)
        dit.sync()
        assert torch.equal(out, again)
        orc = Oracle(cfg, {k: v.astype(np.float64) for k, v in w.items()}, **opt)
        want = orc.full_step(x, mod, 0)
        delta = orc.dev[0].reshape(-1, D)
        # the entry's rounding beside the step's own: half a step of 2^e, max|x| > 63.5 * 2^e
        step = np.abs(delta).reshape(-1, D // 32, 32).max(axis=2).max() / 63.5
        g = host(out)
        assert np.max(np.abs(g - want)) <= 2e-2 * max(1.0, np.abs(want).max() / 4) + step / 2 + 1e-2 * np.abs(delta).max()
    finally:
        dit.close()


@pytest.mark.parametrize("cfg,opt", OPTIONS)
def test_steps_match_oracle(cfg, opt):
    dit, w = make(cfg, **opt, token_chunk=100)
    try:
        x, mod = synth.make_dit_hidden(cfg, 1), synth.make_dit_modulation(cfg, 2)
        out = dit.empty(*x.shape)
        dit.full_step(dit.to_device(x), dit.to_device(mod), out, 0)
        dit.sync()
        orc = Oracle(cfg, {k: v.astype(np.float64) for k, v in w.items()}, **opt)
        check("normal step", host(out), orc.full_step(x, mod, 0), cfg.dtype, wide_range=True)
        check("Delta", host(dit.dev_entry(0)), orc.dev[0], cfg.dtype)
    finally:
        dit.close()


@pytest.mark.parametrize("fmt", ["mxint8", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("cfg", [F32, BF16], ids=lambda c: c.name)
def test_entries_are_what_the_accumulated_delta_packs_to(cfg, fmt):
    """The entry is that of the Delta a stack without options leaves, to the bit; steps on it are the plain stack's on its values."""
    dit, _ = make(cfg)
    try:
        x, md = dit.to_device(synth.make_dit_hidden(cfg, 1)), dit.to_device(synth.make_dit_modulation(cfg, 2))
        full, cached, other = (dit.empty(cfg.B, cfg.T, cfg.D) for _ in range(3))
        dit.full_step(x, md, full, 0)
        dit.sync()
        delta = dit.dev_entry(0)
        flat = delta.reshape(-1, cfg.D)
        entry = tokens.entry_pack(flat, fmt)
        values = tokens.entry_unpack(entry, *flat.shape, fmt).reshape(delta.shape)
        assert 0 < float((values - delta).abs().max()) <= float(delta.abs().max()) * {"mxint8": 2 ** -6, "mxfp8": 2 ** -4, "mxfp4": 2 ** -2}[fmt]
        dit.cache_write(1, values)
        dit.cached_step(x, md, other, 1)
        dit.sync()
        dit.set_options(lcb.make_dit_options(entry=fmt))
        with pytest.raises(lcb.LcError):  # options empty the slots
            dit.cached_step(x, md, cached, 1)
        dit.full_step(x, md, full, 0)
        dit.cached_step(x, md, cached, 0)
        dit.sync()
        assert torch.equal(full, cached) and torch.equal(full, other)
        assert torch.equal(dit.dev_entry(0), values)
        # through the bank and back into a poisoned slot
        dit.swap_out(0, 0)
        dit.cache_write(1, torch.full_like(delta, float("nan")))
        assert torch.all(torch.isnan(dit.dev_entry(1)))
        dit.sync()
        assert dit.host_entry_bytes(0) == entry.cpu().numpy().tobytes()
        dit.swap_in(0, 1)
        dit.cached_step(x, md, cached, 1)
        dit.sync()
        assert torch.equal(full, cached)
        dit.cache_write(1, delta)
        assert torch.equal(dit.dev_entry(1), values)
        dit.set_options(None)
        dit.cache_write(0, values)
        dit.cached_step(x, md, cached, 0)
        dit.sync()
        assert torch.equal(full, cached)
    finally:
        dit.close()


def test_chunks_never_change_a_bit():
    opt = dict(entry="mxint8", sparse=dict(keep=2, q_block=64, sink=1), axes=(32, 32), grid=(16, 18))
    dit, _ = make(BF16_W, **opt, token_chunk=0)
    try:
        x, md = dit.to_device(synth.make_dit_hidden(BF16_W, 1)), dit.to_device(synth.make_dit_modulation(BF16_W, 2))
        full, other = (dit.empty(*x.shape) for _ in range(2))
        dit.full_step(x, md, full, 0)
        dit.sync()
        assert bool(torch.isfinite(full).all())
        for chunk in (1, 100, 575):
            dit.set_chunk(chunk)
            dit.full_step(x, md, other, 1)
            dit.sync()
            assert torch.equal(full, other), chunk
            dit.cached_step(x, md, other, 1)
            dit.sync()
            assert torch.equal(full, other), chunk
    finally:
        dit.close()


def test_refused_options_leave_those_in_force():
    dit, _ = make(F32, entry="mxint8")
    try:
        x, md = dit.to_device(synth.make_dit_hidden(F32, 1)), dit.to_device(synth.make_dit_modulation(F32, 2))
        a, b = dit.empty(*x.shape), dit.empty(*x.shape)
        dit.arena = torch.empty(lcb.lc_dit_options_workspace_bytes(dit.ccfg, dit.options, 0), dtype=torch.uint8, device="cuda")
        dit.sync()
        lcb.lc_dit_set_workspace(dit.ctx, dit.arena.data_ptr(), dit.arena.numel())
        dit.full_step(x, md, a, 0)
        for bad in (lcb.make_dit_options(keep=4, block=1), lcb.make_dit_options()):  # (plain slots do not fit into this workspace)
            with pytest.raises(lcb.LcError) as e:
                lcb.lc_dit_set_options(dit.ctx, bad)
            assert e.value.status in (lcb.LC_ERR_SHAPE, lcb.LC_ERR_NOMEM)
            dit.cached_step(x, md, b, 0)
            dit.sync()
            assert torch.equal(a, b)
    finally:
        dit.close()
