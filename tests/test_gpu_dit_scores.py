"""The transformer stack in bf16 with lists that the score chooses: tokens of a block resemble each other, so that the scores lie further
apart than rounding moves them, which is checked on the oracle."""
import numpy as np
import pytest

from oracle import dit_oracle as dito
from paper_2510_05367_amd import synth
from tests.gpu_util import check, host
from tests.test_gpu_dit_options import Oracle, make

pytestmark = pytest.mark.gpu
CFG = synth.DitConfig("dit_bf16_s", B=1, T=256, D=256, heads=4, head_dim=64, L=1, cache_a=0, cache_b=1, dtype="bf16")


def margin(cfg, w, x, m, keep):
    """The least distance between the last score that is listed and the first that is not, as a share of |mean q| max |mean k|."""
    h = dito.layer_norm(x.astype(np.float64), cfg.ln_eps) * (1 + m[1]) + m[0]
    q, k, _ = np.split((h @ w["blk0.wqkv"].T + w["blk0.bqkv"]).reshape(cfg.T, 3 * cfg.heads, cfg.head_dim), 3, axis=1)
    worst = np.inf
    for hd in range(cfg.heads):
        mk, mq = (np.array([t[i:i + 64, hd].mean(0) for i in range(0, cfg.T, 64)]) for t in (k, q))
        for g in mq:
            s = np.sort(mk @ g)[::-1]
            worst = min(worst, (s[keep - 1] - s[keep]) / (np.linalg.norm(g) * np.linalg.norm(mk, axis=1).max()))
    return worst


@pytest.mark.parametrize("T,keep,seed", [(256, 2, 233), (230, 1, 8)])
def test_lists_that_the_score_chooses(T, keep, seed):
    cfg = CFG.with_(T=T)
    dit, w = make(cfg, sparse=dict(keep=keep, q_block=64))
    try:
        rng = np.random.default_rng(seed)
        x = (np.repeat(rng.standard_normal((1, 4, cfg.D)), 64, axis=1)[:, :T] + 0.3 * rng.standard_normal((1, T, cfg.D))).astype(np.float32)
        mod = synth.make_dit_modulation(cfg, 2)
        w64 = {k: v.astype(np.float64) for k, v in w.items()}
        # h, q and k are rounded to bf16: elements off by 0.41 * 2^-8 of themselves (rms) each time, so q and k by 2.3e-3 of their norms and a
        # distance of two scores by 4 * 2.3e-3 at the very most
        assert margin(cfg, w64, x[0], mod[0, 0].astype(np.float64), keep) > 2 * 4 * 2.3e-3
        out = dit.empty(*x.shape)
        dit.full_step(dit.to_device(x), dit.to_device(mod), out, 0)
        dit.sync()
        orc = Oracle(cfg, w64, sparse=dict(keep=keep, q_block=64))
        check("normal step", host(out), orc.full_step(x, mod, 0), cfg.dtype, wide_range=True)
        check("Delta", host(dit.dev_entry(0)), orc.dev[0], cfg.dtype)
    finally:
        dit.close()
