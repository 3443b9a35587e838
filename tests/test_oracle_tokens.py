"""Pins of the oracle of the operators over the tokens of long videos: closed forms, symmetries, and dense attention."""
import math

import numpy as np
import pytest
import torch

from oracle import tokens_oracle as tko


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_is_a_rotation_that_depends_on_distance_alone(layout):
    rng = np.random.default_rng(0)
    q, k = rng.normal(size=(2, 1, 1, 1, 12))
    at = lambda x, p: tko.rope(x, np.full((1, 1, 2), p), (8, 4), layout)[0, 0, 0]  # noqa: E731
    assert np.allclose(at(q, 0), q[0, 0, 0])
    assert math.isclose(np.linalg.norm(at(q, 77)), np.linalg.norm(q), rel_tol=1e-12)
    assert math.isclose(at(q, 1000009) @ at(k, 1000001), at(q, 8) @ at(k, 0), rel_tol=1e-6, abs_tol=1e-6)
    back = tko.rope(tko.rope(q, np.full((1, 1, 2), 5), (8, 4), layout), np.full((1, 1, 2), 5), (8, 4), layout, inverse=True)
    assert np.allclose(back, q)


def test_rope_by_hand_and_scalings():
    x = np.array([1.0, 2.0, 3.0, 4.0, 9.0]).reshape(1, 1, 1, 5)
    c, s, c2, s2 = math.cos(3), math.sin(3), math.cos(0.03), math.sin(0.03)
    y = tko.rope(x, np.full((1, 1, 1), 3), (4,), "half")[0, 0, 0]
    assert np.allclose(y, [c - 3 * s, 2 * c2 - 4 * s2, s + 3 * c, 2 * s2 + 4 * c2, 9.0])
    y = tko.rope(x, np.full((1, 1, 1), 3), (4,), "interleaved")[0, 0, 0]
    assert np.allclose(y, [c - 2 * s, s + 2 * c, 3 * c2 - 4 * s2, 3 * s2 + 4 * c2, 9.0])
    assert tko.rope_frequency(8, 1, scaling="linear", factor=4.0) == pytest.approx(0.1 / 4)
    assert tko.rope_frequency(8, 3, scaling="base", factor=8.0) == pytest.approx((10000 * 8 ** (8 / 6)) ** -0.75)
    # parts: a pair that turns often within the original length stays, one that does not turn once is slowed by the factor
    assert tko.rope_frequency(64, 0, scaling="parts", factor=4.0, orig_len=4096) == 1.0
    assert tko.rope_frequency(64, 31, scaling="parts", factor=4.0, orig_len=4096) == pytest.approx(10000 ** (-62 / 64) / 4)


def test_everything_listed_is_dense_attention():
    rng = np.random.default_rng(1)
    q, k, v = (rng.normal(size=(2, 150, 4, 8)) for _ in range(3))
    index = np.tile(np.arange(3, dtype=np.int32), (2, 4, 2, 1))
    out = tko.block_attention(q, k[:, :, :2], v[:, :, :2], index, 64, 100)[0]
    t = lambda x: torch.from_numpy(x).transpose(1, 2)  # noqa: E731
    kk, vv = t(k[:, :, :2]).repeat_interleave(2, 1), t(v[:, :, :2]).repeat_interleave(2, 1)
    ref = torch.softmax(t(q) @ kk.transpose(2, 3) / math.sqrt(8), -1) @ vv
    assert np.allclose(out, ref.transpose(1, 2).numpy())


def test_selection_by_hand():
    k = np.zeros((1, 320, 1, 8))
    for j, s in enumerate([1.0, 3.0, 2.0, 3.0, -1.0]):
        k[0, j * 64:(j + 1) * 64, 0, 0] = s
    m = tko.block_means(k, 64)
    assert m.shape == (1, 1, 8, 5) and list(m[0, 0, 0]) == [1.0, 3.0, 2.0, 3.0, -1.0]
    q = np.zeros((1, 1, 1, 8))
    q[..., 0] = 2.0
    pick = lambda keep, **kw: list(tko.block_select(q, m, 320, keep, 64, 16, **kw)[0, 0, 0])  # noqa: E731
    assert pick(1) == [1]  # equal scores: the lower index
    assert pick(2) == [1, 3] and pick(3) == [1, 2, 3]
    assert pick(2, sink=1) == [0, 1]
    assert pick(2, window=0, q_pos0=319) == [1, 4] and pick(3, window=1, q_pos0=319) == [1, 3, 4]
    assert pick(7) == [0, 1, 2, 3, 4, -1, -1]
    assert pick(2, k_len=[65]) == [0, 1] and pick(2, k_len=[0]) == [-1, -1] and pick(2, q_len=[0]) == [-1, -1]
    m[0, 0, 0, 1] = math.nan
    assert pick(4) == [0, 2, 3, 4]
    assert tko.listed_blocks([0, 2, 2, 3], 64, 320) == [0, 2] and tko.listed_blocks([4, 5], 64, 320) == [4]
    assert tko.listed_blocks([-1, 0], 64, 320) == [] and tko.listed_blocks([1], 64, 64) == []


@pytest.mark.parametrize("fmt,top,n", [("mxint8", 127.0, 128), ("mxfp8", 448.0, 127), ("mxfp4", 6.0, 8)])
def test_entries_hold_what_their_codes_hold(fmt, top, n):
    steps = tko.magnitudes(fmt)
    assert len(steps) == n and steps[-1] == top and np.all(np.diff(steps) > 0)
    x = np.zeros((1, 32))
    x[0, 0], x[0, 1], x[0, 2] = top, -steps[1], steps[-2]
    values, exps = tko.entry(x * 2.0 ** 5, fmt)
    assert exps[0, 0] == 5 and np.array_equal(values, x * 32)
    values, exps = tko.entry(np.full((1, 3), top * 1.0001), fmt)  # one step of the scale up, no saturation
    assert exps[0, 0] == 1 and np.all(np.abs(values / top - 1) < 0.2)
    assert tko.entry(np.zeros((1, 1)), fmt)[1][0, 0] == -127
    if fmt == "mxfp8":
        ref = torch.linspace(-448, 448, 5001).to(torch.float8_e4m3fn).double().numpy()
        got = tko.entry(np.concatenate([np.linspace(-448, 448, 5001, dtype=np.float32), np.full(23, 448, np.float32)]).reshape(157, 32).astype(np.float64), fmt)
        # groups that hold 448 have the scale one: elsewhere the scale is smaller and the values no less exact
        assert np.array_equal(got[0].reshape(-1)[4992:5001], ref[4992:])
