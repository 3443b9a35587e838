"""The bytes of quantised entries, decoded by their formats' definitions: integers, e4m3, e2m1 with the first of two in the low bits;
rows of whole groups with zeros behind the last column, then the scale bytes."""
import numpy as np
import pytest
import torch

from oracle import tokens_oracle as tko
from paper_2510_05367_amd import tokens
from tests.test_gpu_tokens import BF, F32, entry_input, f64

pytestmark = pytest.mark.gpu
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def decoded(raw, fmt):
    """What code bytes count, in units of their group's scale."""
    if fmt == "mxint8":
        return raw.view(np.int8).astype(np.float64)
    if fmt == "mxfp8":
        sign, e, f = np.where(raw >> 7, -1.0, 1.0), (raw >> 3 & 15).astype(int), (raw & 7) / 8.0
        assert not np.any((raw & 127) == 127)  # (the one NaN of the format)
        return sign * np.where(e == 0, f * 2.0 ** -6, (1 + f) * 2.0 ** (e - 7.0))
    nibbles = np.stack([raw & 15, raw >> 4], axis=-1).reshape(*raw.shape[:-1], -1)
    return np.where(nibbles >> 3, -1.0, 1.0) * E2M1[nibbles & 7]


@pytest.mark.parametrize("fmt", ["mxint8", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 100), (5, 64), (2, 33), (9, 320), (4, 32)])
def test_bytes_of_an_entry(fmt, dtype, rows, cols):
    rng = np.random.default_rng(rows * 1000 + cols)
    x = entry_input(rng, rows, cols, dtype)
    groups = -(-cols // 32)
    width = groups * (16 if fmt == "mxfp4" else 32)
    values, exps = tko.entry(f64(x), fmt)
    for t in (x, torch.nn.functional.pad(x, (1, 2), value=9.0)[:, 1:cols + 1]):  # rows of whole packets, and others
        raw = tokens.entry_pack(t, fmt).cpu().numpy()
        assert raw.size == rows * (width + groups)
        assert np.array_equal(raw[rows * width:].reshape(rows, groups), exps + 127)
        codes = decoded(raw[:rows * width].reshape(rows, width), fmt)
        assert codes.shape == (rows, groups * 32) and np.all(codes[:, cols:] == 0)
        assert np.array_equal(codes[:, :cols] * np.exp2(np.repeat(exps, 32, axis=1)[:, :cols]), values)


def test_codes_by_hand():
    """One group of each format, byte by byte."""
    x = torch.zeros(1, 32, device="cuda")
    x[0, :6] = torch.tensor([127.0, -1.0, 2.5, 3.5, -128.0 + 1.0, 64.0])
    assert tokens.entry_pack(x, "mxint8").tolist() == [127, 255, 2, 4, 129, 64] + [0] * 26 + [127]
    x[0, :6] = torch.tensor([448.0, -1.0, 0.5, 2.0 ** -9, 1.125, 240.0])
    assert tokens.entry_pack(x, "mxfp8").tolist() == [0x7e, 0xb8, 0x30, 0x01, 0x39, 0x77] + [0] * 26 + [127]
    x[0, :6] = torch.tensor([6.0, -0.5, 1.0, 1.5, -4.0, 3.0])
    assert tokens.entry_pack(x * 0.25, "mxfp4").tolist() == [0x97, 0x32, 0x5e] + [0] * 13 + [125]
