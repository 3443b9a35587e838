"""Pins of the oracle of the operators of long videos at the ends of sequences and of number ranges, by hand."""
import numpy as np
import pytest

from oracle import tokens_oracle as tko


def select_first(length, padded, keep, **kw):
    """The lists of the first group of queries that holds queries 0 .. length - 1, padded to `padded`; the last of 8 blocks scores highest."""
    k = np.zeros((1, 512, 1, 8))
    k[..., 0] = np.repeat(np.arange(8.0), 64)[None, :, None]
    q = np.ones((1, padded, 1, 8))
    return list(tko.block_select(q, tko.block_means(k, 64), 512, keep, 64, 128, q_len=[length], **kw)[0, 0, 0])


def test_forced_blocks_are_those_of_queries_that_exist():
    assert select_first(1, 1, 2, window=0) == [0, 7]
    for padded in (1, 64, 65, 128, 500):  # what a sequence is padded to does not matter
        assert select_first(1, padded, 2, window=0) == [0, 7], padded
    assert select_first(65, 128, 2, window=0) == [0, 1]
    assert select_first(3, 128, 3, window=1, q_pos0=126) == [0, 1, 2] and select_first(2, 128, 3, window=0, q_pos0=126) == [1, 6, 7]


@pytest.mark.parametrize("fmt,last,exp", [("mxint8", 63, 122), ("mxfp8", 240, 120), ("mxfp4", 3, 126)])
def test_finite_values_stay_finite(fmt, last, exp):
    """The largest float is nearest to a code that stands for 2^128; it is held as the code below, and that again as itself."""
    big = np.finfo(np.float32).max
    x = np.zeros((1, 32), dtype=np.float32)
    x[0, :5] = big, -big, big / 2, np.float32(2.0) ** 127, -big / 3
    values, exps = tko.entry(x, fmt)
    assert exps[0, 0] == exp and values[0, 0] == last * 2.0 ** exp == -values[0, 1] and values[0, 3] == 2.0 ** 127
    kept = values.astype(np.float32)
    assert np.all(np.isfinite(kept)) and np.array_equal(kept, values)
    assert np.array_equal(tko.entry(kept, fmt)[0], values)
