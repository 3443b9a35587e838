"""Options of the transformer stack, as far as no GPU is needed: what is refused, and what entries and workspaces take."""
import ctypes

import pytest

from paper_2510_05367_amd import binding as lcb
from paper_2510_05367_amd import synth, tokens

BIG = synth.DITS["video_dit"]


def test_struct_layout_and_names():
    assert ctypes.sizeof(lcb.lc_dit_options) == 24 + 8 + 16
    with pytest.raises(ValueError):
        lcb.make_dit_options(entry="int8")


@pytest.mark.parametrize("kw,status,words", [
    (dict(keep=-1), 1, "keep"), (dict(keep=4, block=60), 2, "block"), (dict(keep=4, q_block=0), 2, "q_block"), (dict(keep=4, sink=-1), 1, "sink"),
    (dict(rope=tokens.make_rope(32)), 2, "channels"), (dict(rope=lcb.lc_rope_table()), 1, "lc_rope_make"),
    (dict(rope=tokens.make_rope(64, axes=(16, 24, 24))), 2, "grid"),
    (dict(rope=tokens.make_rope(64, axes=(16, 24, 24)), grid=(4, 32, 31)), 2, "fewer cells"),
    (dict(rope=tokens.make_rope(64, axes=(32, 32)), grid=(1 << 20, 1 << 20)), 2, "2^31")])
def test_refusals(kw, status, words):
    cfg, opt = lcb.make_dit_config(BIG, 0, 1), lcb.make_dit_options(**kw)
    with pytest.raises(lcb.LcError) as e:
        lcb.lc_dit_check_options(cfg, opt)
    assert e.value.status == status and words in str(e.value)
    assert lcb.lc_dit_options_workspace_bytes(cfg, opt, 0) == 0 and lcb.lc_dit_options_entry_bytes(cfg, opt) == 0


def test_bad_enum_null_and_config():
    cfg, opt = lcb.make_dit_config(BIG, 0, 1), lcb.make_dit_options()
    for f in (-2, 3):
        opt.entry_format = f
        with pytest.raises(lcb.LcError, match="entry_format"):
            lcb.lc_dit_check_options(cfg, opt)
    assert lcb.lib().lc_dit_check_options(cfg, None) == lcb.LC_ERR_ARG
    assert lcb.lib().lc_dit_set_options(None, None) == lcb.LC_ERR_ARG
    cfg.T = 0
    assert lcb.lc_dit_options_workspace_bytes(cfg, lcb.make_dit_options(), 0) == 0


@pytest.mark.parametrize("fmt,share", [("mxint8", 33 / 128), ("mxfp8", 33 / 128), ("mxfp4", 17 / 128)])
def test_entries_take_what_their_codes_take(fmt, share):
    cfg = lcb.make_dit_config(BIG, 0, 2)
    plain = lcb.lc_dit_entry_bytes(cfg)
    assert plain == BIG.B * BIG.T * BIG.D * 4 == lcb.lc_dit_options_entry_bytes(cfg, None) == lcb.lc_dit_options_entry_bytes(cfg, lcb.make_dit_options())
    packed = lcb.lc_dit_options_entry_bytes(cfg, lcb.make_dit_options(entry=fmt))
    assert packed == plain * share
    # two slots of it and one accumulator in place of two plain slots
    for chunk in (0, 1024):
        assert lcb.lc_dit_options_workspace_bytes(cfg, lcb.make_dit_options(entry=fmt), chunk) == lcb.lc_dit_workspace_bytes(cfg, chunk) - plain + 2 * packed


@pytest.mark.parametrize("fmt", ["mxint8", "mxfp8", "mxfp4"])
def test_entries_beyond_their_sizes_are_refused(fmt):
    """2^24 tokens of 2048 channels are a stack's limits, and more values than an entry holds."""
    cfg = lcb.make_dit_config(BIG, 0, 1)
    cfg.B, cfg.T, cfg.D, cfg.heads, cfg.head_dim = 1, 1 << 24, 2048, 32, 64
    assert lcb.lc_dit_entry_bytes(cfg) == 1 << 37
    with pytest.raises(lcb.LcError, match="values") as e:
        lcb.lc_dit_check_options(cfg, lcb.make_dit_options(entry=fmt))
    assert e.value.status == 2 and lcb.lc_dit_options_workspace_bytes(cfg, lcb.make_dit_options(entry=fmt), 0) == 0
    cfg.T = (1 << 23) - 1
    lcb.lc_dit_check_options(cfg, lcb.make_dit_options(entry=fmt))


def test_selection_takes_no_transposed_values():
    cfg = lcb.make_dit_config(BIG, 0, 1)
    R, D = BIG.B * BIG.T, BIG.D
    opt = lcb.make_dit_options(keep=16)
    means, lists = BIG.B * D * 64 * 8, BIG.B * 16 * 32 * 16 * 4
    need = lcb.lc_dit_options_workspace_bytes(cfg, opt, 0)
    assert need == 2 * R * D * 4 + max(8 * R * D + means + lists, 10 * R * D)  # hidden states, the entry; attention or the MLP of all rows
    assert lcb.lc_dit_options_workspace_bytes(cfg, lcb.make_dit_options(rope=tokens.make_rope(64)), 0) == lcb.lc_dit_workspace_bytes(cfg, 0)
