"""The attention over listed blocks writes m0 in its own requests, and cannot declare that (the compiler reserves the register): what it
counts on is that nothing else in the compiled kernels reads or writes it."""
import re

from tests.test_kernel_resources import kernel_meta

# instructions that take m0 without naming it
HIDDEN = re.compile(r"^(v_movrel|s_movrel|s_sendmsg|ds_gws|ds_\w*addtid|s_set_gpr_idx|v_interp|global_load_lds|\w+ .*\blds$)")


def test_m0_belongs_to_the_requests(tmp_path):
    meta = kernel_meta(tmp_path, "lc_battn.hip")
    text = (tmp_path / "lc_battn.hip.s").read_text()
    seen = 0
    for name in meta:
        body = text[text.index("\n" + name + ":"):]
        lines = [l.split(";")[0].strip() for l in body[:body.index(".Lfunc_end")].splitlines()]
        lines = [l for l in lines if l]
        requests = set()
        for i, l in enumerate(lines):
            if re.search(r"\bm0\b", l):
                assert l.startswith("s_mov_b32 m0, s") and lines[i + 1] == "s_nop 0", (name, lines[i:i + 3])
                assert lines[i + 2].startswith("buffer_load_dwordx4") and lines[i + 2].endswith("lds"), (name, lines[i:i + 3])
                requests.add(i + 2)
        others = [l for i, l in enumerate(lines) if HIDDEN.match(l) and i not in requests]
        assert not others, (name, others)
        seen += len(requests)
        assert bool(requests) == ("block_attn_kernel" in name), name
    assert seen > 0
