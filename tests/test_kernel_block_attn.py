"""What the attention over listed blocks counts on, read from the compiled gfx950 code: the requests for the next stage stay in
flight while a stage is contracted, and registers leave room for four wavefronts a SIMD where the kernel is bound by them."""
import re

import pytest

from tests.test_kernel_resources import CSRC, kernel_meta  # noqa: F401


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("asm")
    meta = kernel_meta(tmp, "lc_battn.hip")
    return meta, (tmp / "lc_battn.hip.s").read_text()


def attention(meta):
    return {k: v for k, v in meta.items() if "block_attn_kernel" in k}


def test_registers(asm):
    kernels = attention(asm[0])
    assert len(kernels) == 36 + 15  # two types, six head sizes, three ways to share a tile; prescaled queries of five sizes
    for name, (vg, scratch) in kernels.items():
        d = int(re.search(r"Li(\d+)ELi", name).group(1))
        assert scratch == 0 and vg <= (128 if d <= 64 and "DF16b" in name else 256), (name, vg, scratch)


def test_requests_stay_in_flight(asm):
    """From the requests of a stage to the barrier in front of the next one nothing waits for loads: every wait names LDS alone."""
    meta, text = asm
    for name in attention(meta):
        body = text[text.index("\n" + name + ":"):]
        lines = [l.split(";")[0].strip() for l in body[:body.index(".Lfunc_end")].splitlines()]
        loads = [i for i, l in enumerate(lines) if l.startswith("buffer_load") and l.endswith("lds")]
        assert loads, name
        mfma = [i for i, l in enumerate(lines) if "mfma" in l]
        last = max(i for i in loads if i < mfma[0])  # the loop's own requests are in front of its first product
        between = [l for l in lines[last + 1:mfma[-1]] if l.startswith("s_waitcnt") and "vmcnt" in l]
        assert not between, (name, between)
        barrier = max(i for i in range(last) if lines[i] == "s_barrier")
        assert re.search(r"vmcnt\(0\)", lines[barrier - 1]), (name, lines[barrier - 1])
