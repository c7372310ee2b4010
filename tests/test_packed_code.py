"""The machine code of the packed kernels that hold hand-written instructions (attn_bwd_wide.h), as test_attn_bwd_code.py looks at the
dense ones: rows have strides there, and their addresses are made in scalar registers in front of every request."""
import re
import subprocess

import pytest

from paper_2509_10406_amd import build
from tests.test_attn_bwd_code import faults, functions


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    src, out = f"{build.CSRC}/packed_attn.hip", str(tmp_path_factory.mktemp("asm") / "packed_attn.s")
    subprocess.run(["hipcc", *build.FLAGS, *build.FILE_FLAGS["packed_attn.hip"], "--offload-device-only", "-S", src, "-o", out], check=True,
                   stderr=subprocess.DEVNULL)
    return open(out).read()


def test_hand_written_instructions(code):
    wide = {n: v for n, v in functions(code).items() if "_wide" in n}
    assert len(wide) == 8  # dK / dV at either head dimension and dQ at either, for two types of gradients
    for name, (ins, pred) in wide.items():
        assert sum(x.mfma and x.asm for x in ins) >= 24 and any(x.op.startswith("global_load_lds") for x in ins), name
        assert not (f := faults(ins, pred)), (name, f[:5])
    for what in ("vgpr_spill_count", "private_segment_fixed_size"):  # a few addresses of heads wait in lanes of a vector register
        assert set(re.findall(rf"\.{what}:\s+(\d+)", code)) == {"0"}, what
