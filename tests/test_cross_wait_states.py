"""The gradient products of cross_attention.hip are written in inline asm like those of attention_mfma.hip: the same wait states, read
from this build's own assembly along every path (no GPU)."""
import os
import subprocess

from paper_2006_16668_amd import build
from test_attention_wait_states import check


def test_products_in_asm_have_their_wait_states(tmp_path):
    out, src = str(tmp_path / "cross.s"), "cross_attention.hip"
    subprocess.run([build._hipcc(), *build.FLAGS, *build.EXTRA_FLAGS[src], "-S", "--cuda-device-only", os.path.join(build.CSRC, src),
                    "-o", out], check=True, capture_output=True)
    with_products = {k: v for k, v in check(open(out).read()).items() if v[0]}
    assert len(with_products) == 7                       # dq, and dK and dV in two forms or three, of d 64 and 128
    for name, (products, wrong) in with_products.items():
        assert not wrong, (name, wrong[:5])
