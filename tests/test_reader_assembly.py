"""What the compiler made of the int8 layer's kernels, from their assembly: the
copies into LDS are inline assembly whose waits the kernels place themselves,
so a wait of the compiler's between the MFMAs would drain copies in flight."""
import os

import pytest

from paper_2605_01060_amd import build as B
from test_kernel_assembly import _assembly, _kernels


@pytest.fixture(scope="module")
def kernels():
    try:
        B.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    return list(_kernels(_assembly(os.path.join(B.CSRC, "linear_i8.hip"))))


def test_no_kernel_of_the_int8_layer_spills(kernels):
    assert len(kernels) == 21  # seven kernels, three epilogues
    for name, res, _ in kernels:
        assert not any(res.values()), (name, res)


def test_no_wait_of_the_compilers_between_the_int8_tiles_mfmas(kernels):
    checked = 0
    for name, _, body in kernels:
        if "tokens" in name:  # loads into registers, which the compiler waits for
            continue
        mfmas, waits, inline = 0, 0, False
        for line in body.split("\n") + [".LBB_end:"]:
            op = line.strip()
            if op.startswith(".LBB"):
                assert not (mfmas and waits), (name, mfmas, waits)
                checked += mfmas
                mfmas = waits = 0
            inline = op == ";;#ASMSTART" or (inline and op != ";;#ASMEND")
            mfmas += op.startswith("v_mfma_i32")
            waits += not inline and op.startswith("s_waitcnt") and "vmcnt" in op
    assert checked >= 18 * 16
