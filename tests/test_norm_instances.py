"""Every instance of the norm's kernels for single tokens is one that some group's size reaches."""

import re
import shutil
import subprocess

import pytest

ll = pytest.importorskip("paper_2506_04761_amd", reason="libloglinear.so not built")


def _shape(cg, V):
    """Lanes of a group of cg channels and vectors of V channels of a lane; None where a workgroup cannot hold it."""
    vectors = -(-cg // V)
    if vectors > 1024:
        return None
    lanes = 256 if vectors > 256 else min(64, 1 << (vectors - 1).bit_length())
    per = 1
    while lanes * per < vectors:
        per *= 2
    return V, lanes, per


def test_no_instance_is_out_of_reach():
    if not shutil.which("nm"):
        pytest.skip("no nm")
    names = subprocess.run(["nm", ll._lib.LIB_PATH], check=True, capture_output=True, text=True).stdout
    compiled = {"fwd": set(), "bwd": set()}
    for bwd, dtype, V, lanes, per in re.findall(r"__device_stub__k_norm_rows(_bwd)?I(DF16b|f)Li(\d+)ELi(\d+)ELi(\d+)E", names):
        compiled["bwd" if bwd else "fwd"].add((dtype, int(V), int(lanes), int(per)))
    reached = {"fwd": set(), "bwd": set()}
    for dtype, V in (("f", 4), ("DF16b", 8)):
        for cg in range(1, 1024 * V + 1):
            reached["fwd"].add((dtype, *_shape(cg, V)))
            reached["bwd"].add((dtype, *(_shape(cg, V // 2) or _shape(cg, V))))
    assert compiled == reached
