"""Register constraints of the backward scan's inline assembly, from the assembly that the compiler makes of it: a block
that writes results before it has read its last input says so, or the compiler may give both one register where it
knows them to be equal."""

import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

# the carried gradients, the states and dy are one value: one register would do for all of them
KERNEL = """
#include "ll_layer_device.hpp"
namespace ll {
__global__ void k(float* p, const float* q) {
  const float v = p[threadIdx.x], b = q[threadIdx.x], c = q[threadIdx.x + 64];
  float g[4] = {v, v, v, v}, h[4] = {v, v, v, v}, x, y;
  grad_token<0, %s>(g, b, c, v, h, x, y);
  p[threadIdx.x] = g[0] + g[1] + g[2] + g[3] + x + y;
}
}  // namespace ll
"""


@pytest.mark.parametrize("with_states", ["true", "false"])
def test_a_token_of_the_backward_scan(with_states, tmp_path):
    if not shutil.which(HIPCC):
        pytest.skip("no hipcc")
    src, out = tmp_path / "k.hip", tmp_path / "k.s"
    src.write_text(KERNEL % with_states)
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
                    "-packed-fp32-ops", "-I" + os.path.join(ROOT, "paper_2506_04761_amd", "csrc"), "--cuda-device-only", "-S",
                    str(src), "-o", str(out)], check=True, capture_output=True, timeout=100)
    block = re.findall(r"v_(?:fmac|mul)_f32_dpp (v\d+), (v\d+), (v\d+) row_newbcast", out.read_text())
    assert len(block) == (12 if with_states == "true" else 8)
    carried, dy = [d for d, _, _ in block[:4]], block[0][2]  # the first four: g_i += c_i dy
    assert len(set(carried)) == 4
    # no register of a later input (the rows of B and C, dy, a state) is among those written by then
    written = set()
    for d, row, factor in block:
        assert row not in written
        assert factor not in written or factor in carried and d not in carried  # the sums of b_i g_i read the new g_i
        written.add(d)
    assert dy not in carried
    if with_states == "true":
        products = [f for d, r, f in block[4:] if r == block[0][1]]  # c_i h_i
        assert len(products) == 4 and not set(products) & set(carried)
