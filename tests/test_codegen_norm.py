"""Generated-code checks of the norms' kernels and of the loss's products in parts (no GPU needed): a row, the next one and the columns' sums stay in
registers, and so do a tile's operands and sums inside its loop."""
import functools
import os
import re
import subprocess
import tempfile

import pytest

from paper_2502_02406_amd import build as B
from test_codegen_xent import kernel as xent_kernel

SRC = "lvx_norm.hip"


@functools.lru_cache(maxsize=None)
def scratch():
    """Bytes of scratch a lane, by kernel."""
    with tempfile.TemporaryDirectory() as tmp:
        out = os.path.join(tmp, "k.s")
        cmd = [B.HIPCC] + B.FLAGS + B.FILE_FLAGS.get(SRC, []) + ["--cuda-device-only", "-S", os.path.join(B.CSRC, SRC), "-o", out]
        r = subprocess.run(cmd, capture_output=True, text=True, timeout=900)
        assert r.returncode == 0, r.stderr[-2000:]
        text = open(out).read()
    return {m.group(1): int(m.group(2)) for m in re.finditer(r"^(_ZN[^\n:]*):.*?^\.Lfunc_end\d+:.*?^; ScratchSize: (\d+)", text, re.S | re.M)}


@pytest.mark.parametrize("name", ["norm_fwd_kernel", "norm_bwd_kernel", "norm_fwd_any_kernel", "norm_bwd_any_kernel", "norm_param_any_kernel", "norm_param_sum_kernel",
                                  "pack_kernel", "unpack_kernel", "pack_narrow_kernel"])
def test_no_spills(name):
    """(but for the gradients of rows of 8193 to 16384 features together with those of the weights)"""
    found = {k: v for k, v in scratch().items() if re.search(r"\d" + name + "I|\\d" + name + "E", k)}
    assert found
    assert not {k: v for k, v in found.items() if v and not re.search(r"norm_bwd_kernelI\w+Li512ELi4ELb1E", k)}


def test_tile_loop_of_dw_in_parts():
    body, _ = xent_kernel("xent_bf16_kernelILi4ELi2E")
    loops = [b for b in re.split(r"^\.LBB\d+_\d+:.*$", body, flags=re.M) if b.count("v_mfma_f32_32x32x16_bf16") >= 16]
    assert loops, "tile loop not found as basic blocks"
    for loop in loops:
        assert "v_accvgpr" not in loop and "scratch_" not in loop
