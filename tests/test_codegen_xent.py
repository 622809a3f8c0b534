"""Generated-code checks of the cross entropy's kernels (no GPU needed): the tile loops keep their accumulators in the accumulation file, where the
matrix instructions written out by hand expect them, and none of the loops spills."""
import functools
import os
import re
import subprocess
import tempfile

import pytest

from paper_2502_02406_amd import build as B

SRC = "lvx_xent.hip"


@functools.lru_cache(maxsize=None)
def asm():
    with tempfile.TemporaryDirectory() as tmp:
        out = os.path.join(tmp, "k.s")
        cmd = [B.HIPCC] + B.FLAGS + B.FILE_FLAGS.get(SRC, []) + ["--cuda-device-only", "-S", os.path.join(B.CSRC, SRC), "-o", out]
        r = subprocess.run(cmd, capture_output=True, text=True, timeout=900)
        assert r.returncode == 0, r.stderr[-2000:]
        return open(out).read()


def kernel(name):
    m = re.search(r"^(_ZN[^\n]*" + name + r"[^\n]*):.*?^\.Lfunc_end\d+:.*?^; ScratchSize: (\d+)", asm(), re.S | re.M)
    assert m, name
    return m.group(0), int(m.group(2))


@pytest.mark.parametrize("mode", [0, 1, 2, 3])
@pytest.mark.parametrize("row_blocks", [2, 4])
def test_tile_loop_moves_no_accumulator(mode, row_blocks):
    body, _ = kernel(f"xent_bf16_kernelILi{mode}ELi{row_blocks}E")          # (a tile's own few spills stand before and behind its loop)
    blocks = re.split(r"^\.LBB\d+_\d+:.*$", body, flags=re.M)
    loops = [b for b in blocks if b.count("v_mfma_f32_32x32x16_bf16") >= 8 * row_blocks]      # a tile pair: 4 k-steps x 2 x row_blocks
    assert loops, "tile loop not found as basic blocks"
    for loop in loops:
        assert "v_accvgpr" not in loop, "an accumulator leaves the accumulation file inside the loop"
        assert "scratch_" not in loop, "register spill inside the loop"


@pytest.mark.parametrize("name", ["xent_few_bf16_kernelILi0ELi1ELi6ELb1E", "xent_few_bf16_kernelILi0ELi2ELi3ELb0E", "xent_few_bf16_kernelILi1ELi2ELi6ELb1E",
                                  "xent_few_bf16_kernelILi1ELi4ELi4ELb0E", "xent_few_dx_bf16_kernelILi2ELi6E", "xent_few_f32_kernelILi1E", "xent_f32_kernelILi0ELi128E", "xent_f32_kernelILi2ELi64E"])
def test_no_spills(name):
    assert kernel(name)[1] == 0
