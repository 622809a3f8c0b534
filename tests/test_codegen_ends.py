"""Generated-code checks of the distillation's, the embedding's and the sequence losses' kernels (no GPU needed): the tile loop that hands out a teacher's
entries keeps its accumulators where they are and touches no scratch memory, and the others have no spills."""
import functools
import os
import re
import subprocess
import tempfile

import pytest

from paper_2502_02406_amd import build as B


@functools.lru_cache(maxsize=None)
def asm(src):
    with tempfile.TemporaryDirectory() as tmp:
        out = os.path.join(tmp, "k.s")
        cmd = [B.HIPCC] + B.FLAGS + B.FILE_FLAGS.get(src, []) + ["--cuda-device-only", "-S", os.path.join(B.CSRC, src), "-o", out]
        r = subprocess.run(cmd, capture_output=True, text=True, timeout=900)
        assert r.returncode == 0, r.stderr[-2000:]
        return open(out).read()


def kernels(src):
    """name -> (code, bytes of scratch memory)"""
    found = re.finditer(r"^(_ZN\S+):.*?^\.Lfunc_end\d+:.*?^; ScratchSize: (\d+)", asm(src), re.S | re.M)
    return {m.group(1): (m.group(0), int(m.group(2))) for m in found}


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("row_blocks", [2, 4])
def test_tile_loop_moves_no_accumulator(mode, row_blocks):
    code = [c for n, (c, _) in kernels("lvx_distil.hip").items() if f"xent_bf16_kernelILi{mode}ELi{row_blocks}ELi1E" in n]
    assert len(code) == 1
    loops = [b for b in re.split(r"^\.LBB\d+_\d+:.*$", code[0], flags=re.M) if b.count("v_mfma_f32_32x32x16_bf16") >= 8 * row_blocks]
    assert loops, "tile loop not found as basic blocks"
    for loop in loops:
        assert "v_accvgpr" not in loop and "scratch_" not in loop


@pytest.mark.parametrize("src,most", [("lvx_distil.hip", 0), ("lvx_embed.hip", 0), ("lvx_sequence_loss.hip", 16)])
def test_no_spills(src, most):
    """(of the products only those on one tile of few tokens and in float32; one sequence loss keeps a few numbers of a whole sequence, outside its loop)"""
    for name, (_, scratch) in kernels(src).items():
        if "xent_bf16_kernel" not in name:
            assert scratch <= most, name
