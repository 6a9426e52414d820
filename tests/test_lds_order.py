"""The epilogues that pass sums from lane to lane of a wave through LDS say so to the compiler (no GPU needed).

The hardware carries a wave's LDS operations out in order, so a missing order changes no
result until a compiler moves a lane's read over another lane's write: it is looked for
in what the compiler is given, the code before any of its passes.
"""
import os
import re
import subprocess

import pytest

from paper_2309_17224_amd import build as B

ORDER = "wave_lds_order"


def functions(source, tmp_path):
    """Bodies of the device functions of a source, by mangled name."""
    out = tmp_path / "device.ll"
    cmd = [B.hipcc()] + B.flags() + ["--cuda-device-only", "-S", "-emit-llvm", "-Xclang", "-disable-llvm-passes",
                                     os.path.join(B.CSRC, source), "-o", str(out)]
    subprocess.run(cmd, check=True, stderr=subprocess.DEVNULL)
    return {m.group(1): m.group(2) for m in re.finditer(r"^define [^\n]*?@(\w+)\([^\n]*\{\n(.*?)^\}", out.read_text(), re.M | re.S)}


def test_the_order_is_a_fence_on_both_sides_of_a_wave_barrier(tmp_path):
    body = next(b for n, b in functions("fp8lin_ffn_act.hip", tmp_path).items() if ORDER in n)
    seen = re.findall(r'fence syncscope\("wavefront"\) (\w+)|call void @(llvm\.amdgcn\.wave\.barrier)', body)
    assert [a or b for a, b in seen] == ["release", "llvm.amdgcn.wave.barrier", "acquire"]


@pytest.mark.parametrize("source", ["fp8lin_ffn_act.hip", "fp8lin_ffn_glu.hip", "fp8lin_ffn_act_bwd.hip", "fp8lin_ffn_glu_bwd.hip"])
def test_staged_sums(source, tmp_path):
    """After the rows before have been read, and before these are."""
    staged = [b for n, b in functions(source, tmp_path).items() if "stage_sums" in n]
    assert len(staged) >= 2
    for body in staged:
        seen = re.findall(r"call [^\n]*(%s|ldexpf)" % ORDER, body)
        assert "ldexpf" in seen and seen[0] == seen[-1] == ORDER


def test_staged_outputs_of_the_plain_matmul(tmp_path):
    tiles = [b for n, b in functions("fp8lin_gemm.hip", tmp_path).items() if "gemm_tile" in n]
    assert len(tiles) >= 8
    for body in tiles:
        seen = re.findall(r"call [^\n]*(%s|ldexpf)" % ORDER, body)
        assert seen.count(ORDER) == 2 and seen[0] == ORDER and "ldexpf" in seen[1:-1] and seen[-1] == ORDER
