"""Sums along the line of all pairs have 64 bits in every kernel that attends: pairs of 2^31 tokens, 64 of them side by side (CPU only: hipcc cross-compiles
gfx950).  What a sum decides is only which pairs one wave has alone, so no output shows its width; the steps between lanes do, two for every one of 64 bits."""
import os
import re
import shutil
import subprocess

import pytest

import asm_hazards

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("steps", ["row_shr:1", "row_shr:8", "row_bcast:15", "row_bcast:31"])
def test_sums_of_the_tree_attention_have_64_bits(code, steps):
    """Two sums of the kernel that gives short pairs to a wave, one of the others."""
    for name, lines in code.items():
        sums = 2 if re.search(r"Lb1ELi1ELi4E", name) else 1
        assert sum(re.search(r"_dpp .*" + steps + r"(\D|$)", t) is not None for t in lines) == 2 * sums, name


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("no hipcc")
    out = str(tmp_path_factory.mktemp("asm") / "k.s")
    res = subprocess.run([hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-mllvm",
                          "-amdgpu-mfma-vgpr-form=1", "-Wno-inline-asm", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2502_15804_amd", "csrc"),
                          "--cuda-device-only", "-S", "-x", "hip", os.path.join(ROOT, "tests", "line_kernels.hip"), "-o", out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    return {name: lines for name, lines in asm_hazards.functions(open(out).read()) if "decode_tree" in name}
