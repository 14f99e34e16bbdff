"""The compiler's resource report and assembly of the kernels of a step over a growing cache (CPU only: hipcc cross-compiles gfx950)."""
import os
import re
import shutil
import subprocess

import pytest

import asm_hazards

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    """{kernel: (a function that reads a figure of its resource report, its lines of assembly)}"""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("no hipcc")
    out = str(tmp_path_factory.mktemp("asm") / "k.s")
    res = subprocess.run([hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
                          "-packed-fp32-ops", "-mllvm", "-amdgpu-mfma-vgpr-form=1", "-Wno-inline-asm",
                          "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2502_15804_amd", "csrc"),
                          "--cuda-device-only", "-S", "-x", "hip", os.path.join(ROOT, "tests", "step_kernels.hip"),
                          "-o", out, "-Rpass-analysis=kernel-resource-usage"], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    code = dict(asm_hazards.functions(open(out).read()))
    reports = {k.split()[0]: k for k in re.split(r"remark: Function Name: ", res.stderr)[1:]}
    assert set(reports) == set(code) and len(code) == 11
    figure = lambda report: lambda key: int(re.search(key + r": (\d+)", report).group(1))
    return {name: (figure(report), code[name]) for name, report in reports.items()}


def test_no_wait_state_is_broken(compiled):
    for name, (_, code) in compiled.items():
        assert asm_hazards.hazards(code) == set(), name


def test_the_case_of_a_base_from_a_vector_instruction_is_there(compiled):
    for name in ("chunks2", "chunks4"):
        assert any("v_readfirstlane" in t for t in compiled[name][1])


def test_registers_and_lds(compiled):
    """What spills, waits for every load that is on its way: nothing, but for the two widths in between, which hold 8 waves' registers."""
    for name, (val, code) in compiled.items():
        assert val(r"LDS Size \[bytes/block\]") <= 160 * 1024, name
        between = "Lb0ELi2ELi4E" in name or "Lb0ELi4ELi2E" in name
        assert val("VGPRs Spill") <= (40 if between else 0), name
        assert between or val(r"ScratchSize \[bytes/lane\]") == 0, name


def test_no_packed_arithmetic_of_32_bits(compiled):
    for name, (_, code) in compiled.items():
        assert not any(re.match(r"v_pk_(add|mul|fma)_f32", t) for t in code), name
