"""Every kernel of the attention of a draft tree with heads of 128: the compiler's resource report and wait states (CPU only: hipcc
cross-compiles gfx950).  Those of heads of 64 have 186 to 206 vector registers and spill none."""
import os
import re
import shutil
import subprocess

import pytest

import asm_hazards

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# Vector registers that a kernel spills, by its waves side by side: no more than these.
SPILLS = {"false": {1: 0, 2: 9, 4: 24, 8: 1}, "true": {1: 0, 2: 2, 4: 22, 8: 0}}


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    """{8-bit rows: [(kernel, a function that reads a figure of its resource report, its lines of assembly)]}"""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("no hipcc")
    runs = {}
    for kv8 in SPILLS:                       # side by side
        out = str(tmp_path_factory.mktemp("asm") / f"{kv8}.s")
        runs[kv8] = out, subprocess.Popen(
            [hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-mllvm",
             "-amdgpu-mfma-vgpr-form=1", "-Wno-inline-asm", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2502_15804_amd", "csrc"),
             "--cuda-device-only", "-S", "-x", "hip", os.path.join(ROOT, "tests", "tree_kernels.hip"), f"-DROWS_OF_8_BITS={kv8}", "-o", out,
             "-Rpass-analysis=kernel-resource-usage"], stdout=subprocess.DEVNULL, stderr=subprocess.PIPE, text=True)
    found = {}
    for kv8, (out, run) in runs.items():
        err = run.communicate()[1]
        assert run.returncode == 0, err[-3000:]
        code = dict(asm_hazards.functions(open(out).read()))
        reports = {k.split()[0]: k for k in re.split(r"remark: Function Name: ", err)[1:]}
        assert set(reports) == set(code) and len(code) == 8
        figure = lambda report: lambda key: int(re.search(key + r": (\d+)", report).group(1))
        found[kv8] = [(name, figure(report), code[name]) for name, report in reports.items()]
    return found


@pytest.mark.parametrize("kv8", SPILLS)
def test_registers_lds_and_wait_states(compiled, kv8):
    for name, val, code in compiled[kv8]:
        waves = int(re.search(r"ELb[01]ELi(\d)E", name).group(1))
        assert val("VGPRs Spill") <= SPILLS[kv8][waves], name
        assert val(r"LDS Size \[bytes/block\]") <= 160 * 1024, name
        assert asm_hazards.hazards(code) == set(), name
        assert not any(re.match(r"v_pk_(add|mul|fma)_f32", t) for t in code), name
