"""Every kernel of the compression of a growing cache: the compiler's resource report and wait states (CPU only: hipcc cross-compiles gfx950)."""
import os
import re
import shutil
import subprocess

import pytest

import asm_hazards

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2502_15804_amd", "csrc")


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    """{kernel: (a function that reads a figure of its resource report, its lines of assembly)}"""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("no hipcc")
    out = str(tmp_path_factory.mktemp("asm") / "k.s")
    res = subprocess.run([hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-mllvm",
                          "-amdgpu-mfma-vgpr-form=1", "-Wno-inline-asm", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "--cuda-device-only", "-S", "-x", "hip",
                          os.path.join(CSRC, "fairkv_compress.hip"), "-o", out, "-Rpass-analysis=kernel-resource-usage"], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    code = dict(asm_hazards.functions(open(out).read()))
    reports = {k.split()[0]: k for k in re.split(r"remark: Function Name: ", res.stderr)[1:]}
    assert set(reports) == set(code)
    figure = lambda report: lambda key: int(re.search(key + r": (\d+)", report).group(1))
    return {name: (figure(report), code[name]) for name, report in reports.items()}


def test_every_variant_is_there(compiled):
    count = lambda part: sum(part in name for name in compiled)
    assert count("attn_weights") == 16 and count("select_kernel") == 6 and count("select_first") == 2 and count("select_large") == 3
    assert count("evict_into") == 8 and count("evict_kernel") == 15 and count("evict_lengths") == 1


def test_registers_lds_and_wait_states(compiled):
    for name, (val, code) in compiled.items():
        assert val("VGPRs Spill") == 0 and val(r"ScratchSize \[bytes/lane\]") == 0, name
        assert val(r"LDS Size \[bytes/block\]") <= 160 * 1024, name
        assert asm_hazards.hazards(code) == set(), name
        assert not any(re.match(r"v_pk_(add|mul|fma)_f32", t) for t in code), name


def test_sixteen_waves_of_a_compute_unit(compiled):
    """The waves that the attention weights' launches count on, four of a SIMD or five, their workgroups' LDS side by side."""
    for name, (val, _) in compiled.items():
        m = re.search(r"attn_weights_kernelILi(\d+)ELb[01]ELi(\d+)ELi\d+E", name)
        if m:
            waves = 5 if (int(m.group(1)), int(m.group(2))) == (64, 4) else 4
            assert val(r"Occupancy \[waves/SIMD\]") >= waves, name
            assert val(r"LDS Size \[bytes/block\]") * (4 * waves // int(m.group(2))) <= 160 * 1024, name
