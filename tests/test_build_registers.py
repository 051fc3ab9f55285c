"""The build's check of registers: no kernel spills vector registers to memory while it has matrix registers in use."""
import os
import subprocess

import pytest

from paper_2511_18191_amd import build

SOURCE = os.path.join(build.CSRC, "caller", "keep_path.hip")


def said(name, agprs, spilled, scratch=80):
    lines = [f"Function Name: {name}", "    TotalSGPRs: 42", "    VGPRs: 256", f"    AGPRs: {agprs}", f"    ScratchSize [bytes/lane]: {scratch}", "    SGPRs Spill: 7",
             f"    VGPRs Spill: {spilled}", "    LDS Size [bytes/block]: 0"]
    return "".join(f"a.hip:24:1: remark: {l} [-Rpass-analysis=kernel-resource-usage]\n" for l in lines)


def test_spills_beside_matrix_registers_are_refused():
    good = said("few", 0, 0, 0) + said("array", 8, 0) + said("slow", 0, 6)
    assert build._check_registers(SOURCE, good) == ""
    # (what the fp32 attention of heads above 128 dims had where its scores were wrong)
    with pytest.raises(RuntimeError, match="keep_path.hip.*matrix registers.*: bad, worse$"):
        build._check_registers(SOURCE, good + said("bad", 256, 19) + said("slow", 0, 1) + said("worse", 16, 1))


def test_what_else_the_compiler_says_is_kept():
    assert build._check_registers(SOURCE, said("few", 0, 0) + "a.hip:3:1: warning: unused\n" + said("few", 8, 0)) == "a.hip:3:1: warning: unused"
    with pytest.raises(RuntimeError, match="said nothing"):
        build._check_registers(SOURCE, "a.hip:3:1: warning: unused\n")


def test_the_compiler_speaks_of_every_kernel(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    r = subprocess.run([hipcc, *build.FLAGS, "-c", SOURCE, "-o", str(tmp_path / "a.o")], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    found = build.REMARK.findall(r.stderr)
    assert [what for what, _ in found] == ["Function Name", "AGPRs", "VGPRs Spill"] and "keep_path_kernel" in found[0][1]
    build._check_registers(SOURCE, r.stderr)
