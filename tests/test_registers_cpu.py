"""The kernels of the gated delta rule hold states, sums and what is on its way in registers, near the end of those that a wave has.  What does not fit
goes to memory without a word, a step of every loop: the built library says how much of it a kernel asks for."""
import os
import re
import subprocess

import pytest

from paper_2604_25422_amd import _build
from test_mfma_waits_cpu import code_objects

READELF = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-readelf")


def scratch_of(path):
    """{kernel: bytes of memory that each of its lanes has for registers}, from a code object's notes."""
    r = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    out, name = {}, None
    for line in r.stdout.splitlines():
        # (a kernel's fields are in the order of their names)
        if m := re.match(r"\s+\.name:\s+(_Z\S+)\s*$", line):
            name = m[1]
        elif (m := re.match(r"\s+\.private_segment_fixed_size:\s+(\d+)", line)) and name:
            out[name], name = int(m[1]), None
    return out


def test_the_delta_rule_s_kernels_keep_to_registers(tmp_path):
    if not os.path.exists(READELF):
        pytest.skip("no llvm-readelf")
    if not os.path.exists(_build.LIB_PATH):
        _build.build()
    kernels = {}
    for n, code in enumerate(code_objects(_build.LIB_PATH)):
        path = tmp_path / f"{n}.co"
        path.write_bytes(code)
        kernels.update({k: v for k, v in scratch_of(path).items() if "delta_" in k})
    # fp32 and bf16, keys of up to 32, 64 and 128 channels
    assert sum("delta_bwd_chunk_kernel" in k for k in kernels) == 12 and sum("delta_fwd_kernel" in k for k in kernels) == 12
    assert not {k: v for k, v in kernels.items() if v}


def remark(name, scratch):
    at = "csrc/x.hip:1:1: remark: "
    return f"{at}Function Name: {name} [-Rpass-analysis=kernel-resource-usage]\n{at}    ScratchSize [bytes/lane]: {scratch} [-Rpass-analysis=kernel-resource-usage]\n"


def test_the_build_says_which_spill(capsys):
    _build.check_no_scratch(remark("_ZN6dwconv22delta_bwd_chunk_kernelIfLi8ELb0EEEvv", 0) + remark("_ZN6dwconv16norm_fwd_kernelIfEEvv", 16), "x.hip")
    assert capsys.readouterr().out == ""
    _build.check_no_scratch(remark("_ZN6dwconv22delta_bwd_chunk_kernelIfLi8ELb0EEEvv", 108), "x.hip")
    said = capsys.readouterr().out
    assert "x.hip" in said and "delta_bwd_chunk_kernelIfLi8ELb0E" in said and "108" in said
    with pytest.raises(RuntimeError, match="corr_mfma_kernel"):
        _build.check_no_scratch(remark("_ZN6dwconv16corr_mfma_kernelIfEEvv", 4), "x.hip")
