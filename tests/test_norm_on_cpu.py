"""The norms' kernels in place, run on the host from their own source with the wavefronts of a workgroup as far apart as its barriers allow (no GPU needed)."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_1807_11205_amd", "csrc")
CLANG = os.environ.get("JZ_HOST_CLANG", "/opt/rocm/llvm/bin/clang++")     # the vector types are clang's


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("norm_on_cpu")
    with open(os.path.join(CSRC, "jz_norm.hip")) as f:
        text = f.read()
    begin, end = text.index('#include "jz_vec.h"') + len('#include "jz_vec.h"'), text.index("// ---- host")
    kernels = d / "kernels.inc"
    kernels.write_text(text[begin:end])
    out = d / "norm_on_cpu"
    subprocess.run([CLANG, "-std=c++17", "-O1", "-w", "-DKERNELS=\"%s\"" % kernels, "-I", CSRC, "-o", str(out), os.path.join(HERE, "norm_on_cpu.cpp")], check=True)
    return str(out)


@pytest.mark.parametrize("backward", [0, 1])
def test_in_place_whatever_the_order_of_the_wavefronts(program, backward):
    r = subprocess.run([program, str(backward)], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout
