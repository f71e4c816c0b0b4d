"""Outputs whose alignment the interface does not ask for are declared so: the stores of kv_read's keys and values and
of the decode's outputs carry no more than an element's alignment in the compiler's intermediate code."""
import os
import re
import subprocess

import pytest

from paper_2604_23996_amd import build as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.HIPCC), reason="hipcc not installed")


def kernels(source, name, tmp_path):
    """{mangled name: [(stored type, alignment) of every store to global memory]} of a source's kernels."""
    out = str(tmp_path / "ir.ll")
    r = subprocess.run([B.HIPCC, *B.COMMON, "--cuda-device-only", "-S", "-emit-llvm", os.path.join(B.CSRC, source),
                        "-o", out], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    found = {}
    for f in re.split(r"\ndefine ", open(out).read())[1:]:
        head = f.split("(")[0]
        if "amdgpu_kernel" in head and name in head:
            found[head.split("@")[-1]] = [(t, int(a)) for t, a in re.findall(
                r"store (<[^>]*>|\w+) [^\n]*?, ptr addrspace\(1\) [^\n]*?, align (\d+)", f)]
    assert found and all(found.values())
    return found


def test_rows_read_back(tmp_path):
    for name, stores in kernels("kvcache.hip", "kv_read_kernel", tmp_path).items():
        bf16 = name.split("kv_read_kernelI")[1].split("EEEv")[0].endswith("Lb1")
        rows = [a for t, a in stores if t != "float"]  # the scores are single floats
        assert rows and max(rows) <= (2 if bf16 else 4), (name, stores)


def test_outputs_of_the_decode(tmp_path):
    for name in ("decode_kernel", "decode_join_kernel"):
        for kernel, stores in kernels("decode.hip", name, tmp_path).items():
            rows = [a for t, a in stores if t not in ("float", "<4 x float>", "i64")]  # those: scores, and the workspace
            assert rows and max(rows) <= 2, (kernel, stores)
            assert all(a == 4 for t, a in stores if t == "float")
