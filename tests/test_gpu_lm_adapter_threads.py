"""Calls of the C ABI from several host threads at once, without the interpreter's lock."""

import os
import shutil
import subprocess

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                              # noqa: E402

HERE = os.path.dirname(os.path.abspath(__file__))
NVCC = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"


@pytest.mark.skipif(not os.path.exists(NVCC), reason="needs nvcc")
def test_single_rows_of_other_sizes_at_the_same_time(tmp_path):
    lib, program = os.path.dirname(g.__file__), str(tmp_path / "threads")
    subprocess.run([NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-O2", "-std=c++17", "-I", os.path.join(os.path.dirname(HERE), "include"),
                    os.path.join(HERE, "c_abi_threads.cpp"), "-o", program, "-L", lib, "-lgpd", "-lpthread", "-Xlinker", "-rpath", "-Xlinker", lib],
                   check=True, timeout=300)
    r = subprocess.run([program], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
