"""Calls of the C ABI from several host threads at once, without the interpreter's lock."""

import os
import shutil
import subprocess
import threading

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import paper_1811_10751_b200 as g                              # noqa: E402
from test_gpu_lm_adapters import CASES, Case                   # noqa: E402

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


def in_a_new_thread(call):
    """What the call raises in a thread that has made no other one."""
    raised = []

    def work():
        try:
            call()
        except Exception as e:                         # noqa: BLE001
            raised.append(e)
    t = threading.Thread(target=work)
    t.start()
    t.join()
    return raised


@pytest.mark.parametrize("name", ["one row each", "ragged", "rows off boundaries"])
def test_the_first_call_of_a_thread(name):
    c = Case(**CASES[name])
    out, h = c.forward()
    c.backward(h)
    dx, dA, dB = c.dx.clone(), c.dA.clone(), c.dB.clone()
    for t in (c.dx, c.dA, c.dB):
        t.zero_()
    out2, h2, ws = torch.zeros_like(out), torch.zeros_like(h), c.workspace()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    assert not in_a_new_thread(lambda: g.gpd_adapter(c.x, c.A, c.B, c.offsets, c.index, out2, h2, base=c.base, scale=c.scale, stream=st))
    assert not in_a_new_thread(lambda: g.gpd_adapter_backward(c.dout, c.x, c.A, c.B, h, c.offsets, c.index, c.dx, c.dA, c.dB, ws, dbase=c.dbase,
                                                              scale=c.scale, stream=st))
    st.synchronize()
    assert torch.equal(out2, out) and torch.equal(h2, h)
    assert torch.equal(c.dx, dx) and torch.equal(c.dA, dA) and torch.equal(c.dB, dB)


def test_the_first_call_of_a_thread_to_the_8_bit_product():
    a, a_scales = g.new_fp8(256, 512, torch.float8_e4m3fn)
    b, b_scales = g.new_fp8(384, 512, torch.float8_e4m3fn, 128)
    gen = torch.Generator(device="cuda").manual_seed(1)
    g.gpd_quantize_blocks(torch.randn(256, 512, device="cuda", generator=gen), q=a, scales=a_scales)
    g.gpd_quantize_blocks(torch.randn(384, 512, device="cuda", generator=gen), q=b, scales=b_scales, block_rows=128)
    want, got = torch.empty(256, 384, device="cuda"), torch.zeros(256, 384, device="cuda")
    g.gpd_gemm_fp8(a, a_scales, b, b_scales, want)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    assert not in_a_new_thread(lambda: g.gpd_gemm_fp8(a, a_scales, b, b_scales, got, stream=st))
    st.synchronize()
    assert torch.equal(got, want)
