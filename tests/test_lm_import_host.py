"""CPU-only: the coded products do not need the compiled part of the low-precision operators' binding, and a call of one of
these operators says what is missing."""

import os
import shutil
import subprocess
import sys

import pytest

pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = "paper_1811_10751_b200"

PROGRAM = """
import torch
import paper_1811_10751_b200 as g
assert g.__file__.startswith({where!r}), g.__file__
plan = g.gpd_plan((64, 64, 8), (2, 1, 2, 1), 8)
print("nodes", plan.query(g.GPD_Q_NODES))
x = torch.zeros((2, 16))
for call in (lambda: g.gpd_rmsnorm_quant(x, x[0], 1e-5, y=x), lambda: g.gpd_gemm_fp8(x, x, x, x, x),
             lambda: g.gpd_token_logprobs(x, x[0], x[0], x[0]), lambda: g.gpd_distill_topk(x, x, x, None, x[0])):
    try:
        call()
    except ImportError as e:
        print("ImportError:", e)
"""


@pytest.mark.parametrize("binding", ["absent", "damaged"])
def test_package_without_the_compiled_binding(tmp_path, binding):
    pkg = tmp_path / PKG
    pkg.mkdir()
    for f in os.listdir(os.path.join(ROOT, PKG)):
        if f.endswith(".py"):
            shutil.copy(os.path.join(ROOT, PKG, f), pkg)
    os.symlink(os.path.join(ROOT, PKG, "libgpd.so"), pkg / "libgpd.so")
    if binding == "damaged":
        (pkg / "_lm.so").write_bytes(b"not a library")
    r = subprocess.run([sys.executable, "-c", PROGRAM.format(where=str(tmp_path))], cwd=tmp_path, capture_output=True, text=True,
                       env={**os.environ, "PYTHONPATH": str(tmp_path)}, timeout=300)
    assert r.returncode == 0, r.stderr
    lines = r.stdout.splitlines()
    assert lines[0] == "nodes 8"
    assert len(lines) == 5 and all(ln.startswith("ImportError:") and "build.py" in ln for ln in lines[1:]), lines
