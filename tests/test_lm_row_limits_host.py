"""CPU-only: numbers of rows, segments and adapters that leave no room for the steps of loops over them in 32 bits are refused."""

import ctypes as C

import pytest

pytest.importorskip("torch")
import paper_1811_10751_b200 as g            # noqa: E402

P = C.c_void_p(4096)                          # never dereferenced: the checks come first
L = g.lib


@pytest.mark.parametrize("T", [(1 << 31) - (1 << 16) + 1, (1 << 31) - 1, 1 << 31, 1 << 40])
def test_rows(T):
    size = C.c_int64()
    assert L.gpd_head_norm_rope(1, P, 256, 2, P, 128, 1, 128, 1, P, P, 1e-6, P, 128, 10, 128, 0, 4, P, 1, 1, None, P, 256, P, 128, T, None) == g.GPD_ERR_SHAPE
    assert L.gpd_head_norm_rope_backward(1, P, 256, P, 128, P, 256, 2, P, 128, 1, 128, 1, P, P, 1e-6, P, 128, 10, 128, 0, 4, P, 1, 1, None, P, 256, P, 128, P,
                                         P, T, P, 1 << 30, None) == g.GPD_ERR_SHAPE
    assert L.gpd_adapter(1, P, 64, 2, 8, P, 64, 512, P, 8, 384, None, 4, P, P, 3, P, 1, None, 0, P, 48, T, 64, 48, None) == g.GPD_ERR_SHAPE
    assert L.gpd_adapter_backward_workspace(T, 64, 48, 2, 8, C.byref(size)) == g.GPD_ERR_SHAPE


@pytest.mark.parametrize("n,S", [((1 << 30) + 1, 3), ((1 << 31) - 1, 3), (2, (1 << 30) + 1), (2, (1 << 31) - 1)])
def test_adapters_and_segments(n, S):
    assert L.gpd_adapter(1, P, 64, n, 8, P, 64, 512, P, 8, 384, None, 4, P, P, S, P, 1, None, 0, P, 48, 10, 64, 48, None) == g.GPD_ERR_SHAPE
    assert L.gpd_adapter_backward(1, P, 48, P, 64, n, 8, P, 64, 512, P, 8, 384, None, P, 4, P, P, S, 1, None, 0, P, 64, 0, P, 64, 512, P, 8, 384, 0, 10, 64,
                                  48, P, 1 << 62, None) == g.GPD_ERR_SHAPE
