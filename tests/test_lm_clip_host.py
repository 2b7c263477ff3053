"""CPU-only: which overlaps gpd_clip_grads refuses before it would touch a GPU."""

import ctypes as C

import pytest

pytest.importorskip("torch")
import paper_1811_10751_b200 as g            # noqa: E402


def clip(ptrs, outs, counts, norm):
    n = len(ptrs)
    types = (C.c_int32 * n)()
    return g.lib.gpd_clip_grads(n, types, (C.c_void_p * n)(*ptrs), types, (C.c_void_p * n)(*outs), (C.c_int64 * n)(*counts), C.c_void_p(norm), 1.0, None)


@pytest.mark.parametrize("ptrs,outs,counts", [([4096], [4096], [8]), ([4096], [8192], [8]), ([4096, 16384, 256], [4096, 20480, 128], [8, 3, 2])])
def test_the_norm_is_no_part_of_an_output(ptrs, outs, counts):
    """In place, to other buffers and mixed; the norm at the beginning, inside and at the end of an output."""
    for o, n in zip(outs, counts):
        for at in (o, o + 4 * (n // 2), o + 4 * (n - 1)):
            assert clip(ptrs, outs, counts, at) == g.GPD_ERR_ARG
