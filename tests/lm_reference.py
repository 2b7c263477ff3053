"""Plain 64-bit forms of the low-precision layer operators, and helpers of their tests."""

import math

import torch

TOP = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}
# largest relative rounding error of a normal number (2 to the minus significant bits), and half the spacing of the smallest ones
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11,
            torch.float8_e4m3fn: 2.0 ** -4, torch.float8_e5m2: 2.0 ** -3}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25,
        torch.float8_e4m3fn: 2.0 ** -10, torch.float8_e5m2: 2.0 ** -17}


def strided(rows, cols, dtype, pad=0, offset=0, device="cuda"):
    """[rows, cols] view whose rows are `pad` elements apart from each other, `offset` elements into its buffer."""
    buf = torch.empty(offset + rows * (cols + pad) + 16, dtype=dtype, device=device)
    return buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]


def like(values, dtype, pad=0, offset=0):
    t = strided(values.shape[0], values.shape[1], dtype, pad, offset)
    t.copy_(values)
    return t


def block_amax(x, block_rows):
    """Largest magnitude of every block_rows x 128 block."""
    rows, cols = x.shape
    out = torch.zeros((-(-rows // block_rows), -(-cols // 128)), dtype=torch.float64, device=x.device)
    for i in range(out.shape[0]):
        for j in range(out.shape[1]):
            out[i, j] = x[i * block_rows:(i + 1) * block_rows, 128 * j:128 * (j + 1)].abs().max()
    return out


def spread(blocks, block_rows, rows, cols):
    return blocks.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def scale_values(s):
    """The numbers that scale bytes stand for."""
    b = s.view(torch.uint8).double()
    return torch.where(b == 255, math.nan, torch.exp2(b - 127))


def check_cut(q, scales, y, y_err, block_rows=1):
    """q, scales: a cut of y (64 bits), of which the kernel saw a value within y_err * |y|."""
    amax = block_amax(y, block_rows)
    s = scale_values(scales)
    top = TOP[q.dtype]
    zero = amax == 0
    assert torch.equal(s[zero], torch.ones_like(s[zero]))
    m, s_, lo = amax[~zero], s[~zero], 2.0 ** -127
    assert bool((m <= top * s_ * (1 + y_err)).all()), "the largest magnitude does not fit"
    assert bool(((m > top * s_ / 2 * (1 - y_err)) | (s_ == lo)).all()), "a smaller scale would do"
    s_el = spread(s, block_rows, *y.shape)
    got = q.double() * s_el
    # one rounding of the number, or half a step of the type's smallest numbers
    bound = y.abs() * (HALF_ULP[q.dtype] * (1 + 1e-6) + 2 * y_err) + TINY[q.dtype] * s_el
    # a value just above the largest number may have been cut back to it
    assert bool(((got - y).abs() <= bound).all()), float(((got - y).abs() - bound).max())


def check_close(got, ref, rel, scale=None):
    """|got - ref| <= (rel + the type's rounding) |ref|, or of `scale` where that is given (sums of larger terms)."""
    size = ref.abs() if scale is None else torch.maximum(ref.abs(), scale)
    bound = size * rel + ref.abs() * HALF_ULP[got.dtype] * (1 + 1e-6) + TINY[got.dtype]
    d = (got.double() - ref).abs()
    assert bool((d <= bound).all()), float((d / bound.clamp(min=1e-300)).max())
