"""How far halves are from the rows of the 4-bit product, as the header bounds it:
the kernel's arithmetic in numpy (CPU only).  A value is scaled by 2^up, up = 14 less
its block's largest exponent (at least -112); an fp32 value then leaves at most 2^12
steps of its last bit to a second half of 11 bits: one step, 2^-23 of it, is lost at
most, or half of a half's smallest step, 2^-25, 2^-39 of a largest of 2^14 and more."""
import numpy as np
import pytest
import torch

BF16, F32 = torch.bfloat16, torch.float32


def halves(x, top, dtype):
    """What the product takes for x (fp32 array) in a block whose largest value is top."""
    e = max(int(np.frexp(np.float32(top))[1]) - 1, -112)
    t = np.ldexp(x.astype(np.float32), 14 - e).astype(np.float32)
    h = t.astype(np.float16)
    got = h.astype(np.float64)
    if dtype == F32:
        got = got + (t - h.astype(np.float32)).astype(np.float16).astype(np.float64)
    return np.ldexp(got, e - 14)


def bound(x, top, dtype):
    far = np.full(x.shape, 2.0 ** -39 * float(top))
    return np.maximum(far, 2.0 ** -23 * np.abs(x.astype(np.float64))) if dtype == F32 else far


def _off(x, top, dtype):
    return np.abs(halves(x, top, dtype) - x.astype(np.float64))


def test_a_binade_of_fp32():
    """Every float of one: within 2^-23, and more than 2^-24 for some."""
    x = (np.arange(1 << 23, 1 << 24, dtype=np.uint32)).astype(np.float32)   # 2^23 .. 2^24 in steps of 1
    for top in (x[-1], np.float32(2.0 ** 24), np.float32(2.0 ** 38)):
        off = _off(x, top, F32)
        assert (off <= bound(x, top, F32)).all()
        assert (off / x).max() > 1.9 * 2.0 ** -24
    assert _off(np.float32([16384 + 4 + 2.0 ** -9]), 16384, F32)[0] == 2.0 ** -9


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_small_values_beside_large_ones(dtype):
    g = torch.Generator().manual_seed(1)
    for e in (-140, -126, -113, -112, -111, -60, 0, 60, 114):
        for top in (2.0 ** e, 2.0 ** e * 1.9921875):
            x = torch.randn(60000, generator=g) * torch.exp2(-50 * torch.rand(60000, generator=g)) * 2.0 ** (e - 3)
            x = x.to(dtype).float().clamp(-top, top).numpy()
            off = _off(x, top, dtype)
            assert (off <= bound(x, top, dtype)).all(), e
            if dtype == BF16:
                assert not off[np.abs(x) >= 2.0 ** -31 * top].any(), e


def test_where_values_begin_to_lose_bits():
    """bf16 below 2^-31 of a power of two, fp32 (but for its last bit) below some 2^-16."""
    x = np.float32([2.0 ** -31 * (1 + 2.0 ** -7), 2.0 ** -32 * (1 + 2.0 ** -7)])
    off = _off(x, 1.0, BF16)
    assert off[0] == 0 and off[1] == 2.0 ** -39
    x = np.float32([2.0 ** -20 * (1 + 2.0 ** -19 - 2.0 ** -23)])
    assert _off(x, 1.0, F32)[0] > 2.0 ** -21 * x[0]
