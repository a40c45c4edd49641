"""The plain model of the 8- and 4-bit formats against torch's own conversions and
by hand (no GPU)."""
import numpy as np
import pytest
import torch

import perf.more_operators as cases
from tests import mx_util as mx


def test_values_of_the_codes():
    c = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(mx.code_values(8), c)
    assert mx.code_values(4).tolist()[:8] == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    assert mx.code_values(4).tolist()[8:] == [0, -0.5, -1, -1.5, -2, -3, -4, -6]
    s = torch.tensor([1, 100, 127, 254], dtype=torch.uint8)
    want = s.view(torch.float8_e8m0fnu).double().numpy()
    got = mx.values(np.full((4, 32), 0x38), s.numpy()[:, None], 8)        # 0x38: 1.0
    np.testing.assert_array_equal(got[:, 0], want)
    assert np.isnan(mx.values(np.zeros((1, 32), dtype=int), np.array([[255]]), 4)).all()


@pytest.mark.parametrize("bits,high,byte", [(8, 448, 127), (8, 449, 128), (8, 224, 126), (8, 0, 27),
                                            (8, 1e-31, 27), (4, 6, 127), (4, 6.5, 128), (4, 3, 126),
                                            (4, 4, 127), (8, 65504, 135), (4, 65504, 140),
                                            (4, 49152, 140), (4, 48000, 140)])
def test_scales(bits, high, byte):
    x = np.zeros((1, 32))
    x[0, 7] = -high
    code, scale = mx.quantise(x, bits, torch.float16)
    assert scale.tolist() == [[byte]]


def test_elements():
    x = np.zeros((1, 32))
    x[0, :12] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.01, -0.2, -0.3, 4.99]
    code, scale = mx.quantise(x, 4, torch.bfloat16)
    assert mx.values(code, scale, 4)[0, :12].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 6, 0, -0.5, 4]
    x[0, 3] = np.inf
    code, scale = mx.quantise(x, 4, torch.bfloat16)
    assert scale.tolist() == [[255]] and not code.any()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_rows_against_the_measured_form(bits, dtype):
    """Two models written apart: codes and scales are the same, and every value is
    one of the 16-bit type's."""
    t = cases.TYPES[dtype]
    g = torch.Generator().manual_seed(bits)
    x = torch.randn((300, 2, 96), generator=g) * torch.exp(4 * torch.randn((300, 2, 1), generator=g))
    x = x.to(t)
    x[0], x[1], x[2] = 0.0, torch.finfo(t).max, -torch.finfo(t).max * 0.95
    x[3, :, ::7] = torch.finfo(t).smallest_normal
    x = torch.where(torch.isfinite(x), x, torch.ones_like(x))
    code, scale = mx.quantise(x.double().numpy(), bits, t)
    other, other_scale = cases._quantise(x.float(), dict(code=f"fp{bits}", dtype=dtype))
    np.testing.assert_array_equal(mx.pack(code, bits), other.numpy())
    np.testing.assert_array_equal(scale, other_scale.numpy())
    v = mx.values(code, scale, bits)
    np.testing.assert_array_equal(torch.from_numpy(v).to(t).double().numpy(), v)
    # half a step of a normal code is 2^-4 or 2^-2 of it, and below the normal ones
    # 2^-10 or 2^-2 of the scale
    step = np.maximum(np.abs(x.double().numpy()) * (2.0 ** -4 if bits == 8 else 0.25),
                      np.repeat(2.0 ** (scale - 127.0), 32, -1) * (2.0 ** -10 if bits == 8 else 0.25))
    inside = np.abs(x.double().numpy()) <= torch.finfo(t).max * 0.7
    assert np.all((np.abs(v - x.double().numpy()) <= step)[inside])
