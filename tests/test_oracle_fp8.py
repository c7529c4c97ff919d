"""Pins of the reference of the 8-bit format and of the rotation (oracle/fp8_model.py): published values of the format, an
independent decoder, hand-worked rows, and what a rotation must do."""
import numpy as np
import pytest
import torch

from oracle import fp8_model as F


def test_code_values_are_the_formats():
    v = F.code_values()
    assert v[0x7E] == 448.0 and v[0x01] == 2.0 ** -9 and v[0x08] == 2.0 ** -6 and v[0x38] == 1.0 and v[0xB8] == -1.0
    assert np.isnan(v[0x7F]) and np.isnan(v[0xFF])
    other = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, other, equal_nan=True)


def test_quantise_agrees_with_another_rounding():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((400, 64)) * np.exp2(rng.integers(-30, 30, (400, 1)))).astype(np.float32)
    codes, scales = F.quantise(x)
    scaled = x.astype(np.float64) / np.exp2(scales.astype(np.float64) - 127)[:, None]
    other = torch.from_numpy(scaled.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(codes, other)
    most = np.abs(scaled).max(axis=1)
    assert (most <= 448).all() and (most > 224).all()


def test_hand_worked_rows():
    codes, scales = F.quantise(np.array([[448.0, 1.0, -1.0, 0.0], [448.5, 0, 0, 0], [0, 0, 0, -0.0], [1.75, 1.0625, 1.1875, 0.875],
                                         [np.inf, 2.0, np.nan, 1.0]]))
    assert scales.tolist() == [127, 128, 10, 119, 120]
    assert codes[0].tolist() == [0x7E, 0x38, 0xB8, 0]
    assert codes[1][0] == 0x76                                # 224.25 -> 224
    assert codes[2].tolist() == [0, 0, 0, 0x80]
    # 1.75 = 448 * 2^-8; 272 and 304 lie half way between codes (256 | 288 | 320): to the even ones, 256 and 320
    assert F.code_values()[codes[3]].tolist() == [448.0, 256.0, 320.0, 224.0]
    # not finite: the format's NaN, and the other values of the row keep theirs: 2.0 = 256 * 2^-7, byte 120
    assert codes[4].tolist()[0] == codes[4].tolist()[2] == 0x7F


def test_least_exponent_and_largest_values():
    codes, scales = F.quantise(np.array([[2.0 ** -126, 0], [3.3e38, -1e38]]))
    assert scales[0] == 10 and F.values_of(codes, scales)[0, 0] == 2.0 ** -126
    # 448 * 2^119 is finite in 32 bits and bf16; the next value up, 256 * 2^120, would not be
    assert scales[1] == 246 and F.values_of(codes, scales)[1, 0] == 448 * 2.0 ** 119 < 3.38e38
    assert abs(F.values_of(codes, scales)[1, 1] / -1e38 - 1) <= 2.0 ** -4


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_properties(layout):
    rng = np.random.default_rng(2)
    x, inv = rng.standard_normal((5, 3, 64)), 10000.0 ** (-2 * np.arange(16) / 32)
    at = np.repeat(np.arange(5)[:, None], 16, 1)
    y = F.rotate(x, at, inv, 32, layout)
    assert np.allclose(y[0], x[0]) and np.array_equal(y[..., 32:], x[..., 32:])
    assert np.allclose(F.rotate(y, at, inv, 32, layout, inverse=True), x)
    assert np.allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1))
    # scores depend on the difference of positions alone
    far = F.rotate(x, at + 1000, inv, 32, layout)
    assert np.allclose(np.einsum("thd,shd->hts", y, y), np.einsum("thd,shd->hts", far, far))
    # the first frequency turns (1, 0) by the position in radians
    one = np.zeros((1, 1, 64))
    one[0, 0, 0] = 1
    r = F.rotate(one, np.full((1, 16), 2), inv, 32, layout)
    assert np.allclose([r[0, 0, 0], r[0, 0, 16 if layout == "half" else 1]], [np.cos(2), np.sin(2)])
