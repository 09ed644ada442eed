"""Pins of the 8-bit floating-point oracle: hand-worked values, torch's own conversions, exact scaling, the place of the scales."""
import numpy as np
import pytest
import torch

from oracle import f8

TYPES = [(f8.E4M3, torch.float8_e4m3fn), (f8.E5M2, torch.float8_e5m2)]


@pytest.mark.parametrize("name,dt", TYPES)
def test_formats_are_those_of_torch(name, dt):
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(codes.view(dt).double().numpy(), f8.TABLE[name], equal_nan=True)
    x = torch.randn(20000, generator=torch.Generator().manual_seed(3)).bfloat16().float()
    x = torch.cat([x, x * 2.0 ** -9, torch.tensor([0.0, -0.0, float(f8.MAX[name]), -float(f8.MAX[name])])])
    assert np.array_equal(x.to(dt).view(torch.uint8).numpy(), f8.encode(x.double().numpy(), name))


def test_hand_worked_values():
    assert [f8.value(c, f8.E4M3) for c in (0x00, 0x01, 0x08, 0x38, 0x7E, 0xC0)] == [0.0, 2.0 ** -9, 2.0 ** -6, 1.0, 448.0, -2.0]
    assert [f8.value(c, f8.E5M2) for c in (0x01, 0x04, 0x3C, 0x7B, 0x7C)] == [2.0 ** -16, 2.0 ** -14, 1.0, 57344.0, float("inf")]
    # ties go to the even code: 17 lies between 16 (0x58) and 18 (0x59), 19 between 18 and 20 (0x5A)
    assert list(f8.encode(np.array([17.0, 19.0, -17.0, np.nan]), f8.E4M3)) == [0x58, 0x5A, 0xD8, 0x7F]


@pytest.mark.parametrize("name,log2", [(f8.E4M3, 8), (f8.E5M2, 15)])
def test_scales(name, log2):
    top = f8.MAX[name]
    assert f8.scale_byte(0.0, name) == 127
    assert f8.scale_byte(top, name) == 127 and f8.scale_byte(np.nextafter(top, 1e9), name) == 128
    assert f8.scale_byte(top / 2, name) == 126 and f8.scale_byte(1.0, name) == 127 - log2
    assert f8.scale_byte(2.0 ** -149, name) == 0 and f8.scale_byte(3.4e38, name) == 127 + 127 - log2 + 1


def test_quantize_is_off_by_half_a_step_and_exact_on_the_grid():
    x = np.random.default_rng(5).standard_normal((7, 300)) * np.exp2(np.arange(7) * 9 - 30)[:, None]
    for name, half in ((f8.E4M3, 2.0 ** -4), (f8.E5M2, 2.0 ** -3)):
        codes, scales = f8.quantize(x, name)
        back = f8.dequantize(codes, scales, name)
        amax = np.abs(np.pad(x, ((0, 0), (0, 84))).reshape(7, 3, 128)).max(2)
        floor = np.repeat(amax, 128, axis=1)[:, :300] * 2.0 ** -15                  # (entries below the normal range of their block)
        assert (np.abs(back - x) <= np.maximum(half * np.abs(x), floor)).all()
        again = f8.quantize(back, name)
        assert np.array_equal(f8.dequantize(*again, name), back)


def test_non_finite_entries_enter_no_scale():
    x = np.ones((1, 128))
    x[0, 3], x[0, 4], x[0, 5] = np.nan, np.inf, -np.inf
    codes, scales = f8.quantize(x, f8.E4M3)
    assert scales[0, 0] == 119 and list(codes[0, 3:6] & 0x7F) == [0x7F] * 3 and f8.TABLE[f8.E4M3][codes[0, 0]] == 256.0
    codes, scales = f8.quantize(np.full((1, 4), np.nan), f8.E4M3)
    assert scales[0, 0] == 127 and list(codes[0]) == [0x7F] * 4


def test_places_of_scales_are_a_permutation():
    R, cols = 300, 1100
    s = np.arange(R * 9, dtype=np.int64).reshape(R, 9) % 251
    packed = f8.pack_scales(s.astype(np.uint8), cols)
    assert packed.size == 3 * 3 * 512 and np.array_equal(f8.unpack_scales(packed, R, cols), s)
    assert (f8.scale_at(0, 0, cols), f8.scale_at(1, 0, cols), f8.scale_at(32, 0, cols), f8.scale_at(0, 1, cols), f8.scale_at(0, 4, cols), f8.scale_at(128, 0, cols)) == (0, 16, 4, 1, 512, 1536)
