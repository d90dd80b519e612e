"""Pins of the 64-bit definition of the 8-bit floating-point layer (oracle/f8.py) against independent sources: torch's own
E4M3 conversion, the properties that define the scale, hand-computed values."""
import numpy as np
import torch

from oracle import f8


def test_element_values_are_the_formats():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    got = f8.e4m3_values()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])
    assert np.nanmax(got) == 448.0 and got[1] == 2.0 ** -9


def test_encode_matches_torch_and_saturates():
    g = np.random.default_rng(0)
    v = np.concatenate([g.standard_normal(20000) * np.exp2(g.uniform(-11, 8, 20000)), f8._MID, -f8._MID, f8._POS, [0.0, -0.0, 1e-6]])
    v = v[np.abs(v) <= 448].astype(np.float32)
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(f8.encode(v), want)
    assert list(f8.encode(np.array([1e9, -1e9, np.inf, np.nan]))) == [0x7E, 0xFE, 0x7E, 0x7F]


def test_scale_is_the_smallest_power_of_two_that_fits():
    g = np.random.default_rng(1)
    a = np.concatenate([np.abs(g.standard_normal(5000)) * np.exp2(g.uniform(-100, 100, 5000)), 448 * np.exp2(np.arange(-30.0, 30.0)),
                        np.nextafter(448.0, 500.0) * np.exp2(np.arange(-30.0, 30.0))])
    b = f8.scale_byte(a)
    assert np.all(a <= 448 * f8.pow2(b)) and np.all(a > 448 * f8.pow2(b - 1))
    assert f8.scale_byte(np.array([0.0]))[0] == 127 and f8.scale_byte(np.array([448.0, 449.0]))[1] == 128
    assert f8.scale_byte(np.array([1e-45]))[0] == 0


def test_rows_and_blocks_round_trip_within_half_a_step():
    g = np.random.default_rng(2)
    v = g.standard_normal((7, 300)) * np.exp2(g.uniform(-3, 3, (7, 1)))
    v[3] = 0
    codes, scales = f8.quantize_rows(v)
    assert codes.shape == (7, 384) and scales.shape == (7, 4) and np.all(scales[:, 3] == 127) and np.all(codes[:, 300:] == 0)
    back = f8.dequantize_rows(codes, scales, 300)
    s = np.repeat(f8.pow2(scales[:, :3]), 128, axis=1)[:, :300]
    # three mantissa bits: half a step is at most 2^-4 of the value, or half of the subnormal step 2^-9
    assert np.all(np.abs(back - v) <= np.maximum(np.abs(v) * 2.0 ** -4, s * 2.0 ** -10))
    assert np.all(scales[3] == 127) and np.all(codes[3] == 0)
    again, scales2 = f8.quantize_rows(back)
    assert np.array_equal(f8.dequantize_rows(again, scales2, 300), back)
    W = g.standard_normal((200, 260))
    c, b = f8.quantize_blocks(W)
    assert b.shape == (2, 3)
    Wb = f8.dequantize_blocks(c, b)
    big = np.zeros((256, 384))
    big[:200, :260] = W
    for i in range(2):
        for j in range(3):
            assert f8.scale_byte(np.abs(big[128 * i : 128 * i + 128, 128 * j : 128 * j + 128]).max()) == b[i, j]
    assert np.linalg.norm(Wb - W) / np.linalg.norm(W) < 0.04


def test_norm_and_silu_by_hand():
    t, y = f8.norm(np.array([[3.0, 4.0]]), np.array([[0.0, 0.0]]), np.array([1.0, 2.0]), 0.0)
    assert np.allclose(y, [[3 / np.sqrt(12.5), 8 / np.sqrt(12.5)]], rtol=1e-15) and np.array_equal(t, [[3.0, 4.0]])
    _, y = f8.norm(np.array([[1.0, -1.0]]), np.array([[-1.0, 1.0]]), np.array([1.0, 1.0]), 1e-5)
    assert np.array_equal(y, [[0.0, 0.0]])
    assert f8.silu(np.array([0.0]))[0] == 0 and abs(f8.silu(np.array([1.0]))[0] - 1 / (1 + np.exp(-1))) < 1e-15
    assert f8.silu(np.array([-2000.0]))[0] == 0
