"""Pins of the 8-bit oracle: worked examples and closed forms."""
import numpy as np

from oracle import int8 as o8


def test_codes_of_a_worked_row():
    # largest 254 -> scale 2; 3 / 2 = 1.5 and 5 / 2 = 2.5 are ties and go to the even 2
    q, s = o8.quant_rows([[254.0, 3.0, 5.0, -3.0, -254.0, 0.9, 1.1]])
    assert s.dtype == np.float32 and s[0] == 2.0
    assert q.tolist() == [[127, 2, 2, -2, -127, 0, 1]]


def test_scale_is_rounded_once_and_has_a_floor():
    q, s = o8.quant_rows([[1.0, -0.5], [0.0, 0.0], [1e-40, 0.0]])
    assert s[0] == np.float32(1.0 / 127.0)
    assert s[1] == s[2] == np.float32(2.0 ** -126)
    assert q.tolist() == [[127, -64], [0, 0], [0, 0]]   # -0.5 / fl(1/127) = -63.500000189: beyond the tie


def test_rows_that_are_not_finite():
    q, s = o8.quant_rows([[1.0, np.inf], [np.nan, 2.0], [3.0, -127.0]])
    assert np.isnan(s[:2]).all() and s[2] == 1.0
    assert q.tolist() == [[0, 0], [0, 0], [3, -127]]


def test_codes_stand_for_values_within_half_a_step():
    v = np.random.default_rng(1).standard_normal((20, 300))
    q, s = o8.quant_rows(v)
    assert (np.abs(q * s[:, None].astype(np.float64) - v) <= 0.5 * s[:, None] * (1 + 1e-7)).all()
    assert (np.abs(q.astype(int)).max(1) == 127).all()


def test_linear_by_hand():
    v = o8.linear([[1, -2], [127, 3]], [0.5, 2.0], [[3, 4], [-128, 1]], [1.0, 0.25], [10.0, 20.0])
    assert v.tolist() == [[-2.5 + 10, 0.125 * -130 + 20], [2 * 393 + 10, 0.5 * (3 - 127 * 128) + 20]]


def test_seam_by_hand():
    x, y = np.array([[1.0, 2.0]]), np.array([[3.0, -4.0]])
    h, a = o8.seam(x, y, 0.5, o8.NONE, [2.0, 1.0], [1.0, -1.0], o8.LAYER, [0.0, 1.0], [0.0, 1.0], 1e-30)
    assert h.tolist() == [[6.5, 5.0]]
    assert np.allclose(a, [[1.0, -1.0 * 2 + 1]], atol=1e-12)
    # RMS of (3, -4): sqrt(12.5)
    h, a = o8.seam(x, y, 1.0, o8.RMS, None, None, o8.NONE, None, None, 1e-30)
    assert np.allclose(h, [[1 + 3 / np.sqrt(12.5), 2 - 4 / np.sqrt(12.5)]], atol=1e-12)
    assert np.array_equal(a, h.astype(np.float32))


def test_seam_invariants():
    r = np.random.default_rng(2)
    x, y = r.standard_normal((5, 40)), r.standard_normal((5, 40))
    h, _ = o8.seam(x, y, 1.0, o8.LAYER, None, None, o8.RMS, None, None, 1e-12)
    h2, _ = o8.seam(x, 7 * y + 3, 1.0, o8.LAYER, None, None, o8.RMS, None, None, 1e-12)
    assert np.allclose(h, h2, atol=1e-9)                       # LayerNorm forgets scale and offset
    h0, a0 = o8.seam(x, None, 1.0, o8.NONE, None, None, o8.RMS, None, None, 1e-12)
    assert np.array_equal(h0, x)
    assert np.allclose((a0 ** 2).mean(1), 1.0, atol=1e-6)
