"""Pins of the 4-bit oracle: hand-worked groups, ties, borders, the scale's rule,
and the tests' fast form against the plain one."""
import numpy as np
import pytest

from oracle import entmtp_oracle as orc
from oracle import fp4_oracle as fo
from paper_2606_27550_amd import synth
from tests.fp4_helpers import quantize_fast


def group(*head):
    return np.array(list(head) + [0.0] * (32 - len(head)))


def test_hand_worked_group():
    # largest 6: e = 2, mantissa 1.5, scale 1; ties go to the even code
    x = group(6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.3, -5.01, -0.0)
    codes, s = fo.quantize_group(x)
    assert s == 127
    assert codes[:11].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8 + 1, 8 + 7, 8]
    packed, scales = fo.quantize(x)
    assert packed[0] == 0x07 and packed[1] == 0x22   # (the first value in the lower half)
    np.testing.assert_array_equal(fo.values(packed, scales)[:8], [6, 0, 1, 1, 2, 2, 4, 4])


@pytest.mark.parametrize("top,step,held", [(1.0, 0.25, 1.0), (1.5, 0.25, 1.5), (1.7421875, 0.25, 1.5), (1.75, 0.5, 2.0),
                                           (1.9921875, 0.5, 2.0), (2.0, 0.5, 2.0), (7.0, 2.0, 8.0), (6.96875, 1.0, 6.0)])
def test_scale_rule(top, step, held):
    """The largest value of a group is off by at most one step of its scale."""
    x = group(top)
    codes, s = fo.quantize_group(x)
    assert 2.0 ** (s - 127) == step
    assert fo.values(*fo.quantize(x))[0] == held and abs(held - top) <= step


def test_ends_of_the_range():
    for x, want in ((2.0 ** -133, 2), (0.0, 2), (2.0 ** 127 * 1.9921875, 252)):
        assert fo.quantize_group(group(x))[1] == want
    assert fo.values(*fo.quantize(group(2.0 ** 127 * 1.9921875)))[0] == 6 * 2.0 ** 125
    for bad in (np.nan, np.inf, -np.inf):
        codes, s = fo.quantize_group(group(1.0, bad))
        assert s == 255 and not codes.any()
        assert np.isnan(fo.values(*fo.quantize(group(1.0, bad)))).all()


def test_error_of_normal_numbers():
    """Half a step of the level above or below, so at most 1/4 of the value above one step, and 1/4 step below it."""
    x = orc.bf16_to_f64(synth.normal_bf16(np.random.default_rng(3), (40, 128)))
    codes, s = fo.quantize(x)
    step = np.repeat(2.0 ** (s.astype(float) - 127), 32, -1)
    assert (np.abs(fo.values(codes, s) - x) <= np.maximum(step / 4, np.abs(x) / 4)).all()


def test_fast_form():
    g = np.random.default_rng(4)
    x = orc.bf16_to_f64(synth.normal_bf16(g, (60, 96))) * 2.0 ** g.integers(-120, 110, (60, 1))
    x = orc.round_to_bf16(x)
    x[0] = 0
    x[1, :40] = -0.0
    for a, b in zip(fo.quantize(x), quantize_fast(x)):
        np.testing.assert_array_equal(a, b)


def test_pages():
    g = np.random.default_rng(5)
    codes, scales = g.integers(0, 256, (3, 2, 16, 64), dtype=np.uint8), g.integers(2, 253, (3, 2, 16, 4), dtype=np.uint8)
    pool = fo.join(codes, scales)
    assert pool.shape == (3, 2, 16 * 68)
    for a, b in zip(fo.planes(pool), (codes, scales)):
        np.testing.assert_array_equal(a, b)
    np.testing.assert_array_equal(pool[1, 1, 5 * 64:6 * 64], codes[1, 1, 5])
    np.testing.assert_array_equal(pool[1, 1, 16 * 64 + 5 * 4:16 * 64 + 6 * 4], scales[1, 1, 5])


def test_norm_and_turn():
    x = np.random.default_rng(6).standard_normal((2, 128))
    y = fo.norm_turn(x, 0, None, 1e-6, 1e4)
    np.testing.assert_allclose(y, x, rtol=0, atol=1e-15)
    y = fo.norm_turn(x, 7, np.ones(128), 0.0, 1e4)   # a turn keeps the norm's length sqrt(d)
    np.testing.assert_allclose((y * y).sum(1), [128, 128], rtol=1e-12)
    y = fo.norm_turn(x * 1000, 7, np.ones(128), 0.0, 1e4)
    np.testing.assert_allclose(y, fo.norm_turn(x, 7, np.ones(128), 0.0, 1e4), rtol=1e-9)
