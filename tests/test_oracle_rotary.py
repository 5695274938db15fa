"""Pins of the oracle of rotations and of appends with scales, by hand and by properties."""
import math

import numpy as np
import pytest

from oracle import rotary as R


def test_a_quarter_turn():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 9.0]]])
    f = [math.pi / 2, math.pi]
    np.testing.assert_allclose(R.rotate(x, [1], f)[0, 0], [-3, -2, 1, -4, 9], atol=1e-15)  # (1, 3), (2, 4)
    np.testing.assert_allclose(R.rotate(x, [1], f, interleaved=True)[0, 0], [-2, 1, -3, -4, 9], atol=1e-15)  # (1, 2), (3, 4)
    np.testing.assert_allclose(R.rotate(x, [1], f, magnitude=2.0, reverse=True)[0, 0], [6, -4, -2, -8, 9], atol=1e-15)


@pytest.mark.parametrize("interleaved", [False, True])
def test_scores_go_by_the_distance(interleaved):
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 1, 16))
    f, _ = R.frequencies(16)
    dot = lambda p, r: float((R.rotate(q, [p], f, interleaved=interleaved) * R.rotate(k, [r], f, interleaved=interleaved)).sum())  # noqa: E731
    assert dot(1000, 990) == pytest.approx(dot(17, 7), rel=1e-12)
    back = R.rotate(R.rotate(q, [12345], f, interleaved=interleaved), [12345], f, interleaved=interleaved, reverse=True)
    np.testing.assert_allclose(back, q, rtol=1e-12)


def test_reverse_is_the_gradient():
    rng = np.random.default_rng(1)
    x, g = rng.standard_normal((2, 3, 2, 8))
    f, pos, step = R.frequencies(6)[0], [3, 0, 70], 1e-6
    grad = R.rotate(g, pos, f, 1.3, reverse=True)
    for at in [(0, 0, 0), (0, 1, 5), (2, 1, 2), (2, 0, 7), (1, 1, 3)]:
        d = np.zeros_like(x)
        d[at] = step
        slope = ((R.rotate(x + d, pos, f, 1.3) - R.rotate(x - d, pos, f, 1.3)) * g).sum() / (2 * step)
        assert grad[at] == pytest.approx(slope, abs=1e-8)


def test_frequencies_by_hand():
    f, m = R.frequencies(4, base=100.0)
    np.testing.assert_allclose(f, [1.0, 0.1])
    assert m == 1.0
    np.testing.assert_allclose(R.frequencies(4, 100.0, "linear", 4.0)[0], [0.25, 0.025])
    f, _ = R.frequencies(4, 100.0, "base", 4.0)  # base 100 * 4^2
    np.testing.assert_allclose(f, [1.0, 1.0 / 40.0])
    # Turns over 1000 positions: 159 and 15.9.  All above high stays, all below low goes `factor` times slower; but a ramp
    # begins at the first pair at the earliest, and that stays.
    np.testing.assert_allclose(R.frequencies(4, 100.0, "bands", 4.0, 1000.0, 200.0, 300.0)[0], [0.25, 0.025])
    np.testing.assert_allclose(R.frequencies(4, 100.0, "ramp", 4.0, 1000.0, 200.0, 300.0)[0], [1.0, 0.025])
    np.testing.assert_allclose(R.frequencies(4, 100.0, "bands", 4.0, 1000.0, 1.0, 10.0)[0], [1.0, 0.1])
    keep = (1000 * 0.1 / (2 * math.pi) - 10) / 90
    np.testing.assert_allclose(R.frequencies(4, 100.0, "bands", 4.0, 1000.0, 10.0, 100.0)[0], [1.0, 0.1 * (keep + (1 - keep) / 4)])
    assert R.frequencies(4, 100.0, "ramp", math.e, 1000.0, 1.0, 10.0)[1] == pytest.approx(1.1)


@pytest.mark.parametrize("x,e", [(0.0, -64), (448.0, 0), (448.0001, 1), (447.0, 0), (224.0, -1), (224.001, 0), (1.0, -8), (1e30, 64), (2.0 ** -56, -64)])
def test_powers_of_two(x, e):
    assert R.power_of_two(x) == 2.0 ** e


def test_a_scale_grows_and_earlier_values_stay():
    codes, scales = np.zeros((2, 1, 8, 2)), np.full((2, 1), 0.5, dtype=np.float32)
    codes[1, 0, :3] = [[448, -1], [2 ** -6, 3 * 2 ** -9], [1, 0]]
    x = np.array([[[300.0, 2.0]], [[1.0, 896.0]]])
    got, s, fresh = R.append_scaled(x, [11, 12], codes, scales)  # block 1, places 3 and 4
    assert s.tolist() == [[0.5], [2.0]]
    np.testing.assert_array_equal(got[1, 0, :5], [[112, -0.25], [2 ** -8, 2 ** -9], [0.25, 0], [150, 1], [0.5, 448]])
    assert fresh[1].tolist() == [False] * 3 + [True] * 2 + [False] * 3 and not fresh[0].any()
    got, s, _ = R.append_scaled(x[:1] / 300, [11], codes, scales)
    assert s[1, 0] == 0.5 and got[1, 0, 0, 0] == 448  # the scale suffices
    got, s, _ = R.append_scaled(x[:1], [8], codes, scales)
    assert s[1, 0] == 1.0 and got[1, 0, 1, 0] == 2 ** -6  # a first place: nothing before counts, nothing after changes
