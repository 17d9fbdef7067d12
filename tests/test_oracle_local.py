"""The oracles of the local step's operators, against hand values and difference quotients (CPU)."""
import numpy as np
import pytest

from oracle import mxfp4, preference


def test_codes_at_and_about_the_midpoints():
    # the representable magnitudes, their midpoints (ties to the even code) and the neighbours of these
    for c, v in enumerate(mxfp4.MAGNITUDES):
        assert mxfp4.round_code(np.array([v]))[0] == c
    for i, mid in enumerate([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]):
        even = i if i % 2 == 0 else i + 1
        assert list(mxfp4.round_code(np.array([np.nextafter(mid, 0), mid, np.nextafter(mid, 9)]))) == [i, even, i + 1]
    assert mxfp4.round_code(np.array([7.99]))[0] == 7


def test_scales():
    x = np.zeros((6, 33))
    x[0, 0] = 1.0        # 2^-2
    x[1, 3] = -7.99      # 2^0
    x[2, 31] = 2.0 ** -149
    x[3, 32] = 6.0       # the second block, 2^0
    x[4, 1] = np.inf
    x[5, 0] = 3.4e38     # 2^125
    _, s = mxfp4.quantize(x)
    assert s.tolist() == [[125, 127], [127, 127], [0, 127], [127, 127], [255, 127], [252, 127]]
    assert mxfp4.rounded(x)[1, 3] == -6.0 and np.all(np.isnan(mxfp4.rounded(x)[4, :32]))


def test_small_example_by_hand():
    # max 1.0: scale 1/4; 0.3 -> 1.2 -> 1.0 -> 0.25; -0.07 -> -0.28 -> -0.5 -> -0.125; 0.0625 -> 0.25 -> tie -> 0
    assert mxfp4.rounded(np.array([[1.0, 0.3, -0.07, 0.0625]])).tolist() == [[1.0, 0.25, -0.125, 0.0]]


def test_pack():
    codes, scales = mxfp4.quantize(np.array([[4.0, -6.0, 0.5]]))
    b, s = mxfp4.pack(codes, scales)
    assert b.shape == (1, 64) and b[0, 0] == 0x6 | 0xF << 4 and b[0, 1] == 0x1 and not b[0, 2:].any()
    assert s.shape == (1, 1, 4) and s[0, 0].tolist() == [127] * 4


def test_preference_of_equal_pairs_is_log_two():
    x = np.zeros((2, 5))
    losses, logps, g, w, _ = preference.preference(x, [1, 1], [0, 1, 2], [-0.5, -0.5], 0.3, 0.0, 1.0)
    assert losses[0] == pytest.approx(np.log(2)) and logps == pytest.approx([-np.log(5)] * 2)
    assert w == pytest.approx([-0.15, 0.15]) and g[0] == pytest.approx([0.03, -0.12, 0.03, 0.03, 0.03])


@pytest.mark.parametrize("smoothing", [0.0, 0.2, 1.0])
def test_preference_gradient_against_differences(smoothing):
    rng = np.random.default_rng(3)
    x = rng.normal(0, 2, (9, 7))
    labels = rng.integers(-1, 8, 9)
    off, ref = [0, 3, 3, 7, 9], rng.normal(0, 3, 4)
    args = (labels, off, ref, 0.4, smoothing, 0.5)
    _, _, g, _, _ = preference.preference(x, *args)
    h = 1e-5
    for r in range(9):
        for v in range(7):
            up, down = x.copy(), x.copy()
            up[r, v] += h
            down[r, v] -= h
            d = 0.5 * (preference.preference(up, *args)[0].sum() - preference.preference(down, *args)[0].sum()) / (2 * h)
            assert d == pytest.approx(g[r, v], abs=1e-8)


def test_clip_by_hand():
    (n, c, t), (n2, c2, t2) = preference.clip([[np.array([3.0]), np.array([[4.0]])], [np.array([0.1])]], 1.0)
    assert n == 5.0 and c == pytest.approx(0.2, rel=1e-6) and t[1][0, 0] == pytest.approx(0.8, rel=1e-6)
    assert n2 == pytest.approx(0.1) and c2 == 1.0 and t2[0][0] == 0.1
