"""The oracle of norms and of the 4-bit form, against what it is by definition."""
import numpy as np
import pytest

from oracle import project_oracle as po


def test_norm_is_its_definition():
    x = np.array([[[3.0, 4.0, 0.0, 0.0]]])
    assert np.allclose(po.norm(x, None, 0.0), x / 2.5)
    assert np.allclose(po.norm(x, [1, 2, 3, 4], 0.0), [[[1.2, 3.2, 0, 0]]])
    assert np.allclose(po.norm(np.zeros((1, 1, 4)), None, 1e-6), 0)


@pytest.mark.parametrize("weighted", [False, True])
def test_norm_gradient_by_differences(weighted):
    rng = np.random.default_rng(0)
    x, dy = rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 2, 8))
    w = 1 + 0.3 * rng.standard_normal(8) if weighted else None
    dx, dw = po.norm_backward(x, w, 1e-3, dy)
    h = 1e-5                                             # (the error of a central difference: h^2 times a third derivative of order one)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        assert abs(((po.norm(up, w, 1e-3) - po.norm(down, w, 1e-3)) * dy).sum() / (2 * h) - dx[i]) < 1e-7
    base = np.ones(8) if w is None else w
    for i in range(8):
        e = np.eye(8)[i] * h
        assert abs(((po.norm(x, base + e, 1e-3) - po.norm(x, base - e, 1e-3)) * dy).sum() / (2 * h) - dw[i]) < 1e-7


def test_four_bits_by_search():
    """The nearest of all values that there are, under the least power that holds the block below seven."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 128)) * 10.0 ** rng.integers(-12, 12, (50, 1))
    x[:5] = np.round(x[:5] * 4) / 4                      # with ties
    got = po.to_mx4(x).reshape(50, 4, 32)
    b = x.reshape(50, 4, 32)
    for r in range(50):
        for k in range(4):
            e = min(e for e in range(-60, 61) if np.abs(b[r, k]).max() < 7 * 2.0 ** e)
            values = np.concatenate([po.GRID, -po.GRID]) * 2.0 ** e
            assert (np.abs(got[r, k] - b[r, k]) == np.abs(values[:, None] - b[r, k]).min(axis=0)).all()


def test_four_bits_edges():
    one = np.zeros(32)
    for top, want in ((6.9, 6), (7.0, 8), (5.0, 4), (2.5, 2), (3.5, 4), (0.25, 0.25), (0.0, 0)):
        one[0] = top
        assert po.to_mx4(one)[0] == want, top            # (7: the power doubles, and 3.5 of it is a tie that goes to 4)
    one[0], one[1], one[2], one[3] = 6, 0.25, 0.75, 1.25
    assert list(po.to_mx4(one)[:4]) == [6, 0, 1, 1]
    one[:4] = -6, -1.75, -2.5, -5
    assert list(po.to_mx4(one)[:4]) == [-6, -2, -2, -4]
    one[:4] = 1e30, 0, 0, 0
    assert po.to_mx4(one)[0] == 6 * 2.0 ** 60
    one[:4] = 1e-30, 0, 0, 0
    assert po.to_mx4(one)[0] == 0
