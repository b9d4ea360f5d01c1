"""Pins of the windowed oracle (CPU)."""
import numpy as np
import pytest

from oracle import choreo_oracle as orc
from oracle import window_oracle as win

THETA = 10000.0


def data(seed, lens, n_q, h_q=4, h_kv=2, D=8):
    r = np.random.default_rng(seed)
    ks = [r.standard_normal((n, h_kv, D)) for n in lens]
    vs = [r.standard_normal((n, h_kv, D)) for n in lens]
    return ks, vs, r.standard_normal((n_q, h_q, D)), r.standard_normal((n_q, h_q, D))


CALL = ([(0, 3), (2, 40), (1, 20), (0, 90)], 3, 100, 5)


def test_a_window_over_everything_is_the_plain_attention():
    ks, vs, q, d_o = data(1, [7, 12, 5, 6], 5)
    sel, me, start, n_q = CALL
    a = win.attend_call_window(ks, vs, sel, me, start, n_q, None, q, THETA, 1 << 30, 0)
    b = orc.attend_call(ks, vs, sel, me, start, n_q, None, q, THETA)
    np.testing.assert_allclose(a[0], b[0], atol=1e-13)
    np.testing.assert_allclose(a[1], b[1], atol=1e-13)
    ga = win.attend_call_window_backward(ks, vs, sel, me, start, n_q, None, q, d_o, THETA, 1 << 30, 0)
    gb = orc.attend_call_backward(ks, vs, sel, me, start, n_q, None, q, d_o, THETA)
    np.testing.assert_allclose(ga[0], gb[0], atol=1e-12)
    for x, y in zip(ga[1] + ga[2], gb[1] + gb[2]):
        np.testing.assert_allclose(x, y, atol=1e-12)


def test_a_window_of_one_is_the_own_value():
    ks, vs, q, _ = data(2, [6], 6)
    out, lse = win.attend_call_window(ks, vs, [], 0, 10, 6, None, q, THETA, 1, 0)
    np.testing.assert_allclose(out, np.repeat(vs[0], 2, axis=1), atol=1e-14)
    np.testing.assert_allclose(lse, np.einsum("nhd,nhd->nh", q, np.repeat(ks[0], 2, axis=1)) / np.sqrt(8), atol=1e-12)


def test_the_mask_by_hand():
    # a parent of three tokens at 0, one of two at 10, own three at 5 (an overlap in positions is no matter)
    pos = np.array([0, 1, 2, 10, 11, 5, 6, 7])
    vis = win.visible(pos, np.array([5, 6, 7]), np.array([5, 6, 7]), 5, 1)
    want = np.array([[1, 1, 1, 1, 1, 1, 0, 0],           # 5: above 0; the first token is a sink
                     [1, 0, 1, 1, 1, 1, 1, 0],
                     [1, 0, 0, 1, 1, 1, 1, 1]], dtype=bool)
    assert np.array_equal(vis, want)


def test_rows_that_see_nothing():
    ks, vs, q, d_o = data(3, [4], 3)
    out, lse = win.attend_call_window(ks, vs, [(0, 0)], -1, 0, 3, np.array([3, 50, 4]), q, THETA, 2, 0)
    assert (out[1] == 0).all() and (lse[1] == -np.inf).all() and np.isfinite(lse[[0, 2]]).all()
    d_q, _, _ = win.attend_call_window_backward(ks, vs, [(0, 0)], -1, 0, 3, np.array([3, 50, 4]), q, d_o, THETA, 2, 0)
    assert (d_q[1] == 0).all()


@pytest.mark.parametrize("window,n_sink", [(1, 0), (4, 2), (30, 9), (1000, 0)])
def test_gradient_by_central_differences(window, n_sink):
    ks, vs, q, d_o = data(4, [7, 12, 5, 6], 5)
    sel, me, start, n_q = CALL

    def value():
        return (win.attend_call_window(ks, vs, sel, me, start, n_q, None, q, THETA, window, n_sink)[0] * d_o).sum()
    d_q, d_k, d_v = win.attend_call_window_backward(ks, vs, sel, me, start, n_q, None, q, d_o, THETA, window, n_sink)
    r = np.random.default_rng(5)
    for x, g in [(q, d_q)] + list(zip(ks, d_k)) + list(zip(vs, d_v)):
        for _ in range(6):
            at = tuple(int(r.integers(0, n)) for n in x.shape)
            keep, e = x[at], 1e-5
            x[at] = keep + e
            up = value()
            x[at] = keep - e
            down = value()
            x[at] = keep
            assert abs((up - down) / (2 * e) - g[at]) < 1e-7
