"""The bars of the windowed gradient see mistakes: planted in the oracle's results, in the sizes the GPU tests use."""
import numpy as np
import pytest

from oracle import window_oracle as win
from tests.window_gradient_bars import BAR, LONG, LONG_LENS, LONG_SEL, in_pieces, worst

H_Q, H, D = 2, 1, 64


@pytest.mark.parametrize("n_q,window,n_sink", LONG)
def test_a_tile_that_is_lost_or_counted_twice_is_seen(n_q, window, n_sink):
    rng = np.random.default_rng(n_q)
    ks, vs = [[rng.standard_normal((n, H, D)) for n in LONG_LENS] for _ in range(2)]
    q, d_out = rng.standard_normal((n_q, H_Q, D)), rng.standard_normal((n_q, H_Q, D))

    def grad(rows, d_o, some_vs=None):
        """of the rows [rows[0], rows[1]) alone"""
        keep = np.zeros(n_q, bool)
        keep[rows[0]:rows[1]] = True
        return win.attend_call_window_backward(ks, some_vs or vs, LONG_SEL, 4, 2650, n_q, None, q, d_o * keep[:, None, None], 10000.0, window, n_sink)
    want = grad((0, n_q), d_out)
    assert worst(want, want, [n_q])[0] == 0.0
    zero = [np.zeros_like(x) for x in want[2]]
    assert worst((want[0], want[1], zero), want, [n_q])[0] == 1.0                    # no d_v at all
    # half of the rows that a tile of keys collects from: lost, or taken twice
    part = grad((0, max(1, n_q // 2)), d_out)
    for sign in (-1, 1):
        for which in (1, 2):
            got = [want[0], list(want[1]), list(want[2])]
            got[which][4] = want[which][4] + sign * part[which][4]
            assert worst(got, want, [n_q])[0] > 10 * BAR["bf16"]
    # a tile of 32 keys that a row's split leaves out: d_q without what those keys bring
    pos = np.concatenate([650 * m + np.arange(700) for m in range(4)] + [2650 + np.arange(900)])
    k, v = np.concatenate(ks), np.concatenate(vs)
    at = int(np.nonzero(pos > 2650 + 899 - window)[0][64])
    from oracle.choreo_oracle import rope
    p_rows = 2650 + 900 - n_q + np.arange(n_q)
    kr, qr = rope(k, pos, 10000.0), rope(q, p_rows, 10000.0)
    last = 2800 + 900 - n_q + np.arange(n_q)
    vis = win.visible(pos, p_rows, last, window, n_sink)
    lost = np.zeros_like(q)
    for h in range(H_Q):
        p, _ = win._probabilities(qr[:, h], kr[:, 0], vis, 1 / np.sqrt(D))
        d_p = d_out[:, h] @ v[:, 0].T
        d_s = p * (d_p - (p * d_p).sum(axis=1, keepdims=True)) / np.sqrt(D)
        lost[:, h] = d_s[:, at:at + 32] @ kr[at:at + 32, 0]
    lost = rope(lost, -p_rows, 10000.0)
    assert worst((want[0] - lost, want[1], want[2]), want, [n_q])[0] > 2 * BAR["bf16"]


def test_the_oracle_in_pieces_is_the_oracle():
    rng = np.random.default_rng(1)
    lens = [40, 300]
    ks, vs = [[rng.standard_normal((n, H, D)) for n in lens] for _ in range(2)]
    q, d_out = rng.standard_normal((300, H_Q, D)), rng.standard_normal((300, H_Q, D))
    for window, n_sink in [(50, 20), (7, 0), (1, 3)]:
        a = in_pieces(ks, vs, 1, 0, 0, 40, q, d_out, 10000.0, window, n_sink, 32)
        b = win.attend_call_window_backward(ks, vs, [(0, 0)], 1, 40, 300, None, q, d_out, 10000.0, window, n_sink)
        for x, y in zip([a[0], *a[1], *a[2]], [b[0], *b[1], *b[2]]):
            assert np.abs(x - y).max() <= 1e-12 * max(1.0, np.abs(y).max())
