"""Gradient of the windowed attention where a row sees a few keys (window and sinks 32 at most), against the fp64 oracle: what a bf16
gradient is made of there is what is left when Delta is taken off, so that scores other than the forward's would show.

The bar for d_k and d_v, in the 2-norm: a stored key and a turned query, rounded once each, move a score of N(0,1) data by 2.3e-3, the same in the
forward and here, so that of two keys a probability moves by 2.3e-3 of itself at most; Delta comes from a rounded output, 1.7e-3 of terms as
large as what is left; the probability's gradient and the query in the product are rounded once each, 1.7e-3: 4e-3 together, the bar is 5e-3
(keys rounded once more than in the forward give 5.1e-3)."""
import numpy as np
import pytest

from tests.test_gpu_window_backward import by_message, check, gradients, want
from tests.window_cases import Layer, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("h_q,h_kv", [(8, 2), (4, 4), (16, 1)])
def test_few_keys(h_q, h_kv):
    layer = Layer("bf16", [40, 70, 33, 500, 20, 300], h_q, h_kv, 128)
    layer.cache.reposition(1, 555)
    calls = [([(0, 0), (1, 40), (2, 110)], 3, 143, 500), ([(2, 7), (0, 30), (1, 60)], 4, 130, 20), ([(1, 0)], -1, 0, 3, [69, 5, 900]),
             ([(0, 0), (1, 40), (2, 110)], 5, 143, 300)]
    for window, n_sink in [(1, 1), (2, 0), (3, 29), (30, 2), (1, 0), (32, 0), (31, 2)]:
        check(layer, calls, window, n_sink)
    layer.cache.close()


def test_tiles_of_sinks_that_are_cut():
    """Rows enough for the sinks' tile to go in several parts, and several runs of tiles a block."""
    layer = Layer("bf16", [64, 2500], 4, 1, 128)
    for window, n_sink in [(1, 4), (20, 12)]:
        check(layer, [([(0, 0)], 1, 64, 2500)], window, n_sink)
    layer.cache.close()


@pytest.mark.parametrize("window,n_sink", [(2, 0), (1, 1), (3, 0), (1, 3)])
def test_the_scores_are_the_forwards(window, n_sink):
    layer = Layer("bf16", [300, 400], 8, 2, 128)
    calls = [([(0, 0)], 1, 300, 400)]
    q, d_out = layer.normal(400, 8, 128), layer.normal(400, 8, 128)
    _, d_k, d_v = gradients(layer, calls, window, n_sink, q, d_out)
    _, wk, wv = want(layer, calls, window, n_sink, q, d_out)
    for name, got, w in (("d_k", d_k, wk), ("d_v", d_v, wv)):
        got = np.concatenate(by_message(layer, got)[0])
        w = np.concatenate(w)
        err = np.linalg.norm(got - w) / np.linalg.norm(w)
        say(f"  w {window} s {n_sink}: {name} {err:.2e}")
        assert err <= 5e-3
    layer.cache.close()
