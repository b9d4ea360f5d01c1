"""pc_attend_window_backward on long walks, on tiles that many rows see and in batches of several runs, place by place against the
fp64 oracle (bars and where they come from: window_gradient_bars.py; that they see mistakes: test_window_gradient_bars.py)."""
import numpy as np
import pytest

from tests.test_gpu_window_backward import by_message, gradients, want
from tests.window_cases import Layer, say
from tests.window_gradient_bars import BAR, LONG, LONG_LENS, LONG_SEL, in_pieces, worst

pytestmark = pytest.mark.gpu


def check(layer, got, ref, n_qs, what=""):
    got = (got[0].double().cpu().numpy(), by_message(layer, got[1])[0], by_message(layer, got[2])[0])
    err, where = worst(got, ref, n_qs)
    say(f"  {what} {layer.dtype}: {err:.2e} at {where}")
    assert err <= BAR[layer.dtype], where
    return got


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 4, 1, 128), ("bf16", 8, 2, 128), ("bf16", 3, 3, 128), ("f32", 2, 1, 64), ("f32", 6, 2, 128)])
def test_long_walks_and_tiles_that_every_row_sees(dtype, h_q, h_kv, D):
    layer = Layer(dtype, LONG_LENS, h_q, h_kv, D)
    for n_q, window, n_sink in LONG + [(33, 1 << 30, 0), (1, 1 << 30, 0)]:
        calls = [(LONG_SEL, 4, 2650, n_q)]
        q, d_out = layer.normal(n_q, h_q, D), layer.normal(n_q, h_q, D)
        check(layer, gradients(layer, calls, window, n_sink, q, d_out), want(layer, calls, window, n_sink, q, d_out), [n_q], f"n_q {n_q} w {window} s {n_sink}")
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 8, 2, 128), ("f32", 6, 2, 64)])
def test_many_calls_over_the_same_messages(dtype, h_q, h_kv, D):
    """Tiles that forty calls list are cut into parts; some calls list a message twice at one place."""
    layer = Layer(dtype, [300, 33, 500] + [40] * 10, h_q, h_kv, D)
    calls = [([(0, 0), (1, 300), (2, 333)] + ([(1, 300)] if i % 4 == 0 else []), 3 + i % 10, 833, 1 + 13 * (i % 4)) for i in range(40)]
    n_qs = [c[3] for c in calls]
    for window, n_sink in [(1 << 30, 0), (400, 70)]:
        q, d_out = layer.normal(sum(n_qs), h_q, D), layer.normal(sum(n_qs), h_q, D)
        check(layer, gradients(layer, calls, window, n_sink, q, d_out), want(layer, calls, window, n_sink, q, d_out), n_qs, f"w {window} s {n_sink}")
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,n_q,window,n_sink", [("bf16", 64, 4, 9000, 50, 20), ("bf16", 64, 4, 4500, 20, 12), ("f32", 24, 1, 11000, 50, 20)])
def test_batches_that_go_in_several_runs(dtype, h_q, h_kv, n_q, window, n_sink):
    """Blocks for more than the 256 MB of workspace that a run takes (a quarter as many where rows see few keys): every row's gradient and
    every key's, over the runs' borders, the sinks that all of the runs add to among them."""
    D = 128
    layer = Layer(dtype, [64, n_q, 200], h_q, h_kv, D)
    calls = [([(0, 0)], 2, 64, 70), ([(0, 0)], 1, 64, n_q), ([(0, 5)], 2, 64, 200)]
    few = 4 if dtype == "bf16" and window + n_sink <= 32 else 1
    assert (n_q + 270) / 32 * h_q * (17 * 1024 if dtype == "bf16" else 33 * 1024) * few > 256 << 20
    q, d_out = layer.normal(n_q + 270, h_q, D), layer.normal(n_q + 270, h_q, D)
    got = gradients(layer, calls, window, n_sink, q, d_out)
    ref_q, ref_k, ref_v = in_pieces(layer.ks, layer.vs, 1, 0, 0, 64, q[70:70 + n_q], d_out[70:70 + n_q], layer.theta, window, n_sink)
    rest = np.concatenate([np.arange(70), np.arange(70 + n_q, n_q + 270)])
    a, b, e = want(layer, [calls[0], calls[2]], window, n_sink, q[rest], d_out[rest])
    ref = (np.concatenate([a[:70], ref_q, a[70:]]), [ref_k[0] + b[0], ref_k[1], b[2]], [ref_v[0] + e[0], ref_v[1], e[2]])
    got = check(layer, got, ref, [70, n_q, 200], f"w {window} s {n_sink}")
    if few > 1:                                          # (the forward's own scores: see test_gpu_window_backward_few.py)
        for i in (1, 2):
            err = np.linalg.norm(got[i][1] - ref[i][1]) / np.linalg.norm(ref[i][1])
            say(f"  {err:.2e}")
            assert err <= 5e-3
    layer.cache.close()
