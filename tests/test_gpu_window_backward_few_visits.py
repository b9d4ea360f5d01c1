"""Gradient under a window and sinks of 32 at most where blocks of rows see more extents than queries are turned for (eight tiles of keys a
block in the mean): keys are turned then, with one more rounding, and what holds is the bar of the gradient in general (1.2e-2; see
test_gpu_window_backward.py), not the 5e-3 of the forward's own scores.  Rows of a message without parents see few keys under any window."""
import numpy as np
import pytest

from tests.test_gpu_window_backward import by_message, gradients, want
from tests.window_cases import Layer, say
from tests.window_gradient_bars import BAR, worst

pytestmark = pytest.mark.gpu


def check(layer, calls, window, n_sink, what):
    n_qs = [c[3] for c in calls]
    q, d_out = layer.normal(sum(n_qs), layer.h_q, 128), layer.normal(sum(n_qs), layer.h_q, 128)
    got, ref = gradients(layer, calls, window, n_sink, q, d_out), want(layer, calls, window, n_sink, q, d_out)
    got = (got[0].double().cpu().numpy(), by_message(layer, got[1])[0], by_message(layer, got[2])[0])
    err, where = worst(got, ref, n_qs)
    say(f"  {what} w {window} s {n_sink}: {err:.2e} at {where}")
    assert err <= BAR["bf16"]


@pytest.mark.parametrize("h_q,h_kv", [(8, 2), (4, 4)])
def test_more_extents_than_queries_are_turned_for(h_q, h_kv):
    layer = Layer("bf16", [60] * 12 + [2] * 12 + [20, 90], h_q, h_kv, 128)
    overlapping = [(m, 3 * m) for m in range(12)]
    short = [(12 + m, 40 + 2 * m) for m in range(12)]
    for name, sel, own, at, n_q in [("overlapping", overlapping, 24, 70, 20), ("short", short, 24, 64, 20), ("short", short, 25, 64, 1), ("both", overlapping + short, 25, 80, 60)]:
        for window, n_sink in [(30, 2), (32, 0), (20, 12)]:
            check(layer, [(sel, own, at, n_q)], window, n_sink, f"{name} {n_q}")
    layer.cache.close()


@pytest.mark.parametrize("window,n_sink", [(1 << 30, 0), (200, 4)])
def test_the_first_rows_of_a_message_without_parents(window, n_sink):
    layer = Layer("bf16", [300], 8, 2, 128)
    check(layer, [([], 0, 0, 300)], window, n_sink, "no parents")
    layer.cache.close()
