"""Gradient of the windowed attention where rows see one key: the probability is 1 whatever the score, so that d_q and d_k are 0, to the
last bit (dp and Delta are the same sum of the same numbers, made in the same order); d_v is the sum of the rows' output gradients."""
import numpy as np
import pytest

from tests.test_gpu_window_backward import gradients, want
from tests.window_cases import Layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 8, 2, 128), ("bf16", 5, 5, 128), ("bf16", 32, 2, 128), ("f32", 6, 2, 64), ("f32", 3, 1, 128), ("f32", 40, 2, 64)])
@pytest.mark.parametrize("n_q", [1, 33, 300])
def test_one_key(dtype, h_q, h_kv, D, n_q):
    layer = Layer(dtype, [40, 90, 20, n_q], h_q, h_kv, D)
    layer.cache.reposition(1, 333)
    calls = [([(0, 0), (1, 40)], 3, 130, n_q), ([(1, 0)], 3, 90, n_q), ([(2, 5)], -1, 0, 2, [24, 24])]
    q, d_out = layer.normal(layer.rows(calls), h_q, D), layer.normal(layer.rows(calls), h_q, D)
    d_q, d_k, d_v = gradients(layer, calls, 1, 0, q, d_out)
    assert not d_q.any() and not d_k.any()
    wv = np.concatenate(want(layer, calls, 1, 0, q, d_out)[2])
    got = np.concatenate([np.concatenate([d_v.double().cpu().numpy()[s:s + n] for s, n in layer.cache.message_extents(m, 64)]) for m in range(4)])
    assert np.linalg.norm(got - wv) <= {"f32": 4e-6, "bf16": 1.2e-2}[dtype] * np.linalg.norm(wv)
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 8, 2, 128), ("f32", 6, 2, 64)])
def test_the_first_row_of_more(dtype, h_q, h_kv, D):
    """A message alone: its first row sees itself; the others see more."""
    layer = Layer(dtype, [70], h_q, h_kv, D)
    calls = [([], 0, 0, 70)]
    for window, n_sink in [(20, 0), (500, 3)]:
        q, d_out = layer.normal(70, h_q, D), layer.normal(70, h_q, D)
        d_q = gradients(layer, calls, window, n_sink, q, d_out)[0]
        assert not d_q[0].any() and d_q[1:].any(dim=-1).all()
    layer.cache.close()
