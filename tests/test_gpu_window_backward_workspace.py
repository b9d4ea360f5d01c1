"""The workspace of pc_attend_window_backward: batches longer than a run holds go in runs of about 256 MB, whatever the length of the calls that
they are a part of; what the cache then holds is a quarter more at most (pc_ensure_ws), and the tables of keys' parts."""
import numpy as np
import pytest

from tests.test_gpu_window_backward import BARS
from tests.window_cases import Layer, say

pytestmark = pytest.mark.gpu
MB = 1 << 20


def taken(layer, calls, window, n_sink, q, d_out):
    """The gradient of the calls, and the device memory that it made the cache take."""
    import torch
    out, lse = layer.attend(calls, window, n_sink, q)
    tq, td = layer.dev(q), layer.dev(d_out)
    d_q = torch.full(q.shape, 9.0, device="cuda:0")
    d_k, d_v = (torch.zeros(layer.cache.cache_info()[2], layer.h_kv, layer.D, device="cuda:0") for _ in range(2))
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    layer.cache.attend_window_backward(layer.calls(calls), window, n_sink, tq.data_ptr(), out.data_ptr(), lse.data_ptr(), td.data_ptr(), d_q.data_ptr(),
                                       d_k.data_ptr(), d_v.data_ptr())
    torch.cuda.synchronize()
    return d_q, before - torch.cuda.mem_get_info()[0]


# (rows, window): the last run has 8 blocks of a call of 31 thousand rows, whose walks of 130 tiles are split; the same in fp32
@pytest.mark.parametrize("dtype,h_q,h_kv,n_q", [("bf16", 16, 2, 30976), ("f32", 16, 2, 32064)])
def test_a_run_of_a_few_rows_of_a_long_call(dtype, h_q, h_kv, n_q):
    from oracle import window_oracle as win
    window = 4096
    layer = Layer(dtype, [n_q], h_q, h_kv, 128)
    q, d_out = layer.normal(n_q, h_q, 128), layer.normal(n_q, h_q, 128)
    d_q, extra = taken(layer, [([], 0, 0, n_q)], window, 0, q, d_out)
    say(f"  {dtype}: {extra / MB:.0f} MB")
    assert extra <= 512 * MB
    for r0 in (12345, n_q - 300, n_q - 40):              # (of each run, against the oracle over the keys the rows see)
        rows = slice(r0, r0 + 40)
        k, v = layer.ks[0][r0 - window:r0 + 40], layer.vs[0][r0 - window:r0 + 40]
        a, _, _ = win.attend_call_window_backward([k], [v], [], 0, r0 - window, 40, None, q[rows], d_out[rows], layer.theta, window, 0)
        got = d_q[rows].double().cpu().numpy()
        err = np.linalg.norm(got - a) / np.linalg.norm(a)
        say(f"  rows {r0}: {err:.2e}")
        assert err <= BARS[dtype][0]
    layer.cache.close()


@pytest.mark.parametrize("window", [20, 40])
def test_rotations_are_those_of_a_runs_rows(window):
    """One head, half a million rows: a row's rotations are more memory than its share of a block."""
    n_q = 520000
    layer = Layer("bf16", [64], 1, 1, 128)
    calls = [([(0, 0)], -1, 0, n_q, [40 + i % 24 for i in range(n_q)])]
    q = layer.normal(n_q, 1, 128)
    d_q, extra = taken(layer, calls, window, 2, q, q)
    say(f"  {extra / MB:.0f} MB")
    assert extra <= 400 * MB
    from oracle import window_oracle as win
    for r0 in (0, 255000, n_q - 40):
        rows = slice(r0, r0 + 40)
        a, _, _ = win.attend_call_window_backward(layer.ks, layer.vs, [(0, 0)], -1, 0, 40, calls[0][4][rows], q[rows], q[rows], layer.theta, window, 2)
        err = np.linalg.norm(d_q[rows].double().cpu().numpy() - a) / np.linalg.norm(a)
        say(f"  rows {r0}: {err:.2e}")
        assert err <= BARS["bf16"][0]
    layer.cache.close()
