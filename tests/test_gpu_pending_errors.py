"""An error that the program's earlier work left with the runtime (a device that there is none of, say) is not the next call's: forks, the cache
closing up and the windowed attention succeed, and what the host knows is what the device holds."""
import numpy as np
import pytest

from tests.test_gpu_fork_and_compact import Store
from tests.window_cases import Layer, compare

pytestmark = pytest.mark.gpu


def leave_an_error():
    """The runtime's last error, of a call that did nothing."""
    from paper_2512_23049_amd.binding import lib
    assert lib().hipSetDevice(4096) != 0
    assert lib().hipPeekAtLastError() != 0


def no_error():
    from paper_2512_23049_amd.binding import lib
    return lib().hipPeekAtLastError() == 0


@pytest.mark.parametrize("dtype,h_kv,D", [("bf16", 3, 128), ("f32", 2, 64)])
@pytest.mark.parametrize("n", [12, 400])
@pytest.mark.parametrize("profile", [False, True])
def test_closing_up_three_times(dtype, h_kv, D, n, profile):
    """Short lists (in the launch's arguments) and long ones (staged); each closing up goes by what the one before it counted."""
    s = Store(dtype, h_kv, D, 64 * n + 4096)
    s.cache.profile_enable(profile)
    ids = [s.put(20 + i % 40, i) for i in range(n)]
    stores = s.read()
    kept = {m: s.message(m, stores) for m in ids}
    for step in range(3):
        for m in ids[step::4]:
            s.cache.message_free(m)
            kept.pop(m)
        leave_an_error()
        moved = s.cache.compact()
        assert moved > 0 and no_error()
        stores = s.read()
        at = 0
        for m in kept:
            length, slot, _ = s.cache.message_info(m)
            assert slot == at
            at += (length + 31) // 32 * 32
            assert s.same(s.message(m, stores), kept[m])
    s.cache.close()


@pytest.mark.parametrize("dtype,h_kv,D", [("bf16", 3, 128), ("f32", 2, 64)])
@pytest.mark.parametrize("n", [3, 300])
def test_forks(dtype, h_kv, D, n):
    s = Store(dtype, h_kv, D, 64 * n + 4096)
    m = s.put(50, 1)
    leave_an_error()
    ids = s.cache.message_fork([(m, i % 40, 10, 0, None) for i in range(n)])
    assert no_error() and ids == list(range(1, n + 1))
    stores = s.read()
    k, v = s.message(m, stores)
    for i, f in enumerate(ids):
        assert s.same(s.message(f, stores), (k[:, i % 40:i % 40 + 10].contiguous(), v[:, i % 40:i % 40 + 10].contiguous()))
    s.cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_windowed_attention_and_its_gradient(dtype):
    import torch
    layer = Layer(dtype, [100, 70, 40], 8, 2, 128)
    for n_calls, n_q in [(1, 1), (90, 1), (2, 40)]:      # lists in the launch's arguments, and staged ones
        calls = [([(0, 0), (1, 100)], 2, 170, n_q)] * n_calls
        rows = layer.rows(calls)
        q, d_out = layer.normal(rows, 8, 128), layer.normal(rows, 8, 128)
        for static in (False, True):
            tq, out, lse = layer.dev(q), torch.empty(q.shape, device="cuda:0", dtype=layer.kind), torch.empty(q.shape[:2], device="cuda:0")
            torch.cuda.synchronize()
            leave_an_error()
            (layer.cache.attend_window_static if static else layer.cache.attend_window)(layer.calls(calls), 90, 5, tq.data_ptr(), out.data_ptr(), lse.data_ptr())
            assert no_error()
            torch.cuda.synchronize()
            compare(dtype, out, lse, *layer.want(calls, 90, 5, q), f"{n_calls} calls of {n_q}")
        d, got = layer.dev(d_out), []
        for pending in (False, True):
            d_q, d_k, d_v = torch.zeros(q.shape, device="cuda:0"), *(torch.zeros(layer.cache.cache_info()[2], 2, 128, device="cuda:0") for _ in range(2))
            torch.cuda.synchronize()
            if pending:
                leave_an_error()
            layer.cache.attend_window_backward(layer.calls(calls), 90, 5, tq.data_ptr(), out.data_ptr(), lse.data_ptr(), d.data_ptr(), d_q.data_ptr(), d_k.data_ptr(), d_v.data_ptr())
            assert no_error()
            torch.cuda.synchronize()
            got.append((d_q, d_k, d_v))
        assert all(torch.equal(x, y) and np.isfinite(x.cpu().numpy()).all() for x, y in zip(*got))
    layer.cache.close()
