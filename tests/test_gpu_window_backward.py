"""pc_attend_window_backward against the fp64 oracle and against differences of pc_attend_window.

Bars, in the 2-norm of each gradient.  fp32: about ten roundings of 2^-24 a term, 6e-7, and as much again through the forward's
log-sum-exp and Delta: the bar is 4e-6.  bf16 (a rounding is 1.6e-3 in the mean square): a stored key, a turned key and a turned
query move a score of N(0,1) data by 2.8e-3, the probability and its gradient are rounded once each, and Delta comes from an output
that was rounded: 4e-3 together; the bar is 1.2e-2.  A single element: 5e-2 of the largest.  Where a gradient is zero by cancellation (one visible
key) what is left are those errors of terms of order one: 3e-3 an element in bf16, 1e-5 in fp32."""
import numpy as np
import pytest

from tests.window_cases import Layer, say

pytestmark = pytest.mark.gpu
BARS = {"f32": (4e-6, 1e-5), "bf16": (1.2e-2, 3e-3)}


def gradients(layer, calls, window, n_sink, q, d_out, stream=0, into=None, finalize=True):
    import torch
    out, lse = layer.attend(calls, window, n_sink, q, stream=stream)
    tq, td = layer.dev(q), layer.dev(d_out)
    slots = layer.cache.cache_info()[2]
    d_q = torch.full(q.shape, 9.0, device="cuda:0")
    d_k, d_v = into or (torch.zeros(slots, layer.h_kv, layer.D, device="cuda:0") for _ in range(2))
    layer.cache.attend_window_backward(layer.calls(calls), window, n_sink, tq.data_ptr(), out.data_ptr(), lse.data_ptr(), td.data_ptr(), d_q.data_ptr(),
                                       d_k.data_ptr(), d_v.data_ptr(), stream)
    if finalize:
        layer.cache.grad_keys_finalize(d_k.data_ptr(), stream)
    torch.cuda.synchronize()
    return d_q, d_k, d_v


def want(layer, calls, window, n_sink, q, d_out):
    from oracle import window_oracle as win
    at, dq = 0, []
    dk, dv = [np.zeros(np.shape(k)) for k in layer.ks], [np.zeros(np.shape(k)) for k in layer.ks]
    for c in calls:
        a, b, e = win.attend_call_window_backward(layer.ks, layer.vs, c[0], c[1], c[2], c[3], c[4] if len(c) > 4 else None, q[at:at + c[3]], d_out[at:at + c[3]],
                                                  layer.theta, window, n_sink)
        dq.append(a)
        for m in range(len(dk)):
            dk[m] += b[m]
            dv[m] += e[m]
        at += c[3]
    return np.concatenate(dq), dk, dv


def by_message(layer, x):
    x = x.double().cpu().numpy()
    return [np.concatenate([x[s:s + n] for s, n in layer.cache.message_extents(m, 64)]) for m in range(len(layer.ks))], x


def check(layer, calls, window, n_sink, what=""):
    q, d_out = layer.normal(layer.rows(calls), layer.h_q, layer.D), layer.normal(layer.rows(calls), layer.h_q, layer.D)
    d_q, d_k, d_v = gradients(layer, calls, window, n_sink, q, d_out)
    wq, wk, wv = want(layer, calls, window, n_sink, q, d_out)
    norm, floor = BARS[layer.dtype]
    (gk, rest_k), (gv, rest_v) = by_message(layer, d_k), by_message(layer, d_v)
    used = np.zeros(rest_k.shape[0], bool)
    for m in range(len(layer.ks)):
        for s, n in layer.cache.message_extents(m, 64):
            used[s:s + n] = True
    assert (rest_k[~used] == 0).all() and (rest_v[~used] == 0).all()
    for name, got, ref in [("d_q", d_q.double().cpu().numpy(), wq), ("d_k", np.concatenate(gk), np.concatenate(wk)), ("d_v", np.concatenate(gv), np.concatenate(wv))]:
        assert np.isfinite(got).all()
        size = np.linalg.norm(ref)
        err, far = np.linalg.norm(got - ref), np.abs(got - ref).max()
        say(f"  {what} w {window} s {n_sink} {name}: {err / max(size, 1e-30):.2e} of {size:.3g}, max {far:.2e} of {np.abs(ref).max():.3g}")
        assert err <= norm * size + floor * np.sqrt(np.count_nonzero(np.abs(got) + np.abs(ref))), name
        assert far <= 5e-2 * np.abs(ref).max() + 10 * floor, name


LENS = [31, 1, 64, 33, 100, 90]
SEL = [(0, 0), (4, 40), (1, 7), (2, 300), (0, 500), (3, 140)]


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 4, 4, 128), ("bf16", 8, 2, 128), ("bf16", 6, 2, 128), ("bf16", 5, 1, 128), ("bf16", 16, 1, 128),
                                              ("f32", 4, 2, 64), ("f32", 3, 1, 128), ("f32", 40, 2, 64), ("f32", 8, 2, 128)])
@pytest.mark.parametrize("n_q", [1, 33, 90])
def test_windows_and_sinks(dtype, h_q, h_kv, D, n_q):
    layer = Layer(dtype, LENS, h_q, h_kv, D)
    for window, n_sink in [(1, 0), (2, 1), (33, 32), (100, 40), (1 << 30, 0), (5, 1 << 30)]:
        check(layer, [(SEL, 5, 600, n_q)], window, n_sink)
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 8, 2, 128), ("bf16", 3, 3, 128), ("f32", 6, 2, 64), ("f32", 4, 1, 128)])
def test_batches(dtype, h_q, h_kv, D):
    """Calls that share messages, list one twice, list their new message as a parent too, see nothing, have no new message."""
    lens = [int(x) for x in np.random.default_rng(3).integers(20, 300, size=12)] + [20, 70, 150]
    layer = Layer(dtype, lens, h_q, h_kv, D)
    long = [(m, 300 * m) for m in range(12)]
    calls = [(long, 14, 3700, 1), (long[::-1], 13, 100, 70), ([(0, 5)], -1, 0, 3, [900, 5, 700]), ([], 12, 0, 20), ([(0, -5000)], -1, 9000, 1),
             ([(3, 50), (3, 50), (13, 10)], 13, 80, 40), (long[:3], -1, 0, 5, [-40, 3, 3, 10 ** 6, 90]), ([], -1, 7, 2), (long, 14, 3650, 150), (long[4:], 13, 2000, 33)]
    for window, n_sink in [(50, 0), (333, 7), (4000, 500)]:
        check(layer, calls, window, n_sink)
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 4, 1, 128), ("f32", 2, 1, 64)])
def test_long_walks_and_tiles_that_every_row_sees(dtype, h_q, h_kv, D):
    """Rows' walks are split, and so are the units of tiles with sinks."""
    lens = [700] * 4 + [900]
    layer = Layer(dtype, lens, h_q, h_kv, D)
    sel = [(m, 650 * m) for m in range(4)]
    for n_q, window, n_sink in [(1, 2500, 40), (20, 3000, 0), (900, 200, 150)]:
        check(layer, [(sel, 4, 2650, n_q)], window, n_sink, f"n_q {n_q}")
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 8, 2, 128), ("f32", 6, 2, 64)])
def test_moved_messages_and_extents(dtype, h_q, h_kv, D):
    import torch
    from paper_2512_23049_amd.binding import PC_FLAG_GROW_EXTENTS
    layer = Layer(dtype, [40, 70, 33, 20], h_q, h_kv, D, flags=PC_FLAG_GROW_EXTENTS, room=2000)
    layer.cache.reposition(0, 1000)
    layer.cache.reposition(1, -77)
    for n in (50, 45):
        k, v = layer.normal(n, h_kv, D), layer.normal(n, h_kv, D)
        tk, tv = layer.dev(k), layer.dev(v)
        layer.cache.append_tokens(3, tk.data_ptr(), tv.data_ptr(), n)
        torch.cuda.synchronize()
        layer.ks[3], layer.vs[3] = np.concatenate([layer.ks[3], k]), np.concatenate([layer.vs[3], v])
    assert len(layer.cache.message_extents(3)) > 1
    for n_q in (1, 12):
        for window, n_sink in [(60, 3), (150, 45)]:
            check(layer, [([(0, 0), (2, 40), (3, 100), (1, 77)], 3, 300, n_q), ([(1, 5), (0, 3)], 2, 60, n_q)], window, n_sink)
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 8, 2, 128), ("f32", 6, 2, 64), ("f32", 2, 1, 128)])
def test_what_is_not_finite_stays_with_the_rows_that_see_it(dtype, h_q, h_kv, D):
    """Keys and values that some rows do not see, infinite or no numbers: those rows' gradients, and those of the keys that only
    they see, are what they are without."""
    bad = [np.inf, -np.inf, np.nan]

    def spoil(ks, vs):
        for i, t in enumerate((0, 3, 64, 70)):
            vs[0][t, :, i::7] = bad[i % 3]
            ks[0][t, 0, 5 + i] = bad[i % 3]
        ks[1][66, 0, 9], vs[1][67, 0, 9] = np.nan, np.inf                      # own tokens of the last rows
    spoiled, clean = Layer(dtype, [100, 70], h_q, h_kv, D, spoil=spoil), Layer(dtype, [100, 70], h_q, h_kv, D)
    calls, window = [([(0, 0)], 1, 100, 70)], 30                              # own token t: positions 71 + t .. 100 + t
    q, d_out = clean.normal(70, h_q, D), clean.normal(70, h_q, D)
    a, b = gradients(spoiled, calls, window, 0, q, d_out), gradients(clean, calls, window, 0, q, d_out)
    rows = slice(0, 66)                                                      # (position 70 is out of every row's window)
    x, y = a[0][rows].double().cpu().numpy(), b[0][rows].double().cpu().numpy()
    assert np.isfinite(x).all() and np.array_equal(x, y)
    # keys that no row with such a token in its window sees: tokens 71.. of the parent, own tokens up to 65 - 29
    for u, v in zip(a[1:], b[1:]):
        u, v = u.double().cpu().numpy(), v.double().cpu().numpy()
        own = spoiled.cache.message_info(1)[1]
        keys = np.concatenate([np.arange(71, 100), own + np.arange(0, 36)])
        assert np.isfinite(u[keys]).all() and np.array_equal(u[keys], v[keys])
        assert (u[:71] == 0).all()                                           # nobody sees them
    spoiled.cache.close()
    clean.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 8, 2, 128), ("f32", 6, 2, 64)])
def test_the_same_calls_give_the_same_bits_and_collect(dtype, h_q, h_kv, D):
    import torch
    lens = [300, 200, 250, 400]
    layer = Layer(dtype, lens, h_q, h_kv, D)
    calls = [([(0, 0), (1, 300)], 3, 500, 400), ([(1, 0), (0, 200)], 2, 500, 250)]
    q, d_out = layer.normal(650, h_q, D), layer.normal(650, h_q, D)
    first = gradients(layer, calls, 120, 50, q, d_out, finalize=False)
    for _ in range(4):
        again = gradients(layer, calls, 120, 50, q, d_out, finalize=False)
        assert all(torch.equal(x, y) for x, y in zip(first, again))
    base = [torch.randn_like(first[1]) for _ in range(2)]
    kept = [x.clone() for x in base]
    gradients(layer, calls, 120, 50, q, d_out, into=base, finalize=False)
    for x, y, z in zip(base, kept, first[1:]):
        assert torch.allclose(x, y + z, rtol=2e-6, atol=2e-6 * float(z.abs().max()))
        assert torch.equal(x[z.abs().sum((1, 2)) == 0], y[z.abs().sum((1, 2)) == 0])
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 64, 4, 128), ("f32", 24, 1, 128)])
def test_batches_that_go_in_several_runs(dtype, h_q, h_kv, D):
    """A workspace of 256 MB holds fewer blocks than the batch has: gradients against those of the calls one by one."""
    import torch
    n_q = 9000 if dtype == "bf16" else 11000
    layer = Layer(dtype, [64, n_q, 200], h_q, h_kv, D)
    calls = [([(0, 0)], 2, 64, 70), ([(0, 0)], 1, 64, n_q), ([(0, 5)], 2, 64, 200)]
    blocks = (70 + n_q + 200) / 32 * h_q * (17 * 1024 if dtype == "bf16" else 33 * 1024)
    assert blocks > 256 << 20
    q, d_out = layer.normal(n_q + 270, h_q, D), layer.normal(n_q + 270, h_q, D)
    d_q, d_k, d_v = gradients(layer, calls, 50, 20, q, d_out, finalize=False)
    slots, at = d_k.shape[0], 0
    parts = [torch.zeros_like(d_k), torch.zeros_like(d_v)]
    for c in calls:
        if c[3] == n_q:                                  # (the long one in pieces of its own: its last rows, as the last rows of the message, are the same call)
            at += c[3]
            continue
        x = gradients(layer, [c], 50, 20, q[at:at + c[3]], d_out[at:at + c[3]], into=parts, finalize=False)
        assert torch.equal(x[0], d_q[at:at + c[3]])
        at += c[3]
    # of the long call, rows near a run's border and at its end, against the oracle's over the tokens they see
    from oracle import window_oracle as win
    for r0 in (5000, 7350, 7450, n_q - 40):
        n = 40
        k, v = layer.ks[1][r0 - 60:r0 + n], layer.vs[1][r0 - 60:r0 + n]
        rows = slice(70 + r0, 70 + r0 + n)
        a, _, _ = win.attend_call_window_backward([layer.ks[0], k], [layer.vs[0], v], [(0, 0)], 1, 64 + r0 - 60, n, None, q[rows], d_out[rows], layer.theta, 50, 20)
        got = d_q[rows].double().cpu().numpy()
        err = np.linalg.norm(got - a) / np.linalg.norm(a)
        say(f"  {dtype} rows {r0}: {err:.2e}")
        assert err <= BARS[dtype][0]
    assert torch.isfinite(d_k).all() and torch.isfinite(d_v).all() and torch.isfinite(d_q).all()
    layer.cache.close()


def test_against_differences_of_the_forward():
    """fp32: a step of 1e-2 in one number moves the sum by its gradient, to the second order of the step and the forward's precision."""
    import torch
    layer = Layer("f32", [40, 30], 4, 2, 64)
    calls, window, n_sink = [([(0, 0)], 1, 45, 30)], 25, 3
    q, d_out = layer.normal(30, 4, 64), layer.normal(30, 4, 64)
    d_q, _, _ = gradients(layer, calls, window, n_sink, q, d_out)
    rng = np.random.default_rng(1)
    for _ in range(8):
        at = (int(rng.integers(0, 30)), int(rng.integers(0, 4)), int(rng.integers(0, 64)))
        val = []
        for e in (1e-2, -1e-2):
            p = q.copy()
            p[at] += e
            val.append(float((layer.attend(calls, window, n_sink, p)[0].double().cpu().numpy() * d_out).sum()))
        assert abs((val[0] - val[1]) / 2e-2 - float(d_q[at])) <= 2e-3 * max(1.0, abs(float(d_q[at])))
    layer.cache.close()


def test_captured_streams_are_refused():
    import torch
    from paper_2512_23049_amd.binding import PC_ERR_INVALID_ARG, PcError
    layer = Layer("bf16", [40, 20], 4, 2, 128)
    calls = layer.calls([([(0, 0)], 1, 40, 20)])
    x = [torch.zeros(20, 4, 128, device="cuda:0", dtype=t) for t in (torch.bfloat16,) * 3 + (torch.float32,)]
    lse, dk = torch.zeros(20, 4, device="cuda:0"), torch.zeros(layer.cache.cache_info()[2], 2, 128, device="cuda:0")
    g, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=st):
        for f in (lambda: layer.cache.attend_window_backward(calls, 9, 0, x[0].data_ptr(), x[1].data_ptr(), lse.data_ptr(), x[2].data_ptr(), x[3].data_ptr(), dk.data_ptr(),
                                                             dk.data_ptr(), st.cuda_stream),
                  lambda: layer.cache.attend_window(calls, 9, 0, x[0].data_ptr(), x[1].data_ptr(), 0, st.cuda_stream)):
            with pytest.raises(PcError) as e:
                f()
            assert e.value.code == PC_ERR_INVALID_ARG and "captured" in str(e.value)
        lse.add_(1)
    g.replay()
    torch.cuda.synchronize()
    assert (lse == 1).all()
    layer.cache.close()
