"""pc_attend_window_static recorded into a HIP graph and replayed, with eager calls in between that use the staging ring, the fixed
array and the cache's own workspace: every replay gives the bits of the eager call for the queries it finds.  Side streams, and what is refused
of pointers."""
import numpy as np
import pytest

from pc_inputs import Call
from tests.window_cases import Layer, compare

pytestmark = pytest.mark.gpu

LENS = [200, 31, 64, 333, 1, 150, 290, 97, 400, 128, 77, 260]


def whole(n, gap=0):
    at, sel = 0, []
    for m in range(n):
        sel.append((m, at))
        at += LENS[m] + gap
    return sel, at


def batches():
    sel, end = whole(12)
    few = [(sel[:3], 12, 300, 1), (sel[5:8], -1, 900, 1)]
    rows = [(sel, 13, end, 90), (sel[2:4], -1, 900, 40, list(range(800, 840))), (sel[:2], 12, 250, 1)]
    shared = [(sel if i % 2 else whole(12, i)[0][::-1], -1, end + 40 * i, 1) for i in range(30)]
    own = [([(i % 12, 7 * i)], -1, 500, 1) for i in range(90)]           # lists longer than a kernel's arguments, nothing shared
    return {"a few single tokens": few, "prefill and a token": rows, "shared messages": shared, "many single tokens": own}


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 16, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("which", list(batches()))
def test_replays_give_the_eager_bits(dtype, h_q, h_kv, D, which):
    import torch
    layer = Layer(dtype, LENS + [40, 90], h_q, h_kv, D)
    layer.cache.set_decode_sharing(2 if which == "shared messages" else 0)
    calls = batches()[which]
    rows, window, n_sink = layer.rows(calls), 700, 5
    qs = [layer.normal(rows, h_q, D) for _ in range(4)]
    wants = [layer.attend(calls, window, n_sink, q, static=True) for q in qs]
    compare(dtype, *wants[0], *layer.want(calls, window, n_sink, qs[0]), which)
    q, out, lse = layer.dev(qs[0]), torch.empty_like(wants[0][0]), torch.empty_like(wants[0][1])
    stream, graph, listed = torch.cuda.Stream(), torch.cuda.CUDAGraph(), layer.calls(calls)
    with torch.cuda.graph(graph, stream=stream):
        layer.cache.attend_window_static(listed, window, n_sink, q.data_ptr(), out.data_ptr(), lse.data_ptr(), stream.cuda_stream)
    del listed
    for x, (want, want_lse) in zip(qs, wants):
        for name, other in batches().items():            # (other lists through the ring and both workspaces)
            layer.attend(other, 90, 0, layer.normal(layer.rows(other), h_q, D), static=name != which)
        q.copy_(layer.dev(x))
        out.fill_(7.0)
        lse.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 16, 2, 128), ("f32", 4, 2, 64)])
def test_two_caches_on_two_streams(dtype, h_q, h_kv, D):
    """Calls of two caches that overlap in time, each on a stream of its own, give what they give alone."""
    import torch
    layers = [Layer(dtype, LENS + [40, 90], h_q, h_kv, D, seed=s) for s in (1, 2)]
    for name, calls in batches().items():
        qs = [layer.normal(layer.rows(calls), h_q, D) for layer in layers]
        alone = [layer.attend(calls, 700, 5, q) for layer, q in zip(layers, qs)]
        streams, tqs = [torch.cuda.Stream() for _ in layers], [layer.dev(q) for layer, q in zip(layers, qs)]
        outs, listed = [[torch.empty_like(a[0]) for _ in range(20)] for a in alone], [layer.calls(calls) for layer in layers]
        torch.cuda.synchronize()
        for i in range(20):
            for k, layer in enumerate(layers):
                layer.cache.attend_window(listed[k], 700, 5, tqs[k].data_ptr(), outs[k][i].data_ptr(), 0, streams[k].cuda_stream)
        torch.cuda.synchronize()
        for k in range(2):
            assert all(torch.equal(o, alone[k][0]) for o in outs[k]), name
    for layer in layers:
        layer.cache.close()


def test_pointers_that_are_refused():
    import torch
    from paper_2512_23049_amd.binding import PC_ERR_INVALID_ARG, PcError
    layer = Layer("bf16", [40, 20], 4, 2, 128)
    calls = layer.calls([([(0, 0)], 1, 40, 20)])
    x = [torch.zeros(21, 4, 128, device="cuda:0", dtype=t) for t in (torch.bfloat16,) * 3 + (torch.float32,)]
    lse, dk = torch.zeros(21, 4, device="cuda:0"), torch.zeros(layer.cache.cache_info()[2] + 1, 2, 128, device="cuda:0")
    q, o, do, dq = (t.data_ptr() for t in x)
    good = [q, o, lse.data_ptr(), do, dq, dk.data_ptr(), dk.data_ptr()]
    for i, off in [(0, 8), (1, 2), (2, 2), (3, 8), (4, 4), (5, 4), (6, 8)]:
        for bad in (0, good[i] + off):
            p = good[:i] + [bad] + good[i + 1:]
            with pytest.raises(PcError) as e:
                layer.cache.attend_window_backward(calls, 9, 0, *p)
            assert e.value.code == PC_ERR_INVALID_ARG, (i, bad)
            if i < 3 and not (i == 2 and bad == 0):      # (the forward's lse may be null)
                for f in (layer.cache.attend_window, layer.cache.attend_window_static):
                    with pytest.raises(PcError) as e:
                        f(calls, 9, 0, *p[:3])
                    assert e.value.code == PC_ERR_INVALID_ARG, (i, bad)
    torch.cuda.synchronize()
    assert not any(t.any() for t in x + [lse, dk])
    layer.cache.close()


def test_lists_that_a_staging_slot_does_not_hold():
    """The static form, which cannot grow, says so; the other takes them."""
    from paper_2512_23049_amd.binding import PC_ERR_NO_SPACE, PcError
    layer = Layer("bf16", [2] * 340, 2, 2, 128)
    calls = [([(int(m), 3 * i) for i, m in enumerate(np.random.default_rng(j).permutation(340))], -1, 1100 + j, 1) for j in range(110)]
    q = layer.normal(110, 2, 128)
    out, lse = layer.attend(calls, 1 << 20, 0, q)
    for i in (0, 57, 109):
        compare("bf16", out[i:i + 1], lse[i:i + 1], *layer.want([calls[i]], 1 << 20, 0, q[i:i + 1]))
    with pytest.raises(PcError) as e:
        layer.attend(calls, 1 << 20, 0, q, static=True)
    assert e.value.code == PC_ERR_NO_SPACE
    few, few_lse = layer.attend(calls[:40], 1 << 20, 0, q[:40], static=True)
    compare("bf16", few, few_lse, out[:40].double().cpu().numpy(), lse[:40].double().cpu().numpy())
    layer.cache.close()
