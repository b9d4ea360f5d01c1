"""pc_projected_backward against fp64 and against differences; on its own and behind the attention's gradients."""
import numpy as np
import pytest

from oracle import project_oracle as po
from oracle import window_oracle as win
from oracle.choreo_oracle import rope
from tests.project_cases import THETA, Rows, cache_of, read
from tests.window_cases import say

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", 8, 2, 128), ("bf16", 24, 12, 128), ("f32", 4, 2, 64), ("f32", 9, 3, 128)]


class Grads:
    def __init__(self, rows, padded=0, weights=True):
        import torch
        from paper_2512_23049_amd import binding as b
        self.rows, self.D = rows, rows.D
        per = [rows.h_q * rows.D, rows.h_kv * rows.D, rows.h_kv * rows.D]
        if not rows.queries:
            per[0] = 0
        self.t = torch.full((rows.n + 1, sum(per) + padded), 7.0, dtype=rows.kind, device="cuda:0")
        self.at = np.cumsum([0] + per)
        self.w = torch.full((2, rows.D), 7.0, device="cuda:0")
        es = self.t.element_size()
        ptr = [self.t.data_ptr() + int(a) * es for a in self.at[:3]]
        s = self.t.stride(0)
        self.c = b.projected_grad(ptr[0] if rows.queries else 0, ptr[1], ptr[2], s, s, s, self.w[0].data_ptr() if weights and rows.queries else 0,
                                  self.w[1].data_ptr() if weights else 0)

    def get(self):
        assert (self.t[self.rows.n:] == 7).all() and (self.t[:, self.at[3]:] == 7).all()
        x = self.t[:self.rows.n].double().cpu().numpy()
        parts = [x[:, a:b].reshape(self.rows.n, -1, self.D) for a, b in zip(self.at, self.at[1:])]
        return parts, self.w.double().cpu().numpy()


# 32 bits: as the forward's, some 40 roundings of 2^-24 of the largest terms; a result is the difference of two terms as large as the row's
# largest g r, so that is what errors are measured in.  A bf16 result is off by 2^-8 of itself besides.  A weight's gradient is a
# sum of N terms, added up in pieces of 4 to 64 rows and then 64 shares: relative to the root of the sum of their squares 1e-6.
def check_rows(got, want, terms, dtype, what):
    bar = 5e-6 * terms + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)
    far = (np.abs(got - want) / np.maximum(bar, 1e-30)).max()
    say(f"  {what} {dtype}: {far:.3f} of the bar")
    assert far <= 1


def terms_of(x, w, eps, dy):
    r = 1 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    g = np.abs(dy * (1 if w is None else w)).max(axis=-1, keepdims=True)
    return r * (g + np.abs(x * r).max(axis=-1, keepdims=True) * g)


@pytest.mark.parametrize("dtype,h_q,h_kv,D", SHAPES)
@pytest.mark.parametrize("fused,padded,queries,weights", [(True, 0, True, True), (False, 64, True, False), (True, 8, False, True)])
def test_rows_and_weights(dtype, h_q, h_kv, D, fused, padded, queries, weights):
    import torch
    lens, reserves, taken = [1, 33, 64, 200, 7], [0, 60, 0, 0, 0], [1, 30, 64, 200, 7]
    rows = Rows(dtype, sum(lens), h_q, h_kv, D, fused=fused, weights=weights, queries=queries)
    c = cache_of(dtype, h_q, h_kv, D, 1024)
    ids = c.append_projected(rows.c, lens, rows.out_ptr, reserves)
    c.reposition(ids[2], 50)                             # (a message's keys may stand elsewhere: its gradient is of the keys as they are stored)
    gen = torch.Generator().manual_seed(1)
    starts = [c.message_info(m)[1] for m in ids]
    d_q = torch.randn(rows.n, h_q, D, generator=gen)
    d_k, d_v = torch.randn(1024, h_kv, D, generator=gen), torch.randn(1024, h_kv, D, generator=gen)
    dev = [x.to("cuda:0") for x in (d_q, d_k, d_v)]
    # the first tokens of some messages alone: rows are those that are asked for
    pick = np.concatenate([a + np.arange(n) for a, n in zip(np.cumsum([0] + lens), taken)])
    part = Rows(dtype, sum(lens), h_q, h_kv, D, fused=fused, weights=weights, queries=queries)
    tensors = [p[torch.from_numpy(pick).to("cuda:0")].contiguous() for p in rows.parts]
    from paper_2512_23049_amd import binding as b
    ptr = [t.data_ptr() for t in tensors]
    part.c = b.projected(ptr[0] if queries else 0, ptr[1], 0, *(t.stride(0) for t in tensors), *(w.data_ptr() if weights else 0 for w in rows.w), rows.eps)
    part.n = len(pick)
    out = [Grads(part, padded, weights) for _ in range(2)]
    d_qp = dev[0][torch.from_numpy(pick).to("cuda:0")].contiguous()
    for g in out:
        c.projected_backward(part.c, ids, taken, d_qp.data_ptr() if queries else 0, dev[1].data_ptr(), dev[2].data_ptr(), g.c)
    torch.cuda.synchronize()
    assert torch.equal(out[0].t, out[1].t) and torch.equal(out[0].w, out[1].w)           # the same call, the same bits
    assert torch.equal(dev[1].cpu(), d_k) and torch.equal(dev[2].cpu(), d_v)
    (gq, gk, gv), gw = out[0].get()
    slots = np.concatenate([s + np.arange(n) for s, n in zip(starts, taken)])
    pos = np.concatenate([(50 if i == 2 else 0) + np.arange(n) for i, n in enumerate(taken)])
    assert np.array_equal(gv, d_v[slots].to(rows.kind).double().numpy())
    dk = rope(d_k[slots].double().numpy(), -pos, THETA)
    for name, x, w, dy, got, got_w in (("k", rows.k[pick], rows.kw, dk, gk, gw[1]), ("q", rows.q[pick], rows.qw, d_q.double().numpy()[pick], gq, gw[0])):
        if name == "q" and not queries:
            assert (got_w == 7).all()
            continue
        dx, dw = po.norm_backward(x, w, rows.eps, dy)
        check_rows(got, dx, terms_of(x, w, rows.eps, dy), dtype, name)
        if weights:
            u = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + rows.eps)
            assert (np.abs(got_w - dw) <= 1e-6 * np.sqrt(((dy * u) ** 2).sum(axis=(0, 1))) + 1e-7 * np.abs(dw)).all()
        else:
            assert (got_w == 7).all()
    c.close()


def test_long_lists_of_messages():
    """More messages than the arguments hold, each a row or a few."""
    import torch
    lens = [int(x) for x in np.random.default_rng(4).integers(1, 6, size=180)]
    rows = Rows("f32", sum(lens), 4, 2, 64)
    c = cache_of("f32", 4, 2, 64, 32 * 180, messages=200)
    ids = c.append_projected(rows.c, lens, rows.out_ptr)
    gen = torch.Generator().manual_seed(1)
    d_q, d_k, d_v = torch.randn(rows.n, 4, 64, generator=gen), torch.randn(32 * 180, 2, 64, generator=gen), torch.randn(32 * 180, 2, 64, generator=gen)
    dev = [x.to("cuda:0") for x in (d_q, d_k, d_v)]
    g = Grads(rows)
    c.projected_backward(rows.c, ids, lens, *(x.data_ptr() for x in dev), g.c)
    torch.cuda.synchronize()
    (gq, gk, gv), gw = g.get()
    slots = np.concatenate([32 * i + np.arange(n) for i, n in enumerate(lens)])
    dk = rope(d_k[slots].double().numpy(), -np.concatenate([np.arange(n) for n in lens]), THETA)
    dx, dw = po.norm_backward(rows.k, rows.kw, rows.eps, dk)
    check_rows(gk, dx, terms_of(rows.k, rows.kw, rows.eps, dk), "f32", "k")
    dx, dw = po.norm_backward(rows.q, rows.qw, rows.eps, d_q.double().numpy())
    check_rows(gq, dx, terms_of(rows.q, rows.qw, rows.eps, d_q.double().numpy()), "f32", "q")
    assert np.array_equal(gv, d_v[slots].double().numpy())
    c.close()


def test_by_differences():
    """Along a direction: the appends' own outputs, moved by h both ways.  Rounding: outputs of order one are off by 2e-7 each, their sum over N
    terms by 2e-7 sqrt(N), over 2h; the third derivative gives h^2.  With h = 4e-3 both are below 1e-4 of |dx| |direction| / sqrt(N) x sqrt(N)."""
    import torch
    n, h_q, h_kv, D, h = 60, 4, 2, 64, 4e-3
    base = Rows("f32", n, h_q, h_kv, D)
    gen = torch.Generator().manual_seed(8)
    d_q, d_k = torch.randn(n, h_q, D, generator=gen).double().numpy(), torch.randn(64, h_kv, D, generator=gen)
    way = torch.randn(base.fused.shape, generator=gen).to("cuda:0")
    way[:, (h_q + h_kv) * D:] = 0
    c = cache_of("f32", h_q, h_kv, D, 64)

    def value(sign):
        base.fused += sign * h * way
        ids = c.append_projected(base.c, [n], base.out_ptr)
        k, _ = read(c, ids, n, h_kv, D, torch.float32)
        c.message_free(ids[0])
        base.fused -= sign * h * way
        return (base.q_out.double().cpu().numpy() * d_q).sum() + (k * d_k[:n].double().numpy()).sum()
    slope = (value(1) - value(-1)) / (2 * h)
    ids = c.append_projected(base.c, [n], base.out_ptr)
    g = Grads(base)
    dev = [torch.from_numpy(d_q).float().to("cuda:0"), d_k.to("cuda:0"), torch.zeros_like(d_k).to("cuda:0")]
    c.projected_backward(base.c, ids, [n], *(x.data_ptr() for x in dev), g.c)
    torch.cuda.synchronize()
    dx = g.t[:n].double().cpu().numpy()
    want = (dx * way.double().cpu().numpy()).sum()
    size = np.linalg.norm(dx)                            # (a random direction of unit entries: the sum is of this size)
    say(f"  slope {slope:.6f}, gradient {want:.6f}, size {size:.3f}")
    assert abs(slope - want) <= 1e-3 * size
    c.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("f32", 4, 2, 64), ("bf16", 8, 2, 128)])
@pytest.mark.parametrize("window", [0, 40])
def test_a_layer_and_its_gradient(dtype, h_q, h_kv, D, window):
    """As in training: a layer's projected rows are appended, attend to cached messages and themselves, and the gradient of the output goes back
    through the attention and the norms into the rows and the weights."""
    import torch
    from pc_inputs import Call
    cached, lens = [50, 37], [70, 33]
    c = cache_of(dtype, h_q, h_kv, D, 512)
    old = Rows(dtype, sum(cached), h_q, h_kv, D, seed=1, queries=False)
    parents = c.append_projected(old.c, cached, 0)
    rows = Rows(dtype, sum(lens), h_q, h_kv, D, seed=2)
    ids = c.append_projected(rows.c, lens, rows.out_ptr)
    sel = [(parents[1], 0), (parents[0], 45)]
    calls = [Call(sel, ids[0], 100, 70, None), (Call(sel[:1], ids[1], 60, 33, None))]
    q = rows.q_out
    out, lse = torch.empty_like(q), torch.empty(rows.n, h_q, device="cuda:0")
    d_out = torch.randn(q.shape, generator=torch.Generator().manual_seed(4)).to(rows.kind).to("cuda:0")
    d_q = torch.empty(q.shape, device="cuda:0")
    d_k, d_v = torch.zeros(512, h_kv, D, device="cuda:0"), torch.zeros(512, h_kv, D, device="cuda:0")
    p = [x.data_ptr() for x in (q, out, lse, d_out, d_q, d_k, d_v)]
    if window:
        c.attend_window(calls, window, 3, p[0], p[1], p[2])
        c.attend_window_backward(calls, window, 3, *p)
    else:
        c.attend(calls, p[0], p[1], p[2])
        c.attend_backward(calls, p[0], p[2], p[3], p[4], p[5], p[6])
    g = Grads(rows)
    c.projected_backward(rows.c, ids, lens, p[4], p[5], p[6], g.c)
    torch.cuda.synchronize()
    (gq, gk, gv), gw = g.get()
    # the oracle, all of it in fp64
    ks = [po.norm(old.k[:50], old.kw, old.eps), po.norm(old.k[50:], old.kw, old.eps), rows.want_k(0, 70), rows.want_k(70, 103)]
    vs = [old.v[:50], old.v[50:], rows.v[:70], rows.v[70:]]
    wq, wd = rows.want_q(), d_out.double().cpu().numpy()
    of_q, of_k, of_v = np.zeros(wq.shape), [np.zeros(x.shape) for x in ks], [np.zeros(x.shape) for x in vs]
    at, outs = 0, []
    for s, me, start, n in (([(1, 0), (0, 45)], 2, 100, 70), ([(1, 0)], 3, 60, 33)):
        w = window or 1 << 40
        outs.append(win.attend_call_window(ks, vs, s, me, start, n, None, wq[at:at + n], THETA, w, 3 if window else 0)[0])
        a, b, e = win.attend_call_window_backward(ks, vs, s, me, start, n, None, wq[at:at + n], wd[at:at + n], THETA, w, 3 if window else 0)
        of_q[at:at + n] = a
        for i in range(4):
            of_k[i] += b[i]
            of_v[i] += e[i]
        at += n
    dq, dqw = po.norm_backward(rows.q, rows.qw, rows.eps, of_q)
    dk, dkw = po.norm_backward(rows.k, rows.kw, rows.eps, np.concatenate(of_k[2:]))
    # 2-norms.  fp32: the attention's 3e-6 (see its tests), twice.  bf16: queries, keys, probabilities and results of the attention are rounded once each
    # (3.2e-3), the gradient's probabilities and products again: 1.2e-2 is the bar of its own tests; the rows' rounding adds 1.7e-3.
    bar = 6e-6 if dtype == "f32" else 1.4e-2
    got = out.double().cpu().numpy()
    for name, x, y in (("out", got, np.concatenate(outs)), ("q", gq, dq), ("k", gk, dk), ("v", gv, np.concatenate(of_v[2:])), ("q_weight", gw[0], dqw), ("k_weight", gw[1], dkw)):
        err = np.linalg.norm(x - y) / np.linalg.norm(y)
        say(f"  {name}: {err:.2e}")
        assert err <= bar, name
    c.close()
