"""Layers whose messages come from projected rows, and 4-bit layers, with what they hold in fp64 (shared by tests)."""
import numpy as np

from oracle import project_oracle as po
from oracle.choreo_oracle import rope
from tests.window_cases import say

THETA = 10000.0


def kinds():
    import torch
    from paper_2512_23049_amd import binding as b
    return {"bf16": (b.PC_BF16, torch.bfloat16), "f32": (b.PC_F32, torch.float32), "mx4": (b.PC_MX4, torch.bfloat16)}


class Rows:
    """Rows of a projection on the GPU (strided: one fused tensor, or three), and on the host what the tensors hold."""

    def __init__(self, dtype, n, h_q, h_kv, D, seed=3, extra=0, fused=True, weights=True, eps=1e-5, queries=True, spoil=None):
        import torch
        from paper_2512_23049_amd import binding as b
        self.n, self.h_q, self.h_kv, self.D, self.eps = n, h_q, h_kv, D, eps
        self.kind = kinds()[dtype][1]
        g = torch.Generator().manual_seed(seed)
        per = [h_q * D, h_kv * D, h_kv * D]
        x = torch.randn(n, sum(per) + extra, generator=g) * (0.5 + 3 * torch.rand(n, 1, generator=g))
        if spoil:
            spoil(x)
        self.fused = x.to(self.kind).to("cuda:0")
        parts = [self.fused[:, a:a + w] for a, w in zip(np.cumsum([0] + per[:2]), per)]
        if not fused:
            parts = [p.contiguous() for p in parts]
        self.parts = parts
        self.q, self.k, self.v = (p.double().cpu().numpy().reshape(n, -1, D) for p in parts)
        self.w = [(1 + 0.3 * torch.randn(D, generator=g)).to("cuda:0") if weights else None for _ in range(2)]
        self.qw, self.kw = (w.double().cpu().numpy() if weights else None for w in self.w)
        ptr = [p.data_ptr() for p in parts]
        self.queries = queries
        self.c = b.projected(ptr[0] if queries else 0, ptr[1], ptr[2], *(p.stride(0) for p in parts), *(w.data_ptr() if weights else 0 for w in self.w), eps)
        self.q_out = torch.full((n, h_q, D), 7.0, dtype=self.kind, device="cuda:0")
        self.out_ptr = self.q_out.data_ptr() if queries else 0

    def want_q(self):
        return po.norm(self.q, self.qw, self.eps)

    def want_k(self, a, b):
        """Normed keys of rows [a, b), not turned."""
        return po.norm(self.k[a:b], self.kw, self.eps)


def cache_of(dtype, h_q, h_kv, D, capacity, messages=64, **kw):
    from paper_2512_23049_amd import binding as b
    return b.Cache(h_q, h_kv, D, kinds()[dtype][0], THETA, capacity, messages, **kw)


def read(cache, ids, n, h_kv, D, kind):
    import torch
    k, v = (torch.full((n + 3, h_kv, D), 5.0, dtype=kind, device="cuda:0") for _ in range(2))
    cache.messages_read(ids, k.data_ptr(), v.data_ptr())
    torch.cuda.synchronize()
    assert (k[n:] == 5).all() and (v[n:] == 5).all()     # what lies behind the last row stays
    return (x[:n].double().cpu().numpy() for x in (k, v))


# One rounding to bf16 is off by 2^-8 of the value at most.  In 32 bits a norm's sum of 128 squares is added up in a tree (16 in a
# lane, 3 steps: 20 roundings of 2^-24, halved by the root), and norm, weight and turn take six more products and sums of a pair: below
# 2^-24 x 20 of the head's largest value, doubled.
def check(got, want, dtype, what=""):
    assert np.isfinite(got).all()
    top = np.abs(want).max(axis=-1, keepdims=True)
    bar = 2.4e-6 * top + (2.0 ** -8 * np.abs(want) if dtype != "f32" else 0)
    far = (np.abs(got - want) / np.maximum(bar, 1e-30)).max() if want.size else 0
    say(f"  {what} {dtype}: {far:.3f} of the bar")
    assert far <= 1


class Layer4:
    """A 4-bit cache and what it holds: keys as appended (turned back) and values, in fp64."""

    def __init__(self, lens, h_q, h_kv, seed=7, reserves=None, flags=0, spoil=None, room=0, messages=0, scale=1.0):
        import torch
        self.torch, self.h_q, self.h_kv, self.D, self.theta = torch, h_q, h_kv, 128, THETA
        self.rng = np.random.default_rng(seed)
        reserves = reserves or lens
        cap = sum((max(a, b) + 31) // 32 * 32 for a, b in zip(lens, reserves)) + 32 + room
        self.cache = cache_of("mx4", h_q, h_kv, 128, cap, messages or 4 * len(lens) + 64, flags=flags)
        self.raw, self.ks, self.vs, self.ids = [], [], [], []
        for i, (n, r) in enumerate(zip(lens, reserves)):
            k, v = self.normal(n, h_kv, 128) * scale, self.normal(n, h_kv, 128) * scale
            if spoil:
                spoil(i, k, v)
            self.add(k, v, r)

    def add(self, k, v, reserve=0):
        tk, tv = self.dev(k), self.dev(v)
        k, v = tk.float().cpu().numpy(), tv.float().cpu().numpy()          # (the numbers the cache is given)
        self.ids.append(self.cache.append_message(tk.data_ptr(), tv.data_ptr(), len(k), reserve))
        self.torch.cuda.synchronize()
        self.raw.append((k, v))
        a, b = po.held(k, v, THETA)
        self.ks.append(a)
        self.vs.append(b)

    def grow(self, m, k, v):
        """The books after tokens k, v have been appended to message m."""
        k, v = (np.concatenate([a, b]) for a, b in zip(self.raw[m], (k, v)))
        self.raw[m] = (k, v)
        self.ks[m], self.vs[m] = po.held(k, v, THETA)

    def normal(self, *shape):
        x = self.torch.from_numpy(self.rng.standard_normal(shape).astype(np.float32))
        return x.to(self.torch.bfloat16).float().numpy()

    def dev(self, x):
        return self.torch.from_numpy(np.ascontiguousarray(x)).to(device="cuda:0", dtype=self.torch.bfloat16)

    def calls(self, calls):
        from pc_inputs import Call
        return [Call([(self.ids[m], s) for m, s in c[0]], self.ids[c[1]] if c[1] >= 0 else -1, c[2], c[3], c[4] if len(c) > 4 else None) for c in calls]

    def attend(self, calls, q, window=0, n_sink=0, static=False, stream=0):
        t = self.torch
        tq = self.dev(q)
        out, lse = t.full(q.shape, 7.0, device="cuda:0", dtype=t.bfloat16), t.full(q.shape[:2], 7.0, device="cuda:0")
        cs, ptrs = self.calls(calls), (tq.data_ptr(), out.data_ptr(), lse.data_ptr(), stream)
        c = self.cache
        if window:
            (c.attend_window_static if static else c.attend_window)(cs, window, n_sink, *ptrs)
        else:
            (c.attend_static if static else c.attend)(cs, *ptrs)
        t.cuda.synchronize()
        return out, lse

    def want(self, calls, q, window=0, n_sink=0):
        from oracle import window_oracle as win
        at, outs, lses = 0, [], []
        for c in calls:
            o, l = win.attend_call_window(self.ks, self.vs, c[0], c[1], c[2], c[3], c[4] if len(c) > 4 else None, q[at:at + c[3]], THETA, window or 1 << 40, n_sink)
            outs.append(o)
            lses.append(l)
            at += c[3]
        return np.concatenate(outs), np.concatenate(lses)

    def run(self, calls, window=0, n_sink=0, static=False, what="", q=None):
        q = self.normal(sum(c[3] for c in calls), self.h_q, 128) if q is None else q
        out, lse = self.attend(calls, q, window, n_sink, static)
        want, want_lse = self.want(calls, q, window, n_sink)
        same(out, lse, want, want_lse, what or f"w {window} s {n_sink} static {static}")
        return out, lse


# Against the values held, which are exact: a turned query is off by 2^-8 of a value at most (as bf16: 1.7e-3 in the mean square), probabilities and
# the result are rounded to bf16 once each: 2.9e-3 in the 2-norm together; the bar is twice that.  A single element: half a
# step of a result of 4.5 is 1.8e-2, and a score that is four standard deviations off moves a row of two keys by 7e-3 x 1/4 x |v1 - v2| < 1e-2:
# 4e-2.  A log-sum-exp moves by its scores' errors: 4 x 1.7e-3, and 2^-8 of its keys' probabilities where they are few: 1.5e-2.
def same(out, lse, want, want_lse, what=""):
    got, got_lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    seen = np.isfinite(want_lse)
    assert (got_lse[~seen] == -np.inf).all() and (got[~seen] == 0).all()
    assert np.isfinite(got).all()
    if not seen.any():
        return
    err = np.linalg.norm(got - want) / np.linalg.norm(want)
    far, far_lse = np.abs(got - want).max(), np.abs(got_lse[seen] - want_lse[seen]).max()
    say(f"  {what}: 2-norm {err:.2e} max {far:.2e} lse {far_lse:.2e}")
    assert err <= 5.8e-3 and far <= 4e-2 and far_lse <= 1.5e-2
