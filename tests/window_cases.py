"""Runs calls through pc_attend_window and the fp64 oracle (shared by the tests of the windowed attention)."""
import sys

import numpy as np


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


class Layer:
    """A cache on the GPU and the same messages on the host, in the numbers the cache was given."""

    def __init__(self, dtype, lens, h_q, h_kv, D, seed=7, theta=10000.0, spoil=None, reserves=None, flags=0, max_position=0, room=0):
        import torch
        from paper_2512_23049_amd import binding
        self.torch, self.dtype, self.h_q, self.h_kv, self.D, self.theta = torch, dtype, h_q, h_kv, D, theta
        self.rng = np.random.default_rng(seed)
        self.kind = torch.bfloat16 if dtype == "bf16" else torch.float32
        reserves = reserves or lens
        cap = sum((max(a, b) + 31) // 32 * 32 for a, b in zip(lens, reserves)) + 32 + room
        self.cache = binding.Cache(h_q, h_kv, D, binding.PC_BF16 if dtype == "bf16" else binding.PC_F32, theta, cap, 4 * len(lens) + 64,
                                   flags=flags, max_position=max_position)
        self.ks, self.vs = [], []
        for n, r in zip(lens, reserves):
            k, v = self.normal(n, h_kv, D), self.normal(n, h_kv, D)
            self.ks.append(k)
            self.vs.append(v)
        if spoil:
            spoil(self.ks, self.vs)
        for k, v, r in zip(self.ks, self.vs, reserves):
            tk, tv = self.dev(k), self.dev(v)
            self.cache.append_message(tk.data_ptr(), tv.data_ptr(), len(k), r)
            torch.cuda.synchronize()

    def normal(self, *shape):
        """N(0, 1) in numbers the cache's type holds."""
        x = self.rng.standard_normal(shape).astype(np.float32)
        return self.torch.from_numpy(x).to(self.kind).float().numpy()

    def dev(self, x):
        return self.torch.from_numpy(np.ascontiguousarray(x)).to(device="cuda:0", dtype=self.kind)

    def calls(self, calls):
        from pc_inputs import Call
        return [Call(list(c[0]), c[1], c[2], c[3], c[4] if len(c) > 4 else None) for c in calls]

    def attend(self, calls, window, n_sink, q, static=False, stream=0, lse=True):
        t = self.torch
        tq = self.dev(q)
        out = t.full(q.shape, 7.0, device="cuda:0", dtype=self.kind)
        ls = t.full(q.shape[:2], 7.0, device="cuda:0")
        f = self.cache.attend_window_static if static else self.cache.attend_window
        f(self.calls(calls), window, n_sink, tq.data_ptr(), out.data_ptr(), ls.data_ptr() if lse else 0, stream)
        t.cuda.synchronize()
        return out, ls

    def want(self, calls, window, n_sink, q, vs=None):
        from oracle import window_oracle as win
        at, outs, lses = 0, [], []
        for c in calls:
            o, l = win.attend_call_window(self.ks, vs or self.vs, c[0], c[1], c[2], c[3], c[4] if len(c) > 4 else None, q[at:at + c[3]], self.theta, window, n_sink)
            outs.append(o)
            lses.append(l)
            at += c[3]
        return np.concatenate(outs), np.concatenate(lses)

    def rows(self, calls):
        return sum(c[3] for c in calls)


# fp32: about ten roundings of 2^-24 a term (see test_gpu_f32_attend.py): 6e-7 in the 2-norm, the bar is 3e-6.
# bf16 (half a step is 2^-8 of a value, 1.6e-3 in the mean square): a stored key and a turned query rounded once each move a score
# of N(0,1) data by 2.3e-3, the probabilities and the result are rounded once each: 3.2e-3 in the 2-norm together, the bar is 1e-2.  A single
# element: half a step of a result of 4.5 is 1.8e-2, and a score that is four standard deviations off moves a row of two keys
# by 1e-2 x 1/4 x |v1 - v2| < 1.5e-2: 4e-2.  A log-sum-exp moves by its scores' errors: 4 x 2.3e-3, the bar is 2e-2.
BARS = {"f32": (3e-6, 3e-5, 1e-5), "bf16": (1e-2, 4e-2, 2e-2)}


def compare(dtype, out, lse, want, want_lse, what=""):
    norm, most, bar_lse = BARS[dtype]
    got, got_lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    seen = np.isfinite(want_lse)
    assert (got_lse[~seen] == -np.inf).all() and (got[~seen] == 0).all()
    assert np.isfinite(got).all()
    if not seen.any():
        return
    err = np.linalg.norm(got - want) / np.linalg.norm(want)
    far, far_lse = np.abs(got - want).max(), np.abs(got_lse[seen] - want_lse[seen]).max()
    say(f"  {what} {dtype}: 2-norm {err:.2e} max {far:.2e} lse {far_lse:.2e}")
    assert err <= norm and far <= most and far_lse <= bar_lse
