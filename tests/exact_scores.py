"""A 4-bit cache whose scores are exact: the base of its turns is so large that dims 32 to 63 (and their partners, 96 to 127) do not turn, a score is
log2(e) times a sum of q k, and keys and queries are numbers that 4 bits, and the queries' 8-bit pieces, hold (shared by tests)."""
import numpy as np

from oracle import project_oracle as po
from tests.window_cases import say

LN2 = 0.6931471805599453
DIMS = (40, 100)                                         # a score's two parts: each alone in its block of 32


def two_parts(s):
    """s as a sum of two numbers out of {0, 1, 1.5, 2, 3, ...} and their negatives."""
    one = [0.0] + [m * 2.0 ** e for e in range(-1, 8) for m in (1, 1.5)]
    one = sorted(one + [-x for x in one], key=abs)
    return min(((a, s - a) for a in one if s - a in one), key=lambda ab: abs(ab[0]) + abs(ab[1]))


class Exact:
    def __init__(self, messages, h_q=8, h_kv=2, room=0):
        """messages: (scores [tokens], values [tokens, 128]) or (keys [tokens, 128], values) each, the same for all KV heads."""
        import torch
        from paper_2512_23049_amd import binding as b
        self.torch, self.h_q, self.h_kv = torch, h_q, h_kv
        cap = sum((len(s) + 31) // 32 * 32 for s, _ in messages) + 32 + room
        self.cache = b.Cache(h_q, h_kv, 128, b.PC_MX4, 1e30, cap, len(messages) + 64, softmax_scale=LN2)
        self.ids, self.ks, self.vs = [], [], []
        for s, v in messages:
            s, v = np.asarray(s, np.float64), np.asarray(v, np.float64)
            k = s
            if s.ndim == 1:
                k = np.zeros((len(s), 128))
                k[:, DIMS] = [two_parts(x) for x in s]
            assert np.array_equal(po.to_mx4(k), k)
            self.ks.append(k)
            self.vs.append(po.to_mx4(v))
            tk, tv = (self.dev(np.repeat(x[:, None], h_kv, axis=1)) for x in (k, v))
            self.ids.append(self.cache.append_message(tk.data_ptr(), tv.data_ptr(), len(k)))
            torch.cuda.synchronize()

    def dev(self, x):
        return self.torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(device="cuda:0", dtype=self.torch.bfloat16)

    def query(self, rows):
        q = np.zeros((rows, self.h_q, 128))
        q[..., DIMS] = 1
        return q

    def attend(self, calls, q, window=0, static=False):
        """calls: (messages, rows) each, the messages one behind the other, all seen by every row."""
        from pc_inputs import Call
        t = self.torch
        tq = self.dev(q)
        out, lse = t.full(q.shape, 7.0, device="cuda:0", dtype=t.bfloat16), t.full(q.shape[:2], 7.0, device="cuda:0")
        cs = []
        for listed, rows in calls:
            at = np.cumsum([0] + [len(self.ks[m]) for m in listed])
            cs.append(Call([(self.ids[m], int(p)) for m, p in zip(listed, at)], -1, int(at[-1]), rows, None))
        ptrs = (tq.data_ptr(), out.data_ptr(), lse.data_ptr())
        c = self.cache
        if window:
            (c.attend_window_static if static else c.attend_window)(cs, window, 0, *ptrs)
        else:
            (c.attend_static if static else c.attend)(cs, *ptrs)
        t.cuda.synchronize()
        return out.double().cpu().numpy(), lse.double().cpu().numpy()

    def want(self, calls, q):
        at, outs, lses = 0, [], []
        for listed, rows in calls:
            k, v = (np.concatenate([x[m] for m in listed]) for x in (self.ks, self.vs))
            s = q[at:at + rows] @ k.T
            top = s.max(axis=-1, keepdims=True)
            p = 2.0 ** (s - top)
            outs.append(p @ v / p.sum(axis=-1, keepdims=True))
            lses.append((top[..., 0] + np.log2(p.sum(axis=-1))) * LN2)
            at += rows
        return np.concatenate(outs), np.concatenate(lses)


# Probabilities of whole powers of two are exact in bf16 and fp16 (as long as these hold them), so that what is rounded is the result, by 2^-8 of it at
# most, and what splits add up, in 32 bits: 2^-10 for sums of some thousand terms, and for the copy's (or a split's) normed parts.
BAR = 2.0 ** -8 + 2.0 ** -10


def close(got, want, what, bar=BAR, lse_bar=3e-5):
    (out, lse), (want_out, want_lse) = got, want
    assert np.isfinite(out).all(), what
    far = (np.abs(out - want_out) / np.maximum(np.abs(want_out), 1e-300)).max()
    far_lse = (np.abs(lse - want_lse) / np.maximum(1, np.abs(want_lse))).max()
    say(f"  {what}: {far:.2e} of a value, lse {far_lse:.2e}")
    assert far <= bar and far_lse <= lse_bar, what
