"""Bars without a floor for the gradients of the windowed attention, and the oracle of long batches (shared by tests).

A gradient is held against the oracle's in the 2-norm of what one place computes: a call's rows for d_q, 128 consecutive keys of a message for
d_k and d_v.  Errors are relative to what is there (see test_gpu_window_backward.py: 4e-3 in bf16, 6e-7 and as much again in fp32), however
many keys share a row's probability: each term is off by its own share, and terms of random signs add up as their errors do.  The bars are three
times that, 1.2e-2 and 4e-6; a place whose gradient is zero has to be zero.  (Not for rows that see one key, where all terms cancel.)"""
import numpy as np

BAR = {"f32": 4e-6, "bf16": 1.2e-2}
KEYS = 128


def places(d_q, d_k, d_v, n_qs):
    """(name, array) of every place; d_q: rows; d_k, d_v: lists by message."""
    at = 0
    for i, n in enumerate(n_qs):
        for r in range(at, at + n, 1024):
            yield f"d_q call {i} rows {r - at}..", d_q[r:min(r + 1024, at + n)]
        at += n
    for name, d in (("d_k", d_k), ("d_v", d_v)):
        for m, x in enumerate(d):
            for t in range(0, len(x), KEYS):
                yield f"{name} message {m} keys {t}..", x[t:t + KEYS]


def errors(got, want, n_qs):
    """{place: relative error}; infinite where something stands for zero, or what is not a number."""
    out = {}
    for (name, a), (_, b) in zip(places(*got, n_qs), places(*want, n_qs)):
        size, err = np.linalg.norm(b), np.linalg.norm(a - b)
        out[name] = (err / size if size > 0 else 0.0 if err == 0 else np.inf) if np.isfinite(a).all() else np.inf
    return out


def worst(got, want, n_qs):
    e = errors(got, want, n_qs)
    name = max(e, key=e.get)
    return e[name], name


# calls over four parents of 700 tokens and a new message of 900: a row's walk in many splits, tiles with sinks that every row sees
LONG_LENS = [700] * 4 + [900]
LONG_SEL = [(m, 650 * m) for m in range(4)]
LONG = [(1, 2500, 40), (20, 3000, 0), (900, 200, 150)]          # rows, window, sinks


def in_pieces(ks, vs, own, parent, parent_start, own_start, q, d_out, theta, window, n_sink, step=128):
    """The oracle's gradients of the call ([(parent, parent_start)], own, own_start) with all of the new message's rows, n_sink <= the
    parent's length, made of pieces of `step` rows with the keys that they see: (d_q, d_k of the parent and of own, d_v likewise)."""
    from oracle import window_oracle as win
    n = len(ks[own])
    d_q = np.zeros(q.shape)
    d_k, d_v = [np.zeros(ks[parent].shape), np.zeros(ks[own].shape)], [np.zeros(ks[parent].shape), np.zeros(ks[own].shape)]
    for r0 in range(0, n, step):
        r1, first = min(n, r0 + step), max(0, r0 - window)
        a, b, e = win.attend_call_window_backward([ks[parent], ks[own][first:r1]], [vs[parent], vs[own][first:r1]], [(0, parent_start)], 1, own_start + first,
                                                  r1 - r0, None, q[r0:r1], d_out[r0:r1], theta, window, n_sink)
        d_q[r0:r1] = a
        for d, x in ((d_k, b), (d_v, e)):
            d[0] += x[0]
            d[1][first:r1] += x[1]
    return d_q, d_k, d_v
