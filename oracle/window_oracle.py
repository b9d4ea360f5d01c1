"""Windowed attention in fp64 (test infrastructure, not product): the dense statement of what pc_attend_window and its gradient
compute.  A row at position p sees, of the tokens its call shows it (all parent tokens, own tokens up to its own), those at
positions above p - window and the first n_sink tokens of the call's list.

Shares the position rules of choreo_oracle (which parents are where, which tokens the rows are) and states the mask, the
softmax and its gradient anew.  Pinned in tests/test_window_oracle.py: against choreo_oracle where the window holds
everything, by closed forms and by central differences."""
from __future__ import annotations

import numpy as np

from .choreo_oracle import query_positions, resolve_positions, rope


def _gathered(msgs_k, msgs_v, sel, self_msg, self_start, n_q, q_pos):
    lengths = [int(k.shape[0]) for k in msgs_k]
    sel_r, s_self = resolve_positions(sel, lengths, self_start)
    entries = list(sel_r) + ([(self_msg, s_self)] if self_msg >= 0 else [])
    H, D = msgs_k[0].shape[1], msgs_k[0].shape[2]
    n = sum(lengths[m] for m, _ in entries)
    k = np.concatenate([np.asarray(msgs_k[m], np.float64) for m, _ in entries]) if n else np.zeros((0, H, D))
    v = np.concatenate([np.asarray(msgs_v[m], np.float64) for m, _ in entries]) if n else np.zeros((0, H, D))
    pos = np.concatenate([s + np.arange(lengths[m], dtype=np.int64) for m, s in entries]) if n else np.zeros(0, np.int64)
    own = lengths[self_msg] if self_msg >= 0 else 0
    p_rows = np.asarray(query_positions(n_q, own if self_msg >= 0 else n_q, s_self, q_pos), np.int64)
    # in list order, the last token a row may see: its own one, or the last of all
    last = n - own + own - n_q + np.arange(n_q) if self_msg >= 0 else np.full(n_q, n - 1)
    return entries, k, v, pos, p_rows, last


def visible(pos, p_rows, last, window, n_sink):
    i = np.arange(pos.shape[0])
    return (i[None, :] <= last[:, None]) & ((pos[None, :] > p_rows[:, None] - int(window)) | (i[None, :] < n_sink))


def _probabilities(qr, kr, vis, scale):
    s = np.where(vis, scale * (qr @ kr.T), -np.inf) if kr.shape[0] else np.full(vis.shape, -np.inf)
    top = s.max(axis=1, keepdims=True, initial=-np.inf)
    safe = np.where(np.isfinite(top), top, 0.0)
    e = np.where(vis, np.exp(s - safe), 0.0)
    den = e.sum(axis=1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        # (a row that sees nothing: zeros; one with a score that is not a number is none)
        return np.where(den == 0, 0.0, e / den), np.where(den == 0, -np.inf, safe + np.log(den))[:, 0]


def attend_call_window(msgs_k, msgs_v, sel, self_msg, self_start, n_q, q_pos, q, theta, window, n_sink, scale=None):
    """(out [n_q, H_q, D], lse [n_q, H_q]).  Values that no row of a product sees may be anything: they are left out of it."""
    _, k, v, pos, p_rows, last = _gathered(msgs_k, msgs_v, sel, self_msg, self_start, n_q, q_pos)
    H_q, D = q.shape[1], q.shape[2]
    g = H_q // k.shape[1]
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    kr, qr = rope(k, pos, theta), rope(np.asarray(q, np.float64), p_rows, theta)
    vis = visible(pos, p_rows, last, window, n_sink)
    out, lse = np.zeros((n_q, H_q, D)), np.full((n_q, H_q), -np.inf)
    for h in range(H_q):
        with np.errstate(invalid="ignore"):
            p, lse[:, h] = _probabilities(qr[:, h], kr[:, h // g], vis, scale)
        vh = v[:, h // g]
        fine = np.isfinite(vh).all(axis=1)
        out[:, h] = p[:, fine] @ vh[fine]
        for j in np.nonzero(~fine)[0]:                   # a value that is not finite: only for the rows that see it
            rows = vis[:, j]
            with np.errstate(invalid="ignore"):
                out[rows, h] += p[rows, j][:, None] * vh[j][None]
    return out, lse


def attend_call_window_backward(msgs_k, msgs_v, sel, self_msg, self_start, n_q, q_pos, q, d_out, theta, window, n_sink, scale=None):
    """(d_q, d_k, d_v): the gradient of sum(out d_out) with respect to the queries, the keys as appended and the values."""
    entries, k, v, pos, p_rows, last = _gathered(msgs_k, msgs_v, sel, self_msg, self_start, n_q, q_pos)
    H_q, D = q.shape[1], q.shape[2]
    g = H_q // k.shape[1]
    scale = 1.0 / np.sqrt(D) if scale is None else scale
    kr, qr = rope(k, pos, theta), rope(np.asarray(q, np.float64), p_rows, theta)
    vis = visible(pos, p_rows, last, window, n_sink)
    d_o = np.asarray(d_out, np.float64)
    d_qr, d_kr, d_vc = np.zeros_like(qr), np.zeros_like(kr), np.zeros_like(v)
    for h in range(H_q):
        kh = h // g
        p, _ = _probabilities(qr[:, h], kr[:, kh], vis, scale)
        d_p = d_o[:, h] @ v[:, kh].T
        d_s = scale * p * (d_p - (p * d_p).sum(axis=1, keepdims=True))
        d_qr[:, h] = d_s @ kr[:, kh]
        d_kr[:, kh] += d_s.T @ qr[:, h]
        d_vc[:, kh] += p.T @ d_o[:, h]
    d_kc = rope(d_kr, -pos, theta)
    d_k = [np.zeros(np.shape(x)) for x in msgs_k]
    d_v = [np.zeros(np.shape(x)) for x in msgs_v]
    at = 0
    for m, _ in entries:
        n = msgs_k[m].shape[0]
        d_k[m] += d_kc[at:at + n]
        d_v[m] += d_vc[at:at + n]
        at += n
    return rope(d_qr, -p_rows, theta), d_k, d_v
