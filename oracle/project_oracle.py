"""Norms of heads in front of an append, their gradient, and the 4-bit form of a PC_MX4 cache, in fp64 (test infrastructure, not
product).  Pinned in tests/test_project_oracle.py: by closed forms, by central differences and by a search over all codes."""
from __future__ import annotations

import numpy as np

from .choreo_oracle import rope

GRID = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])


def norm(x, weight, eps):
    x = np.asarray(x, np.float64)
    w = 1.0 if weight is None else np.asarray(weight, np.float64)
    return x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * w


def norm_backward(x, weight, eps, dy):
    """(dx, dw): of sum(norm(x) dy); x [rows, heads, D], dw summed over rows and heads."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    w = np.ones(x.shape[-1]) if weight is None else np.asarray(weight, np.float64)
    r = 1 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    u, g = x * r, dy * w
    return r * (g - u * (g * u).mean(axis=-1, keepdims=True)), (dy * u).sum(axis=(0, 1))


def exponents(x):
    """Of blocks [..., 32]: the least e with max|x| < 7 2^e, from -60 to 60, [..., 1]."""
    top = np.abs(x).max(axis=-1, keepdims=True)
    m, e = np.frexp(top)
    e = e - 3 + (m >= 0.875)
    return np.clip(np.where(top == 0, -60, e), -60, 60)


def to_mx4(x):
    """What a 4-bit cache holds for x [..., D] (finite)."""
    x = np.asarray(x, np.float64)
    b = x.reshape(*x.shape[:-1], -1, 32)
    e = exponents(b)
    a = np.abs(b) * 2.0 ** -e
    below = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, 6)
    up = a - GRID[below] > GRID[below + 1] - a           # nearer to the upper one
    tie = a - GRID[below] == GRID[below + 1] - a
    code = below + np.where(tie, below % 2, up)          # (a tie goes to the even code)
    return (np.sign(b) * GRID[code] * 2.0 ** e).reshape(x.shape)


def held(k, v, theta, weight=None, eps=None):
    """(keys as appended that a PC_MX4 cache attends with, values likewise) for a message's rows k, v [tokens, heads, D]: quantised as
    they are stored, turned to their index, and the keys turned back.  eps None: without norms."""
    k, v = np.asarray(k, np.float64), np.asarray(v, np.float64)
    fine = (np.isfinite(k) & np.isfinite(v)).all(axis=-1)
    at = np.arange(len(k))
    y = np.where(fine[..., None], k, 0)
    y = y if eps is None else norm(y, weight, eps)
    y = rope(to_mx4(rope(y, at, theta)), -at, theta)
    y[~fine] = np.nan                                    # a token that holds what is no number
    return y, np.where(fine[..., None], to_mx4(np.where(fine[..., None], v, 0)), 0)
