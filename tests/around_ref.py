"""Rotary positions, the prompt's attention and the cache in 4 bits in plain
64-bit numpy, straight from the definitions: what the kernels are held to."""
from __future__ import annotations

import math

import numpy as np

HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}     # half a step of a rounding, relative
h = 2.0 ** -24


# ---- rotary positions

def frequencies(r, base, scaling="plain", factor=1.0, trained=0, fast=32.0, slow=1.0):
    """Radians a token of every pair, and the magnitude."""
    if scaling == "ntk":
        base = base * factor ** (r / (r - 2))
    w = np.array([base ** (-2.0 * i / r) for i in range(r // 2)])
    if scaling == "linear":
        return w / factor, 1.0
    if scaling == "yarn":
        g = np.clip((trained * w / (2 * math.pi) - slow) / (fast - slow), 0.0, 1.0)
        return (1 - g) * w / factor + g * w, 0.1 * math.log(factor) + 1.0
    return w, 1.0


def rotate(x, pos, f, m, layout, dtype, sections=None, weight=None, eps=0.0):
    """x [T, H, d] at positions [T] or [3, T]: the outputs and their error bounds.

    cos and sin are off by at most 8 half steps (the reduced angle's rounding, a
    polynomial of values up to 1, the magnitude) and by what 64 bits leave of the
    angle; a product and a sum of two add 2 more; a normalised head is off by a
    sum of d squares over chains of 16 and 3 joins, halved by the root, and six
    more roundings."""
    d, r = x.shape[-1], 2 * len(f)
    y = x.astype(np.float64)
    spread = 0.0
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * weight
        spread = 16 * h
    if sections is None:
        p = np.repeat(np.asarray(pos, np.float64)[:, None], r // 2, 1)
    else:
        row = np.repeat(np.arange(3), sections)
        p = np.asarray(pos, np.float64)[row].T
    t = p * f
    c, s = (m * np.cos(t))[:, None], (m * np.sin(t))[:, None]
    i = np.arange(r // 2)
    a, b = (i, i + r // 2) if layout == "half" else (2 * i, 2 * i + 1)
    out, tol = y.copy(), np.abs(y) * spread
    both = np.abs(y[..., a]) + np.abs(y[..., b])
    near = m * both * (10 * h + spread + 4 * 2.0 ** -53 * np.abs(t)[:, None])
    out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    tol[..., a], tol[..., b] = near, near
    copied = np.arange(d) >= r
    tol = 1.01 * tol + HALF[dtype] * np.abs(out) * ~(copied & (weight is None))
    return out, tol


# ---- attention

def attend(q, k, v, ends, dtype):
    """Queries q [m, d] of one head over rows k, v [n, d], query j seeing the first
    ends[j]: out, lse and the error bounds of both.

    In 32 bits: a logit is a sum of d products, off by at most (d + 8) half steps
    of sum |q_i k_i|; a weight by that (twice: its own and its maximum's), by its
    exponential's argument (4 half steps of it and of 8 powers of two) and by
    its rounding to bfloat16 where the second product takes it so; a sum of
    weights runs over chains of at most n / 2 + 64 terms."""
    d, n = q.shape[1], len(k)
    c = 1.0 / math.sqrt(d)
    out, lse = np.zeros((len(q), v.shape[1])), np.full(len(q), -np.inf)
    tol, ltol = np.zeros_like(out), np.zeros(len(q))
    for e in np.unique(ends):
        rows = np.nonzero(ends == e)[0]
        if e <= 0:
            continue
        kk, vv = k[:e], v[:e]
        s = c * (q[rows] @ kk.T)
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        z = p.sum(1, keepdims=True)
        out[rows], lse[rows] = (p / z) @ vv, (top + np.log(z))[:, 0]
        size = c * (np.abs(q[rows]) @ np.abs(kk).T).max(1)
        logit = (d + 8) * h * size + 4 * h * (top[:, 0] - s.min(1)) + 4 * h * np.abs(top[:, 0])
        chain = (e / 2 + 64) * h
        weight = 2 * logit + 32 * h
        each = weight + (2.0 ** -8 if dtype == "bf16" else 0.0)
        mass = (p / z) @ np.abs(vv)
        tol[rows] = HALF[dtype] * np.abs(out[rows]) + ((each + weight + 2 * chain)[:, None]) * mass * 1.01
        ltol[rows] = logit + weight + chain + 4 * h * np.abs(lse[rows]) + 8 * h
    return out, lse, tol, ltol


# ---- the cache in 4 bits

def attend_held(attend, q, k, v, dtype):
    """cache_ref.attend for values that may be 0 exactly, as codes of e2m1 often
    are: where the largest weight's value is 0, an output is made of weights that
    a float need not hold.  A weight below 2^-126, and each of its up to three
    parts, may count as 0: 4 2^-126 sum |v| more."""
    out, lse, tol, ltol = attend(q, k, v, dtype)
    return out, lse, tol + 4 * 2.0 ** -126 * np.abs(v).sum(0), ltol


LOW, HIGH = -100, 125
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def exponents(x):
    """Of every 32 values [.., 32]: the smallest e with max |x| <= 6 2^e, within bounds."""
    a = np.abs(x).max(-1)
    out = np.full(a.shape, LOW)
    for at in np.ndindex(a.shape):
        if a[at] > 0:
            e = math.frexp(a[at])[1] - 5
            while 6.0 * 2.0 ** e < a[at]:
                e += 1
            out[at] = min(max(e, LOW), HIGH)
    return out


def held(x):
    """Rows [n, d] as the cache holds them."""
    x = np.asarray(x, np.float64)
    y = x.reshape(*x.shape[:-1], -1, 32)
    scale = 2.0 ** exponents(y)[..., None].astype(np.float64)
    z = np.abs(y) / scale
    lo = np.clip(np.searchsorted(E2M1, z, side="right") - 1, 0, 6)
    below, above = z - E2M1[lo], E2M1[lo + 1] - z
    up = (above < below) | ((above == below) & (lo % 2 == 1))
    return (np.sign(y) * E2M1[lo + up] * scale).reshape(x.shape)


class Rows4:
    """K or V of one pair, with the interface of the 8-bit reference's Rows."""

    def __init__(self, bt, d):
        self.x = np.zeros((0, d))

    def store(self, x):
        self.x = held(x)

    def append(self, new):
        if len(new):
            self.x = np.concatenate([self.x, held(new)])

    def cut(self, n):
        self.x = self.x[:n]

    def __len__(self):
        return len(self.x)
