"""The 8-bit cache in plain 64-bit numpy: what the kernels are held to.  One
(layer, sequence, KV head) at a time, straight from the definitions."""
from __future__ import annotations

import math

import numpy as np

LOW, HIGH = -100, 120
# the nonnegative e4m3 values in the order of their codes (0 .. 126)
E4M3 = np.array([m * 2.0 ** -9 for m in range(8)] +
                [(8 + m) * 2.0 ** (x - 10) for x in range(1, 16) for m in range(8)])[:127]
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}     # half a step of a rounding, relative


def exponent(a):
    """The smallest integer e with a <= 448 2^e, held to its bounds."""
    if a == 0.0:
        return LOW
    e = math.frexp(a)[1] - 12
    while 448.0 * 2.0 ** e < a:
        e += 1
    return min(max(e, LOW), HIGH)


def round8(x, e):
    """x rounded to the nearest code times 2^e, ties to the even code."""
    y = np.abs(x) / 2.0 ** e
    lo = np.clip(np.searchsorted(E4M3, y, side="right") - 1, 0, 125)
    below, above = y - E4M3[lo], E4M3[lo + 1] - y
    up = (above < below) | ((above == below) & (lo % 2 == 1))
    return np.sign(x) * E4M3[lo + up] * 2.0 ** e


class Rows:
    """K or V of one pair: the values held, and the exponent of every block."""

    def __init__(self, bt, d):
        self.bt, self.x, self.e = bt, np.zeros((0, d)), []

    def store(self, x):
        self.x, self.e = np.zeros(x.shape), []
        for i in range(0, len(x), self.bt):
            part = x[i:i + self.bt].astype(np.float64)
            self.e.append(exponent(np.abs(part).max()))
            self.x[i:i + self.bt] = round8(part, self.e[-1])

    def append(self, new):
        new = new.astype(np.float64)
        while len(new):
            old = len(self.x) % self.bt
            part, new = new[:self.bt - old], new[self.bt - old:]
            e = exponent(np.abs(part).max())
            base = len(self.x) - old
            if old:
                e = max(e, self.e[base // self.bt])
            del self.e[base // self.bt:]
            self.e.append(e)
            self.x = np.concatenate([self.x[:base], round8(np.concatenate([self.x[base:], part]), e)])

    def cut(self, n):
        """The first n rows; a scale that grew for the others stays."""
        self.x = self.x[:n]
        del self.e[(n + self.bt - 1) // self.bt:]

    def __len__(self):
        return len(self.x)


def attend(q, k, v, dtype):
    """One query over rows k, v: out, lse and the error bounds of both.

    The kernels work in 32 bits: a logit is a sum of d products, so it is off
    by at most (d + 8) half steps of sum |q_i k_i| (scale and split of q among
    them); a weight is off by that logit's error (twice: its own and the
    maximum's), the exponential (4 half steps of its argument) and the split of
    the weight (2^-16 of it for bf16 outputs, where it travels as two bf16
    parts); sums run over chains of at most n / 16 + 64 terms."""
    d, n = q.shape[0], len(k)
    if n == 0:
        return np.zeros(v.shape[1]), -np.inf, np.zeros(v.shape[1]), 0.0
    c = 1.0 / math.sqrt(d)
    s = c * (k @ q)
    top = s.max()
    p = np.exp(s - top)
    z = p.sum()
    out, lse = (p / z) @ v, top + math.log(z)
    h = 2.0 ** -24
    logit = (d + 8) * h * c * (np.abs(k) @ np.abs(q)).max() + 4 * h * (top - s.min())
    chain = (n / 16 + 64) * h
    weight = 2 * logit + 8 * h + (2.0 ** -16 if dtype == "bf16" else 2.0 ** -22)
    mass = (p / z) @ np.abs(v)
    return out, lse, HALF[dtype] * np.abs(out) + (2 * weight + 2 * chain) * mass * 1.01, \
        logit + weight + chain + 4 * h * abs(lse) + 8 * h
