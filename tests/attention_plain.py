"""The attention half of a layer in 64-bit numpy, from the definitions in include/itq3s.h: norm and rotation, the rows of the
4-bit cache and where their bits stand, attention row by row."""
import math

import numpy as np

HALF = {"f16": 2.0**-11, "f32": 2.0**-24}  # half a step of a rounding, relative


def hadamard(D):
    i = np.arange(D)
    return np.array([[1 - 2 * (bin(a & b).count("1") & 1) for b in i] for a in i], dtype=np.float64)


_H = {}


def turned(x):
    """H x along the last axis, H orthonormal"""
    D = x.shape[-1]
    if D not in _H:
        _H[D] = hadamard(D)
    return x @ _H[D] / math.sqrt(D)


def coded(x):
    """x [..., D] -> digits (int), steps (fp16), whether the row was not finite"""
    x = np.asarray(x, dtype=np.float64)
    D = x.shape[-1]
    if D not in _H:
        _H[D] = hadamard(D)
    with np.errstate(invalid="ignore", over="ignore"):
        w = x @ _H[D]
        bad = ~np.isfinite(x).all(axis=-1)
        w = np.where(bad[..., None], 0.0, w)
        s = (np.abs(w).max(axis=-1) / (7.5 * math.sqrt(D))).astype(np.float32)
        s = np.minimum(s, np.float32(65504)).astype(np.float16)
        step = s.astype(np.float64)[..., None] * math.sqrt(D)
        c = np.where(step > 0, np.floor(w / np.where(step > 0, step, 1.0) + 0.5), 0.0)
    return np.clip(c, -8, 7).astype(np.int64), s, bad


def stands_for(c, s):
    return turned(c * s.astype(np.float64)[..., None])


def rotated(x, D, weight=None, eps=1e-6, positions=None, freq=None, interleaved=False, gain=1.0):
    """x [T, heads * D] -> the same shape: norm and rotation of every head"""
    x = np.asarray(x, dtype=np.float64).reshape(x.shape[0], -1, D)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(axis=2, keepdims=True) + np.float64(np.float32(eps))) * np.asarray(weight, dtype=np.float64)
    y = x.copy()
    if freq is not None:
        n = len(freq)
        a = np.arange(n) * (2 if interleaved else 1)
        b = a + (1 if interleaved else n)
        angle = positions.astype(np.float64)[:, None, None] * np.asarray(freq, dtype=np.float64)
        cos, sin = gain * np.cos(angle), gain * np.sin(angle)
        y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    return y.reshape(x.shape[0], -1)


class PlainCache:
    """The bytes of a cache, one value at a time by its own address."""

    def __init__(self, pages, page, heads, D, fill=0):
        self.pages, self.page, self.heads, self.D = pages, page, heads, D
        self.block = 32 * D + 128
        self.data = np.full(pages * heads * (page // 32) * self.block, fill, dtype=np.uint8)

    def base(self, slot, head):
        return ((slot // self.page * self.heads + head) * (self.page // 32) + slot % self.page // 32) * self.block

    def places(self, slot, head, value):
        """(byte, shift) of the digits of a row, D of them, and the byte of its step"""
        t, ch, base = slot % 32, np.arange(self.D), self.base(slot, head)
        if not value:
            j = ch % 8
            nib = (j >> 1) + 4 * (j & 1)
            byte, shift = t * self.D // 2 + ch // 8 * 4 + nib // 2, 4 * (nib & 1)
        else:
            h, p, n, c = ch // 64, ch // 32 % 2, ch // 16 % 2, ch % 16
            a, g, b = t // 16, t % 16 // 4, t % 4
            byte, shift = 16 * self.D + 1024 * h + 16 * (16 * g + c) + 8 * p + 4 * a + 2 * (b & 1) + (b >> 1), 4 * n
        return base + byte, shift, base + 32 * self.D + 4 * t + (2 if value else 0)

    def put(self, slot, head, value, digits, step):
        byte, shift, at = self.places(slot, head, value)
        for b, s, c in zip(byte, shift, digits):
            self.data[b] = (int(self.data[b]) & (0xF0 >> s)) | (int(c) + 8) << s
        self.data[at : at + 2] = np.array([step], dtype=np.float16).view(np.uint8)

    def get(self, slot, head, value):
        byte, shift, at = self.places(slot, head, value)
        return (self.data[byte].astype(np.int64) >> shift & 15) - 8, self.data[at : at + 2].copy().view(np.float16)[0]

    def write(self, slots, k, v):
        """k, v [T, heads, D] in 64 bits"""
        for value, x in ((False, k), (True, v)):
            c, s, _ = coded(x)
            for t, slot in enumerate(slots):
                if 0 <= slot < self.pages * self.page:
                    for h in range(self.heads):
                        self.put(int(slot), h, value, c[t, h], s[t, h])

    def rows(self, slots, head, value):
        """-> digits [n, D], steps [n]"""
        got = [self.get(int(s), head, value) for s in slots]
        return np.array([g[0] for g in got]).reshape(-1, self.D), np.array([g[1] for g in got], dtype=np.float16)


def attend(q, k, v, scale):
    """One row over the tokens that it sees: (o, Sum p |v|, the largest Sum |q_i k_i| times |scale|)"""
    if len(k) == 0:
        return np.zeros(len(q)), 0.0, 0.0
    s = scale * (k @ q)
    p = np.exp(s - s.max())
    p /= p.sum()
    return p @ v, float(p @ np.sqrt((v * v).sum(axis=1))), float(abs(scale) * (np.abs(k) @ np.abs(q)).max())


def bound(o, weight, reach):
    """How far (2-norm) a row of fp16 attention may be off.  A score is off by its operands' roundings, at most half a step of fp16
    of Sum |q_i k_i| (and as much again of fp32's for the sums, under 1 % of it), which moves a weight by that
    factor and the sum of weights by as much; a weight is rounded to fp16 once (and weights below fp16's normal range, 2^-14 of a
    row's largest, by 2^-25 of it); the result is rounded once.  Bounds on single values add up to bounds on norms because
    Sum p |v| bounds the norm of a sum of products."""
    d = 1.02 * 2.0**-11 * reach
    return (2 * d + d * d + 1.01 * 2.0**-11 + 2.0**-20) * weight + 1.01 * 2.0**-11 * float(np.sqrt((o * o).sum())) + 2.0**-24 * math.sqrt(len(o))
