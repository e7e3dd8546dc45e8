"""Rotary positions, attention of packed prompts and the paged 8-bit cache, restated in numpy.

Loops over rows, heads and positions; float64, codes from the list of e4m3
values.  Shares no code with the CUDA path.
"""
from __future__ import annotations

import math

import numpy as np

LOW, HIGH = -60, 36

# the 128 magnitudes of e4m3 (fn): the last is NaN
E4M3 = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)])
E4M3[127] = np.nan


# --------------------------------------------------------------- positions --
def frequencies(rot, base=10000.0, scaling="plain", factor=1.0, trained_len=0.0, low=0.0, high=0.0):
    """Radians a position of each pair."""
    if scaling == "base" and rot > 2:
        base *= factor ** (rot / (rot - 2))
    out = []
    for i in range(rot // 2):
        f = base ** (-2 * i / rot)
        if scaling == "linear":
            f /= factor
        elif scaling == "waves":
            w = min(max((f * trained_len / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            f = w * f + (1 - w) * f / factor
        elif scaling == "parts":
            a, b = (rot * math.log(trained_len / (2 * math.pi * n)) / (2 * math.log(base)) for n in (high, low))
            a, b = max(math.floor(a), 0), min(math.ceil(b), rot - 1)
            w = min(max((i - a) / max(b - a, 0.001), 0.0), 1.0)
            f = w * f / factor + (1 - w) * f
        out.append(f)
    return np.array(out)


def rope(x, pos, freq, interleaved=False, gain=1.0, adjoint=False):
    """x [n, heads, dim] float64."""
    y = np.array(x, np.float64)
    half = len(freq)
    for i, p in enumerate(pos):
        for j, f in enumerate(freq):
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
            angle = math.fmod(int(p) * f, 2 * math.pi) * (-1 if adjoint else 1)
            c, s = math.cos(angle) * gain, math.sin(angle) * gain
            y[i, :, a], y[i, :, b] = x[i, :, a] * c - x[i, :, b] * s, x[i, :, a] * s + x[i, :, b] * c
    return y


# --------------------------------------------------------------- attention --
def attention(q, k, v, scale, ends):
    """q [r, hq, d], k and v [t, hkv, d]; row i sees the first ends[i] positions.
    Output, log of the sums and sum of |weight * value| (for tolerances)."""
    r, hq, d = q.shape
    g = hq // k.shape[1]
    out, lse, mass = np.zeros((r, hq, d)), np.full((r, hq), -np.inf), np.zeros((r, hq, d))
    for i in range(r):
        n = min(max(int(ends[i]), 0), len(k))
        for h in range(hq):
            if n == 0:
                continue
            x = k[:n, h // g] @ q[i, h] * scale
            top = x.max()
            if top == -np.inf:
                continue
            e = np.exp(x - top)
            lse[i, h] = top + math.log(e.sum())
            w = e / e.sum()
            out[i, h], mass[i, h] = w @ v[:n, h // g], w @ np.abs(v[:n, h // g])
    return out, lse, mass


# --------------------------------------------------------------- the cache --
def code_of(x):
    """The code of a float64 with |x| <= 448 (beyond: 448), nearest, ties to the even code; NaN 127."""
    if not np.isfinite(x):
        return 127
    a = min(abs(x), 448.0)
    i = int(np.argmin(np.abs(E4M3[:127] - a)))
    for j in (i - 1, i + 1):
        if 0 <= j < 127 and abs(E4M3[j] - a) == abs(E4M3[i] - a) and j % 2 == 0:
            i = j
    return i | (128 if np.signbit(x) else 0)


def value_of(c):
    return -E4M3[c & 127] if c & 128 else E4M3[c & 127]


def place(d, p, is_value):
    """Byte of dim d and position p in a record."""
    if not is_value:
        return d // 64 * 2048 + p * 64 + d % 64
    d0 = d % 64
    return (d // 64 * 2048 + 1024 + 512 * (d0 // 2 % 2) + 64 * (d0 // 8) + 16 * (p // 2 % 4) + 8 * (d0 % 2) + 4 * (p // 8) + 2 * (d0 // 4 % 2) + p % 2)


class Cache:
    """One layer: bytes [blocks][heads][block_size / 16][32 dim + 16]."""

    def __init__(self, blocks, block_size, heads, dim, fill=0):
        self.bs, self.heads, self.dim = block_size, heads, dim
        self.raw = np.full((blocks, heads, block_size // 16, 32 * dim + 16), fill, np.uint8)

    def record(self, slot, head):
        return self.raw[slot // self.bs, head, slot % self.bs // 16]

    def scales(self, slot, head):
        return self.record(slot, head)[32 * self.dim:32 * self.dim + 8].copy().view(np.float32).astype(np.float64)

    def store(self, slots, k, v):
        """Rows k, v [n, heads, dim] float64 at slots, record by record; up to 31 skipped rows between a record's do not part them."""
        i = 0
        while i < len(slots):
            if slots[i] < 0:
                i += 1
                continue
            j, last = i, i
            while j < len(slots) and j - last <= 32 and (slots[j] < 0 or slots[j] // 16 == slots[i] // 16):
                last = j if slots[j] >= 0 else last
                j += 1
            rows = {int(slots[r]) % 16: r for r in range(i, last + 1) if slots[r] >= 0}
            for h in range(self.heads):
                for is_v, x in enumerate((k, v)):
                    self._write(int(slots[i]), h, is_v, {p: x[r, h] for p, r in rows.items()})
            i = j

    def _write(self, slot, head, is_v, new):
        rec, first = self.record(slot, head), min(new)
        fin = np.concatenate([np.abs(x[np.isfinite(x)]) for x in new.values()] + [np.zeros(1)])
        e = next((e for e in range(LOW, HIGH) if fin.max() <= 448 * 2.0 ** e), HIGH)
        old = 0
        if first:
            old = int(np.log2(self.scales(slot, head)[is_v]))
            e = max(e, old)
        where = np.array([[place(d, p, is_v) for d in range(self.dim)] for p in range(16)])
        for p in range(16):
            if p < first:
                x = np.array([value_of(c) for c in rec[where[p]]]) * 2.0 ** (old - e)
            else:
                x = new[p] * 2.0 ** -e if p in new else np.zeros(self.dim)
            rec[where[p]] = [code_of(u) for u in x]
        tail = rec[32 * self.dim:].view(np.float32)
        tail[is_v], tail[2], tail[3] = 2.0 ** e, 0, 0

    def row(self, slot, is_v):
        """[heads, dim] float64."""
        out = []
        for h in range(self.heads):
            rec, s = self.record(slot, h), self.scales(slot, h)[is_v]
            out.append([value_of(rec[place(d, slot % 16, is_v)]) * s for d in range(self.dim)])
        return np.array(out)
