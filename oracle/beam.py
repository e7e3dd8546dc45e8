"""Beam decode over a paged 4-bit cache, restated in numpy.

Loops over requests, beams and positions, one at a time; attention and scores
in float64, the quantiser in float32 as its definition asks.  Shares no code
with the CUDA path.
"""
from __future__ import annotations

import numpy as np

GROUP, RECORD = 64, 1152


# ------------------------------------------------------------- 16-bit types --
def round16(x, dtype):
    """float32 values rounded to the nearest bf16 or fp16, as float32."""
    x = np.asarray(x, np.float32)
    if dtype == "f16":
        with np.errstate(over="ignore"):
            return x.astype(np.float16).astype(np.float32)
    u = x.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32)
    return np.where(np.isnan(x), np.float32(np.nan), r.view(np.float32)).astype(np.float32)


def bits16(x, dtype):
    x = np.asarray(x, np.float32)
    if dtype == "f16":
        return x.astype(np.float16).view(np.uint16)
    return (x.view(np.uint32) >> 16).astype(np.uint16)


def from_bits16(u, dtype):
    u = np.asarray(u, np.uint16)
    if dtype == "f16":
        return u.view(np.float16).astype(np.float32)
    return (u.astype(np.uint32) << 16).view(np.float32)


# ---------------------------------------------------------------- the cache --
def quantise(group, dtype):
    """64 values -> (codes 0..15, s, z)."""
    x = np.asarray(group, np.float32)
    if not np.isfinite(x).all():
        return np.full(GROUP, 8), np.float32(np.nan), np.float32(np.nan)
    hi, lo = x.max(), x.min()
    s = round16((np.float32(0.5) * hi - np.float32(0.5) * lo) / np.float32(7.5), dtype)[()]
    z = round16(hi - np.float32(7) * s, dtype)[()]
    if not s > 0:
        return np.full(GROUP, 8), s, z
    c = np.clip(np.rint((x - z) / s), -8, 7).astype(int) + 8
    return c, s, z


def code_place(position, dim, is_value):
    """(byte, nibble) of a code in its record of 16 positions."""
    if not is_value:
        return position * 32 + dim // 2, dim % 2
    lane = dim // 8 * 4 + position % 8 // 2
    word = position // 8 * 2 + dim // 4 % 2
    return 512 + lane * 16 + word * 4 + position % 2 * 2 + dim % 4 // 2, dim % 2


def scale_place(position, is_value):
    return 1024 + position % 8 * 16 + is_value * 8 + position // 8 * 4


class Cache:
    """One layer: bytes [blocks][heads * groups][block_size / 16][1152]."""

    def __init__(self, blocks, block_size, heads, dim, dtype, fill=0):
        self.bs, self.heads, self.groups, self.dtype = block_size, heads, dim // GROUP, dtype
        self.raw = np.full((blocks, heads * self.groups, block_size // 16, RECORD), fill, np.uint8)

    def _record(self, slot, slab):
        return self.raw[slot // self.bs, slab, slot % self.bs // 16]

    def put(self, slot, row, is_value):
        pos = slot % 16
        for slab, x in enumerate(np.asarray(row, np.float32).reshape(-1, GROUP)):
            rec = self._record(slot, slab)
            c, s, z = quantise(x, self.dtype)
            for d in range(GROUP):
                byte, nib = code_place(pos, d, is_value)
                rec[byte] = (rec[byte] & 0xF0) | c[d] if nib == 0 else (rec[byte] & 0x0F) | (c[d] << 4)
            rec[scale_place(pos, is_value):][:4] = bits16([s, z], self.dtype).view(np.uint8)

    def get(self, slot, is_value):
        """The row at a slot, float32 (exact: 4-bit codes times 16-bit scales)."""
        pos, out = slot % 16, []
        for slab in range(self.raw.shape[1]):
            rec = self._record(slot, slab)
            s, z = from_bits16(rec[scale_place(pos, is_value):][:4].copy().view(np.uint16), self.dtype)
            c = [rec[b] >> 4 if n else rec[b] & 15 for b, n in (code_place(pos, d, is_value) for d in range(GROUP))]
            out.append(s * (np.array(c, np.float32) - 8) + z)
        return np.concatenate(out)


# ---------------------------------------------------------------- attention --
def attention(q, k, v, scale, seen):
    """q [R, D], k and v [n, D], seen bool [R, n], float64; a row that sees nothing is zeros.
    Returns the output and the weights."""
    x = q @ k.T * scale
    w = np.zeros_like(x)
    for r in range(len(q)):
        if seen[r].any():
            e = np.where(seen[r], np.exp(np.where(seen[r], x[r], -np.inf) - x[r][seen[r]].max()), 0.0)
            w[r] = e / e.sum()
    return w @ v, w


# ------------------------------------------------------------------- tables --
def page_plan(old, new, bs, free, n_free, table, slots_cap, n_blocks):
    """Returns table, offsets, slots, lengths, ids left, (capacity, page) errors."""
    table = np.array(table)
    offsets, slots, lens = [0], [], []
    left, closed, cap_err, page_err = n_free, False, False, False
    if not 0 <= n_free <= n_blocks:
        left, page_err = 0, True
    for i, (a, b) in enumerate(zip(old, new)):
        up = lambda v: -(-v // bs)
        if a < 0 or b < a or up(b) > table.shape[1]:
            page_err = True
            offsets.append(offsets[-1])
            lens.append(a)
            continue
        need = up(b) - up(a)
        if closed or need > left or offsets[-1] + b - a > slots_cap:
            closed = cap_err = True
            offsets.append(offsets[-1])
            lens.append(a)
            continue
        for c in range(up(a), up(b)):
            left -= 1
            table[i, c] = free[left]
        for pos in range(a, b):
            slots.append(table[i, pos // bs] * bs + pos % bs)
        offsets.append(offsets[-1] + b - a)
        lens.append(b)
    return table, offsets, slots + [-1] * (slots_cap - len(slots)), lens, left, (cap_err, page_err)


# ---------------------------------------------------------------- selection --
def beam_select(logits, scores, suppress, eos):
    """logits [beams, vocab] float64, scores [beams].  Returns dict of lists and the ranked scores."""
    W, V = logits.shape
    prop = []
    for w in range(W):
        x = np.where(np.isnan(logits[w]) | (suppress != 0), -np.inf, logits[w])
        m = x.max()
        if not np.isfinite(m):
            continue
        rest = np.log(np.exp(x - m).sum())
        for rank, i in enumerate(sorted(range(V), key=lambda i: (-x[i], i))[:2 * W]):
            total = scores[w] + ((x[i] - m) - rest)
            if total > -np.inf:
                prop.append((-total, w, rank, i))
    prop = sorted(prop)
    ranked = prop[:2 * W]
    go = [(i, w, -v) for v, w, _, i in ranked if i != eos][:W]
    fin = [(w, -v) for k, (v, w, _, i) in enumerate(ranked) if i == eos and k < W]
    go += [(-1, w, -np.inf) for w in range(len(go), W)]
    fin += [(-1, -np.inf)] * (W - len(fin))
    return {"token": [g[0] for g in go], "parent": [g[1] for g in go], "score": [g[2] for g in go],
            "fin_parent": [f[0] for f in fin], "fin_score": [f[1] for f in fin]}, [-p[0] for p in prop[:2 * W + 1]]


# --------------------------------------------------------------- reordering --
def beam_reorder(table, length, parent, bs):
    """One request: table [beams, columns].  Returns the new table (used columns), freed ids in
    order, and the copies (source block, destination block, positions)."""
    W = len(parent)
    full, rem = divmod(length, bs)
    new, moves = np.array(table), []
    over = all(p < 0 for p in parent)
    with_child, keeps = set(), []
    for p in parent:
        keeps.append(p >= 0 and p not in with_child)
        if p >= 0:
            with_child.add(p)
    spare = [w for w in range(W) if w not in with_child]
    for w in range(W):
        for c in range(full):
            new[w, c] = table[parent[w], c] if parent[w] >= 0 else -1
        if rem:
            if keeps[w]:
                new[w, full] = table[parent[w], full]
            else:
                s = spare.pop(0)
                new[w, full] = -1 if over else table[s, full]
                if parent[w] >= 0:
                    moves.append((table[parent[w], full], table[s, full], rem))
    freed = []
    for c in range(full + (rem > 0)):
        held = set(new[:, c])
        for w in range(W):
            b = table[w, c]
            if b >= 0 and b not in held and b not in table[:w, c]:
                freed.append(b)
    return new, freed, moves
