"""Attention over the 4-bit cache where a call is cut into chunks of positions (GPU).

A call is one chunk a CTA, a cluster of up to 8 chunks or more chunks joined by a
second kernel, by its sizes; what a row gets must not depend on which."""
import numpy as np
import pytest

from oracle import beam as ob
from test_gpu_beam_ops import ATT, _attend_case, _check_rows, _dev, _err, _filled, _i32, _pool, _rows_of

pytestmark = pytest.mark.gpu

# positions of one sequence of one head: one chunk, a cluster of 6, a second kernel
CUTS = [200, 1500, 5000]


def _run(cache, lens, q, rps, heads, causal, scale, dtype, table=None, most=None):
    """One call; every sequence has its own blocks in order unless `table` says otherwise."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    n, dim, bs = len(lens), cache.groups * 64, cache.bs
    most = most or max(lens)
    if table is None:
        cols = -(-max(lens) // bs)
        table = np.arange(n * cols).reshape(n, cols)
    out, err = torch.full((n * rps, q.shape[1]), 7.0, dtype=_dev(torch, q[:1], dtype).dtype, device="cuda"), _err(torch)
    nb = B.wf_kv4_attention_scratch_bytes(n, rps, heads, cache.heads, dim, most)
    sc = torch.empty(max(nb, 16), dtype=torch.uint8, device="cuda")
    B.wf_kv4_attention(_pool(B, _dev(torch, cache.raw), cache), 0, _dev(torch, q, dtype), q.shape[1], _i32(torch, table), table.shape[1],
                       _i32(torch, lens), n, rps, heads, causal, scale, most, out, q.shape[1], sc, nb, err)
    assert err.item() == 0
    return out.float().cpu().numpy().astype(np.float64), table


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", CUTS)
def test_a_nan_query_gives_a_nan_row(n, dim, dtype):
    """A query that is not finite has no finite score, so its row is NaN, and no other row is."""
    rng = np.random.default_rng(n + dim)
    cache = _filled(rng, -(-n // 16), 16, 1, dim, dtype)
    q = ob.round16(rng.normal(size=(3, dim)), dtype)
    bad = q.copy()
    bad[1, 5] = np.nan
    got, table = _run(cache, [n], bad, 3, 1, 0, 0.125, dtype)
    assert np.isnan(got[1]).all()
    got[1] = _run(cache, [n], q, 3, 1, 0, 0.125, dtype)[0][1]
    _check_rows(got, cache, table, [n], q, 3, 1, 1, 0, 0.125, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", CUTS)
def test_nan_keys_reach_every_row_that_sees_them(n, dtype):
    """A whole chunk (or a whole warp's step) of keys that read back as NaN makes the rows that see it NaN; a head
    beside it, and a causal row that ends before it, keep their values."""
    rng = np.random.default_rng(n)
    rps = 2
    cache = _filled(rng, -(-n // 16), 16, 2, 64, dtype)
    q = ob.round16(rng.normal(size=(rps, 128)), dtype)
    lo, hi = (64, 128) if n < 256 else (256, 512)
    for pos in range(lo, hi):
        p = ob.scale_place(pos % 16, 0)
        cache.raw[pos // 16, 0, 0, p:p + 4] = 0xFF
    got, table = _run(cache, [n], q, rps, 2, 0, 0.125, dtype)
    assert np.isnan(got[:, :64]).all() and np.isfinite(got[:, 64:]).all()
    # causal, two sequences on the same blocks: one ends before the NaN keys
    cols = -(-n // 16)
    got, table = _run(cache, [lo, n], np.concatenate([q, q]), rps, 2, 1, 0.125, dtype, np.tile(np.arange(cols), (2, 1)))
    assert np.isnan(got[2:, :64]).all() and np.isfinite(got[2:, 64:]).all()
    _check_rows(got[:2], cache, table[:1], [lo], q, rps, 2, 2, 1, 0.125, dtype)


# ------------------------------------------------------- value scales of any size --
def _cache_of(rng, kz, vs, codes, dtype, bs=64):
    """One head whose keys are constant rows (s 0, z of group 0 from kz, else 0) and whose values are codes times vs, z 0.
    kz [n], vs [n, groups], codes [n, groups, 64] of 0 .. 15."""
    n, groups = vs.shape
    blocks = -(-n // bs)
    cache = ob.Cache(blocks, bs, 1, groups * 64, dtype)
    full = blocks * bs
    sz = np.zeros((full, groups, 2, 2), np.float32)          # [position][group][keys, values][s, z]
    sz[:n, 0, 0, 1], sz[:n, :, 1, 0] = kz, vs
    bits = ob.bits16(ob.round16(sz, dtype), dtype).reshape(blocks, bs // 16, 2, 8, groups, 2, 2)
    cache.raw[..., 1024:] = np.ascontiguousarray(bits.transpose(0, 4, 1, 3, 5, 2, 6)).view(np.uint8).reshape(blocks, groups, bs // 16, 128)
    place = np.array([[ob.code_place(p, d, 1) for d in range(64)] for p in range(16)])
    rec, pos = cache.raw.reshape(blocks, groups, bs // 16, ob.RECORD), np.arange(n)
    for p16 in range(16):
        at = pos[pos % 16 == p16]
        low = codes[at][:, :, 0::2] | codes[at][:, :, 1::2] << 4         # dims 2 i and 2 i + 1 share a byte
        for i in range(32):
            rec[at // bs, :, at % bs // 16, place[p16, 2 * i, 0]] = low[:, :, i]
    s = ob.round16(vs, dtype).astype(np.float64)
    return cache, ob.round16(kz, dtype).astype(np.float64), (s[:, :, None] * (codes - 8.0)).reshape(n, -1)


def _scales(kind, rng, n):
    """(scores, value scales [n, 2], codes [n, 2, 64])."""
    x, s, codes = rng.uniform(-6, 0, n), 0.1 * rng.uniform(1, 1.1, (n, 2)), rng.integers(0, 16, (n, 2, 64))
    if kind in ("sink", "faint"):          # one position that dominates, its neighbours' scales 64 times the rest's
        x = np.full(n, -16 * np.log(2) if kind == "sink" else -19.2 * np.log(2))
        x[0], s[:32], codes[:] = 0, s[:32] * 64, rng.integers(12, 16, codes.shape)
        codes[0] = 8
    elif kind == "groups":                 # the groups of a head 2^11 apart
        s[:, 1] *= 2.0 ** -11
    elif kind == "outlier":                # a value near the type's end, of no weight, among small ones
        s *= 2.0 ** -7
        s[::29], x[::29] = 8000, -40
    elif kind == "drift":                  # every 32 positions another size, growing and shrinking
        s = (2.0 ** rng.uniform(-18, 12, (-(-n // 32), 2))).repeat(32, 0)[:n] * rng.uniform(1, 1.9, (n, 2))
    elif kind == "any":                    # every position its own, some of them 0
        s = np.where(rng.random((n, 2)) < 0.1, 0, 2.0 ** rng.uniform(-20, 13, (n, 2)))
    return x, s, codes


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rps", [1, 9])
@pytest.mark.parametrize("kind,n,n_seq", [("sink", 65536, 1300), ("faint", 65536, 1300), ("groups", 3000, 1300), ("groups", 700, 1),
                                          ("outlier", 3000, 1300), ("outlier", 20000, 1), ("drift", 3000, 1300), ("drift", 1500, 1),
                                          ("any", 3000, 1300), ("any", 5000, 2)])
@pytest.mark.parametrize("dim", [64, 128])
def test_value_scales_of_any_size(kind, n, n_seq, rps, dim, dtype):
    """The weights' rounding is relative to each weight and its own scale, whatever the other scales are.  1300
    sequences (on one table) leave each warp a quarter of the positions to walk; one sequence is cut into chunks.

    out = sum(w (sc + z)), sc = s (c - 8), z = 0.  The output is rounded once (u), each weight times s once (u, for fp16
    at least 2^-25 of s off for a weight relative to the row's largest); a score of size |x| is off by a few 2^-24 |x|
    and the exponential by 2^-22, so weights by e = 2^-20 (1 + |x|); n / 64 tensor products of a warp and the joins add
    in fp32, each addition to 2^-23 of sums no larger than that of the magnitudes."""
    rng = np.random.default_rng(n + dim)
    groups = dim // 64
    x, s, codes = _scales(kind, rng, n)
    cache, kz, sc = _cache_of(rng, x, s[:, :groups], codes[:, :groups], dtype)
    q = np.zeros((rps, dim))
    q[:, 0] = (1, 0.5, 2, 0.25, 1.5, 0.75, 0, 1, 1.25)[:rps]
    got, _ = _run(cache, [n] * n_seq, np.tile(q, (n_seq, 1)), rps, 1, 0, 1.0, dtype, np.tile(np.arange(cache.raw.shape[0]), (n_seq, 1)))
    got = got.reshape(n_seq, rps, dim)
    assert (got == got[:1]).all()
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
    for j in range(rps):
        y = q[j, 0] * kz
        p = np.exp(y - y.max())
        w = p / p.sum()
        want, size = w @ sc, w @ np.abs(sc)
        tol = 1.01 * u * np.abs(want) + (u + 2.0 ** -19 * (1 + np.abs(y).max()) + n / 64 * 2.0 ** -23) * size
        if dtype == "f16":
            tol += 2.0 ** -25 * (1 + np.abs(sc).sum(0) / p.sum())
        off = np.abs(got[0, j] - want)
        assert (off <= tol).all(), (j, (off / tol).max(), off.max())


# ---------------------------------------------------------- every position, once --
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rps,heads,dim,bs,causal,lens", [
    (1, 1, 64, 16, 1, [30011]), (1, 3, 64, 64, 1, [9000, 1, 0, 5000]), (4, 1, 128, 32, 1, [4000, 77, 2500]), (9, 2, 64, 16, 0, [1500, 1499, 17]),
    (5, 1, 128, 16, 0, [2047]), (20, 1, 64, 32, 1, [700, 5, 333]), (3, 20, 64, 16, 1, [(37 * i) % 460 for i in range(90)])])
def test_every_position_counts_once(rps, heads, dim, bs, causal, lens, dtype):
    """Queries of zeros weigh every position seen by exactly 1, and values of whole numbers add up exactly, so the
    output is the whole number sum / count but for its last rounding (and the quotient's, by a reciprocal): a position
    dropped, doubled or taken from beyond the length shows, in any chunk, step or record."""
    rng = np.random.default_rng(len(lens) + dim)
    cols = -(-max(max(lens), 1) // bs)
    table = rng.permutation(len(lens) * cols).reshape(len(lens), cols)
    cache = _filled(rng, len(lens) * cols, bs, heads, dim, dtype)
    pairs = np.ascontiguousarray(cache.raw[..., 1024:]).view(np.uint16).reshape(*cache.raw.shape[:3], 8, 2, 2, 2)
    pairs[..., 1, :, 0] = ob.bits16(np.float32(1), dtype)                          # values: s 1, z a whole number
    pairs[..., 1, :, 1] = ob.bits16(rng.integers(-3, 4, pairs.shape[:4] + (2,)).astype(np.float32), dtype)
    cache.raw[..., 1024:] = pairs.view(np.uint8).reshape(*cache.raw.shape[:3], 128)
    q = np.zeros((len(lens) * rps, heads * dim), np.float32)
    got, _ = _run(cache, lens, q, rps, heads, causal, 1.0, dtype, table, max(lens))
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
    for s, n in enumerate(lens):
        for h in range(heads):
            _, v = _rows_of(cache, table[s], n, h)
            for j in range(rps):
                m = max(n - (rps - 1 - j) if causal else n, 0)
                want = v[:m].sum(0) / max(m, 1)
                # the output's rounding, the reciprocal's and the product's; below fp16's normal range its spacing
                tol = np.abs(want) * (u + 2.0 ** -22) + (2.0 ** -25 if dtype == "f16" else 0)
                off = np.abs(got[s * rps + j, h * dim:(h + 1) * dim] - want)
                assert (off <= tol).all(), (s, h, j, off.max())


# --------------------------------------------------- every rounding, and no more --
def _pairs(cache, table, length, head):
    """(s, z) of keys and of values [length, groups] each."""
    pos = np.arange(length)
    rec = cache.raw[table[pos // cache.bs], head * cache.groups:(head + 1) * cache.groups, pos % cache.bs // 16]
    out = []
    for is_v in (0, 1):
        at = np.array([ob.scale_place(p, is_v) for p in range(16)])[pos % 16]
        raw = np.stack([rec[np.arange(length), :, at + b] for b in range(4)], -1)
        sz = ob.from_bits16(np.ascontiguousarray(raw).view(np.uint16), cache.dtype).astype(np.float64)
        out += [sz[..., 0], sz[..., 1]]
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("i", range(len(ATT)))
def test_attention_is_off_by_its_roundings_alone(i, dtype):
    """out = sum w_j (sc_j + z_j) with sc = s (c - 8).  A score's error d_j moves the output by sum w_j d_j (v_j - out).
    d_j: products of queries with codes of up to 8 around a bias that is taken off again (136 for bf16, 72 for half of
    them in fp16), eight additions each to 2^-24 of at most s B sum|q|, the same for z; and 2^-22 of the score and of its
    exponential.  Weights times s are rounded once (2^-8 for bf16, 2^-11 for fp16 or 2^-25 of s), the output once; the
    tensor products of a warp and the joins add n / 64 times to 2^-23."""
    rps, hq, hkv, dim, bs, causal, lens = ATT[i]
    cache, table, q = _attend_case(i, dtype)
    scale, g = dim ** -0.5, hq // hkv
    got, _ = _run(cache, lens, q, rps, hq, causal, scale, dtype, table, max(1, max(lens)))
    u, bias = (2.0 ** -8, 144) if dtype == "bf16" else (2.0 ** -11, 80)
    worst = 0
    for s, n in enumerate(lens):
        for head in range(hkv):
            k, v = _rows_of(cache, table[s], n, head)
            ks, kz, vs, vz = _pairs(cache, table[s], n, head)
            z = vz.repeat(64, 1)
            sc = v - z
            for j in range(rps):
                m = max(n - (rps - 1 - j) if causal else n, 0)
                for e in range(g):
                    cols = slice((head * g + e) * dim, (head * g + e + 1) * dim)
                    out, row = got[s * rps + j, cols], q[s * rps + j, cols].astype(np.float64)
                    if not m:
                        assert (out == 0).all()
                        continue
                    x = k[:m] @ row * scale
                    p = np.exp(x - x.max())
                    w, size = p / p.sum(), np.abs(row).reshape(-1, 64).sum(1)
                    d = 8 * 2.0 ** -24 * scale * ((2 * bias * ks[:m] + np.abs(kz[:m])) @ size) + 2.0 ** -22 * (1 + np.abs(x))
                    want = w @ v[:m]
                    tol = 1.01 * u * np.abs(want) + u * (w @ np.abs(sc[:m])) + (w * d) @ np.abs(v[:m] - want) \
                        + m / 64 * 2.0 ** -23 * (w @ (np.abs(sc[:m]) + np.abs(z[:m])))
                    if dtype == "f16":
                        tol = tol + 2.0 ** -25 * (1 + np.abs(sc[:m]).sum(0) / p.sum())
                    worst = max(worst, (np.abs(out - want) / tol).max())
    assert worst <= 1, worst
