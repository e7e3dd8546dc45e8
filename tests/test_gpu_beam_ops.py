"""Paged 4-bit cache and beam operators against the float64 oracle (GPU)."""
import numpy as np
import pytest

from oracle import beam as ob

pytestmark = pytest.mark.gpu

GUARD = 0xA5


def _torch_dt(torch, dtype):
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype]


def _dev(torch, x, dtype=None):
    if dtype is None:
        return torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to(_torch_dt(torch, dtype))


def _i32(torch, x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _err(torch):
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def _pool(B, raw, cache, layers=1, stride=0):
    blocks = cache.raw.shape[0]
    return B.kv4_pool(raw, layers, blocks, cache.bs, cache.heads, cache.groups * 64,
                      B.WF_F16 if cache.dtype == "f16" else B.WF_BF16, stride)


def _filled(rng, blocks, bs, heads, dim, dtype, garbage=None):
    """A cache with every position written (quickly), but for `garbage` blocks of 0xFF."""
    c = ob.Cache(blocks, bs, heads, dim, dtype, fill=0xFF)
    shape = c.raw.shape[:3]
    c.raw[..., :1024] = rng.integers(0, 256, (*shape, 1024))
    s = np.abs(rng.normal(0.2, 0.1, (*shape, 32, 1))) + 0.01
    z = rng.normal(0, 0.3, (*shape, 32, 1))
    sz = ob.bits16(ob.round16(np.concatenate([s, z], -1), dtype), dtype)
    c.raw[..., 1024:] = np.ascontiguousarray(sz).view(np.uint8).reshape(*shape, 128)
    for b in () if garbage is None else garbage:
        c.raw[b] = 0xFF
    return c


# ------------------------------------------------------------- tables, slots --
PLANS = [
    # (old lengths, new lengths, block size, table columns, ids free, slots)
    ([0], [1], 16, 1, 1, 1),
    ([0], [0], 16, 1, 0, 0),
    ([16], [17], 16, 2, 5, 1),
    ([15, 16, 0, 33], [16, 16, 100, 34], 16, 8, 40, 300),
    ([7, 40, 0], [20, 41, 65], 32, 4, 9, 200),
    ([0, 0, 0], [64, 65, 1], 64, 2, 3, 500),         # the second does not fit; the third is refused too
    ([0, 0, 0], [64, 65, 1], 64, 2, 9, 64),          # the slots run out
    ([5, 9, -1, 3], [4, 200, 2, 9], 16, 4, 9, 90),   # a shrunk, a too long and a negative request among good ones
    ([0, 0], [5, 5], 16, 1, 77, 90),                 # a free count past the stack
]


@pytest.mark.parametrize("case", range(len(PLANS)))
def test_page_plan(case):
    import torch
    from paper_2609_32869_gb300 import binding as B
    old, new, bs, cols, n_free, cap = PLANS[case]
    n, blocks = len(old), 64
    rng = np.random.default_rng(case)
    ids = rng.permutation(blocks)
    table = np.full((n, cols), -1)
    at = 63
    for i, v in enumerate(old):
        for c in range(min(cols, -(-max(v, 0) // bs))):
            table[i, c] = ids[at]
            at -= 1
    want = ob.page_plan(old, new, bs, ids, n_free, table, cap, blocks)
    t, slots = _i32(torch, table), torch.full((cap + 3,), 77, dtype=torch.int32, device="cuda")
    off, ln, left, err = _i32(torch, np.zeros(n + 1)), _i32(torch, np.zeros(n)), _err(torch), _err(torch)
    B.wf_page_plan(_i32(torch, old), _i32(torch, new), n, bs, _i32(torch, ids), blocks, _i32(torch, [n_free]), t, cols, off,
                   slots, cap, ln, left, err)
    np.testing.assert_array_equal(t.cpu().numpy(), want[0])
    np.testing.assert_array_equal(off.cpu().numpy(), want[1])
    np.testing.assert_array_equal(slots.cpu().numpy(), want[2] + [77] * 3)
    np.testing.assert_array_equal(ln.cpu().numpy(), want[3])
    assert left.item() == want[4]
    e = err.item()
    assert (bool(e & B.WF_DEV_ERR_CAPACITY), bool(e & B.WF_DEV_ERR_PAGE)) == want[5]


@pytest.mark.parametrize("n,bs,most", [(300, 16, 40), (1000, 64, 300), (2500, 32, 5), (5, 16, 3000)])
def test_page_plan_many(n, bs, most):
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(n)
    old = rng.integers(0, most, n)
    new = old + rng.integers(0, most, n)
    cols = 2 * most // bs + 1
    used = sum(-(-int(v) // bs) for v in old)
    need = sum(-(-int(v) // bs) for v in new)
    blocks = need + 10
    ids = rng.permutation(blocks)
    table = np.full((n, cols), -1)
    at = blocks - 1
    for i, v in enumerate(old):
        for c in range(-(-int(v) // bs)):
            table[i, c] = ids[at]
            at -= 1
    n_free = blocks - used - (need - used) // 3   # about a third of the requests is refused
    cap = int((new - old).sum()) + 7
    want = ob.page_plan(old.tolist(), new.tolist(), bs, ids, n_free, table, cap, blocks)
    t, slots = _i32(torch, table), _i32(torch, np.zeros(cap))
    off, ln, left, err = _i32(torch, np.zeros(n + 1)), _i32(torch, np.zeros(n)), _err(torch), _err(torch)
    B.wf_page_plan(_i32(torch, old), _i32(torch, new), n, bs, _i32(torch, ids), blocks, _i32(torch, [n_free]), t, cols, off,
                   slots, cap, ln, left, err)
    for got, w in zip((t, off, slots, ln), want):
        np.testing.assert_array_equal(got.cpu().numpy(), w)
    assert left.item() == want[4] and err.item() == B.WF_DEV_ERR_CAPACITY * want[5][0]


@pytest.mark.parametrize("n,share", [(300, 0.5), (1300, 0.9), (1300, 0.0), (5000, 0.3)])
def test_page_plan_many_run_out(n, share):
    """Bad requests among good ones, and a stack that holds a share of what all of them need."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(n)
    new = rng.integers(0, 40, n)
    old = np.where(rng.random(n) < 0.02, new + 1, 0)
    bs, cols, cap = 16, 2, 40 * n
    n_free = int(share * sum(-(-int(b) // bs) for a, b in zip(old, new) if b >= a and -(-int(b) // bs) <= cols))
    blocks = n_free + 5
    ids, table = rng.permutation(blocks), np.full((n, cols), -1)
    want = ob.page_plan(list(old), list(new), bs, ids, n_free, table, cap, blocks)
    t, slots = _i32(torch, table), torch.full((cap,), 77, dtype=torch.int32, device="cuda")
    off, ln, left, err = _i32(torch, np.zeros(n + 1)), _i32(torch, np.zeros(n)), _err(torch), _err(torch)
    B.wf_page_plan(_i32(torch, old), _i32(torch, new), n, bs, _i32(torch, ids), blocks, _i32(torch, [n_free]), t, cols, off,
                   slots, cap, ln, left, err)
    for got, w in zip((t, off, slots, ln), want):
        np.testing.assert_array_equal(got.cpu().numpy(), np.asarray(w))
    assert left.item() == want[4] and err.item() == B.WF_DEV_ERR_CAPACITY | B.WF_DEV_ERR_PAGE


# -------------------------------------------------------------- store, load --
@pytest.mark.parametrize("n,bs,heads,dim,dtype,pad", [
    (1, 16, 1, 64, "bf16", 0), (5, 16, 3, 64, "bf16", 64), (33, 32, 2, 128, "f16", 8), (64, 64, 6, 64, "f16", 0),
    (130, 64, 1, 128, "bf16", 0), (48, 16, 2, 64, "bf16", 0), (17, 16, 5, 64, "f16", 0), (95, 32, 3, 64, "bf16", 8),
])
@pytest.mark.parametrize("order", ["runs", "mixed", "requests"])
def test_store_and_load(n, bs, heads, dim, dtype, pad, order):
    """Bytes equal the oracle's: the quantiser is fp32 arithmetic with every rounding named.
    "runs": consecutive slots from an odd start, the order of a prefill; "mixed": any order, skipped rows;
    "requests": runs that begin at a block, end anywhere and leave rows out, whole records from odd rows on."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(n)
    d, blocks = heads * dim, n // bs + 3
    k, v = (ob.round16(rng.normal(rng.normal(size=(1, d)), 1, (n, d)), dtype) for _ in range(2))
    k[0, :64] = 2.5                                   # a constant group
    v[n // 2, :64] = 0
    v[n - 1, 3] = np.inf
    k[n - 1, d - 1] = np.nan
    big = 3.0e38 if dtype == "bf16" else 65504.0
    k[n // 2, -64:] = ob.round16(np.linspace(-big, big, 64), dtype)   # the range's ends
    slots = np.arange(n) + bs - 3 if order == "runs" else rng.permutation(blocks * bs)[:n]
    if order == "requests":
        slots, at, b = np.full(n, -1), n % 3, 0
        while at < n:
            m = min(int(rng.integers(1, 3 * bs)), n - at, (blocks - b) * bs)
            slots[at:at + m] = b * bs + np.arange(m)
            at, b = at + m + int(rng.integers(0, 3)), b + -(-m // bs)
            if b >= blocks:
                break
    slots = slots.astype(np.int32)
    if order == "mixed" and n > 4:
        slots[1] = -1
    cache = ob.Cache(blocks, bs, heads, dim, dtype, fill=GUARD)
    for i, s in enumerate(slots):
        if s >= 0:
            cache.put(s, k[i], 0)
            cache.put(s, v[i], 1)
    raw = torch.full((cache.raw.size,), GUARD, dtype=torch.uint8, device="cuda")
    pool, err = _pool(B, raw, cache), _err(torch)
    wide = lambda x: _dev(torch, np.concatenate([x, np.full((n, pad), 7.0)], 1), dtype)
    tk, tv, ts = wide(k), wide(v), _i32(torch, slots)
    B.wf_kv4_store(pool, 0, tk, d + pad, tv, d + pad, ts, n, err)
    got = raw.cpu().numpy().reshape(cache.raw.shape)
    # a NaN scale may have any NaN's bits
    def canon(b):
        sz = np.ascontiguousarray(b[..., 1024:]).view(np.uint16)
        nan = np.isnan(ob.from_bits16(sz, dtype))
        return np.where(nan, 0x7FFF, sz)
    np.testing.assert_array_equal(got[..., :1024], cache.raw[..., :1024])
    np.testing.assert_array_equal(canon(got), canon(cache.raw))
    ok, ov = (torch.full((n, d + pad), 9.0, dtype=tk.dtype, device="cuda") for _ in range(2))
    B.wf_kv4_load(pool, 0, ts, n, ok, d + pad, ov, d + pad, err)
    for out, is_v in ((ok, 0), (ov, 1)):
        want = np.stack([ob.round16(cache.get(s, is_v), dtype) if s >= 0 else np.zeros(d, np.float32) for s in slots])
        np.testing.assert_array_equal(out.float().cpu().numpy()[:, :d], want)
        assert (out[:, d:] == 9.0).all()
    assert err.item() == 0


def test_store_skips_slots_out_of_bounds():
    import torch
    from paper_2609_32869_gb300 import binding as B
    cache = ob.Cache(2, 16, 1, 64, "bf16", fill=GUARD)
    raw = torch.full((cache.raw.size + 4096,), GUARD, dtype=torch.uint8, device="cuda")
    x, err = torch.ones(3, 64, dtype=torch.bfloat16, device="cuda"), _err(torch)
    slots = _i32(torch, [-5, 32, 2 ** 31 - 1])
    B.wf_kv4_store(_pool(B, raw, cache), 0, x, 64, x, 64, slots, 3, err)
    assert (raw == GUARD).all() and err.item() == B.WF_DEV_ERR_PAGE
    out = torch.ones(3, 64, dtype=torch.bfloat16, device="cuda")
    B.wf_kv4_load(_pool(B, raw, cache), 0, slots, 3, out, 64, out.clone(), 64, err)
    assert (out == 0).all()


def test_layers_and_offsets_past_32_bits():
    """A layer whose bytes lie past 4 GiB, and a block past 2 GiB in it."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    bs, heads, dim = 64, 20, 64
    block = B.wf_kv4_block_bytes(bs, heads, dim)
    blocks = 3 * 2 ** 30 // block
    stride = blocks * block + 2 ** 31 + 1024
    raw = torch.full((stride + blocks * block,), GUARD, dtype=torch.uint8, device="cuda")
    pool = B.kv4_pool(raw, 2, blocks, bs, heads, dim, B.WF_BF16, stride)
    x = torch.randn(17, heads * dim, device="cuda").bfloat16()
    slots = torch.arange(17, dtype=torch.int32, device="cuda") + (blocks - 1) * bs + 20
    B.wf_kv4_store(pool, 1, x, heads * dim, -x, heads * dim, slots, 17)
    k, v = torch.empty_like(x), torch.empty_like(x)
    B.wf_kv4_load(pool, 1, slots, 17, k, heads * dim, v, heads * dim)
    g = x.float().view(17, heads, 64)
    step = (g.amax(-1) - g.amin(-1)) / 15
    # half a step, the clamp's share, z's rounding and the row's own
    tol = step * 0.57 + 2.0 ** -7 * g.abs().amax(-1)
    assert ((k.float().view_as(g) - g).abs().amax(-1) <= tol).all() and ((v.float().view_as(g) + g).abs().amax(-1) <= tol).all()
    start = stride + (blocks - 1) * block
    assert (raw[:start] == GUARD).all()
    n = torch.tensor([(blocks - 1) * bs + 37 - (blocks - 1) * bs], dtype=torch.int32, device="cuda")
    out = torch.empty_like(x[:1])
    nb = B.wf_kv4_attention_scratch_bytes(1, 1, heads, heads, dim, 64)
    sc = torch.empty(max(nb, 256), dtype=torch.uint8, device="cuda")
    table = torch.tensor([blocks - 1], dtype=torch.int32, device="cuda")
    raw[start:start + block] = 0
    B.wf_kv4_store(pool, 1, x, heads * dim, -x, heads * dim, slots, 17)
    B.wf_kv4_attention(pool, 1, torch.zeros_like(x[:1]), heads * dim, table, 1, n, 1, 1, heads, 0, 1.0, 64, out, heads * dim, sc, nb)
    # zero queries: the mean over 37 positions, the first 20 of them zeros
    want = v.float().sum(0) / 37
    assert (out.float()[0] - want).abs().max() <= 2.0 ** -7 * 1.0


# ---------------------------------------------------------------- attention --
ATT = [
    # (rows, query heads, kv heads, dim, block, causal, lengths)
    (1, 1, 1, 64, 16, 1, [1]),
    (1, 2, 2, 64, 16, 1, [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257]),
    (5, 3, 3, 64, 64, 0, [1500]),
    (5, 2, 2, 64, 32, 0, [0, 3, 64, 100]),
    (9, 2, 2, 64, 16, 1, [0, 1, 8, 9, 10, 70, 300]),          # fewer positions than rows: the first rows see nothing
    (8, 1, 1, 64, 16, 1, [130, 8]),
    (16, 1, 1, 64, 16, 0, [130, 8]),
    (40, 2, 1, 64, 64, 1, [40, 333, 39, 1]),
    (200, 2, 2, 64, 16, 1, [200, 431]),
    (1, 8, 2, 128, 32, 1, [1, 77, 1025, 4000]),
    (1, 14, 2, 128, 64, 1, [0, 500]),
    (3, 15, 3, 64, 16, 1, [2, 90]),
    (2, 6, 2, 128, 16, 0, [65, 640]),
    (17, 3, 1, 128, 32, 1, [17, 16, 200]),
    (1, 3, 3, 64, 64, 1, [9000, 1, 0, 5000]),
    (4, 10, 10, 64, 16, 1, [44] * 40),
    # many units: a warp walks each alone
    (1, 20, 20, 64, 16, 1, [(37 * i) % 230 for i in range(70)]),
    (12, 7, 7, 64, 64, 0, [(13 * i) % 150 for i in range(175)]),
    (2, 5, 5, 128, 32, 1, [(29 * i) % 200 for i in range(250)]),
    (3, 12, 4, 128, 16, 1, [(31 * i) % 99 for i in range(310)]),
    # few long ones: clusters of chunks, and more chunks than a cluster
    (2, 4, 4, 64, 32, 1, [2047, 1030, 300]),
    (11, 2, 1, 128, 64, 1, [5, 2048, 700]),
    (1, 12, 1, 64, 16, 1, [30011]),
]


def _attend_case(i, dtype):
    rps, hq, hkv, dim, bs, causal, lens = ATT[i]
    rng = np.random.default_rng(100 + i)
    cols = max(1, -(-max(lens) // bs))
    counts = [-(-v // bs) for v in lens]
    blocks = sum(counts) + 2
    ids = rng.permutation(blocks)
    table = np.full((len(lens), cols + 1), -1)
    at = 0
    for s, c in enumerate(counts):
        table[s, :c] = ids[at:at + c]
        at += c
    cache = _filled(rng, blocks, bs, hkv, dim, dtype, garbage=ids[at:])
    # past each length: NaN scales
    for s, v in enumerate(lens):
        for pos in range(v, counts[s] * bs):
            for is_v in (0, 1):
                p = ob.scale_place(pos % 16, is_v)
                cache.raw[table[s, pos // bs], :, pos % bs // 16, p:p + 4] = 0xFF
    q = ob.round16(rng.normal(size=(len(lens) * rps, hq * dim)) * 1.5, dtype)
    return cache, table, q


def _rows_of(cache, table, length, head):
    g, D = cache.groups, cache.groups * 64
    k, v = np.zeros((length, D)), np.zeros((length, D))
    pos = np.arange(length)
    rec = cache.raw[table[pos // cache.bs], :, pos % cache.bs // 16]           # [n, slabs, 1152]
    p16 = pos % 16
    for is_v, out in ((0, k), (1, v)):
        for gi in range(g):
            r = rec[:, head * g + gi]
            place = np.array([[ob.code_place(p, d, is_v) for d in range(64)] for p in range(16)])
            byte = np.take_along_axis(r, place[p16, :, 0], 1)
            code = np.where(place[p16, :, 1] == 1, byte >> 4, byte & 15).astype(np.float64) - 8
            sp = np.array([ob.scale_place(p, is_v) for p in range(16)])[p16]
            sz = np.stack([r[np.arange(length), sp + b] for b in range(4)], 1)
            sz = ob.from_bits16(np.ascontiguousarray(sz).view(np.uint16), cache.dtype).astype(np.float64)
            out[:, gi * 64:(gi + 1) * 64] = code * sz[:, :1] + sz[:, 1:]
    return k, v


def _check_rows(got, cache, table, lens, q, rps, hq, hkv, causal, scale, dtype, hide=None):
    D, g = cache.groups * 64, hq // hkv
    unit = 2.0 ** -9 if dtype == "bf16" else 2.0 ** -12         # half an ulp of the output
    weight = 2.0 ** -9 if dtype == "bf16" else 2.0 ** -17       # of a weight (fp16 caches: two bf16 terms)
    for s, n in enumerate(lens):
        for head in range(hkv):
            k, v = _rows_of(cache, table[s], n, head)
            rows = [s * rps + j for j in range(rps) for _ in range(g)]
            cols = [slice((head * g + e) * D, (head * g + e + 1) * D) for _ in range(rps) for e in range(g)]
            qq = np.stack([q[r, c] for r, c in zip(rows, cols)]).astype(np.float64)
            end = np.array([n - (rps - 1 - j) if causal else n for j in range(rps) for _ in range(g)])
            seen = np.arange(n)[None] < end[:, None]
            if hide is not None:
                seen &= ~hide(s, np.arange(n))[None]
                k, v = np.where(hide(s, np.arange(n))[:, None], 0, k), np.where(hide(s, np.arange(n))[:, None], 0, v)
            want, w = ob.attention(qq, k, v, scale, seen)
            out = np.stack([got[r, c] for r, c in zip(rows, cols)])
            # fp32 scores: D products of up to |q||k| and their sums, each to 2^-23 (cached values are up to 3
            # times their group's z-free part); a score off by e moves a weight by 2 e of itself
            e = 4 * D * 2.0 ** -23 * (np.abs(qq) @ (np.abs(k).T + 1)).max(initial=0) * abs(scale) + 2.0 ** -20
            tol = unit * 1.01 * np.abs(want) + (weight + 2 * e) * (w @ (np.abs(v) + 1)) + 1e-7
            bad = np.abs(out - want) > tol
            assert not bad.any(), (s, head, np.abs(out - want).max(), tol.min())
            assert (out[~seen.any(1)] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("i", range(len(ATT)))
def test_attention(i, dtype):
    import torch
    from paper_2609_32869_gb300 import binding as B
    rps, hq, hkv, dim, bs, causal, lens = ATT[i]
    cache, table, q = _attend_case(i, dtype)
    n, d, scale = len(lens), hq * dim, dim ** -0.5
    raw, err = _dev(torch, cache.raw), _err(torch)
    most = max(1, max(lens))
    nb = B.wf_kv4_attention_scratch_bytes(n, rps, hq, hkv, dim, most)
    sc = torch.full((max(nb, 16) + 64,), GUARD, dtype=torch.uint8, device="cuda")
    qd = _dev(torch, np.concatenate([q, np.full((len(q), 24), 5.0)], 1), dtype)
    out = torch.full((n * rps, d + 8), 3.0, dtype=qd.dtype, device="cuda")
    args = (_pool(B, raw, cache), 0, qd, d + 24, _i32(torch, table), table.shape[1], _i32(torch, lens), n, rps, hq, causal, scale,
            most, out, d + 8, sc, nb, err)
    B.wf_kv4_attention(*args)
    got = out.float().cpu().numpy().astype(np.float64)
    assert (got[:, d:] == 3.0).all() and (sc[max(nb, 0):] == GUARD).all() and err.item() == 0
    _check_rows(got[:, :d], cache, table, lens, q, rps, hq, hkv, causal, scale, dtype)
    first = out.clone()
    B.wf_kv4_attention(*args)          # the same bits again
    assert torch.equal(first, out)


def test_attention_blocks_out_of_bounds_are_not_seen():
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(7)
    bs, hkv, dim, lens = 16, 2, 64, [100, 40, 16]
    cache = _filled(rng, 12, bs, hkv, dim, "bf16")
    table = np.array([[0, 12, 2, -1, 4, 5, 6], [7, 8, 2 ** 31 - 1, 0, 0, 0, 0], [-7, 0, 0, 0, 0, 0, 0]])
    q = ob.round16(rng.normal(size=(3, hkv * dim)), "bf16")
    out, err = torch.empty(3, hkv * dim, dtype=torch.bfloat16, device="cuda"), _err(torch)
    nb = B.wf_kv4_attention_scratch_bytes(3, 1, hkv, hkv, dim, 112)
    sc = torch.empty(max(nb, 16), dtype=torch.uint8, device="cuda")
    B.wf_kv4_attention(_pool(B, _dev(torch, cache.raw), cache), 0, _dev(torch, q, "bf16"), 128, _i32(torch, table), 7,
                       _i32(torch, lens), 3, 1, hkv, 1, 0.125, 112, out, 128, sc, nb, err)
    assert err.item() == B.WF_DEV_ERR_PAGE
    bad = (table < 0) | (table >= 12)
    safe = np.where(bad, 0, table)
    _check_rows(out.float().cpu().numpy().astype(np.float64), cache, safe, lens, q, 1, hkv, hkv, 1, 0.125, "bf16",
                hide=lambda s, pos: bad[s, pos // bs])


def test_attention_cuts_to_max_len_and_shares_a_table():
    """Lengths past max_len are cut; stride 0 gives every sequence the same blocks; another stream works."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(8)
    cache = _filled(rng, 8, 32, 1, 64, "f16")
    table = np.array([[3, 1, 5, 0]])
    q = ob.round16(rng.normal(size=(3, 64)), "f16")
    raw, qd, td, ln = _dev(torch, cache.raw), _dev(torch, q, "f16"), _i32(torch, table), _i32(torch, [70, 99, -3])
    out, err = torch.empty(3, 64, dtype=torch.float16, device="cuda"), _err(torch)
    nb = B.wf_kv4_attention_scratch_bytes(3, 1, 1, 1, 64, 90)
    sc = torch.empty(max(nb, 16), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.wf_kv4_attention(_pool(B, raw, cache), 0, qd, 64, td, 0, ln, 3, 1, 1, 1, 0.2, 90, out, 64, sc, nb, err, stream=side)
    side.synchronize()
    assert err.item() == B.WF_DEV_ERR_CAPACITY | B.WF_DEV_ERR_PAGE
    _check_rows(out.float().cpu().numpy().astype(np.float64), cache, np.repeat(table, 3, 0), [70, 90, 0], q, 1, 1, 1, 1, 0.2, "f16")


def test_attention_non_finite_positions_reach_only_rows_that_see_them():
    import torch
    from paper_2609_32869_gb300 import binding as B
    bs, n, rps = 16, 37, 4
    cache = ob.Cache(3, bs, 1, 64, "bf16")
    rng = np.random.default_rng(9)
    for pos in range(n):
        row = ob.round16(rng.normal(size=64), "bf16")
        cache.put(pos, row, 0)
        cache.put(pos, np.where(np.arange(64) == 3, np.inf, row) if pos == n - 1 else row, 1)
    q = ob.round16(rng.normal(size=(rps, 64)), "bf16")
    out, err = torch.empty(rps, 64, dtype=torch.bfloat16, device="cuda"), _err(torch)
    nb = B.wf_kv4_attention_scratch_bytes(1, rps, 1, 1, 64, 48)
    sc = torch.empty(max(nb, 16), dtype=torch.uint8, device="cuda")
    B.wf_kv4_attention(_pool(B, _dev(torch, cache.raw), cache), 0, _dev(torch, q, "bf16"), 64, _i32(torch, [[0, 1, 2]]), 3,
                       _i32(torch, [n]), 1, rps, 1, 1, 0.125, 48, out, 64, sc, nb, err)
    assert torch.isnan(out[-1].float()).all()
    got = out.float().cpu().numpy().astype(np.float64)[:-1]
    _check_rows(got, cache, np.array([[0, 1, 2]]), [n - 1], q[:-1], rps - 1, 1, 1, 1, 0.125, "bf16")


# ---------------------------------------------------------------- selection --
def _select(torch, B, logits, scores, suppress, eos, dtype, pad=0):
    n, W = scores.shape
    V = logits.shape[-1]
    x = np.concatenate([logits.reshape(n * W, V), np.full((n * W, pad), 99.0)], 1)
    ld, code = V + pad, {"f32": B.WF_F32, "bf16": B.WF_BF16, "f16": B.WF_F16}[dtype]
    x = _dev(torch, x, dtype)
    nb = B.wf_beam_select_scratch_bytes(n, W, V)
    sc = torch.full((nb + 64,), GUARD, dtype=torch.uint8, device="cuda")
    out = {"token": _i32(torch, np.full((n, W), 55)), "parent": _i32(torch, np.full((n, W), 55)),
           "score": torch.full((n, W), 5.0, device="cuda"), "fin_parent": _i32(torch, np.full((n, W), 55)),
           "fin_score": torch.full((n, W), 5.0, device="cuda")}
    sup = None if suppress is None else _dev(torch, suppress.astype(np.uint8))
    B.wf_beam_select(x, code, ld, _dev(torch, scores.astype(np.float32)), sup, n, W, V, eos, out["token"], out["parent"], out["score"],
                     out["fin_parent"], out["fin_score"], sc, nb)
    assert (sc[nb:] == GUARD).all()
    return {k: v.cpu().numpy() for k, v in out.items()}, x.float().cpu().numpy()[:, :V].reshape(n, W, V)


def _check_select(got, logits, scores, suppress, eos):
    n, W, V = logits.shape
    sup = np.zeros(V) if suppress is None else suppress
    for i in range(n):
        want, ranked = ob.beam_select(logits[i].astype(np.float64), scores[i].astype(np.float64), sup, eos)
        # fp32: the difference with the maximum, the logarithm and the sums, each rounded once, and the sum of exponentials
        big = 1 + np.abs(scores[i][np.isfinite(scores[i])]).max(initial=0) + 2 * np.abs(logits[i][np.isfinite(logits[i])]).max(initial=0)
        tol = 4 * 2.0 ** -23 * big
        for name in ("score", "fin_score"):
            w = np.array(want[name])
            np.testing.assert_array_equal(np.isinf(got[name][i]), np.isinf(w))
            f = np.isfinite(w)
            assert np.abs(got[name][i][f] - w[f]).max(initial=0) <= tol
        gaps = -np.diff(ranked)
        if len(gaps) and (gaps[gaps > 0].min(initial=1) <= 2 * tol or (gaps == 0).any() and not _exact(logits[i])):
            continue    # which of two equal candidates comes first turns on a rounding
        for name in ("token", "parent", "fin_parent"):
            assert got[name][i].tolist() == want[name], (i, name)


def _exact(x):
    return (np.abs(x[np.isfinite(x)] * 4) % 1 == 0).all()


@pytest.mark.parametrize("n,W,V,dtype", [(1, 1, 2, "f32"), (3, 1, 1000, "bf16"), (2, 2, 4, "f32"), (4, 5, 33, "f16"), (2, 5, 51866, "f32"),
                                         (3, 4, 51865, "bf16"), (2, 16, 40, "f32"), (1, 16, 9001, "f16"), (40, 3, 513, "f32"),
                                         (1, 3, 200001, "f32"), (2, 8, 4096, "f32"), (2, 8, 4097, "bf16"),
                                         # segments of 3 and of 8 tiles, and more than 32 lists' worth of vocabulary
                                         (70, 5, 20011, "f32"), (200, 4, 9000, "f16"), (1, 2, 600007, "bf16")])
def test_select_random(n, W, V, dtype):
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(n * 1000 + W)
    logits = rng.normal(0, 3, (n, W, V))
    scores = -rng.uniform(0, 20, (n, W))
    scores[::2, 1:] = -np.inf
    eos = V // 2
    logits[:, 0, eos] = logits[:, 0].max(-1) + 1
    sup = (rng.random(V) < 0.1) & (np.arange(V) != eos) if V > 100 else None
    got, x = _select(torch, B, logits, scores, sup, eos, dtype, pad=3)
    _check_select(got, x, scores, sup, eos)


@pytest.mark.parametrize("n,W,V,dtype,kind", [(3, 16, 30011, "f32", "ties"), (2, 9, 51866, "f32", "normal"), (2, 12, 20003, "bf16", "ties"),
                                              (3, 13, 12001, "f16", "few"), (1, 16, 9000, "f32", "few"), (4, 16, 51866, "f32", "normal")])
@pytest.mark.parametrize("shift", [0, 3, 13])
def test_select_many_beams(n, W, V, dtype, kind, shift):
    """More than 8 beams: equal logits in many groups, fewer finite ones than places, suppressed ids from any address."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(V + shift)
    if kind == "ties":
        logits = rng.integers(-20, 5, (n, W, V)) / 4.0
    elif kind == "few":
        logits = np.where(rng.random((n, W, V)) < 20 / V, rng.integers(-40, 40, (n, W, V)) / 4.0, -np.inf)
    else:
        logits = rng.normal(0, 3, (n, W, V))
    sup = rng.random(V) < 0.01
    held = torch.zeros(V + 32, dtype=torch.uint8, device="cuda")
    held[:] = 1                                    # what lies around the suppressed ids is not read as one
    held[shift:shift + V] = _dev(torch, sup.astype(np.uint8))
    x, scores = _dev(torch, logits.reshape(n * W, V), dtype), -rng.uniform(0, 10, (n, W)).astype(np.float32)
    code = {"f32": B.WF_F32, "bf16": B.WF_BF16, "f16": B.WF_F16}[dtype]
    nb = B.wf_beam_select_scratch_bytes(n, W, V)
    sc = torch.full((nb + 64,), GUARD, dtype=torch.uint8, device="cuda")
    out = {k: _i32(torch, np.full((n, W), 55)) for k in ("token", "parent", "fin_parent")}
    out.update({k: torch.full((n, W), 5.0, device="cuda") for k in ("score", "fin_score")})
    B.wf_beam_select(x, code, V, _dev(torch, scores), held[shift:shift + V], n, W, V, 7, out["token"], out["parent"], out["score"],
                     out["fin_parent"], out["fin_score"], sc, nb)
    assert (sc[nb:] == GUARD).all()
    _check_select({k: v.cpu().numpy() for k, v in out.items()}, x.float().cpu().numpy().reshape(n, W, V), scores.astype(np.float64), sup, 7)


@pytest.mark.parametrize("n,W,V,dtype", [(20, 8, 1000, "f32"), (9, 8, 3045, "bf16"), (3, 16, 4096, "f32"), (3, 16, 8192, "f16"), (2, 16, 33, "bf16"),
                                         (2, 16, 300, "f32"), (5, 3, 200, "f16")])
@pytest.mark.parametrize("suppressed", [0.0, 0.05, 0.97])
def test_select_few_groups(n, W, V, dtype, suppressed):
    """Vocabularies of about as many groups as places: the bound comes from the logits themselves."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(V + W)
    logits = rng.normal(0, 3, (n, W, V))
    logits[0, 0, ::3] = np.nan
    logits[-1, -1] = -np.inf
    scores, sup = -rng.uniform(0, 10, (n, W)), rng.random(V) < suppressed
    sup[V // 2] = False
    got, x = _select(torch, B, logits, scores, sup, V // 2, dtype, pad=5)
    x = np.where(np.isnan(x), -np.inf, x)          # a NaN is no candidate and no part of the sum
    _check_select(got, x, scores, sup, V // 2)


def test_select_ties_go_to_the_lowest_beam_and_id():
    """Beams with equal rows and equal scores; equal logits all over the row, in one CTA's chunk and across."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    n, W, V = 2, 3, 20000
    logits = np.zeros((n, W, V))
    logits[1, :, 5000:15000:2500] = 2.0
    got, x = _select(torch, B, logits, np.zeros((n, W)), None, -1, "f32")
    assert got["token"][0].tolist() == [0, 1, 2] and got["parent"][0].tolist() == [0, 0, 0]
    assert got["token"][1].tolist() == [5000, 7500, 10000] and got["parent"][1].tolist() == [0, 0, 0]
    assert (got["fin_parent"] == -1).all()
    up = np.arange(V, dtype=np.float64)[None, None] / 64            # every logit larger than the one before
    got, x = _select(torch, B, np.repeat(up, 3, 1), np.array([[0, -100, -100.0]]), None, V - 2, "f32")
    assert got["token"][0].tolist() == [V - 1, V - 3, V - 4] and got["fin_parent"][0].tolist() == [0, -1, -1]
    got, x = _select(torch, B, -np.repeat(up, 3, 1), np.array([[-100, 0, -100.0]]), None, V - 2, "f32")
    assert got["token"][0].tolist() == [0, 1, 2] and got["parent"][0].tolist() == [1, 1, 1]
    # every logit larger than all before it, in every beam: each tile displaces all that came before
    got, x = _select(torch, B, np.repeat(np.arange(60000, dtype=np.float64)[None, None] / 256, 16, 1), np.zeros((1, 16)), None, -1, "f32")
    assert got["token"][0].tolist() == [59999] * 16 and got["parent"][0].tolist() == list(range(16))
    # minus zero equals zero
    z = np.zeros((1, 1, 8))
    z[0, 0, ::2] = -0.0
    got, x = _select(torch, B, z, np.zeros((1, 1)), None, -1, "f32")
    assert got["token"][0].tolist() == [0]


def test_select_rows_without_candidates():
    """Everything suppressed, -inf, NaN or +inf; unused beams; the type's lowest value is a value."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    W, V = 2, 300
    x = np.full((5, W, V), -np.inf)
    x[1] = np.nan
    x[2, 0], x[2, 1] = 0.0, 1.0
    x[2, 0, 7] = np.inf
    x[3, :, :] = np.finfo(np.float32).min
    x[4, 0, 5], x[4, 0, 6] = 1.0, np.nan
    scores = np.zeros((5, W))
    got, _ = _select(torch, B, x, scores, None, 299, "f32")
    for i in (0, 1):
        assert got["token"][i].tolist() == [-1, -1] and got["parent"][i].tolist() == [0, 1] and np.isneginf(got["score"][i]).all()
    assert got["parent"][2].tolist() == [1, 1] and got["token"][2].tolist() == [0, 1]
    assert got["token"][3].tolist() == [0, 1] and got["parent"][3].tolist() == [0, 0]
    np.testing.assert_allclose(got["score"][3], -np.log(V), atol=1e-6)
    assert got["token"][4].tolist() == [5, -1] and got["score"][4, 0] == 0.0
    got, _ = _select(torch, B, np.zeros((1, W, V)), np.full((1, W), -np.inf), None, 3, "bf16")
    assert got["token"][0].tolist() == [-1, -1]
    got, _ = _select(torch, B, np.zeros((1, W, V)), np.zeros((1, W)), np.ones(V), 3, "f16")
    assert got["token"][0].tolist() == [-1, -1] and got["fin_parent"][0].tolist() == [-1, -1]


# --------------------------------------------------------------- reordering --
def _beam_state(rng, n, W, bs, lens, cols):
    """Tables whose beams share blocks the way beams do: each column's holders descend from earlier ones."""
    blocks = n * W * cols + 3
    ids = list(rng.permutation(blocks))
    table = np.full((n * W, cols), -1)
    for i, v in enumerate(lens):
        full, rem = divmod(v, bs)
        for c in range(full):
            for w in range(W):
                share = rng.random() < 0.8 * (1 - c / max(full, 1))
                table[i * W + w, c] = table[i * W, c] if w and share else ids.pop()
        if rem:
            for w in range(W):
                table[i * W + w, full] = ids.pop()
    return table, ids, blocks


@pytest.mark.parametrize("n,W,bs,most,layers,heads,dim", [(1, 1, 16, 20, 1, 1, 64), (3, 5, 16, 100, 3, 2, 64), (2, 4, 64, 200, 2, 1, 128),
                                                          (9, 3, 32, 70, 1, 3, 64), (2, 16, 16, 60, 2, 1, 64), (1, 2, 16, 5000, 1, 1, 64),
                                                          (40, 2, 16, 33, 1, 1, 64)])
@pytest.mark.parametrize("in_place", [False, True])
def test_reorder(n, W, bs, most, layers, heads, dim, in_place):
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(W * 100 + n)
    lens = [most] + [int(v) for v in rng.integers(0, most + 1, n - 1)]
    cols = -(-most // bs) + 1
    table, ids, blocks = _beam_state(rng, n, W, bs, lens, cols)
    parent = rng.integers(0, W, (n, W))
    if n > 2:
        parent[1] = -1                   # a released request
        parent[2, 0] = -1                # a dropped beam
    lens[-1] = lens[-1] // bs * bs       # no partly filled block
    if lens[-1] < most:
        table[-W:, lens[-1] // bs:] = -1
    raw = rng.integers(0, 256, (layers, blocks, heads * dim // 64, bs // 16, 1152)).astype(np.uint8)
    free = np.concatenate([ids, np.full(blocks - len(ids), -9)])
    want_raw, want_table, want_free, left = raw.copy(), table.copy(), free.copy(), len(ids)
    for i in range(n):
        new, freed, moves = ob.beam_reorder(table[i * W:(i + 1) * W], lens[i], parent[i].tolist(), bs)
        used = -(-lens[i] // bs)
        want_table[i * W:(i + 1) * W, :used] = new[:, :used]
        want_free[left:left + len(freed)] = freed
        left += len(freed)
        for a, b, positions in moves:
            t = -(-positions // 16)
            want_raw[:, b, :, :t] = raw[:, a, :, :t]
    guard = torch.full((raw.size + 4096,), GUARD, dtype=torch.uint8, device="cuda")
    guard[:raw.size] = _dev(torch, raw).view(-1)
    pool = B.kv4_pool(guard, layers, blocks, bs, heads, dim)
    t_in = _i32(torch, table)
    t_out = t_in if in_place else t_in.clone()
    fr, n_free = _i32(torch, free), _i32(torch, [len(ids)])
    n_out = n_free if in_place else _err(torch)
    nb, err = B.wf_beam_reorder_scratch_bytes(n, W, cols), _err(torch)
    sc = torch.full((nb + 64,), GUARD, dtype=torch.uint8, device="cuda")
    B.wf_beam_reorder(pool, t_in, t_out, cols, _i32(torch, np.repeat(lens, W)), _i32(torch, parent), n, W, fr, n_free, n_out, sc, nb, err)
    np.testing.assert_array_equal(t_out.cpu().numpy(), want_table)
    assert n_out.item() == left and err.item() == 0
    np.testing.assert_array_equal(fr.cpu().numpy(), want_free)
    np.testing.assert_array_equal(guard[:raw.size].cpu().numpy().reshape(raw.shape), want_raw)
    assert (guard[raw.size:] == GUARD).all() and (sc[nb:] == GUARD).all()


def test_reorder_reports_what_is_out_of_bounds():
    """A parent past the beams, a table entry past the pool and a free stack that is too full: skipped, reported."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    raw = torch.full((4 * 1152,), GUARD, dtype=torch.uint8, device="cuda")
    pool = B.kv4_pool(raw, 1, 4, 16, 1, 64)
    nb, err = B.wf_beam_reorder_scratch_bytes(1, 2, 2), _err(torch)
    sc = torch.empty(nb, dtype=torch.uint8, device="cuda")
    table, free = _i32(torch, [[0, 99], [0, 1]]), _i32(torch, [2, 3, -1, -1])
    out, left = table.clone(), _err(torch)
    B.wf_beam_reorder(pool, table, out, 2, _i32(torch, [20, 20]), _i32(torch, [1, 1]), 1, 2, free, _i32(torch, [2]), left, sc, nb, err)
    assert err.item() == B.WF_DEV_ERR_PAGE and (raw == GUARD).all()
    err.zero_()
    B.wf_beam_reorder(pool, _i32(torch, [[0, 2], [1, 3]]), out, 2, _i32(torch, [20, 20]), _i32(torch, [-1, -1]), 1, 2, free, _i32(torch, [2]),
                      left, sc, nb, err)
    assert err.item() == B.WF_DEV_ERR_PAGE and left.item() == 2 and free.tolist() == [2, 3, -1, -1]
    err.zero_()
    B.wf_beam_reorder(pool, _i32(torch, [[0, 2], [1, 3]]), out, 2, _i32(torch, [20, 20]), _i32(torch, [7, -5]), 1, 2, free, _i32(torch, [0]),
                      left, sc, nb, err)
    assert err.item() == B.WF_DEV_ERR_PAGE and left.item() == 4 and free.tolist() == [0, 1, 2, 3]
