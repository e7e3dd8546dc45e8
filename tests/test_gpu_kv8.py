"""The paged 8-bit cache against its restatement: rows in and out, and attention over it (GPU)."""
import numpy as np
import pytest

from oracle import prompt as op

pytestmark = pytest.mark.gpu


def _dt(torch, name):
    return {"bf16": torch.bfloat16, "f16": torch.float16}[name]


def _rows(torch, rng, n, heads, dim, dtype, size=1.0):
    x = rng.normal(0, 1, (n, heads, dim)) * np.exp(rng.normal(0, 1, (n, heads, 1))) * size
    return torch.from_numpy(x.astype(np.float32)).cuda().to(_dt(torch, dtype))


def _i32(torch, v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _pool(B, raw, c, dtype, layers=1, stride=0):
    return B.kv8_pool(raw, layers, c.raw.shape[0], c.bs, c.heads, c.dim, B.WF_F16 if dtype == "f16" else B.WF_BF16, stride)


def _f64(x):
    return x.double().cpu().numpy()


def _round(torch, x, dtype):
    return torch.from_numpy(np.asarray(x, np.float32)).to(_dt(torch, dtype)).double().numpy()


# slots of a call's rows, call after call; blocks of 32 positions
CALLS = [
    [[0]],
    [list(range(16)), [16], [17, 18], list(range(19, 40))],
    [[5, 6, -1, 64, 65, 66], [7, 67, -1, -7]],
    [[3, 4, 20], [21, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15], [0, 1]],      # begun again at position 0
    [[32, 33, 34, 35], [34], [33, 34, 35]],                                # rolled back and written over
    [[1, 3, 2, 3, 3]],                                                     # out of order, one position three times
    [[9] * 40 + [10]],
    [list(range(96)) + [-1] * 3 + list(range(100, 128))],
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,dim", [(3, 64), (2, 128)])
@pytest.mark.parametrize("calls", range(len(CALLS)))
def test_store_and_load(dtype, heads, dim, calls):
    """Codes and scales equal the restatement's, byte for byte: records that a call does not write to too."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(calls * 10 + dim)
    c = op.Cache(4, 32, heads, dim, fill=0x38)
    c.raw[..., 32 * dim:] = np.array([1.0, 0.5, 0, 0], np.float32).view(np.uint8)
    raw = torch.from_numpy(np.concatenate([c.raw.reshape(-1), np.full(64, 0xA5, np.uint8)])).cuda()
    pool, err = _pool(B, raw, c, dtype), _i32(torch, [0])
    for i, slots in enumerate(CALLS[calls]):
        n = len(slots)
        x = _rows(torch, rng, n, 3 * heads, dim, dtype, 4.0 ** (i - 1))
        k, v = x[:, heads:2 * heads], x[:, 2 * heads:]
        B.wf_kv8_store(pool, 0, k, x.stride(0), v, x.stride(0), _i32(torch, slots), n, err)
        c.store(slots, _f64(k), _f64(v))
    np.testing.assert_array_equal(raw.cpu().numpy()[:-64].reshape(c.raw.shape), c.raw)
    assert (raw[-64:] == 0xA5).all() and err.item() == 0
    see = [s for call in CALLS[calls] for s in call][::-1] + [2, 2, 1]
    ko = torch.full((len(see) + 1, heads * dim + 8), 7.0, dtype=_dt(torch, dtype), device="cuda")
    vo = ko.clone()
    B.wf_kv8_load(pool, 0, _i32(torch, see), len(see), ko, ko.stride(0), vo, vo.stride(0), err)
    for out, is_v in ((ko, 0), (vo, 1)):
        want = np.array([_round(torch, c.row(s, is_v), dtype).reshape(-1) if s >= 0 else np.zeros(heads * dim) for s in see])
        np.testing.assert_array_equal(_f64(out[:len(see), :heads * dim]), want)
        assert (out[len(see):] == 7).all() and (out[:, heads * dim:] == 7).all()


# slots of a call whose rows are partly skipped, as of a block of proposals of which some are taken
SKIPPED = [
    [3, -1, 4, -1, -1, 5, 6],
    [-1] * 5 + [0] + [-1] * 31 + [1] + [-1] * 31 + [2, 16, -1, 17] + [-1] * 70,  # as many as may be
    [0, 1] + [-1] * 3 + [2] + [-1] * 20 + [3, -1, 3, -2, 5] + [-1] * 14 + [33, -1, 34, 64, -1, 65] + [-1] * 14 + [66],  # over several CTAs' rows
    [-1] * 60 + [40] + [-1] * 9 + [41] + [-1] * 9 + [42] + [-1] * 9 + [43] + [-1] * 9 + [44] + [-1] * 9 + [45, 48],
    [20, -1, 21] * 9 + [-1, 22],
    [-1] * 100,
]


@pytest.mark.parametrize("heads,copies", [(2, 1), (24, 1), (2, 2500)])
@pytest.mark.parametrize("case", range(len(SKIPPED)))
def test_rows_that_are_skipped_do_not_part_a_record(heads, copies, case):
    """Byte for byte as the restatement, in few rows and (`copies`, each in blocks of its own) in many a CTA."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(case)
    slots, dim, blocks = SKIPPED[case], 64, 3
    n = len(slots)
    c = op.Cache(blocks, 32, heads, dim, fill=0x38)
    c.raw[..., 32 * dim:] = np.array([1.0, 0.5, 0, 0], np.float32).view(np.uint8)
    raw = torch.from_numpy(c.raw.copy()).cuda().repeat(copies, 1, 1, 1)
    x = _rows(torch, rng, n, 2 * heads, dim, "bf16")
    k, v = x[:, :heads].reshape(n, -1), x[:, heads:].reshape(n, -1)
    many = [s + 32 * blocks * i if s >= 0 else s for i in range(copies) for s in slots]
    pool = B.kv8_pool(raw, 1, blocks * copies, 32, heads, dim, B.WF_BF16)
    kk, vv = k.repeat(copies, 1), v.repeat(copies, 1)
    B.wf_kv8_store(pool, 0, kk, heads * dim, vv, heads * dim, _i32(torch, many), n * copies)
    c.store(slots, _f64(k).reshape(n, heads, dim), _f64(v).reshape(n, heads, dim))
    got = raw.cpu().numpy().reshape((copies,) + c.raw.shape)
    np.testing.assert_array_equal(got[0], c.raw)
    assert (got == got[0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_values_at_the_ends_of_the_range(dtype):
    """All zero, tiny, huge, not finite: one record each, and such a row behind an ordinary one."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    heads, dim = 1, 64
    top = 65504.0 if dtype == "f16" else 3.3e38
    rows = [np.zeros(64), np.full(64, top), np.full(64, 2.0 ** -24), np.linspace(-448, 448, 64), np.linspace(-449, 460, 64)]
    for bad in (np.nan, np.inf, -np.inf):
        r = np.linspace(-3, 5, 64)
        r[[0, 17, 63]] = bad
        rows.append(r)
    rows.append(np.full(64, np.inf))
    if dtype == "bf16":
        rows += [np.full(64, 1e-38), np.full(64, 448 * 2.0 ** 36), np.full(64, 2.0 ** -66)]
    n = len(rows)
    for behind in (False, True):
        c = op.Cache(n, 16, heads, dim)
        raw = torch.from_numpy(c.raw.copy()).cuda()
        pool = _pool(B, raw, c, dtype)
        calls = [([16 * i for i in range(n)], [np.linspace(-1, 1, 64)] * n)] if behind else []
        calls.append(([16 * i + behind for i in range(n)], rows))
        for slots, x in calls:
            t = torch.tensor(np.array(x), device="cuda").to(_dt(torch, dtype)).contiguous()
            B.wf_kv8_store(pool, 0, t, 64, t, 64, _i32(torch, slots), n)
            c.store(slots, _f64(t)[:, None], _f64(t)[:, None])
        got = raw.cpu().numpy()
        # a NaN has one magnitude and either sign
        np.testing.assert_array_equal(np.where(got[..., :2048] & 127 == 127, 127, got[..., :2048]), np.where(c.raw[..., :2048] & 127 == 127, 127, c.raw[..., :2048]))
        np.testing.assert_array_equal(got[..., 2048:], c.raw[..., 2048:])


def test_slots_outside_the_pool_and_layers():
    import torch
    from paper_2609_32869_gb300 import binding as B
    heads, dim, layers = 2, 64, 3
    c = op.Cache(2, 16, heads, dim)
    stride = c.raw.size + 32
    raw = torch.full((layers * stride,), 0xA5, dtype=torch.uint8, device="cuda")
    pool, err = _pool(B, raw, c, "bf16", layers, stride), _i32(torch, [0])
    x = torch.randn(4, heads * dim, device="cuda").bfloat16()
    B.wf_kv8_store(pool, 1, x, heads * dim, x, heads * dim, _i32(torch, [32, 0, 2 ** 31 - 1, 40]), 4, err)
    assert err.item() == B.WF_DEV_ERR_PAGE
    at = raw.view(layers, stride)
    assert (at[[0, 2]] == 0xA5).all() and (at[1, c.raw.size:] == 0xA5).all() and (at[1, heads * 2064:c.raw.size] == 0xA5).all()
    out = torch.full((4, heads * dim), 7.0, device="cuda").bfloat16()
    err.zero_()
    B.wf_kv8_load(pool, 1, _i32(torch, [0, 32, -1, 2 ** 31 - 1]), 4, out, heads * dim, out.clone(), heads * dim, err)
    assert err.item() == B.WF_DEV_ERR_PAGE and out[0].any() and not out[1:].any()


@pytest.mark.parametrize("n", [300, 5000])
def test_many_rows_equal_few(n):
    """A prompt in one call and in calls of 16 rows: the same bytes."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    heads, dim, bs = 5, 64, 64
    blocks = -(-n // bs)
    rng = np.random.default_rng(n)
    k, v = _rows(torch, rng, n, heads, dim, "bf16"), _rows(torch, rng, n, heads, dim, "bf16")
    perm = rng.permutation(blocks)
    slots = _i32(torch, [perm[p // bs] * bs + p % bs for p in range(n)])
    size = blocks * B.wf_kv8_block_bytes(bs, heads, dim)
    a, b = torch.zeros(size, dtype=torch.uint8, device="cuda"), torch.zeros(size, dtype=torch.uint8, device="cuda")
    B.wf_kv8_store(B.kv8_pool(a, 1, blocks, bs, heads, dim), 0, k, heads * dim, v, heads * dim, slots, n)
    for i in range(0, n, 16):
        B.wf_kv8_store(B.kv8_pool(b, 1, blocks, bs, heads, dim), 0, k[i:], heads * dim, v[i:], heads * dim, slots[i:], min(16, n - i))
    assert torch.equal(a, b)


# ---------------------------------------------------------------- attention --
def _cache(rng, blocks, bs, heads, dim, spread=0.0):
    """Every position written: random codes but NaN, scales around 2^-7 times 2^(+-spread)."""
    c = op.Cache(blocks, bs, heads, dim)
    c.raw[..., :32 * dim] = rng.integers(0, 256, c.raw[..., :32 * dim].shape)
    body = c.raw[..., :32 * dim]
    body[(body & 127) > 0x70] &= 0xF7  # large codes are rarer
    body[(body & 127) == 127] = 0
    e = np.rint(rng.normal(-7, spread, (*c.raw.shape[:3], 2)))
    c.raw[..., 32 * dim:32 * dim + 8] = (2.0 ** e).astype(np.float32).view(np.uint8)
    c.raw[..., 32 * dim + 8:] = 0
    return c


def _dense(c):
    """Every position's keys and values [blocks * bs, heads, dim] float64."""
    dim = c.dim
    where = np.array([[[op.place(d, p, s) for d in range(dim)] for p in range(16)] for s in range(2)])
    vals = np.concatenate([op.E4M3, -op.E4M3])
    sc = c.raw[..., 32 * dim:32 * dim + 8].copy().view(np.float32).astype(np.float64)
    out = []
    for s in range(2):
        x = vals[c.raw[..., where[s]]] * sc[..., s, None, None]          # [blocks, heads, tiles, 16, dim]
        out.append(x.transpose(0, 2, 3, 1, 4).reshape(-1, c.heads, dim))
    return out


def _score_error(q, k, scale):
    """fp32 sums of a row's products in any order and the constants' roundings, in units of the exponent."""
    dim = q.shape[-1]
    return 2.0 ** -24 * (dim + 16) * abs(scale) * np.abs(q).max(-1) * np.abs(k).sum(-1).max() + 2.0 ** -20


def _run(torch, B, c, dtype, q, table, lens, rps, hq, causal, scale, max_len, stride=None):
    raw = torch.from_numpy(c.raw.copy()).cuda()
    n, dim = len(lens), c.dim
    rows = torch.full((n * rps + 1, hq * dim + 8), 3.0, dtype=_dt(torch, dtype), device="cuda")
    rows[:n * rps, :hq * dim] = torch.from_numpy(q.reshape(n * rps, -1)).to(rows)
    out = torch.full((n * rps + 1, hq * dim + 16), 7.0, dtype=_dt(torch, dtype), device="cuda")
    size = B.wf_kv8_attention_scratch_bytes(n, rps, hq, c.heads, dim, max_len)
    scratch = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    err = _i32(torch, [0])
    B.wf_kv8_attention(_pool(B, raw, c, dtype), 0, rows, rows.stride(0), _i32(torch, table), table.shape[1] if stride is None else stride, _i32(torch, lens),
                       n, rps, hq, causal, scale, max_len, out, out.stride(0), scratch, size, err)
    assert (out[n * rps:] == 7).all() and (out[:, hq * dim:] == 7).all() and (scratch[size:] == 0xA5).all()
    return _f64(out[:n * rps, :hq * dim]).reshape(n * rps, hq, dim), err.item()


def _check(torch, c, dtype, q, table, lens, rps, hq, causal, scale, got):
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
    kd, vd = _dense(c)
    for i, t in enumerate(lens):
        at = np.array([table[i][p // c.bs] * c.bs + p % c.bs for p in range(t)], int)
        ends = [t - (rps - 1 - j) if causal else t for j in range(rps)]
        qi, k, v = q[i * rps:(i + 1) * rps], kd[at], vd[at]
        want, _, mass = op.attention(qi, k, v, scale, ends)
        # the output's rounding; 11 bits of each weight (its sums are not of the rounded ones), and twice the scores' error
        dx = _score_error(qi, k, scale)[..., None] if t else 0.0
        tol = u * np.abs(want) + (1 + u) * (2.0 ** -11 + 2 * dx) * mass + 2.0 ** -22 * np.abs(v).max(initial=0) + (2.0 ** -25 if dtype == "f16" else 0)
        err = np.abs(got[i * rps:(i + 1) * rps] - want)
        assert (err <= tol).all(), (i, t, (err / np.maximum(tol, 1e-300)).max())


SHAPES = [
    # rps, hq, hkv, dim, block, lengths, causal
    (1, 1, 1, 64, 16, [1], True), (1, 2, 1, 128, 16, [0, 1, 15, 16, 17], True), (3, 2, 2, 64, 32, [1, 2, 3, 33], True),
    (9, 3, 3, 64, 64, [9, 64, 65, 130], True), (5, 4, 2, 128, 32, [200, 3], False), (1, 14, 2, 64, 16, [300, 31], True),
    (2, 8, 1, 128, 64, [511, 512, 513], True), (40, 2, 1, 64, 16, [90, 40, 7], True), (1, 1, 1, 64, 64, [2600], True),
    (1, 4, 2, 128, 16, [4100, 0, 77], True), (17, 5, 1, 128, 32, [260], False)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention(dtype, shape):
    import torch
    from paper_2609_32869_gb300 import binding as B
    rps, hq, hkv, dim, bs, lens, causal = SHAPES[shape]
    rng = np.random.default_rng(shape)
    need = [-(-t // bs) for t in lens]
    c = _cache(rng, sum(need) + 2, bs, hkv, dim, spread=1.0)
    ids = rng.permutation(sum(need) + 2)
    table = np.full((len(lens), max(need) + 1), -1)
    at = 0
    for i, m in enumerate(need):
        table[i, :m] = ids[at:at + m]
        at += m
    c.raw[ids[at:]] = 0xFF
    q = _round(torch, rng.normal(0, 1, (len(lens) * rps, hq, dim)), dtype)
    got, err = _run(torch, B, c, dtype, q, table, lens, rps, hq, causal, 0.09, max(max(lens), 1))
    assert err == 0
    _check(torch, c, dtype, q, table, lens, rps, hq, causal, 0.09, got)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_scales_far_apart(dtype, dim):
    """Records whose powers of two lie across their whole range: the large ones rule the output, the others still share the weights."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(dim)
    c = _cache(rng, 10, 16, 2, dim)
    lo, hi = (-60, 36) if dtype == "bf16" else (-20, 3)
    ev = np.rint(np.linspace(lo, hi, 10))
    for b in range(10):
        c.raw[b, :, :, 32 * dim:32 * dim + 8] = np.array([2.0 ** -7, 2.0 ** ev[(b * 7) % 10]], np.float32).view(np.uint8)
    table = rng.permutation(10)[None]
    q = _round(torch, rng.normal(0, 1, (3, 4, dim)), dtype)
    got, _ = _run(torch, B, c, dtype, q, table, [160], 3, 4, True, 0.1, 160)
    _check(torch, c, dtype, q, table, [160], 3, 4, True, 0.1, got)
    # nothing but zeros under the smallest power, one row of ones among them: it is worth its weight
    c.raw[..., :32 * dim] = 0
    c.raw[..., 32 * dim:32 * dim + 8] = np.array([2.0 ** -7, 2.0 ** -60], np.float32).view(np.uint8)
    for d in range(dim):
        c.raw[table[0][3], :, 0, op.place(d, 5, 1)] = 0x38
    c.raw[table[0][3], :, 0, 32 * dim + 4:32 * dim + 8] = np.array([1.0], np.float32).view(np.uint8)
    got, _ = _run(torch, B, c, dtype, q, table, [160], 3, 4, False, 0.1, 160)
    np.testing.assert_allclose(got, 1 / 160, rtol=2.0 ** -7 if dtype == "bf16" else 2.0 ** -10)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_queries_of_any_size(dtype):
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(3)
    c = _cache(rng, 3, 16, 1, 64)
    table = np.array([[2, 0, 1]])
    big = 1e30 if dtype == "bf16" else 3e4
    size = np.array([1.0, 0.0, big, 1 / big, 1e-3])[:, None, None]
    q = _round(torch, rng.normal(0, 1, (5, 1, 64)) * size, dtype)
    for scale in (0.1 / big, 0.1, -0.2):
        got, _ = _run(torch, B, c, dtype, q, table, [45], 5, 1, False, scale, 48)
        _check(torch, c, dtype, q[[0, 1, 3, 4]], table, [45], 4, 1, False, scale, got[[0, 1, 3, 4]])
        if scale == 0.1 / big and np.isfinite(q).all():  # (fp16's largest may round to infinity)
            _check(torch, c, dtype, q, table, [45], 5, 1, False, scale, got)
    # a row with a NaN is NaN, and no other
    q[2, 0, 7] = np.nan
    got, _ = _run(torch, B, c, dtype, q, table, [45], 5, 1, False, 0.1, 48)
    assert np.isnan(got[2]).all() and np.isfinite(got[[0, 1, 3, 4]]).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("what", ["keys", "values"])
def test_nan_positions_reach_only_rows_that_see_them(dim, what):
    """Position 20 of 30 reads back as NaN (in one dim of its values): rows 0 .. 3 of 14 end before it."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(dim)
    c = _cache(rng, 3, 16, 1, dim)
    c.raw[2] = 0xFF  # past the length: NaN throughout
    table = np.array([[1, 0, 2]])
    rec, d = c.record(table[0][1] * 16 + 4, 0), 9
    rec[op.place(d, 4, what == "values")] = 0xFF
    q = _round(torch, rng.normal(0, 1, (14, 1, dim)), "bf16")
    got, _ = _run(torch, B, c, "bf16", q, table, [30], 14, 1, True, 0.1, 48)
    ends = np.arange(14) + 17
    clean = op.Cache(3, 16, 1, dim)
    clean.raw[:] = c.raw
    clean.record(table[0][1] * 16 + 4, 0)[op.place(d, 4, what == "values")] = 0
    sees = ends > 20
    if what == "keys":
        assert np.isnan(got[sees]).all()
    else:
        assert np.isnan(got[sees][:, 0, d]).all() and np.isfinite(np.delete(got[sees][:, 0], d, -1)).all()
    kd, vd = _dense(clean)
    at = np.array([table[0][p // 16] * 16 + p % 16 for p in range(30)])
    want, _, mass = op.attention(q, kd[at], vd[at], 0.1, ends)
    dx = _score_error(q, kd[at], 0.1)[..., None]
    tol = 2.0 ** -8 * np.abs(want) + 1.01 * (2.0 ** -11 + 2 * dx) * mass + 2.0 ** -22 * np.abs(vd[at]).max()
    ok = np.abs(got - want) <= tol
    assert ok[~sees].all()
    if what == "values":
        assert np.delete(ok[sees][:, 0], d, -1).all()


def test_pages_and_lengths_that_are_not_there():
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(1)
    c = _cache(rng, 6, 16, 2, 64)
    q = _round(torch, rng.normal(0, 1, (4, 2, 64)), "bf16")
    table = np.array([[0, 1, 2], [3, 99, 4], [5, 1, -3], [2, 3, 4]])
    got, err = _run(torch, B, c, "bf16", q, table, [40, 40, 40, -2], 1, 2, True, 0.1, 48)
    assert err & B.WF_DEV_ERR_PAGE and not got[3].any()
    _check(torch, c, "bf16", q[:1], table[:1], [40], 1, 2, True, 0.1, got[:1])
    # positions of a block that is not there are not seen
    kd, vd = _dense(c)
    for i, blocks in ((1, ((3, 16), (4, 8))), (2, ((5, 16), (1, 16)))):
        at = np.concatenate([np.arange(b * 16, b * 16 + m) for b, m in blocks])
        want, _, mass = op.attention(q[i:i + 1], kd[at], vd[at], 0.1, [len(at)])
        assert (np.abs(got[i:i + 1] - want) <= 2.0 ** -7 * mass).all()
    _, err = _run(torch, B, c, "bf16", q, table[:, :2] % 6, [33, 5, 5, 5], 1, 2, True, 0.1, 32)
    assert err == B.WF_DEV_ERR_CAPACITY


def test_sequences_may_share_one_table_row():
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(2)
    c = _cache(rng, 4, 32, 1, 64)
    q = _round(torch, rng.normal(0, 1, (3, 2, 64)), "f16")
    table = np.array([[3, 1, 0]])
    got, err = _run(torch, B, c, "f16", q, table, [5, 70, 96], 1, 2, True, 0.1, 96, stride=0)
    assert err == 0
    _check(torch, c, "f16", q, np.repeat(table, 3, 0), [5, 70, 96], 1, 2, True, 0.1, got)


@pytest.mark.parametrize("dim", [64, 128])
def test_a_shared_row_is_read_as_far_as_lengths_go(dim):
    """A bound far above the lengths: what lies behind the row's columns is no block, and no error."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(3)
    c = _cache(rng, 4, 16, 1, dim)
    q = _round(torch, rng.normal(0, 1, (3, 2, dim)), "bf16")
    table = np.array([[2, 0] + [10 ** 6] * 40])
    lens = [0, 7, 32]
    got, err = _run(torch, B, c, "bf16", q, table, lens, 1, 2, True, 0.1, 600, stride=0)
    assert err == 0 and not got[0].any()
    _check(torch, c, "bf16", q, np.repeat(table, 3, 0), lens, 1, 2, True, 0.1, got)
    got, err = _run(torch, B, c, "bf16", q, np.repeat(table, 3, 0), lens, 1, 2, True, 0.1, 600)
    assert err == 0 and not got[0].any()
    _check(torch, c, "bf16", q, np.repeat(table, 3, 0), lens, 1, 2, True, 0.1, got)
