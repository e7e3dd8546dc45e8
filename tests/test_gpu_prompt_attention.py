"""Attention of packed prompts against the float64 restatement (GPU)."""
import numpy as np
import pytest

from oracle import prompt as op

pytestmark = pytest.mark.gpu

GAP = 3  # rows before the first sequence and behind the last


def _dt(torch, name):
    return {"bf16": torch.bfloat16, "f16": torch.float16}[name]


def _make(torch, rng, dtype, dim, hq, hkv, lens, keys, size=1.0):
    """Rows of a fused projection; the rows around the sequences are NaN."""
    nq, nk = sum(lens) + 2 * GAP, sum(keys) + 2 * GAP
    q = rng.normal(0, size, (nq, hq * dim + 8))
    kv = rng.normal(0, 1, (nk, 2 * hkv * dim + 16))
    for x in (q, kv):
        x[:GAP], x[-GAP:] = np.nan, np.nan
    put = lambda x: torch.from_numpy(x.astype(np.float32)).cuda().to(_dt(torch, dtype))  # noqa: E731
    q, kv = put(q), put(kv)
    return q[:, :hq * dim], kv[:, :hkv * dim], kv[:, hkv * dim:2 * hkv * dim]


def _starts(torch, lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]) + GAP, dtype=torch.int32, device="cuda")


def _run(torch, B, dtype, dim, hq, hkv, q, k, v, qs, ks, n, causal, scale, max_k, lse=True):
    out = torch.full((q.shape[0], hq * dim + 8), 7.0, dtype=q.dtype, device="cuda")
    ls = torch.full((q.shape[0], hq), 7.0, device="cuda") if lse else None
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    size = B.wf_prompt_attention_scratch_bytes(n, q.shape[0], max_k, hq, hkv, dim)
    scratch = torch.full((size + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    B.wf_prompt_attention(q, q.stride(0), k, k.stride(0), v, v.stride(0), qs, ks, n, q.shape[0], k.shape[0], max_k, hq, hkv, dim,
                          B.WF_F16 if dtype == "f16" else B.WF_BF16, causal, scale, out, out.stride(0), ls, scratch, size, err)
    torch.cuda.synchronize()
    assert (scratch[size:] == 0xA5).all()
    return out, ls, err.item()


def _np(x, heads, dim):
    return x.double().cpu().numpy().reshape(-1, heads, dim)


def _check(dtype, dim, hq, hkv, q, k, v, lens, keys, causal, scale, out, lse, rows=None, bad=()):
    """rows: how many of a sequence's rows are compared (the first, the last and some between)."""
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
    Q, K, V, O = _np(q, hq, dim), _np(k, hkv, dim), _np(v, hkv, dim), _np(out[:, :hq * dim], hq, dim)
    a, b = GAP, GAP
    for i, (r, t) in enumerate(zip(lens, keys)):
        pick = np.arange(r) if rows is None or r <= rows else np.unique(np.concatenate([np.linspace(0, r - 1, rows).astype(int), np.arange(r - 3, r)]))
        ends = (t - (r - 1 - pick)) if causal else np.full(len(pick), t)
        want, wl, mass = op.attention(Q[a + pick], K[b:b + t], V[b:b + t], scale, ends)
        if len(pick) and t:
            # scores: fp32 sums of dim products in any order and the constants' roundings; weights: the type's rounding, the sum is not of
            # the rounded ones; the output's own rounding
            dx = 2.0 ** -24 * (dim + 16) * scale * np.abs(Q[a + pick]).max(-1) * np.abs(K[b:b + t]).sum(-1).max() + 2.0 ** -20
            tol = u * np.abs(want) + (1 + u) * (u + 2 * dx[..., None]) * mass + (2.0 ** -24 if dtype == "f16" else 0.0)
            err = np.abs(O[a + pick] - want)
            assert (err <= tol).all(), (i, r, t, np.nanmax(err / np.maximum(tol, 1e-300)), np.argwhere(~(err <= tol))[:5])
            if lse is not None:
                got = lse[a + pick].double().cpu().numpy()
                assert (np.isinf(got) == np.isinf(wl)).all()
                f = np.isfinite(wl)
                assert (np.abs(got - wl)[f] <= (2 * dx + 2.0 ** -22 * np.abs(wl))[f]).all()
        else:
            assert not O[a + pick].any()
        a, b = a + r, b + t
    for x in (out,) + (() if lse is None else (lse,)):
        assert (x[:GAP] == 7).all() and (x[a:] == 7).all()
    assert (out[:, hq * dim:] == 7).all()


SHAPES = [
    # hq, hkv, dim, query rows, keys beyond them, causal
    (1, 1, 64, [1], [0], True), (2, 1, 128, [1, 0, 2], [0, 0, 0], True), (4, 2, 64, [127, 128, 129, 1], [0] * 4, True),
    (3, 3, 128, [64, 65, 300], [0] * 3, True), (7, 1, 64, [18, 19, 37, 200], [0] * 4, True), (10, 2, 128, [25, 26, 51, 130], [0] * 4, True),
    (8, 1, 128, [16, 33, 257], [0] * 3, True), (4, 1, 64, [1, 5, 40], [130, 1000, 255], True), (8, 2, 128, [3, 1, 70], [2000, 0, 129], True),
    (2, 2, 64, [200, 1, 131], [0, 50, 7], False), (5, 1, 128, [100, 1], [0, 300], False), (6, 2, 64, [0, 0, 9], [5, 0, 0], True),
    (64, 1, 64, [1, 2, 5], [0, 40, 3], True), (33, 1, 128, [4, 7], [0, 129], True), (1, 1, 128, [700], [0], True), (2, 1, 64, [513, 256], [0, 0], False)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_against_the_oracle(dtype, shape):
    import torch
    from paper_2609_32869_gb300 import binding as B
    hq, hkv, dim, lens, more, causal = SHAPES[shape]
    keys = [a + b for a, b in zip(lens, more)]
    rng = np.random.default_rng(shape)
    q, k, v = _make(torch, rng, dtype, dim, hq, hkv, lens, keys)
    out, lse, err = _run(torch, B, dtype, dim, hq, hkv, q, k, v, _starts(torch, lens), _starts(torch, keys), len(lens), causal, dim ** -0.5, max(max(keys), 1))
    assert err == 0
    _check(dtype, dim, hq, hkv, q, k, v, lens, keys, causal, dim ** -0.5, out, lse, rows=40)


@pytest.mark.parametrize("dim", [64, 128])
def test_more_rows_than_keys(dim):
    """Causal, r > t: the first r - t rows see nothing; without causal a sequence without keys gives zeros."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(7)
    lens, keys = [150, 5, 40, 300], [20, 0, 39, 160]
    q, k, v = _make(torch, rng, "bf16", dim, 2, 1, lens, keys)
    for causal in (True, False):
        out, lse, err = _run(torch, B, "bf16", dim, 2, 1, q, k, v, _starts(torch, lens), _starts(torch, keys), 4, causal, 0.1, 160)
        assert err == 0
        _check("bf16", dim, 2, 1, q, k, v, lens, keys, causal, 0.1, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_large_and_rising_scores(dtype, dim):
    """Row maxima that rise along the keys by far more than one rescaling's worth, and weights of a single key."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(11)
    lens = [400]
    q, k, v = _make(torch, rng, dtype, dim, 2, 2, lens, lens, size=3.0)
    k *= torch.linspace(0.1, 4, k.shape[0], device="cuda").to(k.dtype)[:, None]
    out, lse, _ = _run(torch, B, dtype, dim, 2, 2, q, k, v, _starts(torch, lens), _starts(torch, lens), 1, True, 0.5, 400)
    _check(dtype, dim, 2, 2, q, k, v, lens, lens, True, 0.5, out, lse, rows=100)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", ["k", "v"])
def test_what_is_masked_does_not_reach_a_row(dim, value, where):
    """A key or value that is not finite at position 75 of 200 changes no row before it; its rows show it in that dim."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(13)
    lens, at, d = [90, 200], 75, 5
    q, k, v = _make(torch, rng, "bf16", dim, 4, 2, lens, lens)
    qs = _starts(torch, lens)
    clean, _, _ = _run(torch, B, "bf16", dim, 4, 2, q, k, v, qs, qs, 2, True, 0.1, 200)
    (k if where == "k" else v)[GAP + 90 + at, dim + d] = value  # the second head
    got, _, _ = _run(torch, B, "bf16", dim, 4, 2, q, k, v, qs, qs, 2, True, 0.1, 200)
    a, b = _np(clean[:, :4 * dim], 4, dim), _np(got[:, :4 * dim], 4, dim)
    first = GAP + 90 + at
    np.testing.assert_array_equal(a[:first], b[:first])
    np.testing.assert_array_equal(a[:, :2], b[:, :2])
    if where == "v":
        seen = b[first:first + 200 - at, 2:, d]
        assert (np.isnan(seen) if np.isnan(value) else seen == value).all()
        # (the other dims go through other sums: their weights are the same)
        np.testing.assert_array_equal(np.delete(a, d, -1), np.delete(b, d, -1))
    elif np.isnan(value):
        assert np.isnan(b[first:first + 200 - at, 2:]).all()


def test_bounds_and_bad_starts():
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(17)
    lens = [40, 60]
    q, k, v = _make(torch, rng, "bf16", 64, 2, 1, lens, lens)
    qs = _starts(torch, lens)
    # keys past max_k are not seen
    out, lse, err = _run(torch, B, "bf16", 64, 2, 1, q, k, v, qs, qs, 2, False, 0.1, 40)
    assert err == B.WF_DEV_ERR_CAPACITY
    keep = GAP + 40 + 40
    short = torch.tensor([GAP, GAP + 40, keep], dtype=torch.int32, device="cuda")
    want, _, err = _run(torch, B, "bf16", 64, 2, 1, q, k, v, qs, short, 2, False, 0.1, 40)
    assert err == 0 and torch.equal(out, want)
    # starts that descend or leave the buffers: nothing outside is read or written
    for bad in ([GAP, 200, 103], [-5, 20, 10 ** 6], [50, 20, 30], [2 ** 31 - 1, -2 ** 31, 5]):
        s = torch.tensor(bad, dtype=torch.int32, device="cuda")
        for a, b in ((s, qs), (qs, s), (s, s)):
            _, _, err = _run(torch, B, "bf16", 64, 2, 1, q, k, v, a, b, 2, True, 0.1, 60)
            assert err & B.WF_DEV_ERR_PAGE


def test_no_lse_and_many_short_sequences():
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(19)
    lens = [int(x) for x in rng.integers(0, 9, 700)]
    q, k, v = _make(torch, rng, "bf16", 64, 2, 2, lens, lens)
    s = _starts(torch, lens)
    out, _, err = _run(torch, B, "bf16", 64, 2, 2, q, k, v, s, s, len(lens), True, 0.125, 9, lse=False)
    assert err == 0
    _check("bf16", 64, 2, 2, q, k, v, lens, lens, True, 0.125, out, None)


@pytest.mark.parametrize("r,t", [(1, 9000), (20, 9000), (300, 5000)])
def test_few_rows_behind_many_keys(r, t):
    """The keys may be cut up and joined: the same rows as in a call of one row each, within both calls' roundings."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(r)
    q, k, v = _make(torch, rng, "f16", 128, 8, 2, [r], [t])
    out, lse, _ = _run(torch, B, "f16", 128, 8, 2, q, k, v, _starts(torch, [r]), _starts(torch, [t]), 1, True, 128 ** -0.5, t)
    _check("f16", 128, 8, 2, q, k, v, [r], [t], True, 128 ** -0.5, out, lse, rows=8)


def test_runs_are_equal_and_graphs_replay():
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(23)
    lens = [5, 300, 77]
    q, k, v = _make(torch, rng, "bf16", 128, 8, 2, lens, lens)
    s = _starts(torch, lens)
    out = torch.full((q.shape[0], 8 * 128), 7.0, dtype=q.dtype, device="cuda")
    size = B.wf_prompt_attention_scratch_bytes(3, q.shape[0], 300, 8, 2, 128)
    scratch = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")

    def call():
        B.wf_prompt_attention(q, q.stride(0), k, k.stride(0), v, v.stride(0), s, s, 3, q.shape[0], k.shape[0], 300, 8, 2, 128, B.WF_BF16, True, 0.1, out,
                              out.stride(0), None, scratch, size)

    call()
    first = out.clone()
    for _ in range(5):
        out.fill_(7.0)
        call()
        assert torch.equal(out, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    q.mul_(2)
    out.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    doubled = out.clone()
    out.fill_(7.0)
    call()
    assert torch.equal(out, doubled) and not torch.equal(out, first)
