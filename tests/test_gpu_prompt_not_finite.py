"""Prompt attention where keys, values or queries that a row sees are not finite, with the keys in one piece and cut up (GPU)."""
import numpy as np
import pytest

from test_gpu_prompt_attention import GAP, _make, _np, _run, _starts

pytestmark = pytest.mark.gpu


def _cut(B, nq, t, hq, hkv, dim):
    return B.wf_prompt_attention_scratch_bytes(1, nq, t, hq, hkv, dim) > 0


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("top,at", [(5500, 100), (40, 3000), (3000, 5999), (40, 5999)])
@pytest.mark.parametrize("what", ["key", "value", "inf", "-inf"])
def test_a_part_far_below_the_largest_score(dtype, dim, top, at, what):
    """Keys in five parts; one position's score is 256 above all others, so every other part's factor is 0 in fp32.  A NaN that a row sees in one
    of those still makes NaN of it, an infinite value something that is not finite, each in its dim alone."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(top)
    r, t, hq, hkv, d = 2, 6000, 2, 1, 5
    q, k, v = _make(torch, rng, dtype, dim, hq, hkv, [r], [t])
    assert _cut(B, q.shape[0], t, hq, hkv, dim)
    q[GAP:-GAP] = 0
    q[GAP:-GAP, ::dim] = 16.0
    k[GAP:-GAP, 0] = 0
    k[GAP + top, 0] = 16.0
    qs, ks = _starts(torch, [r]), _starts(torch, [t])
    clean, lse, err = _run(torch, B, dtype, dim, hq, hkv, q, k, v, qs, ks, 1, True, 1.0, t)
    assert err == 0
    a = _np(clean[:, :hq * dim], hq, dim)
    # e^-256 is 0 beside 1: the one value and the one score
    np.testing.assert_array_equal(a[GAP:-GAP], np.broadcast_to(_np(v, 1, dim)[GAP + top], (r, hq, dim)))
    assert (lse[GAP:-GAP] == 256).all()
    if what == "key":
        k[GAP + at, 3] = float("nan")
    else:
        v[GAP + at, d] = float("nan") if what == "value" else float(what)
    got, lse, err = _run(torch, B, dtype, dim, hq, hkv, q, k, v, qs, ks, 1, True, 1.0, t)
    assert err == 0
    b = _np(got[:, :hq * dim], hq, dim)
    seen = [j for j in range(r) if at < t - (r - 1 - j)]
    assert len(seen) == (1 if at == t - 1 else r)
    for j in range(r):
        if j not in seen:
            np.testing.assert_array_equal(a[GAP + j], b[GAP + j])
            assert (lse[GAP + j] == 256).all()
        elif what == "key":
            assert np.isnan(b[GAP + j]).all() and torch.isnan(lse[GAP + j]).all()
        else:
            assert (np.isnan if what == "value" else lambda x: ~np.isfinite(x))(b[GAP + j, :, d]).all()
            np.testing.assert_array_equal(np.delete(a[GAP + j], d, -1), np.delete(b[GAP + j], d, -1))
            assert (lse[GAP + j] == 256).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("first", ["value", "-inf", "key", "query"])
@pytest.mark.parametrize("cut", [False, True])
def test_an_infinite_value_hides_no_nan(dtype, dim, first, cut):
    """A NaN (in an earlier value, key or the row's query), or the opposite infinity, and then an infinite value of the same dim in the block where
    the rows' sight ends: NaN, whichever block each lies in."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(3)
    r, t = (70, 6070) if cut else (200, 200)
    hq, hkv, d, late = 2, 1, 7, t - 10
    q, k, v = _make(torch, rng, dtype, dim, hq, hkv, [r], [t])
    assert _cut(B, q.shape[0], t, hq, hkv, dim) == cut
    rows = slice(GAP + r - 10, GAP + r)  # those that see `late`
    v[GAP + late, d] = float("inf")
    qs, ks = _starts(torch, [r]), _starts(torch, [t])
    only, _, _ = _run(torch, B, dtype, dim, hq, hkv, q, k, v, qs, ks, 1, True, 0.1, t)
    o = _np(only[:, :hq * dim], hq, dim)
    assert (o[rows, :, d] == np.inf).all() and np.isfinite(np.delete(o[rows], d, -1)).all() and np.isfinite(o[GAP:GAP + r - 10]).all()
    for at in (10, t - 30):  # in a block that all rows of the last tile see, and in one that they do not
        v2, k2, q2 = v.clone(), k.clone(), q.clone()
        if first == "query":
            q2[GAP + r - 3, 2] = float("nan")
        elif first == "key":
            k2[GAP + at, 2] = float("nan")
        else:
            v2[GAP + at, d] = float("nan") if first == "value" else float(first)
        got, _, _ = _run(torch, B, dtype, dim, hq, hkv, q2, k2, v2, qs, ks, 1, True, 0.1, t)
        g = _np(got[:, :hq * dim], hq, dim)
        if first == "query":
            assert np.isnan(g[GAP + r - 3, 0]).all()
            np.testing.assert_array_equal(g[GAP + r - 3, 1], o[GAP + r - 3, 1])
        elif first == "key":
            assert np.isnan(g[rows]).all()
        else:
            assert np.isnan(g[rows, :, d]).all()
            np.testing.assert_array_equal(np.delete(g[rows], d, -1), np.delete(o[rows], d, -1))
