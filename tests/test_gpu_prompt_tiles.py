"""Prompt attention where a CTA has two tiles with rows, and where keys are cut up, against the float64 restatement (GPU)."""
import numpy as np
import pytest

from oracle import prompt as op
from test_gpu_prompt_attention import GAP, _check, _make, _np, _run, _starts

pytestmark = pytest.mark.gpu

SMS = 152


def _pair(lens, hq, hkv):
    """Tokens of two tiles; the call has to be large enough for CTAs of two."""
    per = 2 * (128 // (hq // hkv))
    n = sum(lens) + 2 * GAP
    assert min(n, n // per + len(lens)) * hkv >= SMS
    return per


def _compare(dtype, dim, hq, hkv, q, k, v, lens, keys, causal, scale, out, lse, per):
    """Rows at the ends of tiles and some between, in a few heads; the bounds are those of _check, written out for chosen rows."""
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
    Q, K, V, O = _np(q, hq, dim), _np(k, hkv, dim), _np(v, hkv, dim), _np(out[:, :hq * dim], hq, dim)
    g, a, b = hq // hkv, GAP, GAP
    heads = sorted({0, hkv // 2, hkv - 1})
    pick_h = [h * g + j for h in heads for j in range(g)]
    for r, t in zip(lens, keys):
        if r == 0:
            b += t
            continue
        near = {x + e for x in range(0, r + per, per // 2) for e in (-1, 0, 1)} | {0, r // 3, r - 2, r - 1}
        near |= {r - t - 1, r - t, r - t + 1}  # the first rows that see something
        pick = np.array(sorted(x for x in near if 0 <= x < r))
        ends = t - (r - 1 - pick) if causal else np.full(len(pick), t)
        qq, kk, vv = Q[a + pick][:, pick_h], K[b:b + t][:, heads], V[b:b + t][:, heads]
        want, wl, mass = op.attention(qq, kk, vv, scale, ends)
        dx = 2.0 ** -24 * (dim + 16) * scale * np.abs(qq).max(-1) * np.abs(kk).sum(-1).max(initial=0) + 2.0 ** -20
        tol = u * np.abs(want) + (1 + u) * (u + 2 * dx[..., None]) * mass + (2.0 ** -24 if dtype == "f16" else 0.0)
        err = np.abs(O[a + pick][:, pick_h] - want)
        assert (err <= tol).all(), (r, t, np.argwhere(~(err <= tol))[:5], pick)
        got = lse[a + pick].double().cpu().numpy()[:, pick_h]
        f = np.isfinite(wl)
        assert (np.isfinite(got) == f).all() and (np.abs(got[f] - wl[f]) <= 2 * dx[f] + 2.0 ** -22 * np.abs(wl[f])).all()
        a, b = a + r, b + t
    for x in (out, lse):
        assert (x[:GAP] == 7).all() and (x[a:] == 7).all()
    assert (out[:, hq * dim:] == 7).all() and not torch_nan(out[GAP:-GAP]) and not torch_nan(lse[GAP:-GAP])


def torch_nan(x):
    return bool((x != x).any())


PAIRS = [
    # hq, hkv, dim, query rows, keys beyond them, causal
    (32, 32, 64, [1280], [0], True), (48, 16, 64, [1219], [130], True), (32, 8, 128, [1249], [1000], True), (20, 20, 128, [2000, 257], [0, 0], False),
    (24, 24, 64, [1500, 129, 1], [0, 700, 33], False), (40, 40, 64, [900], [-400], True), (20, 20, 128, [1537, 200], [-700, -200], True),
    (32, 32, 128, [300, 2304], [5, 0], True), (56, 8, 64, [700, 40], [64, 1300], True), (80, 16, 128, [470, 1], [999, 2303], True),
    (20, 20, 64, [7, 255, 256, 257, 129, 1, 0, 1100], [0, 1, 63, 64, 65, 0, 9, 0], True)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", range(len(PAIRS)))
def test_two_tiles(dtype, shape):
    import torch
    from paper_2609_32869_gb300 import binding as B
    hq, hkv, dim, lens, more, causal = PAIRS[shape]
    keys = [a + b for a, b in zip(lens, more)]
    per = _pair(lens, hq, hkv)
    rng = np.random.default_rng(100 + shape)
    q, k, v = _make(torch, rng, dtype, dim, hq, hkv, lens, keys)
    out, lse, err = _run(torch, B, dtype, dim, hq, hkv, q, k, v, _starts(torch, lens), _starts(torch, keys), len(lens), causal, dim ** -0.5, max(keys))
    assert err == 0
    _compare(dtype, dim, hq, hkv, q, k, v, lens, keys, causal, dim ** -0.5, out, lse, per)


@pytest.mark.parametrize("dim", [64, 128])
def test_two_tiles_with_rising_scores(dim):
    """Rows' references are raised again and again, in both tiles."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    hq, lens = 32, [1111]
    rng = np.random.default_rng(5)
    q, k, v = _make(torch, rng, "f16", dim, hq, hq, lens, lens, size=3.0)
    k *= torch.linspace(0.1, 4, k.shape[0], device="cuda").to(k.dtype)[:, None]
    out, lse, _ = _run(torch, B, "f16", dim, hq, hq, q, k, v, _starts(torch, lens), _starts(torch, lens), 1, True, 0.5, 1111)
    _compare("f16", dim, hq, hq, q, k, v, lens, lens, True, 0.5, out, lse, _pair(lens, hq, hq))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("at", [0, 127, 128, 200, 255, 256, 700])
def test_two_tiles_with_a_value_that_is_not_finite(dim, value, where, at):
    """Before, in and behind the block where the first tile of a CTA ends and the second goes on: rows that do not see it keep their bits."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    hq, lens, d, head = 32, [1111], 11, 3
    _pair(lens, hq, hq)
    rng = np.random.default_rng(6)
    q, k, v = _make(torch, rng, "bf16", dim, hq, hq, lens, lens)
    s = _starts(torch, lens)
    clean, _, _ = _run(torch, B, "bf16", dim, hq, hq, q, k, v, s, s, 1, True, 0.05, 1111)
    (k if where == "k" else v)[GAP + at, head * dim + d] = value
    got, _, _ = _run(torch, B, "bf16", dim, hq, hq, q, k, v, s, s, 1, True, 0.05, 1111)
    bits = lambda x: x[:, :hq * dim].contiguous().view(torch.int16).reshape(-1, hq, dim)  # noqa: E731
    a, b = bits(clean), bits(got)
    others = [h for h in range(hq) if h != head]
    assert torch.equal(a[:, others], b[:, others]) and torch.equal(a[:GAP + at, head], b[:GAP + at, head])
    seen = got[GAP + at:-GAP, head * dim:head * dim + dim]
    if where == "v":
        assert (torch.isnan(seen[:, d]) if value != value else seen[:, d] == value).all()
        rest = [e for e in range(dim) if e != d]
        assert torch.equal(a[:, head][:, rest], b[:, head][:, rest])
    elif value != value:
        assert torch.isnan(seen).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("r,t,causal", [(1, 9000, True), (20, 9000, True), (20, 2048, False), (130, 5001, True)])
def test_keys_cut_up(dtype, dim, r, t, causal):
    """Every row and head against float64, and rows in calls of their own: both differ by no more than both calls' bounds."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    hq, hkv, scale = 4, 2, dim ** -0.5
    rng = np.random.default_rng(r)
    q, k, v = _make(torch, rng, dtype, dim, hq, hkv, [r], [t])
    assert B.wf_prompt_attention_scratch_bytes(1, q.shape[0], t, hq, hkv, dim) > 0
    out, lse, err = _run(torch, B, dtype, dim, hq, hkv, q, k, v, _starts(torch, [r]), _starts(torch, [t]), 1, causal, scale, t)
    assert err == 0
    _check(dtype, dim, hq, hkv, q, k, v, [r], [t], causal, scale, out, lse, rows=40)
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
    for j in sorted({0, r // 2, r - 1}):
        keys = t - (r - 1 - j) if causal else t
        one = torch.tensor([GAP + j, GAP + j + 1], dtype=torch.int32, device="cuda")
        alone, _, err = _run(torch, B, dtype, dim, hq, hkv, q, k, v, one, _starts(torch, [keys]), 1, causal, scale, t)
        assert err == 0
        x, y = (_np(z[GAP + j:GAP + j + 1, :hq * dim], hq, dim)[0] for z in (out, alone))
        _, _, mass = op.attention(_np(q, hq, dim)[GAP + j:GAP + j + 1], _np(k, hkv, dim)[GAP:GAP + keys], _np(v, hkv, dim)[GAP:GAP + keys], scale, [keys])
        dx = 2.0 ** -24 * (dim + 16) * scale * np.abs(_np(q, hq, dim)[GAP + j]).max(-1) * np.abs(_np(k, hkv, dim)[GAP:GAP + t]).sum(-1).max() + 2.0 ** -20
        assert (np.abs(x - y) <= 2 * (1 + u) * (u + 2 * dx[:, None]) * mass[0] + 2 * u * np.maximum(np.abs(x), np.abs(y)) + 2.0 ** -23).all()
        assert (alone[:GAP + j] == 7).all() and (alone[GAP + j + 1:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,keys,causal", [
    ([2300], [2100], True), ([5, 3, 40, 0, 70], [5000, 3, 0, 9, 1029], True), ([33, 1], [2047, 4100], False), ([1] * 9, [1, 0, 2049, 5, 1024, 1025, 64, 4099, 2], True)])
def test_keys_cut_up_of_ragged_sequences(dtype, dim, lens, keys, causal):
    """Sequences whose keys end in an early part, that have none, and rows that see nothing of some parts or of any."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    hq, hkv = 2, 1
    rng = np.random.default_rng(len(lens))
    q, k, v = _make(torch, rng, dtype, dim, hq, hkv, lens, keys)
    assert B.wf_prompt_attention_scratch_bytes(len(lens), q.shape[0], max(keys), hq, hkv, dim) > 0
    out, lse, err = _run(torch, B, dtype, dim, hq, hkv, q, k, v, _starts(torch, lens), _starts(torch, keys), len(lens), causal, dim ** -0.5, max(keys))
    assert err == 0
    _check(dtype, dim, hq, hkv, q, k, v, lens, keys, causal, dim ** -0.5, out, lse, rows=60)
