"""Prompt attention with starts that descend or leave the buffers: what is read and written, and that it is told (GPU)."""
import numpy as np
import pytest

from test_gpu_prompt_attention import GAP, _make, _run

pytestmark = pytest.mark.gpu


def _ascending(starts, n):
    """Query starts as they are taken: within the buffer, none below an earlier one, none above the last."""
    first = min(max(starts[0], 0), n)
    last = max(min(starts[-1], n), first)
    return [min(max(max(starts[:i + 1]), first), last) for i in range(len(starts))]


def _i32(torch, v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


BAD = [[GAP, 200, 103], [-5, 20, 10 ** 6], [50, 20, 30], [2 ** 31 - 1, -2 ** 31, 5], [GAP, 60, 20, 103], [0, 90, 3, 80, 10, 70], [103, 50, 0], [0, 40, 106, 107],
       [0, 106, 0, 106, 0, 106], [-1, 106], list(range(0, 40)) + [12, 50, 45, 106], [0] * 70 + [80, 20, 90], list(range(3, 103)) + [3]]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 64])
@pytest.mark.parametrize("bad", range(len(BAD)))
@pytest.mark.parametrize("cut", [False, True])
def test_query_starts(dim, group, bad, cut):
    """The bits of the call with those starts brought in order; rows of no sequence, and what lies beside rows, are left as they were."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(bad)
    hq, n = group, 106
    t = 3000 if cut else 60
    q, _, _ = _make(torch, rng, "bf16", dim, hq, 1, [100], [100])
    _, k, v = _make(torch, rng, "bf16", dim, hq, 1, [1], [t])
    q[:GAP], q[-GAP:] = 0.5, 0.25  # (rows that a start out of place names are rows)
    s = BAD[bad]
    m = len(s) - 1
    ks = _i32(torch, [GAP + t * i // m for i in range(m + 1)])
    good = _ascending(s, n)
    want, wl, err = _run(torch, B, "bf16", dim, hq, 1, q, k, v, _i32(torch, good), ks, m, True, 0.1, t)
    assert err == 0
    got, gl, err = _run(torch, B, "bf16", dim, hq, 1, q, k, v, _i32(torch, s), ks, m, True, 0.1, t)
    assert err == B.WF_DEV_ERR_PAGE
    assert torch.equal(got, want) and torch.equal(gl, wl)
    for x in (got, gl):
        assert (x[:good[0]] == 7).all() and (x[good[-1]:] == 7).all()
    assert (got[:, hq * dim:] == 7).all() and not (got[good[0]:good[-1], 0] == 7).any()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", [[GAP, 200, 103], [-5, 20, 10 ** 6], [50, 20, 30], [2 ** 31 - 1, -2 ** 31, 5], [90, 3, 2000]])
def test_key_starts(dim, bad):
    """A sequence's keys are from its start, within the buffer, to the next start, or none where that lies before it."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(9)
    hq, lens = 2, [40, 60]
    q, k, v = _make(torch, rng, "bf16", dim, hq, 1, lens, [100])
    k[:GAP], v[:GAP], k[-GAP:], v[-GAP:] = 1.0, 0.5, 0.25, -0.5
    qs = [GAP, GAP + 40, GAP + 100]
    got, gl, err = _run(torch, B, "bf16", dim, hq, 1, q, k, v, _i32(torch, qs), _i32(torch, bad), 2, True, 0.1, 106)
    assert err == B.WF_DEV_ERR_PAGE
    for x in (got, gl):
        assert (x[:GAP] == 7).all() and (x[-GAP:] == 7).all()
    assert (got[:, hq * dim:] == 7).all()
    for i in range(2):
        first = min(max(bad[i], 0), 106)
        keys = [first, max(min(max(bad[i + 1], 0), 106), first)]
        want, wl, err = _run(torch, B, "bf16", dim, hq, 1, q, k, v, _i32(torch, qs[i:i + 2]), _i32(torch, keys), 1, True, 0.1, 106)
        assert err == 0
        a, b = qs[i], qs[i + 1]
        assert torch.equal(got[a:b], want[a:b]) and torch.equal(gl[a:b], wl[a:b])


def test_a_start_behind_all_rows_is_told_of():
    """One row, and a hundred sequences without rows behind it, one of which begins before it; and a key start of a sequence without rows."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(2)
    q, k, v = _make(torch, rng, "bf16", 64, 1, 1, [1], [5])
    ks = [GAP] + [GAP + 5] * 100
    qs = [GAP] + [GAP + 1] * 100
    for a, b in ((qs, ks), (qs[:70] + [GAP] + qs[71:], ks), (qs, ks[:80] + [GAP + 4] + ks[81:])):
        out, _, err = _run(torch, B, "bf16", 64, 1, 1, q, k, v, _i32(torch, a), _i32(torch, b), 100, True, 0.1, 5)
        assert err == (0 if a == qs and b == ks else B.WF_DEV_ERR_PAGE)
        if err == 0:
            want = out
        assert torch.equal(out, want)
