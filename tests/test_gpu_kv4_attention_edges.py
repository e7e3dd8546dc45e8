"""Attention over the 4-bit cache where a call is cut into chunks of positions (GPU).

A call is one chunk a CTA, a cluster of up to 8 chunks or more chunks joined by a
second kernel, by its sizes; what a row gets must not depend on which."""
import numpy as np
import pytest

from oracle import beam as ob
from test_gpu_beam_ops import _check_rows, _dev, _err, _filled, _i32, _pool

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
