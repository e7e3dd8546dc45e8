"""8-bit cache attention reads of a table what the lengths ask for, wherever the table lies (GPU)."""
import numpy as np
import pytest

from test_gpu_kv8 import _cache, _check, _f64, _i32, _pool, _round

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens", [[40, 64, 7], [0, 33, 0], [64], [1]])
def test_the_last_columns_of_a_wider_table(dim, lens):
    """A layer's columns at the end of a table of several, max_len the stride's: the last row has fewer columns behind it than max_len asks for.
    The output is that of a table of its own with every column up to max_len."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(4)
    bs, wide, cols, n, hq = 16, 24, 4, len(lens), 2
    c = _cache(rng, n * cols, bs, 1, dim)
    q = _round(torch, rng.normal(0, 1, (n, hq, dim)), "bf16")
    ids = rng.permutation(n * cols).reshape(n, cols)
    table = torch.full((n, wide), -1, dtype=torch.int32, device="cuda")
    table[:, wide - cols:] = _i32(torch, ids)
    own = torch.full((n, wide), -1, dtype=torch.int32, device="cuda")
    own[:, :cols] = _i32(torch, ids)
    raw, rows = torch.from_numpy(c.raw.copy()).cuda(), torch.from_numpy(q.reshape(n, -1)).cuda().bfloat16()
    outs = []
    for t in (table[:, wide - cols:], own):
        out, err = torch.full_like(rows, 7.0), _i32(torch, [0])
        B.wf_kv8_attention(_pool(B, raw, c, "bf16"), 0, rows, hq * dim, t, wide, _i32(torch, lens), n, 1, hq, True, 0.1, wide * bs, out, hq * dim, None, 0, err)
        assert err.item() == 0
        outs.append(out)
    assert torch.equal(outs[0], outs[1])
    _check(torch, c, "bf16", q, ids, lens, 1, hq, True, 0.1, _f64(outs[0]).reshape(n, hq, dim))
