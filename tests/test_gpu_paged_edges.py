"""Block tables, slots and rows of the paged 4-bit cache at the edges of what the calls promise (GPU)."""
import numpy as np
import pytest

from oracle import beam as ob
from test_gpu_beam_ops import GUARD, _dev, _err, _i32, _pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("W,parent", [(2, [-1, -1]), (2, [0, 0]), (5, [4, 4, 4, 4, 4]), (16, [-1] * 16)])
@pytest.mark.parametrize("bad", [8, 99, 2 ** 31 - 1])
def test_reorder_does_not_free_ids_outside_the_pool(W, parent, bad):
    """A full column of a beam that no child takes names a block past the pool: reported, not pushed; the others are."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    blocks, cols = 8, 3
    raw = torch.full((blocks * 1152,), GUARD, dtype=torch.uint8, device="cuda")
    pool = B.kv4_pool(raw, 1, blocks, 16, 1, 64)
    table = np.tile([0, 1, 2], (W, 1))
    table[1] = [0, bad, 5]                   # full columns 0 to 2, beam 1 apart from column 1 on
    nb, err, left = B.wf_beam_reorder_scratch_bytes(1, W, cols), _err(torch), _err(torch)
    sc, free = torch.empty(nb, dtype=torch.uint8, device="cuda"), _i32(torch, [3, 4, 6, 7, -9, -9, -9, -9])
    out = _i32(torch, table)
    B.wf_beam_reorder(pool, _i32(torch, table), out, cols, _i32(torch, [48] * W), _i32(torch, parent), 1, W, free, _i32(torch, [4]),
                      left, sc, nb, err)
    new, freed, _ = ob.beam_reorder(table, 48, parent, 16)
    freed = [b for b in freed if b < blocks]
    assert err.item() == B.WF_DEV_ERR_PAGE
    np.testing.assert_array_equal(out.cpu().numpy(), new)
    assert left.item() == 4 + len(freed) and free.tolist() == [3, 4, 6, 7] + freed + [-9] * (4 - len(freed))


def test_reorder_reports_ids_outside_the_pool_that_stay():
    """The beam that names one goes on: its row keeps the entry, the call reports it."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    raw = torch.full((4 * 1152,), GUARD, dtype=torch.uint8, device="cuda")
    pool = B.kv4_pool(raw, 1, 4, 16, 1, 64)
    nb, err, left = B.wf_beam_reorder_scratch_bytes(1, 1, 2), _err(torch), _err(torch)
    sc, table, free = torch.empty(nb, dtype=torch.uint8, device="cuda"), _i32(torch, [[4, 1]]), _i32(torch, [2, 3, -1, -1])
    B.wf_beam_reorder(pool, table, table, 2, _i32(torch, [32]), _i32(torch, [0]), 1, 1, free, _i32(torch, [2]), left, sc, nb, err)
    assert err.item() == B.WF_DEV_ERR_PAGE and table.tolist() == [[4, 1]] and left.item() == 2


@pytest.mark.parametrize("n", [2, 16, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_slot_named_twice_leaves_the_others_alone(n, dtype):
    """What such a slot holds is not promised; every other slot is, and so is what lies around the cache.  Both ways of
    storing a row take part: whole records and single rows."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(n)
    heads, bs, blocks, twice = 2, 16, 4, 21
    cache = ob.Cache(blocks, bs, heads, 64, dtype, fill=GUARD)
    k, v = (ob.round16(rng.normal(size=(n, heads * 64)), dtype) for _ in range(2))
    slots = np.array(([twice, twice] + [twice + 16] * 14 if n <= 16 else list(range(16, 32)) + [twice] * 8 + list(range(32, 48)))[:n], np.int32)
    shared = [s for s in set(slots.tolist()) if (slots == s).sum() > 1]
    for i, s in enumerate(slots):
        cache.put(s, k[i], 0)
        cache.put(s, v[i], 1)
    raw = torch.full((cache.raw.size + 4096,), GUARD, dtype=torch.uint8, device="cuda")
    err, d = _err(torch), heads * 64
    B.wf_kv4_store(_pool(B, raw, cache), 0, _dev(torch, k, dtype), d, _dev(torch, v, dtype), d, _i32(torch, slots), n, err)
    got = raw.cpu().numpy()
    assert err.item() == 0 and (got[cache.raw.size:] == GUARD).all()
    got, want = got[:cache.raw.size].reshape(cache.raw.shape).copy(), cache.raw.copy()
    for s in shared:                                     # a shared slot's own bytes may hold anything
        p, record = s % 16, np.s_[s // bs, :, s % bs // 16]
        mine = [ob.code_place(p, d, w)[0] for d in range(64) for w in (0, 1)] + [ob.scale_place(p, w) + b for w in (0, 1) for b in range(4)]
        for x in (got, want):
            x[record][:, mine] = 0
    np.testing.assert_array_equal(got, want)
