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
