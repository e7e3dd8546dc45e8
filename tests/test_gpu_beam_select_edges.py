"""Beam selection where the bound of a row's candidates is hard to find (GPU)."""
import numpy as np
import pytest

from test_gpu_beam_ops import _check_select, _select

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("W", [5, 9, 16])
@pytest.mark.parametrize("V,dtype", [(8192, "f32"), (16384, "bf16"), (16384, "f16")])
def test_groups_of_nan_are_no_candidates(W, V, dtype):
    """The second half of the vocabulary is NaN; of the first, every run of V / 64 logits has one that stands out,
    and eos is among the best.  NaN counts as -inf, so the finite ones fill every place."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    logits, run = np.full((1, W, V), -10.0), V // 64
    logits[:, :, V // 2:] = np.nan
    logits[:, :, 3:V // 2:run] = 5 + np.arange(32) / 4
    scores = np.full((1, W), -np.inf)
    scores[0, W // 2] = -1
    eos = 3 + 30 * run
    got, x = _select(torch, B, logits, scores, None, eos, dtype)
    _check_select(got, np.where(np.isnan(x), -np.inf, x), scores, None, eos)
    best = [3 + g * run for g in range(31, -1, -1) if g != 30][:W]
    assert got["token"][0].tolist() == best and (got["parent"][0] == W // 2).all()
    assert got["fin_parent"][0].tolist() == [W // 2] + [-1] * (W - 1)
