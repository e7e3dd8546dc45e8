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


@pytest.mark.parametrize("n,W,V,dtype", [(3, 4, 51865, "bf16"), (1, 16, 9001, "f16"), (2, 8, 4097, "bf16"), (200, 4, 9000, "f16"), (70, 5, 20011, "f32"),
                                         (1, 2, 600007, "bf16"), (6, 12, 51866, "bf16"), (9, 3, 517, "f16"), (4, 1, 30000, "bf16")])
def test_a_beams_tokens_follow_the_order_of_its_logits(n, W, V, dtype):
    """16-bit logits are full of equal ones.  Which beam is ahead may turn on a rounding; within a beam the order is
    defined (larger logit, then lower id), so the tokens taken from a beam are the first ones of its order, and the k-th
    score is the k-th of the exact ones to within the rounding of a score."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(V + W)
    logits = rng.normal(0, 2, (n, W, V))
    scores, eos = -rng.uniform(0, 4, (n, W)), V // 3
    logits[:, W // 2, eos] = logits[:, W // 2].max(-1)
    sup = rng.random(V) < 0.02
    sup[eos] = False
    got, x = _select(torch, B, logits, scores, sup, eos, dtype, pad=1)
    x, scores = x.astype(np.float64), scores.astype(np.float32).astype(np.float64)
    for i in range(n):
        ranked = []
        order = []
        for w in range(W):
            y = np.where(sup, -np.inf, x[i, w])
            best = np.lexsort((np.arange(V), -y))[:2 * W]
            order.append(best.tolist())
            total = scores[i, w] + (y[best] - y.max()) - np.log(np.exp(y - y.max()).sum())
            ranked += [(-t, w, r, int(b)) for r, (t, b) in enumerate(zip(total, best))]
        # a score: the difference with the maximum, the logarithm and two sums, each rounded to 2^-24 of its size
        tol = 4 * 2.0 ** -23 * (1 + np.abs(scores[i]).max() + 2 * np.abs(x[i]).max())
        exact = sorted(ranked)[:2 * W]
        ended = [(w, s) for w, s in zip(got["fin_parent"][i].tolist(), got["fin_score"][i].tolist()) if w >= 0]
        want = np.array([-t for t, _, _, b in exact if b != eos][:W])
        assert (np.diff(got["score"][i]) <= 0).all()
        if len(ended) == sum(b == eos for _, _, _, b in exact[:W]):
            assert np.abs(got["score"][i] - want).max() <= tol
        for w in range(W):
            mine = got["token"][i][got["parent"][i] == w].tolist()
            rest = [b for b in order[w] if b != eos]
            assert mine == rest[:len(mine)], (i, w)
        for w, s in ended:
            assert any(abs(-t - s) <= tol for t, v, _, b in ranked if v == w and b == eos)
