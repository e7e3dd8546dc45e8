"""Rotary positions of 16-bit rows where a CTA takes several of them (GPU)."""
import numpy as np
import pytest

from test_gpu_rope import _case, _code, _size, _tol, _want
from oracle import prompt as op

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("n,hq,hkv,dim,rot,lead", [
    (2000, 4, 2, 128, 128, 0), (5003, 1, 1, 64, 64, 8), (6001, 3, 1, 64, 32, 0), (2500, 2, 1, 80, 30, 0), (1217, 5, 5, 64, 64, 0), (9001, 2, 0, 256, 254, 2)])
def test_many_rows(dtype, layout, n, hq, hkv, dim, rot, lead):
    """Some rows against float64, and all of them the bits of calls of a few rows each, out of place and in place."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    x, q, k, pos = _case(torch, n, hq, hkv, dim, dtype, n, lead)
    t, code = B.wf_rope_init(dim, rot, layout), _code(B, dtype)
    p = torch.tensor(pos, dtype=torch.int32, device="cuda")
    width = (hq + hkv) * dim
    whole, parts = (torch.full((n + 1, width), 7.0, dtype=x.dtype, device="cuda") for _ in range(2))

    def call(out, a, b):
        B.wf_rope(t, q[a:], x.stride(0), hq, k[a:] if hkv else None, x.stride(0), hkv, p[a:], b - a, code, False, out[a:], width,
                  out[a:, hq * dim:] if hkv else None, width)

    call(whole, 0, n)
    for a in range(0, n, 7):
        call(parts, a, min(a + 7, n))
    assert torch.equal(whole, parts) and (whole[n:] == 7).all()
    rows = np.unique(np.concatenate([np.arange(9), np.linspace(0, n - 1, 30).astype(int), np.arange(n - 9, n)]))
    src = x[torch.tensor(rows, device="cuda"), lead:lead + width]
    want = _want(src, hq + hkv, dim, pos[rows], op.frequencies(rot), interleaved=bool(layout))
    got = whole[torch.tensor(rows, device="cuda")].double().cpu().numpy().reshape(want.shape)
    assert (np.abs(got - want) <= _tol(dtype, _size(src, hq + hkv, dim, rot, bool(layout)))).all()
    B.wf_rope(t, q, x.stride(0), hq, k if hkv else None, x.stride(0), hkv, p, n, code, False, q, x.stride(0), k if hkv else None, x.stride(0))
    assert torch.equal(x[:, lead:lead + width], whole[:n])
