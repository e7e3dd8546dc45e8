"""Prompt attention and the output projection directly behind it, both with accumulators in TMEM (GPU)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,hq,hkv,lens", [(64, 4, 4, [300, 17]), (64, 20, 20, [90] * 16), (128, 8, 2, [700]), (64, 2, 1, [1])])
@pytest.mark.parametrize("m", [160, 900])
def test_projection_right_behind(dim, hq, hkv, lens, m):
    """Calls in a row without a pause, eager and replayed, give the bits of calls that are waited for."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    torch.manual_seed(dim)
    n, w = max(sum(lens), m), hq * dim
    x = torch.randn(n, (hq + 2 * hkv) * dim, device="cuda").bfloat16()
    weight = torch.randn(512, w, device="cuda").bfloat16()
    out, y = torch.zeros(n, w, dtype=torch.bfloat16, device="cuda"), torch.zeros(m, 512, device="cuda")
    start = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    size = B.wf_prompt_attention_scratch_bytes(len(lens), n, max(lens), hq, hkv, dim)
    scratch = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
    need = B.wf_gemm_scratch_bytes(m, 512, w)
    room = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")

    def call(wait):
        s = x.stride(0)
        B.wf_prompt_attention(x, s, x[:, hq * dim:], s, x[:, (hq + hkv) * dim:], s, start, start, len(lens), n, n, max(lens), hq, hkv, dim, B.WF_BF16, True,
                              dim ** -0.5, out, w, None, scratch, size)
        if wait:
            torch.cuda.synchronize()
        B.wf_gemm_bf16(out, weight, None, y, m, 512, w, room, need)
        if wait:
            torch.cuda.synchronize()

    call(True)
    want = out.clone(), y.clone()
    rows = min(m, sum(lens))
    exact = out[:rows].double() @ weight.double().T
    # fp32 sums of w exact products
    assert ((y[:rows].double() - exact).abs() <= 2.0 ** -24 * (w + 2) * (out[:rows].double().abs() @ weight.double().abs().T)).all()
    for _ in range(50):
        out.zero_(), y.zero_()
        call(False)
    assert torch.equal(out, want[0]) and torch.equal(y, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(20):
            call(False)
    out.zero_(), y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(y, want[1])
