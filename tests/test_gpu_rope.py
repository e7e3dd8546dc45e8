"""Rotary positions against the float64 restatement (GPU)."""
import numpy as np
import pytest

from oracle import prompt as op

pytestmark = pytest.mark.gpu

SCALED = {"plain": {}, "linear": dict(factor=8.0), "base": dict(factor=8.0), "waves": dict(factor=8.0, trained_len=8192.0, low=1.0, high=4.0),
          "parts": dict(factor=8.0, trained_len=8192.0, low=1.0, high=32.0)}


def _dt(torch, name):
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[name]


def _code(B, name):
    return {"bf16": B.WF_BF16, "f16": B.WF_F16, "f32": B.WF_F32}[name]


def _tol(dtype, pair_size):
    """fp32: cos and sin within 2^-22 (their own two steps, the angle's 2^-28 of a turn and the gain), two products and a sum: 2^-21 of the pair's size.
    Then the type's own rounding."""
    u = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}[dtype]
    return (2.0 ** -21 + u) * pair_size + (2.0 ** -25 if dtype == "f16" else 0.0)


def _case(torch, n, hq, hkv, dim, dtype, seed, lead=0, far=1 << 20):
    rng = np.random.default_rng(seed)
    width = lead + (hq + 2 * hkv) * dim
    x = torch.from_numpy(rng.normal(0, 2, (n, width)).astype(np.float32)).cuda().to(_dt(torch, dtype))
    pos = rng.integers(-5, far, n)
    pos[:4] = (0, 1, 2 ** 31 - 1, -2 ** 31)[:len(pos[:4])]
    q, k = x[:, lead:lead + hq * dim], x[:, lead + hq * dim:lead + (hq + hkv) * dim]
    return x, q, k, pos


def _want(x, heads, dim, pos, freq, **kw):
    return op.rope(x.double().cpu().numpy().reshape(len(pos), heads, dim), pos, freq, **kw)


def _size(x, heads, dim, rot, inter):
    """Of each value the length of its pair."""
    v = np.abs(x.double().cpu().numpy().reshape(x.shape[0], heads, dim)).copy()
    head = v[..., :rot]
    both = np.hypot(head[..., 0::2], head[..., 1::2]) if inter else np.hypot(head[..., :rot // 2], head[..., rot // 2:])
    v[..., :rot] = np.repeat(both, 2, -1) if inter else np.concatenate([both, both], -1)
    return v


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("n,hq,hkv,dim,rot,lead", [
    (1, 1, 1, 64, 64, 0), (5, 4, 2, 128, 128, 0), (3, 2, 1, 128, 64, 8), (7, 3, 3, 80, 30, 0), (4, 1, 1, 96, 20, 4), (2, 2, 2, 256, 256, 0),
    (3, 5, 1, 65, 64, 1), (2, 1, 1, 2, 2, 0), (2, 3, 1, 66, 2, 2), (9, 7, 1, 64, 8, 0), (2, 1, 1, 600, 256, 0)])
def test_rows(dtype, layout, n, hq, hkv, dim, rot, lead):
    import torch
    from paper_2609_32869_gb300 import binding as B
    x, q, k, pos = _case(torch, n, hq, hkv, dim, dtype, n * dim + rot, lead)
    t = B.wf_rope_init(dim, rot, layout)
    p = torch.tensor(pos, dtype=torch.int32, device="cuda")
    qo, ko = torch.full((n + 1, hq * dim + 3), 7.0, dtype=x.dtype, device="cuda"), torch.full((n + 1, hkv * dim + 5), 7.0, dtype=x.dtype, device="cuda")
    B.wf_rope(t, q, x.stride(0), hq, k, x.stride(0), hkv, p, n, _code(B, dtype), False, qo, qo.stride(0), ko, ko.stride(0))
    freq = op.frequencies(rot)
    for src, out, heads in ((q, qo, hq), (k, ko, hkv)):
        got = out[:n, :heads * dim].double().cpu().numpy().reshape(n, heads, dim)
        err = np.abs(got - _want(src, heads, dim, pos, freq, interleaved=bool(layout)))
        assert (err <= _tol(dtype, _size(src, heads, dim, rot, bool(layout)))).all(), err.max()
        np.testing.assert_array_equal(got[..., rot:], src.double().cpu().numpy().reshape(n, heads, dim)[..., rot:])
        assert (out[n:] == 7).all() and (out[:, heads * dim:] == 7).all()


@pytest.mark.parametrize("name", list(SCALED))
@pytest.mark.parametrize("n", [2, 3000])
def test_scalings_and_gradients(name, n):
    """Every scaling, at far positions; the adjoint is the transposed turn: <g, R x> = <R^T g, x>."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    hq, hkv, dim, gain = 4, 2, 128, 1.25
    x, q, k, pos = _case(torch, n, hq, hkv, dim, "f32", n, far=2_000_000)
    t = B.wf_rope_init(dim, 96, B.WF_ROPE_INTERLEAVED, 10000.0, B.WF_ROPE_PLAIN + list(SCALED).index(name), gain=gain, **SCALED[name])
    p = torch.tensor(pos, dtype=torch.int32, device="cuda")
    out, back = torch.empty(n, (hq + hkv) * dim, device="cuda"), torch.empty(n, (hq + hkv) * dim, device="cuda")
    for o, adjoint in ((out, False), (back, True)):
        B.wf_rope(t, q, x.stride(0), hq, k, x.stride(0), hkv, p, n, B.WF_F32, adjoint, o, o.stride(0), o[:, hq * dim:], o.stride(0))
    freq = op.frequencies(96, scaling=name, **SCALED[name])
    few = slice(0, min(n, 40))
    for o, adjoint in ((out, False), (back, True)):
        want = _want(x[few, :(hq + hkv) * dim], hq + hkv, dim, pos[few], freq, interleaved=True, gain=gain, adjoint=adjoint)
        err = np.abs(o[few].double().cpu().numpy().reshape(want.shape) - want)
        assert (err <= gain * _tol("f32", _size(x[few, :(hq + hkv) * dim], hq + hkv, dim, 96, True))).all(), err.max()
    # a different gradient g: sums of n * 768 products, each off by the two results' errors
    g = torch.randn(n, (hq + hkv) * dim, device="cuda")
    rg = torch.empty_like(g)
    B.wf_rope(t, g, g.stride(0), hq, g[:, hq * dim:], g.stride(0), hkv, p, n, B.WF_F32, True, rg, rg.stride(0), rg[:, hq * dim:], rg.stride(0))
    xs = x[:, :(hq + hkv) * dim].double()
    a, b = (g.double() * out.double()).sum(), (rg.double() * xs).sum()
    assert abs(a - b) <= 2.0 ** -19 * gain * (g.double().norm() * xs.norm())


def test_gradient_against_differences():
    """The derivative of sum(w * rope(x)) along a direction, by differences of the forward call in fp32."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    n, h, dim = 5, 2, 64
    t = B.wf_rope_init(dim, 32)
    p = torch.arange(n, dtype=torch.int32, device="cuda") * 1000
    x, w, d = (torch.randn(n, h * dim, device="cuda") for _ in range(3))

    def call(v, adjoint=False):
        o = torch.empty_like(v)
        B.wf_rope(t, v, h * dim, h, None, 0, 0, p, n, B.WF_F32, adjoint, o, h * dim, None, 0)
        return o.double()

    step = 2.0 ** -4  # linear in x: only rounding is left
    diff = ((call(x + step * d) - call(x - step * d)) * w.double()).sum() / (2 * step)
    grad = (call(w, True) * d.double()).sum()
    assert abs(diff - grad) <= 2.0 ** -20 / step * float(w.norm() * (x.norm() + d.norm()))


@pytest.mark.parametrize("layout", [0, 1])
def test_in_place_and_queries_alone(layout):
    import torch
    from paper_2609_32869_gb300 import binding as B
    n, hq, hkv, dim = 6, 3, 2, 64
    x, q, k, pos = _case(torch, n, hq, hkv, dim, "bf16", 5)
    t = B.wf_rope_init(dim, 32, layout)
    p = torch.tensor(pos, dtype=torch.int32, device="cuda")
    out = torch.empty(n, hq * dim, dtype=x.dtype, device="cuda")
    B.wf_rope(t, q, x.stride(0), hq, None, 0, 0, p, n, B.WF_BF16, False, out, out.stride(0), None, 0)
    before = x.clone()
    B.wf_rope(t, q, x.stride(0), hq, k, x.stride(0), hkv, p, n, B.WF_BF16, False, q, x.stride(0), k, x.stride(0))
    assert torch.equal(x[:, :hq * dim], out)
    assert torch.equal(x[:, (hq + hkv) * dim:], before[:, (hq + hkv) * dim:])
    assert not torch.equal(x[:, hq * dim:(hq + hkv) * dim], before[:, hq * dim:(hq + hkv) * dim])


def test_nan_stays_in_its_pair():
    import torch
    from paper_2609_32869_gb300 import binding as B
    x = torch.ones(2, 64, device="cuda")
    x[0, 3], x[1, 40] = float("nan"), float("inf")
    out = torch.empty_like(x)
    B.wf_rope(B.wf_rope_init(64, 32), x, 64, 1, None, 0, 0, torch.tensor([5, 6], dtype=torch.int32, device="cuda"), 2, B.WF_F32, False, out, 64, None, 0)
    assert sorted(torch.isnan(out[0]).nonzero()[:, 0].tolist()) == [3, 19] and out[1, 40] == float("inf")
    assert torch.isfinite(out).sum() == 128 - 3


def test_as_many_rows_as_an_int_counts():
    """2^31 - 1 rows of one pair, in place: the first, some and the last turned by their positions."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    n = 2 ** 31 - 1
    if torch.cuda.mem_get_info()[0] < 24 * 2 ** 30:
        pytest.skip("24 GiB needed")
    x = torch.ones(n, 2, dtype=torch.float16, device="cuda")
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")
    at = torch.tensor([0, 1, 7, 2 ** 30 + 3, n - 9, n - 8, n - 2, n - 1], device="cuda")
    pos[at] = torch.arange(1, len(at) + 1, dtype=torch.int32, device="cuda")
    B.wf_rope(B.wf_rope_init(2), x, 2, 1, None, 0, 0, pos, n, B.WF_F16, False, x, 2, None, 0)
    p = np.arange(1, len(at) + 1, dtype=np.float64)
    want = np.stack([np.cos(p) - np.sin(p), np.sin(p) + np.cos(p)], 1)
    # half a step of fp16 and fp32 arithmetic
    assert (np.abs(x[at].double().cpu().numpy() - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -20).all()
    assert (x[at[-1] - 6:at[-1] - 1] == 1).all()
