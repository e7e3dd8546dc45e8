"""Prompts and the 8-bit cache where offsets pass 32 bits: the same bits as in small buffers (GPU)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

STRIDE = 1 << 22  # elements between rows: 600 of them are past 2^31


def _room(torch, gib):
    if torch.cuda.mem_get_info()[0] < gib * 2 ** 30:
        pytest.skip(f"{gib} GiB needed")


def _i32(torch, v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _far(torch, rows, cols, at):
    """Rows of `cols` elements, STRIDE apart, the first at element `at`."""
    return torch.empty(rows * STRIDE, dtype=torch.bfloat16, device="cuda").view(rows, STRIDE)[:, at:at + cols]


@pytest.mark.parametrize("dim,lens", [(64, [3, 250, 347]), (128, [600]), (128, [1, 64, 200])])
def test_rows_far_apart(dim, lens):
    """Rotary positions and prompt attention over strided rows, the last behind 2^31 elements."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    _room(torch, 16)
    torch.manual_seed(dim)
    hq, hk, n, past = 4, 2, sum(lens), 5000 if len(lens) == 3 and dim == 128 else 0
    start = _i32(torch, np.cumsum([0] + lens))
    w = (hq + 2 * hk) * dim
    near = torch.randn(n, w, device="cuda").bfloat16()
    keys = torch.randn(past, 2 * hk * dim, device="cuda").bfloat16() if past else None
    far, far_out = _far(torch, n, w, 64), _far(torch, n, hq * dim, 8)
    far.copy_(near)
    pos, table, outs = torch.arange(n, dtype=torch.int32, device="cuda") * 70001, B.wf_rope_init(dim), []
    for x, out in ((near, torch.empty(n, hq * dim, dtype=torch.bfloat16, device="cuda")), (far, far_out)):
        s, k = x.stride(0), x[:, hq * dim:]
        B.wf_rope(table, x, s, hq, k, s, hk, pos, n, B.WF_BF16, False, x, s, k, s)
        kv, kvs, nk, ks, most = (keys, 2 * hk * dim, past, _i32(torch, [0, 100, 1200, past]), past) if past else (k, s, n, start, max(lens))
        size = B.wf_prompt_attention_scratch_bytes(len(lens), n, most, hq, hk, dim)
        scratch = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
        B.wf_prompt_attention(x, s, kv, kvs, kv[:, hk * dim:], kvs, start, ks, len(lens), n, nk, most, hq, hk, dim, B.WF_BF16, True, 0.1,
                              out, out.stride(0), None, scratch, size)
        outs.append((x.clone(), out.clone()))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    assert outs[0][1].float().abs().max() > 0


@pytest.mark.parametrize("dim", [64, 128])
def test_blocks_far_apart(dim):
    """Blocks, rows and layers of the cache behind 4 GiB."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    _room(torch, 32)
    torch.manual_seed(dim)
    hq, hk, bs, n = 8, 4, 64, 600
    block = B.wf_kv8_block_bytes(bs, hk, dim)
    many = 5 * 2 ** 30 // block
    near = torch.randn(n, 2 * hk * dim, device="cuda").bfloat16()
    far, far_back, far_q, far_out = _far(torch, n, 2 * hk * dim, 0), _far(torch, n, 2 * hk * dim, 128), _far(torch, n, hq * dim, 0), _far(torch, n, hq * dim, 16)
    far.copy_(near)
    q = torch.randn(n, hq * dim, device="cuda").bfloat16()
    far_q.copy_(q)
    few = -(-n // bs)
    got = []
    for blocks, layer, x, back, qq, out in (
            (few, 0, near, torch.empty_like(near), q, torch.empty_like(q)), (many, 1, far, far_back, far_q, far_out)):
        raw = torch.empty((layer + 1) * blocks * block, dtype=torch.uint8, device="cuda")
        pool = B.kv8_pool(raw, layer + 1, blocks, bs, hk, dim)
        ids = blocks - 1 - np.arange(few)  # the last blocks
        slots = _i32(torch, [ids[i // bs] * bs + i % bs for i in range(n)])
        err = _i32(torch, [0])
        B.wf_kv8_store(pool, layer, x, x.stride(0), x[:, hk * dim:], x.stride(0), slots, n, err)
        B.wf_kv8_load(pool, layer, slots, n, back, back.stride(0), back[:, hk * dim:], back.stride(0), err)
        B.wf_kv8_attention(pool, layer, qq, qq.stride(0), _i32(torch, ids), 0, _i32(torch, [n]), 1, n, hq, True, 0.1, n, out,
                           out.stride(0), None, 0, err)
        assert err.item() == 0
        got.append((back.clone(), out.clone()))
        del raw, pool
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    # three bits of fraction: half a step of a code is 2^-4 of it, and a record's smallest codes are 2^-9 of 2^e
    err = (got[0][0].float() - near.float()).abs()
    assert (err <= 2.0 ** -4 * near.float().abs() + 2.0 ** -10 * near.float().abs().max() / 224).all()
