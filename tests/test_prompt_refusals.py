"""The rotary, prompt and 8-bit cache calls check their arguments on the host, before any launch."""
import math

import numpy as np
import pytest

from oracle import prompt as op
from paper_2609_32869_gb300 import binding as B

A = 1 << 20   # an aligned address that no call reads: each is refused first
INVALID, CAPACITY, UNSUPPORTED = B.WF_ERR_INVALID, B.WF_ERR_CAPACITY, B.WF_ERR_UNSUPPORTED


def _status(call, **kw):
    try:
        call(**kw)
    except B.WfError as e:
        return e.status
    return B.WF_OK


def _pool(**kw):
    f = dict(base=A, n_layers=2, n_blocks=8, block_size=16, n_kv_heads=2, head_dim=64, dtype=B.WF_BF16, layer_stride=0)
    f.update(kw)
    return B.kv8_pool(**f)


def _store(pool=None, layer=0, k=A, k_stride=128, v=A, v_stride=128, slots=A, n=4):
    B.wf_kv8_store(pool or _pool(), layer, k, k_stride, v, v_stride, slots, n, None, 0)


def _load(pool=None, layer=0, k=A, k_stride=128, v=A, v_stride=128, slots=A, n=4):
    B.wf_kv8_load(pool or _pool(), layer, slots, n, k, k_stride, v, v_stride, None, 0)


def _attend(pool=None, layer=0, q=A, q_stride=256, table=A, table_stride=8, length=A, n_seq=2, rps=1, n_heads=4, max_len=128, out=A,
            out_stride=256, scratch=A, scratch_bytes=1 << 30, scale=0.125):
    B.wf_kv8_attention(pool or _pool(), layer, q, q_stride, table, table_stride, length, n_seq, rps, n_heads, 1, scale, max_len, out, out_stride,
                       scratch, scratch_bytes, None, 0)


def _prompt(q=A, q_stride=256, k=A, k_stride=128, v=A, v_stride=128, q_start=A, k_start=A, n_seq=2, n_q=9, n_k=9, max_k=9, n_heads=4, n_kv_heads=2,
            head_dim=64, dtype=B.WF_BF16, scale=0.125, out=A, out_stride=256, lse=A, scratch=A, scratch_bytes=1 << 30):
    B.wf_prompt_attention(q, q_stride, k, k_stride, v, v_stride, q_start, k_start, n_seq, n_q, n_k, max_k, n_heads, n_kv_heads, head_dim, dtype, True,
                          scale, out, out_stride, lse, scratch, scratch_bytes, None, 0)


def _rope(table=None, q=A, q_stride=256, n_heads=4, k=A, k_stride=128, n_kv_heads=2, pos=A, n=3, dtype=B.WF_BF16, q_out=A, q_out_stride=256, k_out=A,
          k_out_stride=128):
    B.wf_rope(table or B.wf_rope_init(64), q, q_stride, n_heads, k, k_stride, n_kv_heads, pos, n, dtype, False, q_out, q_out_stride, k_out,
              k_out_stride, 0)


@pytest.mark.parametrize("kw,want", [
    (dict(base=A + 8), INVALID), (dict(base=0), INVALID), (dict(n_layers=0), INVALID), (dict(n_blocks=0), INVALID),
    (dict(block_size=24), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(n_kv_heads=0), UNSUPPORTED), (dict(dtype=B.WF_F32), UNSUPPORTED),
    (dict(layer_stride=2064), INVALID), (dict(layer_stride=10 ** 6 + 8), INVALID), (dict(n_blocks=1 << 27), INVALID)])
@pytest.mark.parametrize("call", [_store, _load, _attend])
def test_pools(call, kw, want):
    assert _status(call, pool=_pool(**kw)) == want


@pytest.mark.parametrize("call", [_store, _load])
@pytest.mark.parametrize("kw", [dict(layer=2), dict(layer=-1), dict(k=None), dict(v=A + 4), dict(slots=None), dict(n=-1), dict(k_stride=127),
                                dict(v_stride=132), dict(k_stride=120)])
def test_rows(call, kw):
    assert _status(call, **kw) == INVALID


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), INVALID), (dict(q=A + 2), INVALID), (dict(q_stride=248), INVALID), (dict(q_stride=260), INVALID), (dict(out_stride=255), INVALID),
    (dict(out=None), INVALID), (dict(table=None), INVALID), (dict(length=None), INVALID), (dict(n_seq=0), INVALID), (dict(rps=0), INVALID),
    (dict(n_heads=3), INVALID), (dict(n_heads=0), INVALID), (dict(max_len=0), INVALID), (dict(max_len=129), INVALID),
    (dict(table_stride=-1), INVALID), (dict(scale=float("nan")), INVALID), (dict(layer=2), INVALID), (dict(rps=1 << 20), UNSUPPORTED)])
def test_attention(kw, want):
    assert _status(_attend, **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(q=A + 2), INVALID), (dict(v=A + 8), INVALID),
    (dict(q_stride=248), INVALID), (dict(q_stride=260), INVALID), (dict(k_stride=120), INVALID), (dict(v_stride=132), INVALID),
    (dict(out=None), INVALID), (dict(out=A + 8), INVALID), (dict(out_stride=250), INVALID), (dict(q_start=None), INVALID),
    (dict(k_start=None), INVALID), (dict(n_seq=0), INVALID), (dict(n_q=-1), INVALID), (dict(n_k=-1), INVALID), (dict(max_k=-1), INVALID),
    (dict(n_heads=3), INVALID), (dict(n_kv_heads=0), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(lse=A + 2), INVALID), (dict(head_dim=96), UNSUPPORTED),
    (dict(dtype=B.WF_F32), UNSUPPORTED), (dict(n_heads=130, n_kv_heads=2, q_stride=130 * 64, out_stride=130 * 64), UNSUPPORTED)])
def test_prompt(kw, want):
    assert _status(_prompt, **kw) == want


def test_no_rows_is_no_call():
    assert _status(_prompt, n_q=0) == B.WF_OK and _status(_store, n=0) == B.WF_OK and _status(_load, n=0) == B.WF_OK and _status(_rope, n=0) == B.WF_OK


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(pos=None), INVALID), (dict(n=-1), INVALID), (dict(n_heads=0), INVALID),
    (dict(n_kv_heads=-1), INVALID), (dict(q_stride=255), INVALID), (dict(k_stride=127), INVALID), (dict(q_out=None), INVALID),
    (dict(q_out_stride=100), INVALID), (dict(k_out=None), INVALID), (dict(k_out_stride=64), INVALID), (dict(q=A + 1), INVALID),
    (dict(q=A + 2, dtype=B.WF_F32), INVALID), (dict(q_stride=264), INVALID), (dict(k_stride=136), INVALID),  # in place with two strides
    (dict(dtype=3), UNSUPPORTED), (dict(n_heads=65530, n_kv_heads=6, q_stride=1 << 23, q_out_stride=1 << 23, k_stride=384, k_out_stride=384), UNSUPPORTED)])
def test_rope(kw, want):
    assert _status(_rope, **kw) == want


def test_rope_refuses_a_table_of_no_spec():
    assert _status(_rope, table=B.WfRopeTable()) == INVALID


@pytest.mark.parametrize("kw,want", [
    (dict(head_dim=1, rot_dim=1), INVALID), (dict(head_dim=64, rot_dim=66), INVALID), (dict(head_dim=64, rot_dim=31), INVALID),
    (dict(head_dim=64, rot_dim=0), INVALID), (dict(head_dim=512), UNSUPPORTED), (dict(head_dim=5000, rot_dim=64), UNSUPPORTED),
    (dict(head_dim=64, layout=2), INVALID), (dict(head_dim=64, base=1.0), INVALID), (dict(head_dim=64, base=float("inf")), INVALID),
    (dict(head_dim=64, scaling=5), INVALID), (dict(head_dim=64, scaling=1, factor=0.5), INVALID), (dict(head_dim=64, gain=0.0), INVALID),
    (dict(head_dim=64, gain=float("nan")), INVALID), (dict(head_dim=64, scaling=3, factor=2, trained_len=0, low=1, high=4), INVALID),
    (dict(head_dim=64, scaling=4, factor=2, trained_len=100, low=4, high=4), INVALID),
    (dict(head_dim=64, scaling=3, factor=2, trained_len=100, low=0, high=4), INVALID)])
def test_rope_specs(kw, want):
    assert _status(B.wf_rope_init, **kw) == want


SCALINGS = [("plain", dict()), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)), ("waves", dict(factor=8.0, trained_len=8192.0, low=1.0, high=4.0)),
            ("parts", dict(factor=16.0, trained_len=4096.0, low=1.0, high=32.0))]


@pytest.mark.parametrize("rot", [2, 20, 64, 128, 256])
@pytest.mark.parametrize("name,kw", SCALINGS)
def test_rope_table(rot, name, kw):
    """turns is the frequency in turns, in units of 2^-64.  Two evaluations of base^(-2i/rot) in doubles differ by a few of their
    steps times the exponent's size: 2^-45 relative is beyond both.  The fraction of 2^64 is cut to a whole number of 2^-64, which is
    up to 2^-64 less, whatever the frequency's size."""
    t = B.wf_rope_init(256, rot, scaling=B.WF_ROPE_PLAIN + [n for n, _ in SCALINGS].index(name), base=500000.0, **kw)
    want = op.frequencies(rot, 500000.0, name, **kw) / (2 * math.pi)
    got = np.array([t.turns[i] for i in range(rot // 2)], np.float64) * 2.0 ** -64
    np.testing.assert_allclose(got, want, rtol=2.0 ** -45, atol=2.0 ** -64)
    assert (t.head_dim, t.rot_dim, t.layout, t.gain) == (256, rot, 0, 1.0)
    assert not any(t.turns[rot // 2:])


def test_sizes():
    assert B.wf_kv8_block_bytes(16, 20, 64) == 20 * 2064 and B.wf_kv8_block_bytes(64, 8, 128) == 8 * 4 * 4112
    assert B.wf_kv8_block_bytes(48, 20, 64) == 0 and B.wf_kv8_block_bytes(16, 0, 64) == 0 and B.wf_kv8_block_bytes(16, 1, 80) == 0
    for bad in ((0, 1, 4, 4, 64, 9), (1, 0, 4, 4, 64, 9), (1, 1, 3, 2, 64, 9), (1, 1, 4, 4, 96, 9), (1, 1, 4, 4, 64, 0)):
        assert B.wf_kv8_attention_scratch_bytes(*bad) == 0
    for bad in ((0, 1, 9, 4, 4, 64), (1, 0, 9, 4, 4, 64), (1, 1, 9, 3, 2, 64), (1, 1, 9, 4, 4, 96)):
        assert B.wf_prompt_attention_scratch_bytes(*bad) == 0


def test_the_oracle_codes():
    """Codes round to the nearest, ties to even; the quantiser's e is the least that holds a record."""
    assert [op.code_of(x) for x in (0.0, -0.0, 448.0, 500.0, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, float("nan"))] == [0, 128, 126, 126, 0x58, 0x5A, 0, 2, 127]
    c = op.Cache(1, 16, 1, 64)
    x = np.zeros((1, 1, 64))
    x[0, 0, 3], x[0, 0, 5] = 448.5, -1.0
    c.store([0], x, x * 0.25)
    assert list(c.scales(0, 0)) == [2.0, 0.5] and c.row(0, 0)[0, 5] == -1.0
    y = np.full((1, 1, 64), 4000.0)
    c.store([1], y, y * 0)
    assert c.scales(0, 0)[0] == 16.0 and c.row(0, 0)[0, 5] == -1.0 and c.row(0, 1)[0, 5] == -0.25 and not c.row(2, 0).any()
