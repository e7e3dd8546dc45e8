"""The beam-decode calls check their arguments on the host, before any launch."""
import pytest

from paper_2609_32869_gb300 import binding as B

A = 1 << 20   # an aligned address that no call reads: each is refused first


def _pool(**kw):
    f = dict(base=A, n_layers=2, n_blocks=8, block_size=16, n_kv_heads=2, head_dim=64, dtype=B.WF_BF16, layer_stride=0)
    f.update(kw)
    return B.kv4_pool(**f)


def _status(call, **kw):
    try:
        call(**kw)
    except B.WfError as e:
        return e.status
    return B.WF_OK


BAD_POOLS = [(dict(base=A + 8), B.WF_ERR_INVALID), (dict(base=0), B.WF_ERR_INVALID), (dict(n_layers=0), B.WF_ERR_INVALID),
             (dict(n_blocks=0), B.WF_ERR_INVALID), (dict(block_size=24), B.WF_ERR_UNSUPPORTED), (dict(head_dim=96), B.WF_ERR_UNSUPPORTED),
             (dict(n_kv_heads=0), B.WF_ERR_UNSUPPORTED), (dict(dtype=B.WF_F32), B.WF_ERR_UNSUPPORTED),
             (dict(layer_stride=1152), B.WF_ERR_INVALID), (dict(layer_stride=10 ** 6 + 8), B.WF_ERR_INVALID),
             (dict(n_blocks=1 << 27), B.WF_ERR_INVALID)]


def _store(pool=None, layer=0, k=A, k_stride=128, v=A, v_stride=128, slots=A, n=4):
    B.wf_kv4_store(pool or _pool(), layer, k, k_stride, v, v_stride, slots, n, None, 0)


def _load(pool=None, layer=0, k=A, k_stride=128, v=A, v_stride=128, slots=A, n=4):
    B.wf_kv4_load(pool or _pool(), layer, slots, n, k, k_stride, v, v_stride, None, 0)


def _attend(pool=None, layer=0, q=A, q_stride=256, table=A, table_stride=8, length=A, n_seq=2, rps=1, n_heads=4, max_len=128, out=A,
            out_stride=256, scratch=A, scratch_bytes=1 << 30, scale=0.125):
    B.wf_kv4_attention(pool or _pool(), layer, q, q_stride, table, table_stride, length, n_seq, rps, n_heads, 1, scale, max_len, out, out_stride,
                       scratch, scratch_bytes, None, 0)


def _plan(old=A, new=A + 64, n=2, bs=16, free=A, n_blocks=8, n_free=A, table=A, stride=4, offsets=A, slots=A, cap=8, ln=A + 128, left=A + 192):
    B.wf_page_plan(old, new, n, bs, free, n_blocks, n_free, table, stride, offsets, slots, cap, ln, left, None, 0)


def _select(logits=A, dtype=B.WF_F32, ld=1000, scores=A, n=1, beams=5, vocab=1000, token=A, scratch=A, scratch_bytes=1 << 30):
    B.wf_beam_select(logits, dtype, ld, scores, None, n, beams, vocab, 3, token, A, A, A, A, scratch, scratch_bytes, 0)


def _reorder(pool=None, table=A, stride=4, length=A, parent=A, n=2, beams=3, free=A, scratch=A, scratch_bytes=1 << 30):
    B.wf_beam_reorder(pool or _pool(), table, A, stride, length, parent, n, beams, free, A, A, scratch, scratch_bytes, None, 0)


@pytest.mark.parametrize("kw,want", BAD_POOLS)
@pytest.mark.parametrize("call", [_store, _load, _attend, _reorder])
def test_pools(call, kw, want):
    assert _status(call, pool=_pool(**kw)) == want


@pytest.mark.parametrize("call", [_store, _load])
@pytest.mark.parametrize("kw", [dict(layer=2), dict(layer=-1), dict(k=None), dict(v=A + 4), dict(slots=None), dict(n=-1), dict(k_stride=127),
                                dict(v_stride=132), dict(k_stride=120)])
def test_rows(call, kw):
    assert _status(call, **kw) == B.WF_ERR_INVALID


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), 1), (dict(q=A + 2), 1), (dict(q_stride=248), 1), (dict(q_stride=260), 1), (dict(out_stride=255), 1), (dict(out=None), 1),
    (dict(table=None), 1), (dict(length=None), 1), (dict(n_seq=0), 1), (dict(rps=0), 1), (dict(n_heads=3), 1), (dict(n_heads=0), 1),
    (dict(max_len=0), 1), (dict(max_len=129), 1), (dict(table_stride=-1), 1), (dict(scale=float("nan")), 1), (dict(layer=2), 1),
    (dict(rps=1 << 20, n_heads=4), B.WF_ERR_UNSUPPORTED)])
def test_attention(kw, want):
    assert _status(_attend, **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(old=None), 1), (dict(n=0), 1), (dict(bs=8), B.WF_ERR_UNSUPPORTED), (dict(free=None), 1), (dict(stride=0), 1), (dict(cap=-1), 1),
    (dict(slots=None), 1), (dict(ln=A), 1), (dict(ln=A + 64), 1), (dict(left=A), 1), (dict(n_blocks=1 << 28), 1), (dict(stride=1 << 28), 1)])
def test_plan(kw, want):
    assert _status(_plan, **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(logits=None), 1), (dict(scores=None), 1), (dict(token=None), 1), (dict(n=0), 1), (dict(beams=0), 1), (dict(ld=999), 1),
    (dict(scratch=None), 1), (dict(scratch=A + 4), 1), (dict(dtype=3), B.WF_ERR_UNSUPPORTED), (dict(dtype=-1), B.WF_ERR_UNSUPPORTED),
    (dict(beams=17), B.WF_ERR_UNSUPPORTED), (dict(vocab=9), B.WF_ERR_UNSUPPORTED),
    (dict(vocab=(1 << 22) + 1, ld=1 << 23), B.WF_ERR_UNSUPPORTED), (dict(logits=A + 2), 1), (dict(scratch_bytes=100), B.WF_ERR_CAPACITY)])
def test_select(kw, want):
    assert _status(_select, **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(table=None), 1), (dict(stride=0), 1), (dict(parent=None), 1), (dict(n=0), 1), (dict(beams=0), 1), (dict(free=None), 1),
    (dict(scratch=None), 1), (dict(scratch=A + 2), 1), (dict(beams=17), B.WF_ERR_UNSUPPORTED), (dict(stride=1 << 28), 1),
    (dict(scratch_bytes=16), B.WF_ERR_CAPACITY)])
def test_reorder(kw, want):
    assert _status(_reorder, **kw) == want


def test_sizes():
    assert B.wf_kv4_block_bytes(16, 20, 64) == 20 * 1152 and B.wf_kv4_block_bytes(64, 8, 128) == 8 * 2 * 4 * 1152
    assert B.wf_kv4_block_bytes(48, 20, 64) == 0 and B.wf_kv4_block_bytes(16, 0, 64) == 0 and B.wf_kv4_block_bytes(16, 1, 80) == 0
    assert B.wf_beam_select_scratch_bytes(0, 5, 1000) == 0 and B.wf_beam_select_scratch_bytes(2, 5, 1000) > 0
    assert B.wf_beam_reorder_scratch_bytes(1, 17, 4) == 0


def test_plan_takes_65536_requests():
    assert _status(_plan, n=(1 << 16) + 1) == B.WF_ERR_UNSUPPORTED
