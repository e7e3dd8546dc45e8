"""A step of beam search as a CUDA graph, and the decoder's options (GPU)."""
import numpy as np
import pytest

from paper_2609_32869_gb300 import synthetic as syn
from test_gpu_beam_decode import _cross, _log_probs
from test_gpu_beam_ops import _beam_state, _filled

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("length,max_len", [(37, 448), (48, 1500), (40, 9000)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_step_can_be_captured(length, max_len, dtype):
    """Plan, store, attention (one chunk, a cluster, a second kernel), selection and reordering in one graph: every
    buffer afterwards equals that of the calls made one by one."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    rng = np.random.default_rng(length)
    n, W, bs, heads, V, eos = 3, 4, 16, 2, 700, 5
    cols, rows, d, dt = -(-max_len // bs), n * W, heads * 64, torch.bfloat16 if dtype == "bf16" else torch.float16
    table, ids, blocks = _beam_state(rng, n, W, bs, [length] * n, cols)
    cache = _filled(rng, blocks, bs, heads, 64, dtype)
    code = B.WF_F16 if dtype == "f16" else B.WF_BF16
    start = dict(raw=torch.from_numpy(cache.raw).view(-1), table=torch.tensor(table, dtype=torch.int32),
                 free=torch.tensor(list(ids) + [-9] * (blocks - len(ids)), dtype=torch.int32), left=torch.tensor([len(ids)], dtype=torch.int32),
                 old=torch.full((rows,), length, dtype=torch.int32), new=torch.full((rows,), length + 1, dtype=torch.int32),
                 table_out=torch.full((rows, cols), -1, dtype=torch.int32), offsets=torch.zeros(rows + 1, dtype=torch.int32),
                 slots=torch.zeros(rows, dtype=torch.int32), len=torch.zeros(rows, dtype=torch.int32), left1=torch.zeros(1, dtype=torch.int32),
                 left2=torch.zeros(1, dtype=torch.int32), qkv=torch.randn(rows, 3 * d).to(dt), out=torch.zeros(rows, d, dtype=dt),
                 logits=torch.randn(rows, V), scores=-torch.rand(n, W), token=torch.zeros(n, W, dtype=torch.int32),
                 parent=torch.zeros(n, W, dtype=torch.int32), score=torch.zeros(n, W), fin_parent=torch.zeros(n, W, dtype=torch.int32),
                 fin_score=torch.zeros(n, W), err=torch.zeros(1, dtype=torch.int32))
    s = {k: v.cuda() for k, v in start.items()}
    pool = B.kv4_pool(s["raw"], 1, blocks, bs, heads, 64, code)
    size = max(B.wf_kv4_attention_scratch_bytes(rows, 1, heads, heads, 64, max_len), B.wf_beam_select_scratch_bytes(n, W, V),
               B.wf_beam_reorder_scratch_bytes(n, W, cols), 16)
    sc = torch.empty(size, dtype=torch.uint8, device="cuda")

    def step():
        B.wf_page_plan(s["old"], s["new"], rows, bs, s["free"], blocks, s["left"], s["table"], cols, s["offsets"], s["slots"], rows, s["len"],
                       s["left1"], s["err"])
        B.wf_kv4_store(pool, 0, s["qkv"][:, d:], 3 * d, s["qkv"][:, 2 * d:], 3 * d, s["slots"], rows, s["err"])
        B.wf_kv4_attention(pool, 0, s["qkv"], 3 * d, s["table"], cols, s["len"], rows, 1, heads, True, 0.125, max_len, s["out"], d, sc, size, s["err"])
        B.wf_beam_select(s["logits"], B.WF_F32, V, s["scores"], None, n, W, V, eos, s["token"], s["parent"], s["score"], s["fin_parent"],
                         s["fin_score"], sc, size)
        B.wf_beam_reorder(pool, s["table"], s["table_out"], cols, s["len"], s["parent"], n, W, s["free"], s["left1"], s["left2"], sc, size, s["err"])

    def reset():
        for k, v in start.items():
            s[k].copy_(v)

    step()
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in s.items()}
    assert want["err"].item() == 0 and want["offsets"].tolist() == list(range(rows + 1))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        for k, v in want.items():
            assert torch.equal(s[k].view(torch.uint8), v.view(torch.uint8)), k


def _decoder():
    from paper_2609_32869_gb300.beam import BeamDecoder
    cfg = syn.toy_config()
    ws = syn.make_weights(cfg, seed=7, std=0.05)
    enc, prompt = syn.encoder_output(cfg, 2, seed=8), syn.prompts(cfg, 2, length=5, seed=8)
    return cfg, ws, enc, prompt, BeamDecoder(cfg, ws, 2, 4, max_ctx=24, block_size=32)


def test_suppressed_ids_are_never_proposed_and_take_no_probability():
    """The logits are within 3e-2 of the oracle's, a log-probability within twice that (as without suppressed ids)."""
    import torch
    cfg, ws, enc, prompt, dec = _decoder()
    free = dec.decode(enc, prompt, 10)
    taken = sorted({t for r in free for h in r for t in h.tokens})[::2]
    sup = torch.zeros(cfg.vocab, dtype=torch.uint8, device="cuda")
    sup[taken] = 1
    found = dec.decode(enc, prompt, 10, suppress=sup)
    w, keep = syn.weights_as_float(ws), np.setdiff1d(np.arange(cfg.vocab), taken)
    for i, r in enumerate(found):
        assert len(r) >= 4
        cross = _cross(w, syn.bf16_bits_to_f32(enc[i]).astype(np.float64), cfg.d_model)
        for h in r:
            assert not set(h.tokens) & set(taken)
        for h in r[:2]:
            lp = _log_probs(cfg, w, cross, prompt[i].tolist() + h.tokens)
            lp = lp - np.log(np.exp(lp[:, keep]).sum(-1, keepdims=True))
            out = h.tokens + ([cfg.eos_id] if h.ended else [])
            assert abs(h.score - sum(lp[4 + j, t] for j, t in enumerate(out))) <= 6e-2 * len(out)
    same = dec.decode(enc, prompt, 10, suppress=sup.bool())
    strided = dec.decode(enc, prompt, 10, suppress=torch.stack([sup, 1 - sup], 1)[:, 0])
    key = lambda f: [[(h.tokens, h.score) for h in r] for r in f]  # noqa: E731
    assert key(same) == key(found) == key(strided)


@pytest.mark.parametrize("penalty", [0.0, 0.5, 2.0])
def test_length_penalty_orders_the_same_hypotheses(penalty):
    cfg, ws, enc, prompt, dec = _decoder()
    plain, found = dec.decode(enc, prompt, 8), dec.decode(enc, prompt, 8, length_penalty=penalty)
    for a, b in zip(plain, found):
        assert sorted((h.tokens, h.score, h.ended) for h in a) == sorted((h.tokens, h.score, h.ended) for h in b)
        value = [h.score / max(1, len(h.tokens) + h.ended) ** penalty for h in b]
        assert value == sorted(value, reverse=True)
