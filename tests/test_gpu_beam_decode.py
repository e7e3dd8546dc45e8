"""Beam search end to end: the decoder of `beam.py` against the oracle (GPU)."""
import numpy as np
import pytest

from oracle import beam as ob
from oracle import decoder as od
from paper_2609_32869_gb300 import synthetic as syn

pytestmark = pytest.mark.gpu


def _four_bits(x):
    """Rows [n, d] as the cache holds them: bf16, then 4 bits by groups of 64."""
    x = ob.round16(x, "bf16")
    out = np.empty(x.shape)
    for i, row in enumerate(x):
        for g in range(0, x.shape[1], 64):
            c, s, z = ob.quantise(row[g:g + 64], "bf16")
            out[i, g:g + 64] = s * (c - 8.0) + z
    return out


def _cross(w, enc, d):
    kv = [od.linear(enc, lw["xkv_w"], lw["xkv_b"]) for lw in w["target_layers"]]
    return [(_four_bits(x[:, :d]), _four_bits(x[:, d:])) for x in kv]


def _log_probs(cfg, w, cross, tokens):
    """float64 log-probabilities of every next token along a path, keys and values held in 4 bits."""
    t, d, n = w["target"], cfg.d_model, len(tokens)
    x = t["tok_emb"][tokens] + t["pos_emb"][:n]
    causal = np.tril(np.ones((n, n), bool))
    for lw, (ck, cv) in zip(w["target_layers"], cross):
        qkv = od.linear(od.layer_norm(x, lw["ln1_g"], lw["ln1_b"], cfg.ln_eps), lw["qkv_w"], lw["qkv_b"])
        att = od.multi_head_attention(qkv[:, :d], _four_bits(qkv[:, d:2 * d]), _four_bits(qkv[:, 2 * d:]), cfg.n_heads, causal)
        x = x + od.linear(att, lw["out_w"], lw["out_b"])
        q = od.linear(od.layer_norm(x, lw["ln2_g"], lw["ln2_b"], cfg.ln_eps), lw["xq_w"], lw["xq_b"])
        x = x + od.linear(od.multi_head_attention(q, ck, cv, cfg.n_heads), lw["xout_w"], lw["xout_b"])
        h = od.linear(od.layer_norm(x, lw["ln3_g"], lw["ln3_b"], cfg.ln_eps), lw["fc1_w"], lw["fc1_b"])
        x = x + od.linear(od.gelu(h), lw["fc2_w"], lw["fc2_b"])
    z = od.linear(od.layer_norm(x, t["lnf_g"], t["lnf_b"], cfg.ln_eps), t["tok_emb"])
    z = z - z.max(-1, keepdims=True)
    return z - np.log(np.exp(z).sum(-1, keepdims=True))


@pytest.mark.parametrize("n,beams,P,new,block", [(2, 4, 5, 24, 16), (1, 1, 3, 6, 64), (3, 5, 16, 17, 16)])
def test_scores_are_the_paths_log_probabilities(n, beams, P, new, block):
    """Each hypothesis's score against the oracle's along its tokens.  The framework's logits are within 3e-2 of
    the oracle's in bf16; a log-probability moves by at most twice that.  A beam that read another beam's keys,
    a wrong block or a wrong parent would be off by the spread of the logits, several units a token."""
    import torch
    from paper_2609_32869_gb300.beam import BeamDecoder
    cfg = syn.toy_config()
    ws = syn.make_weights(cfg, seed=3, std=0.05)
    enc, prompt = syn.encoder_output(cfg, n, seed=4), syn.prompts(cfg, n, length=P, seed=4)
    dec = BeamDecoder(cfg, ws, n, beams, max_ctx=P + new, block_size=block)
    w = syn.weights_as_float(ws)
    found = dec.decode(enc, prompt, new)
    for i in range(n):
        cross = _cross(w, syn.bf16_bits_to_f32(enc[i]).astype(np.float64), cfg.d_model)
        assert len(found[i]) >= beams
        for h in found[i][:3] + found[i][-1:]:
            path = prompt[i].tolist() + h.tokens
            lp = _log_probs(cfg, w, cross, path)
            out = h.tokens + ([cfg.eos_id] if h.ended else [])
            want = sum(lp[P - 1 + j, tok] for j, tok in enumerate(out))
            assert abs(h.score - want) <= 6e-2 * len(out), (i, h, want)
        assert len({tuple(h.tokens) for h in found[i] if not h.ended}) == sum(not h.ended for h in found[i])
    # every block came back, once
    assert dec.n_free[0].item() == dec.n_blocks
    assert sorted(dec.free.tolist()) == list(range(dec.n_blocks))
    # and the same search again gives the same hypotheses
    again = dec.decode(enc, prompt, new)
    assert [[(h.tokens, h.score) for h in r] for r in again] == [[(h.tokens, h.score) for h in r] for r in found]
    torch.cuda.synchronize()


def test_wider_search_finds_no_worse_sums():
    """With one beam the search is greedy; its path is one of a wide search's prefixes or loses to one."""
    from paper_2609_32869_gb300.beam import BeamDecoder
    cfg = syn.toy_config()
    ws = syn.make_weights(cfg, seed=5, std=0.05)
    enc, prompt = syn.encoder_output(cfg, 1, seed=6), syn.prompts(cfg, 1, length=4, seed=6)
    one = BeamDecoder(cfg, ws, 1, 1, max_ctx=16).decode(enc, prompt, 2)[0]
    wide = BeamDecoder(cfg, ws, 1, 16, max_ctx=16).decode(enc, prompt, 2)[0]
    assert max(h.score for h in wide) >= max(h.score for h in one if not h.ended) - 0.1


def test_positions_are_checked():
    from paper_2609_32869_gb300.beam import BeamDecoder
    cfg = syn.toy_config()
    dec = BeamDecoder(cfg, syn.make_weights(cfg, seed=5), 1, 2, max_ctx=16)
    with pytest.raises(ValueError):
        dec.decode(syn.encoder_output(cfg, 1), syn.prompts(cfg, 1, length=8), 9)
