"""`BeamDecoder` checks what it is given on the host, before any call that reads by address or indexes with it (CPU)."""
import numpy as np
import pytest

from paper_2609_32869_gb300 import synthetic as syn
from paper_2609_32869_gb300.beam import BeamDecoder

torch = pytest.importorskip("torch")
CFG = syn.toy_config(enc_frames=20)


@pytest.fixture(scope="module")
def decoder():
    return BeamDecoder(CFG, syn.make_weights(CFG, seed=1), 2, 3, max_ctx=16, device="cpu")


def _good():
    return dict(enc=syn.encoder_output(CFG, 2), prompt=syn.prompts(CFG, 2, length=4), max_new=4)


def _tensor(**kw):
    return torch.zeros(2, CFG.enc_frames, CFG.d_model, **{"dtype": torch.bfloat16, **kw})


BAD = {
    "suppress too short": dict(suppress=torch.zeros(CFG.vocab - 1, dtype=torch.uint8)),
    "suppress of four bytes": dict(suppress=torch.zeros(CFG.vocab, dtype=torch.int32)),
    "suppress on another device": dict(suppress=torch.zeros(CFG.vocab, dtype=torch.uint8, device="meta")),
    "suppress of two dimensions": dict(suppress=torch.zeros(1, CFG.vocab, dtype=torch.uint8)),
    "an id past the vocabulary": dict(prompt=np.full((2, 4), CFG.vocab)),
    "a negative id": dict(prompt=np.array([[1, 2, -1, 3]] * 2)),
    "an id past 32 bits": dict(prompt=np.full((2, 4), 2 ** 32 + 5)),
    "ids that are not whole": dict(prompt=np.ones((2, 4))),
    "one prompt for two requests": dict(prompt=np.ones((1, 4), int)),
    "a prompt without tokens": dict(prompt=np.zeros((2, 0), int)),
    "a flat prompt": dict(prompt=np.ones(2, int)),
    "a negative number of tokens": dict(max_new=-1),
    "more positions than there are": dict(max_new=13),
    "frames for one request": dict(enc=np.zeros((1, CFG.enc_frames, CFG.d_model), np.uint16)),
    "frames of four bytes": dict(enc=np.zeros((2, CFG.enc_frames, CFG.d_model), np.float32)),
    "frames as numpy's fp16, which is not the bits of bf16": dict(enc=np.zeros((2, CFG.enc_frames, CFG.d_model), np.float16)),
    "too many frames": dict(enc=np.zeros((2, CFG.enc_frames + 1, CFG.d_model), np.uint16)),
    "a tensor of fp32 frames": dict(enc=_tensor(dtype=torch.float32)),
    "a tensor of fp16 frames": dict(enc=_tensor(dtype=torch.float16)),
    "frames on another device": dict(enc=_tensor(device="meta")),
}


@pytest.mark.parametrize("what", BAD)
def test_decode_refuses(decoder, what):
    with pytest.raises(ValueError):
        decoder.decode(**{**_good(), **BAD[what]})


@pytest.mark.parametrize("kw", [dict(n_req=0), dict(beams=0), dict(beams=17), dict(block_size=24), dict(beams=6, cfg=syn.toy_config(vocab=11)),
                                dict(cfg=syn.toy_config(n_heads=4))])
def test_construction_refuses(kw):
    cfg = kw.pop("cfg", CFG)
    args = {"n_req": 1, "beams": 2, "max_ctx": 16, **kw}
    with pytest.raises(ValueError):
        BeamDecoder(cfg, {}, device="cpu", **args)


def test_no_new_tokens_is_an_empty_transcript(decoder):
    found = decoder.decode(**{**_good(), "max_new": 0})
    assert [[(h.tokens, h.score, h.ended) for h in r] for r in found] == [[([], 0.0, False)]] * 2
