"""Plain forms, inputs and 64-bit values of the beam-decode operators.

The operators serve beam search over a paged key/value cache held in 4 bits:

  plan     block tables and slot maps from request lengths (wf_page_plan)
  store    rows of keys and values into the cache and back (wf_kv4_store, wf_kv4_load)
  attend   attention of query rows over the cache (wf_kv4_attention)
  select   the best continuations over beams and vocabulary (wf_beam_select)
  reorder  the beams' block tables and cache tails after a selection (wf_beam_reorder)

The cache.  Each head of 64 or 128 values is held in groups of 64.  A group of
a row is 4-bit codes c with a scale s and an offset z in the cache's 16-bit
type, for the values s (c - 8) + z:

  s = round((max - min) / 15),  z = round(max - 7 s),  c = clamp(rint((x - z) / s), -8, 7) + 8

(c = 8 where s is 0).  16 positions of a group form a record of 1152 bytes:
512 of key codes, 512 of value codes and 128 of scales and offsets.
"""
import math

import torch

own = False

REC = 1152  # bytes of 16 positions of one group
GROUP = 64


def listed():
    return [
        # one decode step of 16 requests with 5 beams each: one new token per beam
        {"name": "plan_step", "op": "plan", "n": 80, "most_old": 447, "most_new": 1, "bs": 16},
        # admission of many requests at once, ragged prompts of up to 4096 tokens
        {"name": "plan_admit", "op": "plan", "n": 512, "most_old": 0, "most_new": 4096, "bs": 64},
        # the new token of 80 beams in one decoder layer, a slice of the fused projection's output
        {"name": "store_step", "op": "store", "n": 80, "hkv": 20, "dim": 64, "bs": 16, "dtype": "bf16", "fused": True},
        # the encoder frames of 32 requests (1500 each) as one layer's cross-attention keys and values
        {"name": "store_frames", "op": "store", "n": 48000, "hkv": 20, "dim": 64, "bs": 64, "dtype": "bf16", "fused": False},
        # cross-attention of one request's 5 beams over its 1500 frames: latency
        {"name": "attend_frames_1", "op": "attend", "n": 1, "rps": 5, "hq": 20, "hkv": 20, "dim": 64, "least": 1500, "most": 1500,
         "bs": 64, "causal": False, "dtype": "bf16"},
        # self-attention of one decode step of 16 requests with 5 beams, transcripts of up to 448 tokens
        {"name": "attend_beams_80", "op": "attend", "n": 80, "rps": 1, "hq": 20, "hkv": 20, "dim": 64, "least": 4, "most": 448,
         "bs": 16, "causal": True, "dtype": "bf16"},
        # cross-attention of 96 requests, 9 query rows each (a verified block of proposals)
        {"name": "attend_frames_96", "op": "attend", "n": 96, "rps": 9, "hq": 20, "hkv": 20, "dim": 64, "least": 1500, "most": 1500,
         "bs": 64, "causal": False, "dtype": "bf16"},
        # a few long contexts with shared key/value heads, ragged, one new token each
        {"name": "attend_long", "op": "attend", "n": 6, "rps": 1, "hq": 32, "hkv": 8, "dim": 128, "least": 5000, "most": 65001,
         "bs": 32, "causal": True, "dtype": "f16"},
        # one request's 5 beams over the full vocabulary: latency
        {"name": "select_1", "op": "select", "n": 1, "beams": 5, "vocab": 51866, "dtype": "f32"},
        # 96 requests' beams over the full vocabulary
        {"name": "select_96", "op": "select", "n": 96, "beams": 5, "vocab": 51866, "dtype": "f32"},
        # one request's beams after a selection, 4 decoder layers
        {"name": "reorder_1", "op": "reorder", "n": 1, "beams": 5, "least": 100, "most": 100, "bs": 16, "layers": 4, "hkv": 6,
         "dim": 64, "dtype": "bf16"},
        # 16 requests' beams after a selection, all 32 decoder layers, transcripts of up to 448 tokens
        {"name": "reorder_16", "op": "reorder", "n": 16, "beams": 5, "least": 1, "most": 447, "bs": 16, "layers": 32, "hkv": 20,
         "dim": 64, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)) - 0.2)))))


def draw(rng):
    op = rng.choice(["plan", "store", "attend", "attend", "attend", "select", "select", "reorder"])
    bs = rng.choice([16, 32, 64])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if op == "plan":
        return {"op": op, "n": _log_int(rng, 1, 512), "most_old": rng.choice([0, 447, 2000]),
                "most_new": rng.choice([1, 9, _log_int(rng, 1, 4000)]), "bs": bs}
    hkv, dim = rng.choice([(20, 64), (6, 64), (10, 128), (3, 64), (2, 128)])
    if op == "store":
        return {"op": op, "n": _log_int(rng, 1, 40000 * 1280 // (hkv * dim * 2)), "hkv": hkv, "dim": dim, "bs": bs, "dtype": dtype,
                "fused": rng.random() < 0.5}
    if op == "attend":
        kind = rng.choice(["frames", "beams", "long", "prompt"])
        g = rng.choice([1, 1, 2, 4, 5, 7]) if kind != "frames" else 1
        if kind == "frames":
            n, rps, most, causal = _log_int(rng, 1, 64), rng.choice([1, 3, 5, 9]), rng.choice([1500, 750, 1499]), False
            least = most
        elif kind == "beams":
            n, rps, most, causal = _log_int(rng, 1, 160), rng.choice([1, 1, 2, 9]), _log_int(rng, 12, 448), True
            least = rng.choice([0, 1, most])
        elif kind == "long":
            n, rps, most, causal = _log_int(rng, 1, 4), rng.choice([1, 1, 4]), _log_int(rng, 2000, 48000), rng.random() < 0.7
            least = rng.choice([1, most // 2, most])
        else:
            n, rps, most, causal = _log_int(rng, 1, 6), _log_int(rng, 17, 200), _log_int(rng, 200, 900), True
            least = most // 2
        return {"op": op, "n": n, "rps": rps, "hq": hkv * g, "hkv": hkv, "dim": dim, "least": least, "most": most, "bs": bs,
                "causal": causal, "dtype": dtype}
    if op == "select":
        beams = rng.choice([1, 2, 3, 4, 5, 5, 8, 16])
        vocab = rng.choice([51866, 51865, 1000, _log_int(rng, 100, 130000)])
        return {"op": op, "n": _log_int(rng, 1, max(1, 20_000_000 // (beams * vocab))) if beams * vocab * 200 > 20_000_000
                else _log_int(rng, 1, 200), "beams": beams, "vocab": vocab, "dtype": rng.choice(["f32", "f32", "bf16", "f16"])}
    most = _log_int(rng, 5, 447)
    return {"op": op, "n": _log_int(rng, 1, 16), "beams": rng.choice([2, 3, 4, 5, 8]), "least": rng.choice([1, most]), "most": most,
            "bs": bs, "layers": rng.choice([1, 4, 12]), "hkv": hkv if dim == 64 else 4, "dim": dim, "dtype": dtype}


# ------------------------------------------------------------------ inputs --

_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _spread(n, lo, hi):
    """n lengths from lo to hi, the same for every seed up to their order."""
    return [lo + (i * 7919 * 104729 + (hi - lo)) % (hi - lo + 1) for i in range(n)]


def _up(x, m):
    return -(-x // m)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _records(nblocks, slabs, bs, dtype, gen):
    """Cache blocks [nblocks, slabs, bs/16, REC] of rows that a decoder writes, quantised; a few distinct ones repeated."""
    m = min(nblocks, 96)
    out = torch.zeros(m, slabs, bs // 16, REC, dtype=torch.uint8, device="cuda")
    x = torch.randn(2, m, slabs, bs, GROUP, device="cuda", generator=gen)
    x = (x * (0.5 + torch.rand(2, m, slabs, 1, 1, device="cuda", generator=gen)) + 0.3 * torch.randn(2, 1, slabs, 1, GROUP, device="cuda", generator=gen)).to(dtype)
    codes, sz = _quantise(x, dtype)
    _write(out, codes, sz)
    if m < nblocks:
        out = out[torch.randint(0, m, (nblocks,), device="cuda", generator=gen)]
    return out


def _tables(lens, bs, nblocks, width, gen):
    """Block tables [n, width] with the blocks of each length drawn from a permutation of the pool, -1 after them."""
    n = len(lens)
    perm = torch.randperm(nblocks, device="cuda", generator=gen).to(torch.int32)
    counts = torch.tensor([_up(v, bs) for v in lens], device="cuda")
    first = torch.cumsum(counts, 0) - counts
    col = torch.arange(width, device="cuda")[None]
    held = col < counts[:, None]
    return torch.where(held, perm[(first[:, None] + col).clamp(max=nblocks - 1)], -1).to(torch.int32), perm, int(counts.sum())


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case)
    op, n = case["op"], case["n"]
    bs = case.get("bs", 16)
    order = torch.randperm(n, generator=torch.Generator().manual_seed(seed)).tolist()
    if op == "plan":
        held, more = _spread(n, 0, case["most_old"]), _spread(n, 1, case["most_new"])
        old = [held[i] for i in order]
        new = [o + more[i] for o, i in zip(old, order[::-1])]
        width = _up(case["most_old"] + case["most_new"], bs)
        nblocks = sum(_up(v, bs) for v in new) + 64
        table, perm, used = _tables(old, bs, nblocks, width, gen)
        total = sum(new) - sum(old)
        s.update(old=_i32(old), new=_i32(new), table=table, free=perm[used:].clone(), n_free=_i32([nblocks - used]), width=width, cap=total + 5)
        s["free"] = torch.cat([s["free"], torch.zeros(used, dtype=torch.int32, device="cuda")])
        s.update(offsets=_empty(n + 1, torch.int32), slots=_empty(s["cap"], torch.int32), len=_empty(n, torch.int32), left=_empty(1, torch.int32))
        return _handles(s)
    if op == "select":
        W, V, dt = case["beams"], case["vocab"], _DT[case["dtype"]]
        x = torch.randn(n * W, V, device="cuda", generator=gen) * 2.5
        at = torch.randint(0, V, (n * W, 12), device="cuda", generator=gen)
        x.scatter_add_(1, at, torch.rand(n * W, 12, device="cuda", generator=gen) * 9 + 2)
        x[:, V - 7] += torch.where(torch.rand(n * W, device="cuda", generator=gen) < 0.3, 18.0, 0.0)
        scores = -torch.rand(n, W, device="cuda", generator=gen) * 6 - 3
        scores[::5, 1:] = -math.inf  # a request's first step: one live beam
        sup = torch.zeros(V, dtype=torch.uint8, device="cuda")
        sup[torch.randint(0, V - 8, (max(1, min(90, V // 20)),), device="cuda", generator=gen)] = 1
        s.update(logits=x.to(dt).contiguous(), scores=scores.contiguous(), suppress=sup, eos=V - 7)
        s.update(token=_empty((n, W), torch.int32), parent=_empty((n, W), torch.int32), score=_empty((n, W), torch.float32),
                 fin_parent=_empty((n, W), torch.int32), fin_score=_empty((n, W), torch.float32))
        return _handles(s)
    dt = _DT[case["dtype"]]
    hkv, dim = case["hkv"], case["dim"]
    slabs = hkv * dim // GROUP
    if op == "store":
        nblocks = _up(n, bs) + 3
        pool = torch.zeros(1, nblocks, slabs, bs // 16, REC, dtype=torch.uint8, device="cuda")
        perm = torch.randperm(nblocks, device="cuda", generator=gen)
        t = torch.arange(n, device="cuda")
        slots = (perm[t // bs] * bs + t % bs).to(torch.int32)
        d = hkv * dim
        rows = torch.randn(n, 3 * d if case["fused"] else 2 * d, device="cuda", generator=gen).to(dt)
        s.update(pool=pool, slots=slots, k=rows[:, -2 * d:-d], v=rows[:, -d:], nblocks=nblocks, layers=1)
        if not case["fused"]:
            s.update(k=s["k"].contiguous(), v=s["v"].contiguous())
        s.update(k_out=_empty((n, d), dt), v_out=_empty((n, d), dt))
        return _handles(s)
    if op == "attend":
        spread = _spread(n, case["least"], case["most"])
        lens = [spread[i] for i in order]
        width = _up(case["most"], bs)
        nblocks = sum(_up(v, bs) for v in lens) + 2
        table, perm, used = _tables(lens, bs, nblocks, width, gen)
        pool = _records(nblocks, slabs, bs, dt, gen)[None]
        pool[0, perm[used:].long()] = 0xFF  # blocks that nothing was written to
        blocks = table.tolist()
        for i, v in enumerate(lens):  # positions past the length, in the last block: what was there before
            if v % bs:
                at = torch.arange(v % bs, bs, device="cuda")
                rec = pool[0, blocks[i][v // bs]]
                szv = rec.view(slabs, bs // 16, REC)[:, :, 1024:].reshape(slabs, bs // 16, 8, 2, 2, 4)
                keep = torch.ones(bs, dtype=torch.bool, device="cuda")
                keep[at] = False
                keep = keep.view(bs // 16, 2, 8).permute(0, 2, 1)[None, :, :, None, :, None]
                rec[:, :, 1024:] = torch.where(keep, szv, 0xFF).reshape(slabs, bs // 16, 128)
        q = torch.randn(n * case["rps"], case["hq"], dim, device="cuda", generator=gen).to(dt)
        s.update(pool=pool.contiguous(), table=table, len=_i32(lens), q=q, width=width, nblocks=nblocks, scale=dim ** -0.5, layers=1)
        s["out"] = torch.empty_like(q)
        return _handles(s)
    W, L = case["beams"], case["layers"]
    spread = _spread(n, case["least"], case["most"])
    lens = [spread[i] for i in order]
    width = _up(case["most"] + 1, bs)
    rows = [v for v in lens for _ in range(W)]
    nblocks = sum(_up(v, bs) for v in rows) + 4
    table, perm, used = _tables(rows, bs, nblocks, width, gen)
    # beams of a request share the blocks before a point, and pairs of beams share more; the last, partly filled block is each one's own
    t3 = table.view(n, W, width)
    ln = torch.tensor(lens, device="cuda")
    col = torch.arange(width, device="cuda")[None, None]
    full = (ln // bs)[:, None, None]
    shared = (full * torch.rand(n, 1, 1, device="cuda", generator=gen)).long()
    pair = (torch.arange(W, device="cuda") // 2 * 2)[None, :, None].expand(n, W, width)
    table = torch.where(col < shared, t3[:, :1], torch.where((col < shared + 2) & (col < full), t3.gather(1, pair), t3)).reshape(n * W, width).contiguous()
    # W - W // 2 of the beams go on, W // 2 of them twice or more
    alive = torch.rand(n, W, device="cuda", generator=gen).argsort(1)[:, : W - W // 2]
    parent = torch.cat([alive, alive[:, torch.randint(0, W - W // 2, (W // 2,), device="cuda", generator=gen)]], 1)
    parent = parent.gather(1, torch.rand(n, W, device="cuda", generator=gen).argsort(1)).to(torch.int32).contiguous()
    if n > 3:
        parent[order[3] % n] = -1  # a finished request
    pool = _records(nblocks * L, slabs, bs, dt, gen).view(L, nblocks, slabs, bs // 16, REC)
    free = torch.full((nblocks,), -1, dtype=torch.int32, device="cuda")
    gone = torch.ones(nblocks, dtype=torch.bool, device="cuda")
    gone[table[table >= 0].long()] = False
    ids = gone.nonzero()[:, 0].to(torch.int32)
    free[: len(ids)] = ids
    s.update(pool=pool, table=table, len=_i32(rows), parent=parent, free=free, n_free=_i32([len(ids)]), width=width, nblocks=nblocks)
    s.update(table_out=torch.full_like(table, -1), left=_empty(1, torch.int32))
    return _handles(s)


# ------------------------------------------------------- the framework's calls --


def _empty(shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _handles(s):
    """What a program holds between its calls: the cache's descriptor, a workspace of the size that the framework asks for, an error word."""
    if not own:
        return s
    from paper_2609_32869_gb300 import binding as B
    op, size = s["op"], 0
    s["B"], s["err"] = B, torch.zeros(1, dtype=torch.int32, device="cuda")
    if op in ("store", "attend", "reorder"):
        s["p"] = B.kv4_pool(s["pool"], s["layers"], s["nblocks"], s["bs"], s["hkv"], s["dim"], B.WF_F16 if s["dtype"] == "f16" else B.WF_BF16)
    if op == "attend":
        size = B.wf_kv4_attention_scratch_bytes(s["n"], s["rps"], s["hq"], s["hkv"], s["dim"], s["most"])
    elif op == "select":
        s["dt"] = {"f32": B.WF_F32, "bf16": B.WF_BF16, "f16": B.WF_F16}[s["dtype"]]
        size = B.wf_beam_select_scratch_bytes(s["n"], s["beams"], s["vocab"])
    elif op == "reorder":
        size = B.wf_beam_reorder_scratch_bytes(s["n"], s["beams"], s["width"])
    s.update(bytes=size, scratch=_empty(max(256, size), torch.uint8))
    return s


def _run_own(s):
    B, op, n = s["B"], s["op"], s["n"]
    if op == "plan":
        B.wf_page_plan(s["old"], s["new"], n, s["bs"], s["free"], s["free"].numel(), s["n_free"], s["table"], s["width"], s["offsets"], s["slots"],
                       s["cap"], s["len"], s["left"], s["err"])
        return {"table": s["table"], "offsets": s["offsets"], "slots": s["slots"], "len": s["len"], "n_free": s["left"]}
    if op == "store":
        d = s["hkv"] * s["dim"]
        B.wf_kv4_store(s["p"], 0, s["k"], s["k"].stride(0), s["v"], s["v"].stride(0), s["slots"], n, s["err"])
        B.wf_kv4_load(s["p"], 0, s["slots"], n, s["k_out"], d, s["v_out"], d, s["err"])
        return {"k": s["k_out"], "v": s["v_out"]}
    if op == "attend":
        d = s["hq"] * s["dim"]
        B.wf_kv4_attention(s["p"], 0, s["q"], d, s["table"], s["width"], s["len"], n, s["rps"], s["hq"], s["causal"], s["scale"], s["most"], s["out"], d,
                           s["scratch"], s["bytes"], s["err"])
        return {"out": s["out"]}
    if op == "select":
        B.wf_beam_select(s["logits"], s["dt"], s["vocab"], s["scores"], s["suppress"], n, s["beams"], s["vocab"], s["eos"], s["token"], s["parent"],
                         s["score"], s["fin_parent"], s["fin_score"], s["scratch"], s["bytes"])
        return {k: s[k] for k in ("token", "parent", "score", "fin_parent", "fin_score")}
    B.wf_beam_reorder(s["p"], s["table"], s["table_out"], s["width"], s["len"], s["parent"], n, s["beams"], s["free"], s["n_free"], s["left"], s["scratch"],
                      s["bytes"], s["err"])
    return {"table": s["table_out"], "n_free": s["left"], "free": s["free"], "pool": s["pool"].view(torch.int32)}


# -------------------------------------------------------------- plain forms --


def _quantise(x, dtype):
    """x [..., 64] -> codes uint8 [..., 64], (s, z) [..., 2] in dtype."""
    x = x.float()
    hi, lo = x.amax(-1, keepdim=True), x.amin(-1, keepdim=True)
    s = ((0.5 * hi - 0.5 * lo) / 7.5).to(dtype).float()
    z = (hi - 7 * s).to(dtype).float()
    c = torch.where(s > 0, torch.round((x - z) / s), 0.0).clamp(-8, 7) + 8
    return c.to(torch.uint8), torch.cat([s, z], -1).to(dtype)


def _places():
    """Where in a record the 32 code bytes of value row `key` and its scale and offset are."""
    key = torch.arange(16, device="cuda")[:, None]
    b = torch.arange(32, device="cuda")[None]
    value = 512 + ((b // 4) * 4 + key % 8 // 2) * 16 + key // 8 * 8 + b // 2 % 2 * 4 + key % 2 * 2 + b % 2
    sz = 1024 + key % 8 * 16 + key // 8 * 4 + torch.arange(4, device="cuda")[None]
    return value, sz


def _write(blocks, codes, sz):
    """codes [2, m, slabs, bs, 64] and sz [2, m, slabs, bs, 2] (keys, values) into whole blocks [m, slabs, bs/16, REC]."""
    m, slabs, nt = blocks.shape[:3]
    packed = (codes[..., 0::2] | (codes[..., 1::2] << 4)).view(2, m, slabs, nt, 16, 32)
    raw = sz.contiguous().view(torch.uint8).view(2, m, slabs, nt, 16, 4)
    value, at = _places()
    blocks[..., :512] = packed[0].reshape(m, slabs, nt, 512)
    blocks[..., value.reshape(-1)] = packed[1].reshape(m, slabs, nt, 512)
    blocks[..., at.reshape(-1)] = raw[0].reshape(m, slabs, nt, 64)
    blocks[..., (at + 8).reshape(-1)] = raw[1].reshape(m, slabs, nt, 64)


def _read(rec, dtype):
    """Records [..., REC] as fp32 keys and values [..., 16, 64]."""
    lead = rec.shape[:-1]
    kb = rec[..., :512].reshape(*lead, 16, 32)
    # value bytes: [dims / 8][key pair][upper 8 keys][dims / 4 % 2][odd key][byte]
    vb = rec[..., 512:1024].reshape(*lead, 8, 4, 2, 2, 2, 2)
    e = len(lead)
    vb = vb.permute(*range(e), e + 2, e + 1, e + 4, e, e + 3, e + 5).reshape(*lead, 16, 32)
    sz = rec[..., 1024:].contiguous().view(dtype).reshape(*lead, 8, 2, 2, 2)  # [key % 8][keys, values][key / 8][s, z]
    sz = sz.permute(*range(e), e + 1, e + 2, e, e + 3).reshape(*lead, 2, 16, 2).float()

    def one(b, sz):
        c = torch.stack([b & 15, b >> 4], -1).reshape(*lead, 16, 64).float() - 8
        return c * sz[..., :1] + sz[..., 1:]

    return one(kb, sz[..., 0, :, :]), one(vb, sz[..., 1, :, :])


def _plain_plan(s):
    bs, n, cap = s["bs"], s["n"], s["cap"]
    old, new, nf = s["old"].long(), s["new"].long(), s["n_free"].long()
    have, want = (old + bs - 1) // bs, (new + bs - 1) // bs
    cb, ct = torch.cumsum(want - have, 0), torch.cumsum(new - old, 0)
    ok = (cb <= nf) & (ct <= cap)
    ends = torch.cumsum(torch.where(ok, new - old, 0), 0)
    offsets = torch.cat([ends.new_zeros(1), ends])
    left = nf - torch.where(ok, want - have, 0).sum()
    col = torch.arange(s["width"], device="cuda")[None]
    mine = ok[:, None] & (col >= have[:, None]) & (col < want[:, None])
    at = nf - 1 - ((cb - (want - have))[:, None] + col - have[:, None])
    table = torch.where(mine, s["free"][at.clamp(0, s["free"].numel() - 1)], s["table"])
    t = torch.arange(cap, device="cuda")
    i = torch.searchsorted(ends, t, right=True).clamp(max=n - 1)
    pos = old[i] + t - offsets[i]
    slots = torch.where(t < ends[-1], table[i, (pos // bs).clamp(0, s["width"] - 1)] * bs + pos % bs, -1)
    s["table"].copy_(table)
    return {"table": s["table"], "offsets": offsets.int(), "slots": slots.int(), "len": torch.where(ok, new, old).int(), "n_free": left.int()}


def _plain_store(s):
    n, hkv, dim, bs, dt = s["n"], s["hkv"], s["dim"], s["bs"], _DT[s["dtype"]]
    slabs = hkv * dim // GROUP
    slot = s["slots"].long()
    base = (slot // bs)[:, None] * (slabs * (bs // 16)) + torch.arange(slabs, device="cuda")[None] * (bs // 16) + (slot % bs // 16)[:, None]
    key = slot % 16
    value, at = _places()
    keys = key[:, None] * 32 + torch.arange(32, device="cuda")[None]
    flat = s["pool"].view(-1, REC)
    for_k, for_v = _quantise(s["k"].reshape(n, slabs, GROUP), dt), _quantise(s["v"].reshape(n, slabs, GROUP), dt)

    def put(codes, sz, where, plus):
        packed = codes[..., 0::2] | (codes[..., 1::2] << 4)
        flat[base[..., None], where[:, None, :].expand(n, slabs, 32)] = packed
        flat[base[..., None], (at[key] + plus)[:, None, :].expand(n, slabs, 4)] = sz.contiguous().view(torch.uint8).view(n, slabs, 4)

    def get(where, plus):
        b = flat[base[..., None], where[:, None, :].expand(n, slabs, 32)]
        sz = flat[base[..., None], (at[key] + plus)[:, None, :].expand(n, slabs, 4)].view(dt).float()
        c = torch.stack([b & 15, b >> 4], -1).reshape(n, slabs, GROUP).float() - 8
        return (c * sz[..., :1] + sz[..., 1:]).to(dt).view(n, hkv * dim)

    put(*for_k, keys, 0)
    put(*for_v, value[key], 8)
    return {"k": get(keys, 0), "v": get(value[key], 8)}


def _plain_attend(s):
    n, rps, hq, hkv, dim, bs, dt = s["n"], s["rps"], s["hq"], s["hkv"], s["dim"], s["bs"], _DT[s["dtype"]]
    g, G = hq // hkv, dim // GROUP
    T = s["width"] * bs
    rec = s["pool"][0][s["table"].long().clamp(min=0)]  # [n, width, slabs, bs/16, REC]
    k, v = _read(rec, dt)
    shape = lambda x: x.view(n, s["width"], hkv, G, bs, GROUP).permute(0, 2, 1, 4, 3, 5).reshape(n, hkv, T, dim)  # noqa: E731
    pos = torch.arange(T, device="cuda")
    held = (pos[None] < s["len"][:, None])[:, None, :, None]
    k, v = torch.where(held, shape(k), 0.0), torch.where(held, shape(v), 0.0)
    q = s["q"].float().view(n, rps, hkv, g, dim).permute(0, 2, 1, 3, 4).reshape(n, hkv, rps * g, dim)
    x = torch.matmul(q, k.transpose(2, 3)) * s["scale"]
    end = s["len"][:, None] - (rps - 1 - torch.arange(rps, device="cuda")[None] if s["causal"] else 0)
    seen = (pos[None, None] < end.expand(n, rps)[..., None]).repeat_interleave(g, 1)[:, None]
    x = torch.where(seen, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(x - torch.where(m > -math.inf, m, 0.0)), 0.0)
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(l > 0, l, 1.0)
    return {"out": o.view(n, hkv, rps, g, dim).permute(0, 2, 1, 3, 4).reshape(n * rps, hq, dim).to(dt)}


def _best(x, k):
    """The k largest of each row of x (no NaN), descending, equal ones by index: their places."""
    i = (x + 0.0).view(torch.int32)
    rank = (i ^ ((i >> 31) & 0x7FFFFFFF)).long()
    key = rank * (1 << 32) + (0x7FFFFFFF - torch.arange(x.shape[-1], device="cuda"))
    return torch.topk(key, k, dim=-1, sorted=True).indices


def _plain_select(s):
    n, W, V, eos = s["n"], s["beams"], s["vocab"], s["eos"]
    x = s["logits"].float()
    x = torch.where(torch.isnan(x) | (s["suppress"] != 0)[None], -math.inf, x)
    m = x.amax(-1, keepdim=True)
    # the sum in 64 bits: whole numbers come out of its comparison with other beams'
    rest = torch.log(torch.exp(x - m).sum(-1, keepdim=True, dtype=torch.float64)).float()
    at = _best(x, 2 * W)
    total = s["scores"].view(n * W, 1) + ((x.gather(1, at) - m) - rest)
    total = torch.where(torch.isnan(total), -math.inf, total).view(n, 2 * W * W)
    top = _best(total, 2 * W)
    score, beam, token = total.gather(1, top), top // (2 * W), at.view(n, -1).gather(1, top)
    live = score > -math.inf
    ends = live & (token == eos) & (torch.arange(2 * W, device="cuda") < W)[None]
    goes = live & (token != eos)

    def packed(keep, v, none):
        place = torch.where(keep & (torch.cumsum(keep, 1) <= W), torch.cumsum(keep, 1) - 1, W)
        return torch.cat([none, none[:, :1]], 1).scatter(1, place, v.to(none.dtype))[:, :W].contiguous()

    none = torch.full((n, W), -1, dtype=torch.int32, device="cuda")
    low = torch.full((n, W), -math.inf, device="cuda")
    idle = torch.arange(W, device="cuda", dtype=torch.int32)[None].expand(n, W)
    return {"token": packed(goes, token, none), "parent": packed(goes, beam, idle), "score": packed(goes, score, low),
            "fin_parent": packed(ends, beam, none), "fin_score": packed(ends, score, low)}


def _plain_reorder(s):
    n, W, bs, C = s["n"], s["beams"], s["bs"], s["width"]
    old, parent = s["table"].view(n, W, C), s["parent"].view(n, W).long()
    length = s["len"].view(n, W)[:, 0].long()
    full, rem = length // bs, length % bs
    col = torch.arange(C, device="cuda")
    none = parent < 0
    over = none.all(1)
    src = parent.clamp(min=0)
    # full blocks go with the parent
    new = torch.where(none[..., None], -1, old.gather(1, src[..., None].expand(n, W, C)))
    # the first child of a beam keeps its last, partly filled block; the other beams take the blocks of those without children
    w = torch.arange(W, device="cuda")
    child = (parent[:, None, :] == w[None, :, None])  # [n, beam, child]
    keeps = ~none & ~((parent[:, :, None] == parent[:, None, :]) & (w[None, :] < w[:, None])[None]).any(2)
    dead = ~child.any(2)
    dead_order = torch.argsort(torch.where(dead, w[None], W + w[None]), 1)
    from_beam = torch.where(keeps, src, dead_order.gather(1, (torch.cumsum(~keeps, 1) - 1).clamp(min=0)))
    tail = old.gather(1, from_beam[..., None].expand(n, W, C))
    in_full, in_tail = (col[None] < full[:, None])[:, None], ((col[None] == full[:, None]) & (rem > 0)[:, None])[:, None]
    new = torch.where(in_full, new, torch.where(in_tail, torch.where(over[:, None, None], -1, tail), s["table_out"].view(n, W, C)))
    # blocks that no beam holds any more, by request, column, beam
    used = in_full | in_tail
    held = (old[:, :, None] == new[:, None]).any(2)
    again = ((old[:, :, None] == old[:, None]) & (w[None, :] < w[:, None])[None, :, :, None]).any(2)
    gone = (used & (old >= 0) & ~held & ~again).permute(0, 2, 1).reshape(-1)
    rank = torch.cumsum(gone, 0) - 1
    ids, room = old.permute(0, 2, 1).reshape(-1)[gone], s["free"]
    room[(s["n_free"].long() + rank)[gone]] = ids
    left = s["n_free"] + gone.sum().int()
    # the last blocks' contents, in every layer, by 16 positions
    nt = bs // 16
    tile = torch.arange(nt, device="cuda") * 16
    moves = (~keeps & ~none & (rem > 0)[:, None])[..., None] & (tile[None] < rem[:, None])[:, None]
    i, b, t = moves.nonzero(as_tuple=True)
    a = old[i, parent[i, b], full[i]].long()
    z = new[i, b, full[i]].long()
    pool = s["pool"]
    pool[:, z, :, t] = pool[:, a, :, t]
    s["table_out"].copy_(new.reshape(n * W, C))
    return {"table": s["table_out"], "n_free": left, "free": room, "pool": pool.view(torch.int32)}


def run(state):
    if own:
        return _run_own(state)
    return {"plan": _plain_plan, "store": _plain_store, "attend": _plain_attend, "select": _plain_select, "reorder": _plain_reorder}[state["op"]](state)


# --------------------------------------------------------------------- work --


def work(case):
    """Each input read once and each output written once."""
    op, n = case["op"], case["n"]
    bs = case.get("bs", 16)
    if op == "plan":
        tokens = sum(_spread(n, 1, case["most_new"]))
        blocks = sum(_up(v, bs) for v in _spread(n, 1, case["most_new"]))
        return {"bytes": 4 * (3 * n + tokens + 2 * blocks + n), "flops": tokens + 4 * n}
    if op == "select":
        size = 4 if case["dtype"] == "f32" else 2
        rows = n * case["beams"]
        return {"bytes": rows * case["vocab"] * size + case["vocab"] + rows * 24, "flops": 4 * rows * case["vocab"]}
    slabs = case["hkv"] * case["dim"] // GROUP
    if op == "store":
        held = n * slabs * REC // 16 * 2  # keys and values: 72 bytes a position and group
        rows = 2 * n * case["hkv"] * case["dim"] * 2
        return {"bytes": 2 * rows + held + 4 * n, "flops": 10 * n * case["hkv"] * case["dim"]}
    lens = _spread(n, case["least"], case["most"])
    if op == "attend":
        keys = sum(lens)
        rows = n * case["rps"] * case["hq"] * case["dim"] * 2
        return {"bytes": keys * slabs * REC // 16 + 2 * rows + 4 * sum(_up(v, bs) for v in lens), "flops": 4 * keys * case["rps"] * case["hq"] * case["dim"]}
    W = case["beams"]
    tables = 4 * 2 * W * sum(_up(v, bs) for v in lens)
    moved = sum(_up(v % bs, 16) for v in lens) * (W // 2) * slabs * REC * case["layers"]
    return {"bytes": tables + 2 * moved, "flops": W * W * sum(_up(v, bs) for v in lens)}


# -------------------------------------------------------------------- exact --


def _exact_rows(raw, dtype):
    """Records [m, REC] in 64 bits, keys and values [m, 16, 64], each code looked up at its own byte."""
    key, dim = torch.meshgrid(torch.arange(16), torch.arange(64), indexing="ij")
    lane = dim // 8 * 4 + (key // 2) % 4
    half = (key // 8) * 4 + (dim // 4 % 2) * 2 + key % 2
    at = {"k": key * 32 + dim // 2, "v": 512 + lane * 16 + half * 2 + dim % 4 // 2}

    def one(where, plus):
        byte = raw[:, where.reshape(-1).cuda()].view(-1, 16, 64)
        code = torch.where((dim % 2 == 0).cuda(), byte % 16, byte // 16).double() - 8
        place = 1024 + torch.arange(16) % 8 * 16 + torch.arange(16) // 8 * 4 + plus
        pair = torch.stack([raw[:, (place + b).cuda()] for b in range(4)], -1).contiguous().view(dtype).double()
        return code * pair[..., :1] + pair[..., 1:]

    return one(at["k"], 0), one(at["v"], 8)


def exact(case, seed):
    op = case["op"]
    if op in ("plan", "reorder"):
        return None
    s = prepare(case, seed)
    n = case["n"]
    if op == "store":
        dt = _DT[case["dtype"]]

        def back(x):
            x = x.double().reshape(n, -1, GROUP)
            top, low = x.max(-1, keepdim=True).values, x.min(-1, keepdim=True).values
            step = ((top - low) / 15).to(dt).double()
            mid = (top - 7 * step).to(dt).double()
            c = torch.round((x - mid) / torch.where(step == 0, 1.0, step)).clamp(-8, 7)
            return torch.where(step == 0, mid.expand_as(x), step * c + mid).reshape(n, -1)

        return {"k": back(s["k"]), "v": back(s["v"])}
    if op == "attend":
        hkv, dim, bs, rps, g = case["hkv"], case["dim"], case["bs"], case["rps"], case["hq"] // case["hkv"]
        G = dim // GROUP
        out = torch.zeros(n * rps, case["hq"], dim, dtype=torch.float64, device="cuda")
        for i, length in enumerate(s["len"].tolist()):
            if not length:
                continue
            blocks = s["pool"][0, s["table"][i, : _up(length, bs)].long()]  # [nb, slabs, bs/16, REC]
            for h in range(hkv):
                rec = blocks[:, h * G:(h + 1) * G].permute(1, 0, 2, 3).reshape(-1, REC)
                k, v = (x.reshape(G, -1, GROUP).permute(1, 0, 2).reshape(-1, dim)[:length] for x in _exact_rows(rec, _DT[case["dtype"]]))
                for j in range(rps):
                    m = length - (rps - 1 - j) if case["causal"] else length
                    if m <= 0:
                        continue
                    q = s["q"][i * rps + j, h * g:(h + 1) * g].double()
                    a = torch.softmax(q @ k[:m].T * s["scale"], -1)
                    out[i * rps + j, h * g:(h + 1) * g] = a @ v[:m]
        return {"out": out}
    W, V, eos = case["beams"], case["vocab"], s["eos"]
    score, fin = torch.full((n, W), -math.inf, dtype=torch.float64), torch.full((n, W), -math.inf, dtype=torch.float64)
    for i in range(n):
        x = s["logits"][i * W:(i + 1) * W].double()
        x[:, s["suppress"].bool()] = -math.inf
        total = torch.log_softmax(x, -1) + s["scores"][i].double()[:, None]
        best = torch.topk(total.reshape(-1), 2 * W)
        values, tokens = best.values.cpu(), best.indices.cpu() % V
        ends = [v for j, (v, t) in enumerate(zip(values.tolist(), tokens.tolist())) if t == eos and j < W and v > -math.inf]
        goes = [v for v, t in zip(values.tolist(), tokens.tolist()) if t != eos and v > -math.inf][:W]
        score[i, : len(goes)], fin[i, : len(ends)] = torch.tensor(goes, dtype=torch.float64), torch.tensor(ends, dtype=torch.float64)
    return {"token": None, "parent": None, "score": score.cuda(), "fin_parent": None, "fin_score": fin.cuda()}
