"""Plain forms, inputs and 64-bit values of the prompt and 8-bit cache operators.

The operators take a request from its prompt to its first tokens:

  rope     rotary positions of queries and keys, or the gradient's way back (wf_rope)
  prompt   attention over whole prompts, packed one after another (wf_prompt_attention)
  store    rows of keys and values into a paged 8-bit cache and back (wf_kv8_store, wf_kv8_load)
  attend   attention of query rows over that cache (wf_kv8_attention)

Rotary positions.  Pair i of a head's first `rot` dims turns by pos * f_i, f_i =
base ** (-2 i / rot) or one of its scaled forms for long contexts; the pairs are
dims (i, i + rot / 2), or (2 i, 2 i + 1) in the interleaved layout.

The cache.  16 positions of a head form a record: their keys as e4m3 codes c with
one exponent e for the values c 2^e, their values likewise.  e is the least with
max |x| <= 448 * 2^e (and within -60 .. 36).  A stored row ends its record: the
positions before it are kept, under a larger exponent where it needs one, those
after it are zeros.  Bytes of a record: for every 64 dims 1024 of keys [position][dim]
and 1024 of values in the order the tensor instructions take them; then 2^e of the
keys, 2^e of the values (fp32) and 8 zero bytes.
"""
import math

import torch

own = False

LOW, HIGH = -60, 36  # exponents of a record


def listed():
    return [
        # one decode step of 16 requests with 5 beams each, queries and keys in the fused projection's output
        {"name": "rope_step", "op": "rope", "n": 80, "hq": 20, "hkv": 20, "dim": 64, "rot": 64, "pairs": "half", "scaling": "plain", "far": 448,
         "dtype": "bf16", "fused": True, "back": False},
        # a prompt batch of a long-context decoder with shared key/value heads
        {"name": "rope_prompt", "op": "rope", "n": 16384, "hq": 32, "hkv": 8, "dim": 128, "rot": 128, "pairs": "interleaved", "scaling": "parts",
         "far": 131072, "dtype": "bf16", "fused": False, "back": False},
        # the gradients of a training batch's queries and keys in fp32, half of each head rotated
        {"name": "rope_grad", "op": "rope", "n": 6001, "hq": 20, "hkv": 20, "dim": 64, "rot": 32, "pairs": "half", "scaling": "waves", "far": 20000,
         "dtype": "f32", "fused": False, "back": True},
        # 16 prompts of 1 to 224 tokens, admitted together
        {"name": "prompt_short", "op": "prompt", "n": 16, "least": 1, "most": 224, "past": 0, "hq": 20, "hkv": 20, "dim": 64, "causal": True,
         "dtype": "bf16"},
        # the encoder's own attention over 32 windows of 1500 frames
        {"name": "prompt_frames", "op": "prompt", "n": 32, "least": 1500, "most": 1500, "past": 0, "hq": 20, "hkv": 20, "dim": 64, "causal": False,
         "dtype": "bf16"},
        # one long prompt, shared key/value heads
        {"name": "prompt_long", "op": "prompt", "n": 1, "least": 8192, "most": 8192, "past": 0, "hq": 32, "hkv": 8, "dim": 128, "causal": True,
         "dtype": "bf16"},
        # pieces of 1 to 300 new tokens of three requests behind up to 30000 tokens that they hold already
        {"name": "prompt_piece", "op": "prompt", "n": 3, "least": 1, "most": 300, "past": 30000, "hq": 32, "hkv": 8, "dim": 128, "causal": True,
         "dtype": "f16"},
        # the new token of 80 beams in one decoder layer, behind the tokens that its record holds already
        {"name": "store8_step", "op": "store", "n": 80, "new": 1, "hkv": 20, "dim": 64, "bs": 16, "dtype": "bf16", "fused": True},
        # the encoder frames of 32 requests (1500 each) as one layer's cross-attention keys and values
        {"name": "store8_frames", "op": "store", "n": 32, "new": 1500, "hkv": 20, "dim": 64, "bs": 64, "dtype": "bf16", "fused": False},
        # cross-attention of one request's 5 beams over its 1500 frames: latency
        {"name": "attend8_frames_1", "op": "attend", "n": 1, "rps": 5, "hq": 20, "hkv": 20, "dim": 64, "least": 1500, "most": 1500, "bs": 64,
         "causal": False, "dtype": "bf16"},
        # cross-attention of 96 requests, 9 query rows each (a verified block of proposals)
        {"name": "attend8_frames_96", "op": "attend", "n": 96, "rps": 9, "hq": 20, "hkv": 20, "dim": 64, "least": 1500, "most": 1500, "bs": 64,
         "causal": False, "dtype": "bf16"},
        # a few long contexts with shared key/value heads, ragged, one new token each
        {"name": "attend8_long", "op": "attend", "n": 6, "rps": 1, "hq": 32, "hkv": 8, "dim": 128, "least": 5000, "most": 65001, "bs": 32,
         "causal": True, "dtype": "f16"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)) - 0.2)))))


def draw(rng):
    op = rng.choice(["rope", "rope", "prompt", "prompt", "prompt", "store", "store", "attend", "attend", "attend"])
    hkv, dim = rng.choice([(20, 64), (6, 64), (8, 128), (3, 64), (2, 128), (1, 128)])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if op == "rope":
        dim = rng.choice([dim, dim, 80, 96, 256])
        rot = rng.choice([dim, dim, dim // 2, dim // 4 // 2 * 2, 2 * rng.randint(1, dim // 2)])
        return {"op": op, "n": _log_int(rng, 1, 16000 * 5120 // (hkv * dim * 5)), "hq": hkv * rng.choice([1, 1, 4, 3]), "hkv": hkv, "dim": dim,
                "rot": rot, "pairs": rng.choice(["half", "interleaved"]), "scaling": rng.choice(["plain", "plain", "linear", "base", "waves", "parts"]),
                "far": _log_int(rng, 10, 2_000_000), "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "fused": rng.random() < 0.5,
                "back": rng.random() < 0.4}
    if op == "prompt":
        g = rng.choice([1, 1, 2, 4, 5, 7, 8])
        kind = rng.choice(["short", "packed", "frames", "long", "piece"])
        past, causal = 0, kind != "frames"
        if kind == "short":
            n, most = _log_int(rng, 1, 64), _log_int(rng, 1, 300)
            least = rng.choice([0, 1, most])
        elif kind == "packed":
            n, most, least = _log_int(rng, 2, 24), _log_int(rng, 200, 2500), rng.choice([0, 1, 100])
        elif kind == "frames":
            n, most = _log_int(rng, 1, 24), rng.choice([1500, 750, 1499])
            least = most
        elif kind == "long":
            n, most = rng.choice([1, 1, 2]), _log_int(rng, 1500, 6000)
            least = most
        else:
            n, most, least, past = _log_int(rng, 1, 6), _log_int(rng, 1, 400), 1, _log_int(rng, 100, 20000)
        while n * most * (most + past) * hkv * g * dim > 8192 * 8192 * 32 * 128 // 2:
            n, most = max(1, n // 2), (most + 1) // 2
        return {"op": op, "n": n, "least": min(least, most), "most": most, "past": past, "hq": hkv * g, "hkv": hkv, "dim": dim, "causal": causal,
                "dtype": dtype}
    bs = rng.choice([16, 32, 64])
    if op == "store":
        new = rng.choice([1, 1, 9, _log_int(rng, 1, 2000)])
        return {"op": op, "n": _log_int(rng, 1, max(1, min(256, 40000 * 1280 // (hkv * dim * new)))), "new": new, "hkv": hkv, "dim": dim, "bs": bs,
                "dtype": dtype, "fused": rng.random() < 0.5}
    kind = rng.choice(["frames", "beams", "long", "rows"])
    g = rng.choice([1, 1, 2, 4, 5, 7, 8]) if kind != "frames" else 1
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
        n, rps, most, causal = _log_int(rng, 1, 6), _log_int(rng, 17, 100), _log_int(rng, 200, 900), True
        least = most // 2
    return {"op": op, "n": n, "rps": rps, "hq": hkv * g, "hkv": hkv, "dim": dim, "least": least, "most": most, "bs": bs, "causal": causal,
            "dtype": dtype}


# ------------------------------------------------------------------ inputs --

_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

# scaled rotary frequencies: by what, and the context that the plain ones were trained for
FACTOR, TRAINED, BASE = 8.0, 8192, 10000.0
WAVES = (1.0, 4.0)   # turns over the trained context below and above which a frequency is scaled and is not
PARTS = (1.0, 32.0)  # likewise, as bounds of a ramp over the pairs
GAIN = 0.1 * math.log(FACTOR) + 1.0


def _up(x, m):
    return -(-x // m)


def _spread(n, lo, hi):
    """n lengths from lo to hi, the same for every seed up to their order."""
    return [lo + (i * 7919 * 104729 + (hi - lo)) % (hi - lo + 1) for i in range(n)]


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _empty(shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _rows(gen, n, heads, dim, dt):
    """What a projection gives: a channel's own offset and size, and a row's own size."""
    x = torch.randn(n, heads, dim, device="cuda", generator=gen)
    size = 0.5 + torch.rand(1, heads, dim, device="cuda", generator=gen) + torch.rand(n, 1, 1, device="cuda", generator=gen)
    return (x * size + 0.3 * torch.randn(1, heads, dim, device="cuda", generator=gen)).to(dt)


def _record_bytes(dim):
    return 32 * dim + 16


def _records(nblocks, hkv, dim, bs, gen):
    """Cache blocks [nblocks, hkv, bs / 16, bytes] of a decoder's keys and values; a few distinct ones repeated."""
    m = min(nblocks, 96)
    x = _rows(gen, 2 * m * bs, hkv, dim, torch.float32).view(2, m, bs // 16, 16, hkv, dim).permute(0, 1, 4, 2, 3, 5)
    out = _pack(*_quantise(x[0], None), *_quantise(x[1], None))
    if m < nblocks:
        out = out[torch.randint(0, m, (nblocks,), device="cuda", generator=gen)]
    return out.contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case)
    op, n, dim, hkv, dt = case["op"], case["n"], case["dim"], case["hkv"], _DT[case["dtype"]]
    order = torch.randperm(n, generator=torch.Generator().manual_seed(seed)).tolist()
    if op == "rope":
        hq = case["hq"]
        x = _rows(gen, n, hq + 2 * hkv, dim, dt)
        q, k = x[:, :hq], x[:, hq:hq + hkv]
        if not case["fused"]:
            q, k = q.contiguous(), k.contiguous()
        end = torch.randint(case["far"] // 2, case["far"], (1,), device="cuda", generator=gen)
        pos = torch.randint(0, case["far"], (n,), device="cuda", generator=gen) if n < 500 else (end - n + torch.arange(n, device="cuda")).abs()
        s.update(q=q, k=k, pos=pos.to(torch.int32), q_out=_empty((n, hq, dim), dt), k_out=_empty((n, hkv, dim), dt))
        return _handles(s)
    if op == "prompt":
        hq = case["hq"]
        spread, held = _spread(n, case["least"], case["most"]), _spread(n, case["past"] // 2, case["past"])
        lens = [spread[i] for i in order]
        keys = [a + held[i] for a, i in zip(lens, order[::-1])]
        q = _rows(gen, max(1, sum(lens)), hq, dim, dt)
        kv = _rows(gen, max(1, sum(keys)), 2 * hkv, dim, dt)
        s.update(lens=lens, keys=keys, q=q, k=kv[:, :hkv], v=kv[:, hkv:], scale=dim ** -0.5)
        for name, v in (("q_start", lens), ("k_start", keys)):
            s[name] = _i32([sum(v[:i]) for i in range(n + 1)])
        s.update(out=torch.zeros_like(q), lse=torch.zeros(q.shape[0], hq, dtype=torch.float32, device="cuda"))
        return _handles(s)
    bs = case["bs"]
    if op == "store":
        new = case["new"]
        filled = [(i * 7919) % 16 if new < 100 else 0 for i in range(n)]  # of each request's first record
        per = max(_up(f + new, bs) for f in filled)
        nblocks = n * per + 2
        perm = torch.randperm(nblocks, generator=torch.Generator().manual_seed(seed)).tolist()
        slots, see = [], []
        for i in range(n):
            f = filled[order[i]]
            at = [perm[i * per + p // bs] * bs + p % bs for p in range(f + new)]
            slots, see = slots + at[f:], see + at
        total = len(slots)
        x = _rows(gen, total, 3 * hkv if case["fused"] else 2 * hkv, dim, dt)
        k, v = x[:, -2 * hkv:-hkv], x[:, -hkv:]
        if not case["fused"]:
            k, v = k.contiguous(), v.contiguous()
        s.update(pool=_records(nblocks, hkv, dim, bs, gen), k=k, v=v, total=total, slots=_i32(slots), see=_i32(see), nblocks=nblocks)
        s.update(k_out=_empty((len(see), hkv, dim), dt), v_out=_empty((len(see), hkv, dim), dt))
        return _handles(s)
    spread = _spread(n, case["least"], case["most"])
    lens = [spread[i] for i in order]
    width = _up(case["most"], bs)
    nblocks = sum(_up(v, bs) for v in lens) + 2
    perm = torch.randperm(nblocks, device="cuda", generator=gen).to(torch.int32)
    counts = torch.tensor([_up(v, bs) for v in lens], device="cuda")
    first, col = torch.cumsum(counts, 0) - counts, torch.arange(width, device="cuda")[None]
    table = torch.where(col < counts[:, None], perm[(first[:, None] + col).clamp(max=nblocks - 1)], -1).to(torch.int32)
    pool = _records(nblocks, hkv, dim, bs, gen)
    pool[perm[int(counts.sum()):].long()] = 0xFF  # blocks that nothing was written to
    q = _rows(gen, n * case["rps"], case["hq"], dim, dt)
    s.update(pool=pool, table=table, len=_i32(lens), q=q, width=width, nblocks=nblocks, scale=dim ** -0.5, out=torch.empty_like(q))
    return _handles(s)


# ------------------------------------------------------- the framework's calls --


def _handles(s):
    """What a program holds between its calls: the rotary table, the cache's descriptor, a workspace of the size that the framework asks for, an error word."""
    if not own:
        return s
    from paper_2609_32869_gb300 import binding as B
    op, size = s["op"], 0
    s["B"], s["err"] = B, torch.zeros(1, dtype=torch.int32, device="cuda")
    s["dt"] = {"bf16": B.WF_BF16, "f16": B.WF_F16, "f32": B.WF_F32}[s["dtype"]]
    if op == "rope":
        kw = {"plain": {}, "linear": {"scaling": B.WF_ROPE_LINEAR, "factor": FACTOR}, "base": {"scaling": B.WF_ROPE_BASE, "factor": FACTOR},
              "waves": {"scaling": B.WF_ROPE_WAVES, "factor": FACTOR, "trained_len": TRAINED, "low": WAVES[0], "high": WAVES[1]},
              "parts": {"scaling": B.WF_ROPE_PARTS, "factor": FACTOR, "trained_len": TRAINED, "low": PARTS[0], "high": PARTS[1], "gain": GAIN}}[s["scaling"]]
        s["table"] = B.wf_rope_init(s["dim"], s["rot"], B.WF_ROPE_HALF if s["pairs"] == "half" else B.WF_ROPE_INTERLEAVED, BASE, **kw)
    if op in ("store", "attend"):
        s["p"] = B.kv8_pool(s["pool"], 1, s["nblocks"], s["bs"], s["hkv"], s["dim"], s["dt"])
    if op == "attend":
        size = B.wf_kv8_attention_scratch_bytes(s["n"], s["rps"], s["hq"], s["hkv"], s["dim"], s["most"])
    elif op == "prompt":
        size = B.wf_prompt_attention_scratch_bytes(s["n"], s["q"].shape[0], max(s["keys"]), s["hq"], s["hkv"], s["dim"])
    s.update(bytes=size, scratch=_empty(max(256, size), torch.uint8))
    return s


def _run_own(s):
    B, op, n = s["B"], s["op"], s["n"]
    if op == "rope":
        B.wf_rope(s["table"], s["q"], s["q"].stride(0), s["hq"], s["k"], s["k"].stride(0), s["hkv"], s["pos"], n, s["dt"], s["back"],
                  s["q_out"], s["hq"] * s["dim"], s["k_out"], s["hkv"] * s["dim"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "prompt":
        B.wf_prompt_attention(s["q"], s["q"].stride(0), s["k"], s["k"].stride(0), s["v"], s["v"].stride(0), s["q_start"], s["k_start"], n,
                              s["q"].shape[0], s["k"].shape[0], max(s["keys"]), s["hq"], s["hkv"], s["dim"], s["dt"], s["causal"], s["scale"],
                              s["out"], s["hq"] * s["dim"], s["lse"], s["scratch"], s["bytes"], s["err"])
        return {"out": s["out"], "lse": s["lse"]}
    d = s["hkv"] * s["dim"]
    if op == "store":
        B.wf_kv8_store(s["p"], 0, s["k"], s["k"].stride(0), s["v"], s["v"].stride(0), s["slots"], s["total"], s["err"])
        B.wf_kv8_load(s["p"], 0, s["see"], s["see"].numel(), s["k_out"], d, s["v_out"], d, s["err"])
        return {"k": s["k_out"], "v": s["v_out"]}
    d = s["hq"] * s["dim"]
    B.wf_kv8_attention(s["p"], 0, s["q"], d, s["table"], s["width"], s["len"], n, s["rps"], s["hq"], s["causal"], s["scale"], s["most"], s["out"], d,
                       s["scratch"], s["bytes"], s["err"])
    return {"out": s["out"]}


# -------------------------------------------------------------- plain forms --


def _turns(s):
    """f_i in 64 bits, and what cos and sin are multiplied by."""
    rot, kind = s["rot"], s["scaling"]
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    base = BASE * FACTOR ** (rot / (rot - 2)) if kind == "base" and rot > 2 else BASE
    f = base ** (-2 * i / rot)
    if kind == "linear":
        f = f / FACTOR
    if kind == "waves":
        lo, hi = WAVES
        keep = ((f * TRAINED / (2 * math.pi) - lo) / (hi - lo)).clamp(0, 1)
        f = f * (keep + (1 - keep) / FACTOR)
    if kind == "parts":
        pair = [rot * math.log(TRAINED / (2 * math.pi * t)) / (2 * math.log(BASE)) for t in PARTS]
        first, last = max(math.floor(pair[1]), 0), min(math.ceil(pair[0]), rot - 1)
        ramp = ((i - first) / max(last - first, 0.001)).clamp(0, 1)
        f = f * (1 - ramp + ramp / FACTOR)
    return f, GAIN if kind == "parts" else 1.0


def _plain_rope(s):
    rot, half = s["rot"], s["rot"] // 2
    f, gain = _turns(s)
    angle = s["pos"].double()[:, None] * f[None]
    cos, sin = (torch.cos(angle) * gain).float()[:, None], (torch.sin(angle) * gain).float()[:, None]
    sin = -sin if s["back"] else sin

    def turn(x):
        y = x.float().clone()
        a, b = (y[..., :half].clone(), y[..., half:rot].clone()) if s["pairs"] == "half" else (y[..., 0:rot:2].clone(), y[..., 1:rot:2].clone())
        u, v = a * cos - b * sin, a * sin + b * cos
        if s["pairs"] == "half":
            y[..., :half], y[..., half:rot] = u, v
        else:
            y[..., 0:rot:2], y[..., 1:rot:2] = u, v
        return y.to(x.dtype)

    return {"q": turn(s["q"]), "k": turn(s["k"])}


def _softmax_rows(q, k, v, seen, scale):
    """q [h, g, r, d], k and v [h, 1, t, d], seen [r, t]: outputs and the logarithms of the sums, zero and -inf where nothing is seen."""
    x = torch.where(seen, torch.matmul(q, k.transpose(-1, -2)) * scale, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m > -math.inf, m, 0.0)
    p = torch.where(seen, torch.exp(x - m), 0.0)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    return o, (m + torch.log(total))[..., 0]


def _plain_prompt(s):
    hq, hkv, dim, dt = s["hq"], s["hkv"], s["dim"], _DT[s["dtype"]]
    g = hq // hkv
    out, lse = torch.zeros_like(s["q"]), torch.zeros(s["q"].shape[0], hq, device="cuda")
    a, b = 0, 0
    for r, t in zip(s["lens"], s["keys"]):
        k, v = (s[c][b:b + t].float().permute(1, 0, 2)[:, None] for c in ("k", "v"))
        for r0 in range(0, r, 1024):
            r1 = min(r, r0 + 1024)
            q = s["q"][a + r0:a + r1].float().view(r1 - r0, hkv, g, dim).permute(1, 2, 0, 3)
            end = t - r + 1 + torch.arange(r0, r1, device="cuda") if s["causal"] else torch.full((r1 - r0,), t, device="cuda")
            top = min(t, t - r + r1) if s["causal"] else t
            o, l = _softmax_rows(q, k[:, :, :top], v[:, :, :top], torch.arange(top, device="cuda")[None] < end[:, None], s["scale"])
            out[a + r0:a + r1] = o.permute(2, 0, 1, 3).reshape(r1 - r0, hq, dim).to(dt)
            lse[a + r0:a + r1] = l.permute(2, 0, 1).reshape(r1 - r0, hq)
        a, b = a + r, b + t
    return {"out": out, "lse": lse}


def _quantise(x, kept):
    """x [..., 16, dim] -> e4m3 codes (uint8) and 2^e [...].  kept: (codes as fp32, 2^e, which positions), of a record that goes on."""
    x = x.float()
    f, e = torch.frexp(x.abs().amax((-1, -2)))
    e = torch.where(f > 0, torch.where(f <= 0.875, e - 9, e - 8), LOW).clamp(LOW, HIGH)
    if kept is not None:
        e = torch.where(kept[2].any(-1), torch.maximum(e, torch.frexp(kept[1])[1] - 1), e)
    scale = ((e + 127) << 23).to(torch.int32).view(torch.float32)  # 2^e, exactly
    y = x / scale[..., None, None]
    if kept is not None:
        y = torch.where(kept[2][..., None], kept[0] * (kept[1] / scale)[..., None, None], y)
    return y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), scale


def _value_order():
    """Byte i of a record's 1024 value bytes of 64 dims holds the value of position p[i], dim d[i]."""
    i = torch.arange(1024, device="cuda")
    half, r, t, odd, a, e = i // 512, i // 64 % 8, i // 16 % 4, i // 8 % 2, i // 2 % 4, i % 2
    return 2 * t + e + 8 * (a // 2), 8 * r + 4 * (a % 2) + 2 * half + odd


def _pack(k, ks, v, vs):
    """Codes [..., 16, dim] and scales [...] as records [..., bytes]."""
    lead, dim = k.shape[:-2], k.shape[-1]
    p, d = _value_order()
    groups = lambda x: x.reshape(*lead, 16, dim // 64, 64).transpose(-2, -3)  # noqa: E731
    body = torch.cat([groups(k).reshape(*lead, dim // 64, 1024), groups(v)[..., p, d]], -1).reshape(*lead, 32 * dim)
    tail = torch.stack([ks, vs, torch.zeros_like(ks), torch.zeros_like(ks)], -1).contiguous().view(torch.uint8)
    return torch.cat([body, tail], -1)


def _unpack(rec):
    """Records [..., bytes] as codes in fp32 [..., 16, dim] and scales [...], of keys and of values."""
    lead, dim = rec.shape[:-1], (rec.shape[-1] - 16) // 32
    p, d = _value_order()
    body = rec[..., : 32 * dim].reshape(*lead, dim // 64, 2, 1024)
    v = torch.empty(*lead, dim // 64, 16, 64, dtype=torch.uint8, device="cuda")
    v[..., p, d] = body[..., 1, :]
    real = lambda x: x.reshape(*lead, dim // 64, 16, 64).transpose(-2, -3).reshape(*lead, 16, dim).view(torch.float8_e4m3fn).float()  # noqa: E731
    sc = rec[..., 32 * dim:].contiguous().view(torch.float32)
    return real(body[..., 0, :]), sc[..., 0], real(v), sc[..., 1]


def _plain_store(s):
    hkv, dim, dt = s["hkv"], s["dim"], _DT[s["dtype"]]
    tiles = s["bs"] // 16
    slot, see = s["slots"].long(), s["see"].long()
    at, which = torch.unique_consecutive(slot // 16, return_inverse=True)
    m = at.numel()
    flat = s["pool"].view(s["nblocks"], hkv, tiles, _record_bytes(dim))
    old = _unpack(flat[at // tiles, :, at % tiles])  # [m, hkv, ...]
    mine = torch.zeros(m, 16, dtype=torch.bool, device="cuda")
    mine[which, slot % 16] = True
    kept = (torch.cumsum(mine, 1) == 0)[:, None].expand(m, hkv, 16)
    parts = []
    for x, codes, scale in ((s["k"], old[0], old[1]), (s["v"], old[2], old[3])):
        rows = torch.zeros(m, 16, hkv, dim, device="cuda")
        rows[which, slot % 16] = x.float()
        parts += _quantise(rows.transpose(1, 2), (codes, scale, kept))
    flat[at // tiles, :, at % tiles] = _pack(*parts)
    k, ks, v, vs = _unpack(flat[see // s["bs"], :, see % s["bs"] // 16])
    pick = (torch.arange(see.numel(), device="cuda"), slice(None), see % 16)
    return {"k": (k * ks[..., None, None])[pick].to(dt), "v": (v * vs[..., None, None])[pick].to(dt)}


def _plain_attend(s):
    n, rps, hq, hkv, dim, dt = s["n"], s["rps"], s["hq"], s["hkv"], s["dim"], _DT[s["dtype"]]
    g, out = hq // hkv, torch.zeros_like(s["q"])
    per = max(1, 2_000_000_000 // (s["width"] * s["bs"] * hkv * dim * 24))  # requests at a time
    for i in range(0, n, per):
        table, length = s["table"][i:i + per].long().clamp(min=0), s["len"][i:i + per]
        b = table.shape[0]
        k, ks, v, vs = _unpack(s["pool"][table])  # [b, width, hkv, bs / 16, 16, dim]
        shape = lambda x, sc: (x * sc[..., None, None]).permute(0, 2, 1, 3, 4, 5).reshape(b, hkv, 1, -1, dim)  # noqa: E731
        k, v = shape(k, ks), shape(v, vs)
        pos = torch.arange(k.shape[3], device="cuda")
        held = (pos[None] < length[:, None])[:, None, None, :, None]
        k, v = torch.where(held, k, 0.0), torch.where(held, v, 0.0)
        q = s["q"][i * rps:(i + b) * rps].float().view(b, rps, hkv, g, dim).permute(0, 2, 3, 1, 4)
        end = length[:, None] - (rps - 1 - torch.arange(rps, device="cuda")[None] if s["causal"] else 0)
        seen = (pos[None, None] < end.expand(b, rps)[..., None])[:, None, None]
        o, _ = _softmax_rows(q, k, v, seen, s["scale"])
        out[i * rps:(i + b) * rps] = o.permute(0, 3, 1, 2, 4).reshape(b * rps, hq, dim).to(dt)
    return {"out": out}


def run(state):
    if own:
        return _run_own(state)
    return {"rope": _plain_rope, "prompt": _plain_prompt, "store": _plain_store, "attend": _plain_attend}[state["op"]](state)


# --------------------------------------------------------------------- work --


def work(case):
    """Each input read once and each output written once; the products of the keys that a row sees."""
    op, n, dim, hkv = case["op"], case["n"], case["dim"], case["hkv"]
    size = 4 if case["dtype"] == "f32" else 2
    if op == "rope":
        rows = n * (case["hq"] + hkv) * dim
        return {"bytes": 2 * rows * size + 4 * n, "flops": 3 * n * (case["hq"] + hkv) * case["rot"]}
    if op == "prompt":
        lens, held = _spread(n, case["least"], case["most"]), _spread(n, case["past"] // 2, case["past"])
        tokens, past = sum(lens), sum(held)
        pairs = sum(a * (b + (a + 1) / 2 if case["causal"] else a + b) for a, b in zip(lens, [past / n] * n))
        return {"bytes": tokens * case["hq"] * (dim * 4 + 4) + (tokens + past) * hkv * dim * 4, "flops": 4 * pairs * case["hq"] * dim}
    record = hkv * _record_bytes(dim) / 16  # bytes of a position
    if op == "store":
        new, filled = n * case["new"], sum((i * 7919) % 16 for i in range(n)) if case["new"] < 100 else 0
        row = 2 * hkv * dim * 2
        return {"bytes": new * row + 2 * filled * record + new * record + (new + filled) * (record + row), "flops": 4 * new * hkv * dim}
    keys, rows = sum(_spread(n, case["least"], case["most"])), n * case["rps"] * case["hq"] * dim
    return {"bytes": keys * record + 4 * rows + 4 * keys / case["bs"], "flops": 4 * keys * case["rps"] * case["hq"] * dim}


# -------------------------------------------------------------------- exact --


def _two(e):
    """2^e in 64 bits, from a list: a power function on the GPU need not be exact."""
    return torch.tensor([2.0 ** i for i in range(-300, 300)], dtype=torch.float64, device="cuda")[e.long() + 300]


def _grid(x, e):
    """x rounded to the e4m3 values times 2^e, in 64 bits: 3 bits behind the leading one, none below 2^-9."""
    y = x.double() * _two(-e)
    step = _two(torch.frexp(y)[1].clamp(min=-5) - 4)
    return (torch.round(y / step) * step).clamp(-448, 448)


def _exponent(x):
    """The least e of -60 .. 36 with max |x| <= 448 * 2^e over the last two dims."""
    big = x.double().abs().amax((-1, -2))
    e = torch.full(big.shape, LOW, dtype=torch.int64, device=big.device)
    for v in range(LOW, HIGH):
        e[big > 448 * 2.0 ** v] = v + 1
    return e


def _held(rec):
    """Records [m, bytes] in 64 bits: keys and values [m, 16, dim], each code looked up at its own byte, and their exponents."""
    m, dim = rec.shape[0], (rec.shape[1] - 16) // 32
    pos, d = torch.meshgrid(torch.arange(16), torch.arange(dim), indexing="ij")
    r, a, half, odd = d % 64 // 8, d // 4 % 2 + 2 * (pos // 8), d // 2 % 2, d % 2
    at = {"k": d // 64 * 2048 + pos * 64 + d % 64, "v": d // 64 * 2048 + 1024 + half * 512 + (r * 4 + pos % 8 // 2) * 16 + odd * 8 + a * 2 + pos % 2}
    got = []
    for name, off in (("k", 0), ("v", 4)):
        c = rec[:, at[name].reshape(-1).cuda()].view(m, 16, dim).int()
        mant, ex = (c & 7).double(), (c >> 3) & 15
        value = torch.where(ex == 0, mant * 2.0 ** -9, (8 + mant) * _two(ex - 10))
        value = torch.where(c >= 128, -value, value)
        scale = rec[:, 32 * dim + off:32 * dim + off + 4].contiguous().view(torch.float32)[:, 0].double()
        got += [value, torch.frexp(scale)[1].long() - 1]
    return got


def exact(case, seed):
    op = case["op"]
    s = prepare(case, seed)
    n, dim, hkv = case["n"], case["dim"], case["hkv"]
    if op == "rope":
        rot, out = case["rot"], {}
        f = []
        for i in range(rot // 2):
            base = BASE * FACTOR ** (rot / (rot - 2)) if case["scaling"] == "base" and rot > 2 else BASE
            v = math.exp(-2 * i / rot * math.log(base))
            turned = v * TRAINED / (2 * math.pi)
            if case["scaling"] == "linear":
                v /= FACTOR
            elif case["scaling"] == "waves":
                w = min(max((turned - WAVES[0]) / (WAVES[1] - WAVES[0]), 0), 1)
                v = w * v + (1 - w) * v / FACTOR
            elif case["scaling"] == "parts":
                at = [rot * math.log(TRAINED / (2 * math.pi * t)) / (2 * math.log(BASE)) for t in PARTS]
                first, last = max(math.floor(at[1]), 0), min(math.ceil(at[0]), rot - 1)
                w = min(max((i - first) / max(last - first, 0.001), 0), 1)
                v = w * v / FACTOR + (1 - w) * v
            f.append(v)
        angle = s["pos"].double()[:, None] * torch.tensor(f, dtype=torch.float64, device="cuda")
        turn = torch.polar(torch.full_like(angle, GAIN if case["scaling"] == "parts" else 1.0), -angle if case["back"] else angle)[:, None]
        for name in ("q", "k"):
            x = s[name].double()
            head = x[..., :rot]
            pair = head.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if case["pairs"] == "half" else head.unflatten(-1, (rot // 2, 2))
            y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
            y = y.transpose(-1, -2) if case["pairs"] == "half" else y
            out[name] = torch.cat([y.flatten(-2), x[..., rot:]], -1)
        return out
    if op == "store":
        bs, tiles = case["bs"], case["bs"] // 16
        slots, see = s["slots"].long(), s["see"].long()
        recs = torch.unique(slots // 16)
        rows = s["pool"][recs // tiles, :, recs % tiles].reshape(-1, _record_bytes(dim))
        k0, ke, v0, ve = _held(rows)
        place = torch.searchsorted(recs, slots // 16)
        first = torch.full((len(recs),), 16, device="cuda").scatter_reduce(0, place, slots % 16, "amin")
        keep = (torch.arange(16, device="cuda")[None] < first[:, None])
        out = {}
        for name, codes, e0 in (("k", k0, ke), ("v", v0, ve)):
            new = torch.zeros(len(recs), 16, hkv, dim, dtype=torch.float64, device="cuda")
            new[place, slots % 16] = s[name].double()
            new = new.transpose(1, 2)
            e, e0 = _exponent(new), e0.view(-1, hkv)
            e = torch.where(keep.any(1)[:, None], torch.maximum(e, e0), e)[..., None, None]
            old = codes.view(-1, hkv, 16, dim) * _two(e0)[..., None, None]
            val = _grid(torch.where(keep[:, None, :, None], old, new), e) * _two(e)
            out[name] = val[torch.searchsorted(recs, see // 16), :, see % 16]
        return out
    scale, g = s["scale"], case["hq"] // hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")

    def rows(q, k, v, ends):
        """q [r, g, d] on k, v [t, d], row i on the first ends[i] of them."""
        x = torch.einsum("rgd,td->rgt", q.double(), k) * scale
        x = x.masked_fill(torch.arange(k.shape[0], device="cuda") >= ends[:, None, None], -math.inf)
        total = torch.logsumexp(x, -1)
        return torch.einsum("rgt,td->rgd", torch.nan_to_num(torch.exp(x - total[..., None])), v), total

    if op == "prompt":
        lse = torch.full((s["q"].shape[0], case["hq"]), -math.inf, dtype=torch.float64, device="cuda")
        if not sum(s["lens"]):
            lse.zero_()
        a, b = 0, 0
        for r, t in zip(s["lens"], s["keys"]):
            for h in range(hkv):
                k, v = s["k"][b:b + t, h].double(), s["v"][b:b + t, h].double()
                for r0 in range(0, r, 1024):
                    r1 = min(r, r0 + 1024)
                    ends = torch.arange(r0, r1, device="cuda") + t - r + 1 if case["causal"] else torch.full((r1 - r0,), t, device="cuda")
                    top = min(t, t - r + r1) if case["causal"] else t
                    out[a + r0:a + r1, h * g:(h + 1) * g], lse[a + r0:a + r1, h * g:(h + 1) * g] = rows(
                        s["q"][a + r0:a + r1, h * g:(h + 1) * g], k[:top], v[:top], ends)
            a, b = a + r, b + t
        return {"out": out, "lse": lse}
    bs, rps = case["bs"], case["rps"]
    for i, t in enumerate(s["len"].tolist()):
        if not t:
            continue
        blocks = s["pool"][s["table"][i, : _up(t, bs)].long()]
        for h in range(hkv):
            k, ke, v, ve = _held(blocks[:, h].reshape(-1, _record_bytes(dim)))
            k, v = ((c * _two(e)[:, None, None]).reshape(-1, dim)[:t] for c, e in ((k, ke), (v, ve)))
            ends = torch.arange(rps, device="cuda") + t - rps + 1 if case["causal"] else torch.full((rps,), t, device="cuda")
            out[i * rps:(i + 1) * rps, h * g:(h + 1) * g] = rows(s["q"][i * rps:(i + 1) * rps, h * g:(h + 1) * g], k, v, ends)[0]
    return {"out": out}
