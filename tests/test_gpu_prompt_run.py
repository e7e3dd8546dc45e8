"""From packed prompts to tokens: rotary positions, prompt attention, the 8-bit cache and attention over it, one after another (GPU)."""
import numpy as np
import pytest

from oracle import prompt as op

pytestmark = pytest.mark.gpu

HQ, HKV, DIM, BS, COLS = 4, 2, 64, 16, 6
LENS = [5, 40, 17]
U = 2.0 ** -8


class Layer:
    """One layer's state of len(LENS) requests, as a program holds it."""

    def __init__(self, torch, B):
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
        n, blocks = len(LENS), len(LENS) * COLS
        self.torch, self.B, self.n, self.blocks = torch, B, n, blocks
        self.raw = torch.zeros(blocks * B.wf_kv8_block_bytes(BS, HKV, DIM), dtype=torch.uint8, device="cuda")
        self.pool = B.kv8_pool(self.raw, 1, blocks, BS, HKV, DIM)
        self.table = torch.full((n, COLS), -1, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(blocks, device="cuda").to(torch.int32)
        self.n_free, self.len, self.want, self.left, self.new_len = torch.full((1,), blocks, dtype=torch.int32, device="cuda"), i32(n), i32(n), i32(1), i32(n)
        self.offsets, self.err, self.pos = i32(n + 1), i32(1), i32(n)
        self.rope = B.wf_rope_init(DIM, 32, B.WF_ROPE_INTERLEAVED, 500000.0, B.WF_ROPE_WAVES, 8.0, 64.0, 1.0, 4.0)
        self.scratch = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def plan(self, more, cap):
        """Blocks and slots for `more` (device) new tokens of each request."""
        slots = self.torch.empty(cap, dtype=self.torch.int32, device="cuda")
        self.torch.add(self.len, more, out=self.want)
        self.B.wf_page_plan(self.len, self.want, self.n, BS, self.free, self.blocks, self.n_free, self.table, COLS, self.offsets, slots, cap, self.new_len,
                            self.left, self.err)
        self.len.copy_(self.new_len)
        self.n_free.copy_(self.left)
        return slots

    def turn(self, x, pos):
        """Queries and keys of the fused rows turn in place."""
        B, n = self.B, x.shape[0]
        k = x[:, HQ * DIM:]
        B.wf_rope(self.rope, x, x.stride(0), HQ, k, x.stride(0), HKV, pos, n, B.WF_BF16, False, x, x.stride(0), k, x.stride(0))

    def store(self, x, slots):
        k, v = x[:, HQ * DIM:], x[:, (HQ + HKV) * DIM:]
        self.B.wf_kv8_store(self.pool, 0, k, x.stride(0), v, x.stride(0), slots, x.shape[0], self.err)

    def prompt(self, x, start):
        out = self.torch.empty(x.shape[0], HQ * DIM, dtype=x.dtype, device="cuda")
        size = self.B.wf_prompt_attention_scratch_bytes(self.n, x.shape[0], max(LENS), HQ, HKV, DIM)
        assert size <= self.scratch.numel()
        self.B.wf_prompt_attention(x, x.stride(0), x[:, HQ * DIM:], x.stride(0), x[:, (HQ + HKV) * DIM:], x.stride(0), start, start, self.n, x.shape[0],
                                   x.shape[0], max(LENS), HQ, HKV, DIM, self.B.WF_BF16, True, DIM ** -0.5, out, HQ * DIM, None, self.scratch, size, self.err)
        return out

    def step(self, x, out, one):
        """A token of every request; x [n, (HQ + 2 HKV) DIM]."""
        self.pos.copy_(self.len)
        slots = self.plan(one, self.n)
        self.turn(x, self.pos)
        self.store(x, slots)
        size = self.B.wf_kv8_attention_scratch_bytes(self.n, 1, HQ, HKV, DIM, COLS * BS)
        self.B.wf_kv8_attention(self.pool, 0, x, x.stride(0), self.table, COLS, self.len, self.n, 1, HQ, True, DIM ** -0.5, COLS * BS, out, HQ * DIM,
                                self.scratch, size, self.err)


def _f64(x):
    return x.double().cpu().numpy()


def _oracle_step(cache, x, lens, table):
    """x: turned rows float64 [n, heads, DIM]; appends them and attends."""
    want, tol = [], []
    for i, t in enumerate(lens):
        at = [int(table[i, p // BS]) * BS + p % BS for p in range(t)]
        cache.store([at[-1]], x[i:i + 1, HQ:HQ + HKV], x[i:i + 1, HQ + HKV:])
        k, v = (np.array([cache.row(s, is_v) for s in at]) for is_v in (0, 1))
        o, _, mass = op.attention(x[i:i + 1, :HQ], k, v, DIM ** -0.5, [t])
        dx = 2.0 ** -24 * (DIM + 16) * DIM ** -0.5 * np.abs(x[i, :HQ]).max() * np.abs(k).sum(-1).max() + 2.0 ** -20
        want.append(o[0])
        tol.append(U * np.abs(o[0]) + (1 + U) * (2.0 ** -11 + 2 * dx) * mass[0] + 2.0 ** -22 * np.abs(v).max())
    return np.array(want), np.array(tol)


@pytest.mark.parametrize("how", ["plain", "stream", "graph"])
def test_prompts_and_tokens(how):
    import torch
    from paper_2609_32869_gb300 import binding as B
    torch.manual_seed(7)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side if how == "stream" else torch.cuda.current_stream()):
        la = Layer(torch, B)
        total, width, n = sum(LENS), (HQ + 2 * HKV) * DIM, len(LENS)
        x = torch.randn(total, width, device="cuda").bfloat16()
        before = _f64(x)
        pos = torch.cat([torch.arange(v, device="cuda") for v in LENS]).to(torch.int32)
        start = torch.tensor(np.concatenate([[0], np.cumsum(LENS)]), dtype=torch.int32, device="cuda")
        slots = la.plan(torch.tensor(LENS, dtype=torch.int32, device="cuda"), total)
        la.turn(x, pos)
        out = la.prompt(x, start)
        la.store(x, slots)
        # the prompt's rows: turned, attended, stored
        freq = op.frequencies(32, 500000.0, "waves", 8.0, 64.0, 1.0, 4.0)
        turned = _f64(x).reshape(total, -1, DIM)
        want = op.rope(before.reshape(total, -1, DIM)[:, :HQ + HKV], _f64(pos), freq, interleaved=True)
        assert (np.abs(turned[:, :HQ + HKV] - want) <= (U + 2.0 ** -21) * np.abs(before).max()).all()
        cache, table = op.Cache(la.blocks, BS, HKV, DIM), la.table.cpu().numpy()
        got, a = _f64(out).reshape(total, HQ, DIM), 0
        for i, t in enumerate(LENS):
            r = turned[a:a + t]
            o, _, mass = op.attention(r[:, :HQ], r[:, HQ:HQ + HKV], r[:, HQ + HKV:], DIM ** -0.5, np.arange(t) + 1)
            dx = 2.0 ** -24 * (DIM + 16) * DIM ** -0.5 * np.abs(r).max() ** 2 * DIM + 2.0 ** -20
            assert (np.abs(got[a:a + t] - o) <= U * np.abs(o) + (1 + U) * (U + 2 * dx) * mass).all()
            at = [int(table[i, p // BS]) * BS + p % BS for p in range(t)]
            cache.store(at, r[:, HQ:HQ + HKV], r[:, HQ + HKV:])
            a += t
        np.testing.assert_array_equal(la.raw.cpu().numpy()[: cache.raw.size].reshape(cache.raw.shape), cache.raw)
        # tokens
        one = torch.ones(n, dtype=torch.int32, device="cuda")
        buf, res = torch.zeros(n, width, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, HQ * DIM, dtype=torch.bfloat16, device="cuda")
        graph = None
        if how == "graph":
            saved = [v.clone() for v in (la.raw, la.table, la.free, la.n_free, la.len)]
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                la.step(buf, res, one)
            for v, s in zip((la.raw, la.table, la.free, la.n_free, la.len), saved):
                v.copy_(s)
        lens = list(LENS)
        for _ in range(20):
            buf.copy_(torch.randn(n, width, device="cuda").bfloat16())
            if graph is None:
                la.step(buf, res, one)
            else:
                graph.replay()
            lens = [v + 1 for v in lens]
            assert la.len.tolist() == lens
            want, tol = _oracle_step(cache, _f64(buf).reshape(n, -1, DIM), lens, la.table.cpu().numpy())
            assert (np.abs(_f64(res).reshape(n, HQ, DIM) - want) <= tol).all()
        assert la.err.item() == 0
    torch.cuda.synchronize()


def test_two_calls_at_once_with_their_own_scratch():
    """Prompt pieces and cache attention that need a workspace, on two streams at a time, and two graphs of them: each as alone."""
    import torch
    from paper_2609_32869_gb300 import binding as B
    torch.manual_seed(3)
    t, r, hq, hkv, dim = 5000, 3, 8, 2, 128
    k, v = (torch.randn(t, hkv * dim, device="cuda").half() for _ in range(2))
    qs, ks = (torch.tensor([0, x], dtype=torch.int32, device="cuda") for x in (r, t))
    size = B.wf_prompt_attention_scratch_bytes(1, r, t, hq, hkv, dim)
    size8 = B.wf_kv8_attention_scratch_bytes(1, r, hq, hkv, dim, t)
    assert size > 0 and size8 > 0
    blocks = -(-t // 64)
    raw = torch.zeros(blocks * B.wf_kv8_block_bytes(64, hkv, dim), dtype=torch.uint8, device="cuda")
    pool = B.kv8_pool(raw, 1, blocks, 64, hkv, dim, B.WF_F16)
    B.wf_kv8_store(pool, 0, k, hkv * dim, v, hkv * dim, torch.arange(t, dtype=torch.int32, device="cuda"), t)
    table, length = torch.arange(blocks, dtype=torch.int32, device="cuda"), torch.tensor([t], dtype=torch.int32, device="cuda")
    lanes = []
    for i in range(2):
        q = torch.randn(r, hq * dim, device="cuda").half()
        o, o8 = torch.zeros_like(q), torch.zeros_like(q)
        s, s8 = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty(size8, dtype=torch.uint8, device="cuda")

        def call(q=q, o=o, o8=o8, s=s, s8=s8):
            B.wf_prompt_attention(q, hq * dim, k, hkv * dim, v, hkv * dim, qs, ks, 1, r, t, t, hq, hkv, dim, B.WF_F16, True, 0.09, o, hq * dim, None, s, size)
            B.wf_kv8_attention(pool, 0, q, hq * dim, table, blocks, length, 1, r, hq, True, 0.09, t, o8, hq * dim, s8, size8)

        call()
        lanes.append((call, o, o8, o.clone(), o8.clone(), torch.cuda.Stream()))
    assert all(x[3].any() and x[4].any() for x in lanes)
    torch.cuda.synchronize()
    graphs = []
    for call, *_ in lanes:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    for use_graphs in (False, True):
        for _, o, o8, *_ in lanes:
            o.zero_(), o8.zero_()
        torch.cuda.synchronize()
        for _ in range(10):
            for (call, *_, stream), g in zip(lanes, graphs):
                with torch.cuda.stream(stream):
                    g.replay() if use_graphs else call()
        torch.cuda.synchronize()
        for _, o, o8, want, want8, _ in lanes:
            assert torch.equal(o, want) and torch.equal(o8, want8)
