"""The operators of scoring and prefilling prompts together, as a model would call them: norms and rotary positions, the cache's write, attention over the packed prompts, logits and the
log probabilities of the prompts' own tokens; then the prompts' next rows behind the cache that was read back.  Against 64 bits, eager, captured, replayed, on other streams."""
import numpy as np
import pytest

import prompt_oracle
import tree_oracle

pytestmark = pytest.mark.gpu

H, HKV, HD, VOCAB, TOP = 4, 2, 64, 3001, 5


def i32(x):
    import torch
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


def host(t):
    return t.double().cpu().numpy()


class Run:
    """Buffers of fixed sizes for prompts of up to `rows` rows in all, whose contents (lengths among them) change from pass to pass."""

    def __init__(self, dtype, rows=200, seqs=3, seed=0):
        import paper_2512_07503_amd as sjd
        import torch
        self.rng, self.rows, self.seqs, self.dtype = np.random.default_rng(seed), rows, seqs, dtype
        self.td = torch.float32 if dtype == "f32" else torch.bfloat16
        z = lambda *s: torch.zeros(s, dtype=self.td, device="cuda")
        self.qkv, self.tokens = z(rows, (H + 2 * HKV) * HD), i32([0] * rows)
        self.starts, self.first, self.positions = i32([0] * (seqs + 1)), i32([0] * seqs), i32([0] * rows)
        self.gain = [torch.from_numpy(1 + 0.2 * self.rng.standard_normal(HD).astype(np.float32)).cuda().to(self.td) for _ in range(2)]
        self.head = torch.from_numpy(self.rng.standard_normal((H * HD, VOCAB)).astype(np.float32) * 0.3).cuda().to(self.td)
        self.table = sjd.rope_table(HD)
        self.cache = sjd.KvCache("f32" if dtype == "f32" else "bf16", 20, 64, HKV, HD, i32(self.rng.permutation(20)[:12].reshape(3, 4)))

    def feed(self):
        import torch
        n = self.rng.multinomial(self.rows - 10, [0.5, 0.1, 0.4])
        self.n = n.tolist()
        self.at = np.concatenate([[0], np.cumsum(n)])
        self.starts.copy_(i32(self.at))
        positions = np.zeros(self.rows, dtype=np.int32)
        positions[:sum(n)] = np.concatenate([np.arange(m) for m in n])
        self.positions.copy_(i32(positions))
        self.qkv.copy_(torch.from_numpy(self.rng.standard_normal(tuple(self.qkv.shape)).astype(np.float32)).cuda())
        self.tokens.copy_(i32(self.rng.integers(0, VOCAB, self.rows)))

    def step(self):
        import paper_2512_07503_amd as sjd
        x = self.qkv.unflatten(1, (H + 2 * HKV, HD))
        q, k, v = x[:, :H], x[:, H:H + HKV], x[:, H + HKV:]
        q2, k2 = sjd.op_norm_rotary(q, k, self.positions, self.table, *self.gain)
        sjd.op_cache_write(self.cache, k2, v, self.starts, self.first)
        out = sjd.op_prompt_attention(q2, k2, v, self.starts, max_rows=self.rows, max_kv=self.rows)
        logits = out.flatten(1) @ self.head
        return (q2, k2, out, logits) + sjd.op_token_logprobs(logits, self.tokens, n_top=TOP)

    def check(self, outs):
        """Each operator against 64 bits on what came into it (its own tests say how far it may be off; here a quarter of a percent of the largest, and 2^-8 of a bf16 result)."""
        import paper_2512_07503_amd as sjd
        import torch
        torch.cuda.synchronize()
        q2, k2, out, logits = outs[:4]
        n = sum(self.n)
        x = host(self.qkv).reshape(self.rows, H + 2 * HKV, HD)
        f = tree_oracle.frequencies(HD)
        eps = 2.0 ** -20 if self.dtype == "f32" else 2.0 ** -8
        for got, lo, hi, g in ((q2, 0, H, self.gain[0]), (k2, H, H + HKV, self.gain[1])):
            y, _ = prompt_oracle.norm(x[:n, lo:hi], host(g), None, False, 1e-5)
            want, size = tree_oracle.rotary(y, host(self.positions)[:n], f, False)
            assert (np.abs(host(got)[:n] - want) <= 2.0 ** -20 * (1 + size) + eps * np.abs(want)).all()
        v = x[:, H + HKV:]
        kept = sjd.op_cache_read(self.cache, self.starts, self.first, self.rows, dtype=self.td)
        assert torch.equal(kept[0][:n], k2[:n])
        for b in range(self.seqs):
            rows = slice(self.at[b], self.at[b + 1])
            want, size, dot = prompt_oracle.attention(host(q2)[rows], host(k2)[rows], v[rows], HD ** -0.5)
            if want.size:
                tol = 2.0 ** -18 * (1 + dot) * size if self.dtype == "f32" else 2.0 ** -7 * (size + np.abs(want))
                assert (np.abs(host(out)[rows] - want) <= tol).all()
        r = prompt_oracle.logprobs(host(logits)[:n], self.tokens.cpu().numpy()[:n], TOP)
        assert np.array_equal(outs[5].cpu().numpy()[:n], r["rank"]) and np.array_equal(outs[7].cpu().numpy()[:n], r["ids"])
        for got, want in ((outs[4], r["logprob"]), (outs[6], r["entropy"]), (outs[8], r["top"])):
            assert np.abs(host(got)[:n] - want).max() <= 2.0 ** -16 * (1 + np.abs(want).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_eager(dtype):
    l = Run(dtype)
    for _ in range(3):
        l.feed()
        l.check(l.step())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_agrees_with_attention_over_the_cache(dtype):
    """A prompt is a window without a context: op_tree_attention over the cache that was written gives the same, to either's rounding.  And the rows of a second part of the prompt give what
    they gave in one pass, behind the first part's keys and values as the cache returns them."""
    import paper_2512_07503_amd as sjd
    l = Run(dtype, seed=1)
    l.feed()
    q2, k2, out = l.step()[:3]
    n = sum(l.n)
    again = sjd.op_tree_attention(q2, l.cache, l.starts, l.first, max_rows=l.rows, max_ctx=0)
    d = np.abs(host(again)[:n] - host(out)[:n])
    v = host(l.qkv).reshape(l.rows, H + 2 * HKV, HD)[:n, H + HKV:]
    # (each is at most 2^-8 (sum p |v| + |out|) and a rounding off in bf16)
    assert d.max() <= (2.0 ** -16 if dtype == "f32" else 2.0 ** -5) * np.abs(v).max()
    half = [m // 2 for m in l.n]
    pick = np.concatenate([np.arange(l.at[b] + h, l.at[b + 1]) for b, h in enumerate(half)])
    late = np.concatenate([[0], np.cumsum([m - h for m, h in zip(l.n, half)])])
    k, v = sjd.op_cache_read(l.cache, l.starts, l.first, l.rows, dtype=l.td)
    part = sjd.op_prompt_attention(q2[pick].contiguous(), k, v, i32(late), kv_start=l.starts, max_rows=l.rows, max_kv=l.rows)
    d = np.abs(host(part) - host(out)[pick])
    assert d.max() <= (2.0 ** -16 if dtype == "f32" else 2.0 ** -5) * np.abs(host(v)).max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_and_replayed(dtype):
    """One graph, replayed with eager work and synchronizations in between; lengths change on the device."""
    import torch
    l = Run(dtype, seed=2)
    l.feed()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        l.check(l.step())                # warm-up: an eager pass on another stream
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = l.step()
    for i in range(5):
        l.feed()
        graph.replay()
        l.check(outs)
        if i == 2:
            l.feed()
            l.check(l.step())


def test_splits_captured_and_two_graphs():
    """Calls with workspaces (few rows behind many keys, few rows of many logits), two of each captured into a graph of their own, replayed in turn and on two streams at once."""
    import paper_2512_07503_amd as sjd
    import torch
    rng = np.random.default_rng(3)
    runs = []
    for s in range(2):
        g = torch.Generator(device="cuda").manual_seed(s)
        q = torch.zeros((3, 8, 64), dtype=torch.bfloat16, device="cuda")
        k, v = (torch.randn((5000, 2, 64), generator=g, device="cuda").bfloat16() for _ in range(2))
        z, tokens = torch.zeros((2, 60000), device="cuda"), i32([7, 59999])
        starts, kv = i32([0, 3]), i32([0, 5000])

        def step(q=q, k=k, v=v, z=z, tokens=tokens, starts=starts, kv=kv):
            return (sjd.op_prompt_attention(q, k, v, starts, kv_start=kv, max_rows=3, max_kv=5000),) + sjd.op_token_logprobs(z, tokens, n_top=9)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = step()
        runs.append((q, z, kv, step, graph, outs))
    streams = [torch.cuda.Stream() for _ in runs]
    for i in range(4):
        for q, z, kv, *_ in runs:
            q.copy_(torch.from_numpy(rng.standard_normal((3, 8, 64)).astype(np.float32)))
            z.copy_(torch.from_numpy(rng.standard_normal((2, 60000)).astype(np.float32)))
            kv.copy_(i32([0, int(rng.integers(3, 5001))]))
        torch.cuda.synchronize()
        for (*_, graph, _), s in zip(runs, streams):
            with torch.cuda.stream(s if i % 2 else torch.cuda.default_stream()):
                graph.replay()
        torch.cuda.synchronize()
        for *_, step, _, outs in runs:
            for a, b in zip(outs, step()):
                assert torch.equal(a, b)


def test_on_a_stream_that_is_behind():
    """Work is enqueued on the current stream, and waits for what is ahead of it there."""
    import paper_2512_07503_amd as sjd
    import torch
    l = Run("bf16", seed=4)
    l.feed()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    source = l.qkv.clone()
    l.qkv.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        l.qkv.copy_(source)
        outs = l.step()
    s.synchronize()
    l.check(outs)
