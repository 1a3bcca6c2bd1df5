"""The operators in eight bits together, as the serving example runs them, against plain 64-bit arithmetic on what the library's codes stand
for; and a step of theirs captured into a graph."""
import os
import sys

import numpy as np
import pytest
import torch

import tests.eight_bit as eb
import tests.four_bit as fb
from paper_2410_09687_amd import moin
from tests.gpu_common import ctx

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import serve_eight_bit as example  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, I32 = torch.bfloat16, torch.int32


def f64(t):
    return t.detach().cpu().double().numpy()


def bf16(x):
    return f64(torch.tensor(x).to(BF16))


class Plain:
    """The layer in 64 bits; tokens in 8-bit integers, keys and values in E4M3 blocks, results rounded to bf16 where the library's are."""

    def __init__(self, layer):
        self.layer = layer
        self.W = {n: f64(w.codes[:, :w.d_in]) * f64(w.scales)[:, None] for n, w in layer.base.items()}
        self.past = {}

    def project(self, name, x, e):
        A, B = (f64(t[e]) for t in self.layer.adapters[name])
        q, s = eb.integers(x)
        return bf16((q * s[:, None]) @ self.W[name].T + self.layer.scale * ((x @ A.T) @ B.T))

    def step(self, s, x, e):
        lay = self.layer
        h, g, D = lay.n_heads, lay.n_kv, lay.head_dim
        qkv = self.project("qkv", x, e).reshape(len(x), h + 2 * g, D)
        cache, n = self.past.get(s, (eb.Cache(np.zeros((8, moin.KV8Pages.page_bytes(g, D))), 8, g, D, 64), 0))
        pos, f = np.arange(n, n + len(x)), f64(lay.freqs)
        q = bf16(eb.norm_rope(qkv[:, :h], pos, f, f64(lay.q_gain), 1e-6, True, False)[0])
        k = bf16(eb.norm_rope(qkv[:, h:h + g], pos, f, f64(lay.k_gain), 1e-6, True, False)[0])
        cache.append(k, qkv[:, h + g:], [0, len(x)], pos)
        self.past[s] = cache, n + len(x)
        k, v = cache.values()
        y = fb.attention(q, k[:n + len(x)], v[:n + len(x)], n, D ** -0.5, 0)[0]
        return self.project("o", bf16(y).reshape(len(x), h * D), e)


@pytest.mark.parametrize("n_heads,n_kv,head_dim", [(8, 2, 64), (2, 1, 128)])
def test_steps_against_plain_arithmetic(n_heads, n_kv, head_dim):
    """Bar: 3 % of the rms.  Where a projection differs by a rounding, a code of the cache may fall to its neighbour (a step of at most an eighth of it,
    one time in tens), a code of a token of the second projection by one of 127; the rest are bf16 roundings of 2^-8: all well below
    1 % of the rms in Frobenius norm; a token, position, page, expert or mask taken wrongly is an error of the order of the rms itself."""
    g = torch.Generator(device="cuda").manual_seed(5)
    layer = example.EightBitAttention(ctx(), 256, n_heads, n_kv, head_dim, 64, 4, g)
    centroids = torch.randn((4, 64), generator=g, device="cuda")
    server = example.Server(ctx(), layer, centroids, 4, n_pages=12, max_tokens=256)
    topics = torch.tensor([3, 1, 0, 1], device="cuda")
    server.admit(slice(None), centroids[topics] + 0.05)
    plain = Plain(layer)
    for step, lens in enumerate([[70, 1, 0, 33], [1, 1, 64, 1], [1, 1, 1, 0], [2, 0, 40, 1], [1, 1, 1, 1]]):
        if step == 3:
            server.finish([0, 1, 0, 1])
            for s in (1, 3):
                plain.past.pop(s)
        x = torch.randn((sum(lens), 256), generator=g, device="cuda").to(BF16)
        y, offsets = server.step(x, lens)
        ctx().check()
        off = offsets.tolist()
        want = np.concatenate([plain.step(s, f64(x[off[s]:off[s + 1]]), int(topics[s])) for s in range(4) if lens[s]])
        assert np.linalg.norm(f64(y) - want) <= 0.03 * np.linalg.norm(want)
        assert server.lens.tolist() == [plain.past.get(s, (None, 0))[1] for s in range(4)]
    server.finish([1] * 4)
    ctx().check()
    assert int(server.n_free) == 12 and sorted(server.free.tolist()) == list(range(12))


def test_a_captured_step_replays_token_after_token():
    """The whole step of a decode batch -- plans, projections, norms and rotation, append, attention -- as one graph, against the same calls made
    one after the other on a context and a cache of their own."""
    h, g, D, S, E = 4, 2, 64, 5, 3

    class Batch:
        def __init__(self, own):
            gen = torch.Generator(device="cuda").manual_seed(7)
            self.layer = example.EightBitAttention(own, 256, h, g, D, 64, E, gen)
            dev = lambda x: torch.tensor(x, dtype=I32).cuda()   # noqa: E731
            self.kv_plan, self.plan = moin.KVPlan(own), moin.Plan(own)
            self.pages = moin.KV8Pages.empty(24, g, D)
            self.pages.data.fill_(0xFF)
            self.lens, self.one, self.ids = dev([0, 60, 63, 64, 130]), dev([1] * S), dev([0, 1, 2, 0, -1])
            self.table = torch.full((S, 4), -1, dtype=I32, device="cuda")
            self.free, self.n_free = dev(list(range(24))), dev([24])
            self.off, self.slots = dev([0] * (S + 1)), dev([0] * S)
            self.x = torch.empty((S, 256), dtype=BF16, device="cuda")
            self.pos = torch.empty(S, dtype=I32, device="cuda")
            # the keys that the requests begin with
            k = torch.randn((317, 2 * g, D), generator=gen, device="cuda").to(BF16)
            zero = torch.zeros_like(self.lens)
            off, _, slots, _ = self.kv_plan.build(zero, self.lens.clone(), 317, self.table, self.free, self.n_free, n_pages=24, page_tokens=64, n_heads=h,
                                                  n_kv=g, max_new=130, out=(dev([0] * (S + 1)), zero, dev([0] * 317), self.n_free))
            moin.moin_kv8_append(own, self.pages, k[:, :g], k[:, g:], off, slots)
            own.check()

        def step(self):
            self.pos.copy_(self.lens)
            self.kv_plan.build(self.lens, self.one, S, self.table, self.free, self.n_free, n_pages=24, page_tokens=64, n_heads=h, n_kv=g, max_new=1,
                               out=(self.off, self.lens, self.slots, self.n_free))
            self.plan.build(self.off, self.ids, S, E)
            self.y = self.layer(self.plan, self.kv_plan, self.pages, self.table, self.off, self.slots, self.pos, self.x)

    own = moin.Context(0)
    try:
        a, b = Batch(own), Batch(ctx())
        x0 = torch.randn((S, 256), device="cuda").to(BF16)
        for q in (a, b):      # one step eagerly: it sizes the workspaces
            q.x.copy_(x0)
            q.step()
        own.check()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            a.step()
        for i in range(6):
            x = torch.randn((S, 256), device="cuda").to(BF16)
            a.x.copy_(x)
            b.x.copy_(x)
            graph.replay()
            b.step()
            own.check()
            ctx().check()
            assert torch.equal(a.y, b.y) and torch.equal(a.lens, b.lens) and torch.equal(a.pages.data, b.pages.data)
            assert torch.isfinite(a.y).all()
        del graph
        a.kv_plan.close()
        a.plan.close()
    finally:
        torch.cuda.synchronize()
        own.close()


def test_the_example_runs():
    example.main(n_requests=3, steps=4, prompt=70)
