"""An eager step with the most requests and tokens prepares captured ones of fewer: their requests may have other tiles (of few rows, of many,
or both), whose lists and partial results take other room."""
import pytest
import torch

from paper_2410_09687_amd import moin
from tests.gpu_common import ctx as common

pytestmark = pytest.mark.gpu
BF16, I32 = torch.bfloat16, torch.int32

CASES = [
    ([2048] * 2, [2048, 1], 2048, 32, 4, 64),      # tiles of many rows / both
    ([512] * 8, [512] * 7 + [3], 512, 32, 4, 64),
    ([512] * 8, [1] * 8, 512, 32, 4, 64),          # / tiles of few rows alone
    ([33, 33], [33, 7], 33, 1, 1, 64),
    ([300, 300, 300], [1, 300], 300, 16, 2, 128),
    ([40] * 3, [40, 4], 40, 8, 1, 256),
    ([1] * 64, [1] * 63, 1, 32, 4, 64),
    ([100, 1, 1], [100, 1], 100, 64, 1, 64)]       # 64 heads of a kv head: no tiles of few rows at all


class Step:
    """New requests, whose keys and values are given; everything that a call writes has its place beforehand."""

    def __init__(self, ctx, plan, new, max_new, heads, H, D):
        S, T, per = len(new), sum(new), -(-max(new) // 64)
        n_pages = S * per + 1
        g = torch.Generator(device="cuda").manual_seed(T)
        self.ctx, self.plan = ctx, plan
        self.kw = dict(n_pages=n_pages, page_tokens=64, n_heads=heads, n_kv=H, max_new=max_new)
        dev = lambda x: torch.tensor(x, dtype=I32).cuda()   # noqa: E731
        self.kv, self.new, self.T = dev([0] * S), dev(new), T
        self.table = torch.full((S, per), -1, dtype=I32, device="cuda")
        self.free, self.n_free = dev(list(range(n_pages))), dev([n_pages])
        self.out = (dev([0] * (S + 1)), dev([0] * S), dev([0] * T), dev([0]))
        self.pages = moin.KVPages.empty(n_pages, H, D)
        self.qkv = torch.randn((T, heads + 2 * H, D), device="cuda", generator=g).to(BF16)
        self.heads, self.H = heads, H
        self.y = torch.empty((T, heads, D), dtype=BF16, device="cuda")

    def build(self):
        self.plan.build(self.kv, self.new, self.T, self.table, self.free, self.n_free, out=self.out, **self.kw)

    def attend(self):
        h, g = self.heads, self.H
        moin.moin_kv_append(self.ctx, self.pages, self.qkv[:, h:h + g], self.qkv[:, h + g:], self.out[2])
        moin.moin_kv_attention(self.ctx, self.plan, self.pages, self.qkv[:, :h], self.table, out=self.y)


def captured(first, then, max_new, heads, H, D, whole):
    """The largest step eagerly, then the other one captured: its plan, or (`whole`) its attention as well."""
    ctx = moin.Context(0)
    try:
        plan = moin.KVPlan(ctx)
        big = Step(ctx, plan, first, max_new, heads, H, D)
        big.build()
        if whole:
            big.attend()
        ctx.check()
        other = moin.KVPlan(common())
        want = Step(common(), other, then, max_new, heads, H, D)
        want.build()
        want.attend()
        common().check()
        own = Step(ctx, plan, then, max_new, heads, H, D)
        torch.cuda.synchronize()
        print(f"[gpu] captured step of {len(then)} requests, {sum(then)} tokens after {sum(first)}, {heads} on {H} heads of {D}", flush=True)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            own.build()
            if whole:
                own.attend()
        for _ in range(3):
            own.table.fill_(-1)
            own.y.fill_(float("nan"))
            graph.replay()
            ctx.check()
            assert torch.equal(own.table, want.table) and all(torch.equal(a, b) for a, b in zip(own.out, want.out))
            if whole:
                assert torch.equal(own.y.view(torch.int16), want.y.view(torch.int16))
        del graph
        plan.close()
    finally:
        torch.cuda.synchronize()
        ctx.close()


@pytest.mark.parametrize("first,then,max_new,heads,H,D", CASES)
def test_a_plan_captured_after_the_largest_eager_one(first, then, max_new, heads, H, D):
    captured(first, then, max_new, heads, H, D, False)


@pytest.mark.parametrize("first,then,max_new,heads,H,D", CASES)
def test_attention_captured_after_the_largest_eager_step(first, then, max_new, heads, H, D):
    captured(first, then, max_new, heads, H, D, True)
