"""A serving step in four bits: requests of different topics through one attention layer whose base weights and cache are MXFP4.

    python examples/serve_four_bit.py [--requests 6] [--steps 8]

Each request is routed to its expert by its prompt's embedding.  A step then takes whatever tokens the requests bring (whole prompts, one
token each, nothing from those that wait) through
    plans (cache pages, attention, grouping by expert) -> q, k, v (4-bit base + the expert's adapters) -> append -> attention -> o,
and requests that are done give their pages back.  Everything of a step stays on the device; sizes are the only thing the host knows.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2410_09687_amd import moin  # noqa: E402

BF16, I32 = torch.bfloat16, torch.int32


class FourBitAttention:
    """One attention layer: q, k, v and o projections in MXFP4, a rank-r adapter of every expert on each."""

    def __init__(self, ctx, d_model, n_heads, n_kv, head_dim, rank, n_experts, generator, device="cuda"):
        self.ctx, self.n_heads, self.n_kv, self.head_dim, self.n_experts, self.scale = ctx, n_heads, n_kv, head_dim, n_experts, 2.0
        q, kv = n_heads * head_dim, n_kv * head_dim
        draw = lambda *s: torch.randn(s, generator=generator, device=device)   # noqa: E731
        self.base, self.adapters = {}, {}
        for name, d_in, d_out in (("qkv", d_model, q + 2 * kv), ("o", q, d_model)):
            W = (draw(d_out, d_in) * d_in ** -0.5).to(BF16)
            self.base[name] = moin.moin_mx4_quantize(ctx, W)
            self.adapters[name] = ((draw(n_experts, rank, d_in) * d_in ** -0.5).to(BF16), (draw(n_experts, d_out, rank) * 0.1).to(BF16))

    def project(self, name, plan, x):
        A, B = self.adapters[name]
        return moin.moin_lora_linear_mx4_planned(self.ctx, plan, x, self.base[name], A, B, self.scale)

    def __call__(self, plan, kv_plan, pages, table, slots, x):
        h, g, D = self.n_heads, self.n_kv, self.head_dim
        qkv = self.project("qkv", plan, x).view(-1, h + 2 * g, D)
        moin.moin_kv_append(self.ctx, pages, qkv[:, h:h + g], qkv[:, h + g:], slots)
        y, _ = moin.moin_kv_attention(self.ctx, kv_plan, pages, qkv[:, :h], table)
        return self.project("o", plan, y.view(-1, h * D))


class Server:
    """Places for `n_requests` requests, `n_pages` pages of 64 tokens between them."""

    def __init__(self, ctx, layer, centroids, n_requests, n_pages, max_tokens, device="cuda"):
        self.ctx, self.layer, self.centroids = ctx, layer, centroids
        self.pages = moin.KVPages.empty(n_pages, layer.n_kv, layer.head_dim)
        self.lens = torch.zeros(n_requests, dtype=I32, device=device)
        self.table = torch.full((n_requests, -(-max_tokens // 64)), -1, dtype=I32, device=device)
        self.free = torch.arange(n_pages, dtype=I32, device=device)
        self.n_free = torch.tensor([n_pages], dtype=I32, device=device)
        self.experts = torch.zeros(n_requests, dtype=I32, device=device)
        self.kv_plan, self.plan = moin.KVPlan(ctx), moin.Plan(ctx)

    def admit(self, places, embeddings):
        """New requests in `places`, each to the expert of the topic nearest its embedding."""
        experts, _, _ = moin.moin_route(self.ctx, embeddings, self.centroids)
        self.experts[places] = experts

    def step(self, x, new_lens):
        """x: the new tokens of all requests, one request after the other; new_lens: how many each brings (a list)."""
        new = torch.tensor(new_lens, dtype=I32, device=x.device)
        offsets, self.lens, slots, self.n_free = self.kv_plan.build(
            self.lens, new, x.shape[0], self.table, self.free, self.n_free, n_pages=self.pages.n_pages, page_tokens=64,
            n_heads=self.layer.n_heads, n_kv=self.layer.n_kv, max_new=max(new_lens))
        self.plan.build(offsets, self.experts, x.shape[0], self.layer.n_experts)
        return self.layer(self.plan, self.kv_plan, self.pages, self.table, slots, x), offsets

    def finish(self, done):
        """Requests with done[i] != 0 give back their pages."""
        moin.moin_kv_release(self.ctx, torch.tensor(done, dtype=I32, device=self.lens.device), self.lens, self.table, self.free, self.n_free,
                             n_pages=self.pages.n_pages, page_tokens=64)


def main(n_requests=6, steps=8, d_model=512, n_heads=8, n_kv=2, head_dim=64, rank=16, n_experts=8, prompt=150, seed=0):
    ctx = moin.Context(0)
    g = torch.Generator(device="cuda").manual_seed(seed)
    layer = FourBitAttention(ctx, d_model, n_heads, n_kv, head_dim, rank, n_experts, g)
    centroids = torch.randn((n_experts, 64), generator=g, device="cuda")
    server = Server(ctx, layer, centroids, n_requests, n_pages=n_requests * 8, max_tokens=512)
    topics = torch.arange(n_requests, device="cuda") % n_experts
    server.admit(slice(None), centroids[topics] + 0.1 * torch.randn((n_requests, 64), generator=g, device="cuda"))
    # prompts of different lengths, then a token a step; every other request ends half way and a new one takes its place
    lens = [max(1, prompt - 37 * i % prompt) for i in range(n_requests)]
    for step in range(steps):
        if step == steps // 2:
            done = [i % 2 for i in range(n_requests)]
            server.finish(done)
            places = torch.tensor(done, device="cuda").nonzero()[:, 0]
            server.admit(places, centroids[(topics[places] + 3) % n_experts])
            lens = [33 if d else 1 for d in done]
        x = torch.randn((sum(lens), d_model), generator=g, device="cuda").to(BF16)
        y, offsets = server.step(x, lens)
        ctx.check()
        print(f"step {step}: {x.shape[0]} tokens, keys {server.lens.tolist()}, pages free {int(server.n_free)}, rms {float(y.float().square().mean().sqrt()):.4f}",
              flush=True)
        lens = [1] * n_requests
    server.finish([1] * n_requests)
    ctx.check()
    assert int(server.n_free) == server.pages.n_pages and torch.equal(server.free.sort().values, torch.arange(server.pages.n_pages, device="cuda", dtype=I32))
    ctx.close()


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--requests", type=int, default=6)
    a.add_argument("--steps", type=int, default=8)
    args = a.parse_args()
    main(args.requests, args.steps)
