"""A serving step in eight bits: requests of different topics through one attention layer whose base weights are 8-bit integers and
whose cache is E4M3, with norms of queries and keys and a rotation by position between them.

    python examples/serve_eight_bit.py [--requests 6] [--steps 8]

A step takes whatever tokens the requests bring through
    plans (cache pages, attention, grouping by expert) -> q, k, v (integer base + the expert's adapters) -> norms and rotation -> append ->
    attention -> o,
as examples/serve_four_bit.py does in four bits; its server admits requests and takes their pages back here, too.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import serve_four_bit as four  # noqa: E402
from serve_four_bit import BF16, I32, moin  # noqa: E402


class EightBitAttention:
    """One attention layer: q, k, v and o projections in 8-bit integers, a rank-r adapter (a multiple of 64) of every expert on each."""

    def __init__(self, ctx, d_model, n_heads, n_kv, head_dim, rank, n_experts, generator, device="cuda"):
        self.ctx, self.n_heads, self.n_kv, self.head_dim, self.n_experts, self.scale = ctx, n_heads, n_kv, head_dim, n_experts, 2.0
        q, kv = n_heads * head_dim, n_kv * head_dim
        draw = lambda *s: torch.randn(s, generator=generator, device=device)   # noqa: E731
        self.base, self.adapters = {}, {}
        for name, d_in, d_out in (("qkv", d_model, q + 2 * kv), ("o", q, d_model)):
            self.base[name] = moin.moin_i8_quantize(ctx, (draw(d_out, d_in) * d_in ** -0.5).to(BF16))
            self.adapters[name] = ((draw(n_experts, rank, d_in) * d_in ** -0.5).to(BF16), (draw(n_experts, d_out, rank) * 0.1).to(BF16))
        self.q_gain, self.k_gain = ((1 + 0.2 * draw(head_dim)).to(BF16) for _ in range(2))
        self.freqs = moin.rope_frequencies(head_dim, device=device)

    def project(self, name, plan, x):
        A, B = self.adapters[name]
        return moin.moin_lora_linear_i8_planned(self.ctx, plan, x, self.base[name], A, B, self.scale)

    def __call__(self, plan, kv_plan, pages, table, offsets, slots, positions, x):
        h, g, D = self.n_heads, self.n_kv, self.head_dim
        qkv = self.project("qkv", plan, x).view(-1, h + 2 * g, D)
        q, k = qkv[:, :h], qkv[:, h:h + g]
        moin.moin_qk_norm_rope(self.ctx, q, k, positions=positions, freqs=self.freqs, q_gain=self.q_gain, k_gain=self.k_gain, out=(q, k))
        moin.moin_kv8_append(self.ctx, pages, k, qkv[:, h + g:], offsets, slots)
        y, _ = moin.moin_kv8_attention(self.ctx, kv_plan, pages, q, table)
        return self.project("o", plan, y.view(-1, h * D))


class Server(four.Server):
    """Places for `n_requests` requests, `n_pages` pages of 64 tokens between them, in eight bits."""

    def __init__(self, ctx, layer, centroids, n_requests, n_pages, max_tokens, device="cuda"):
        super().__init__(ctx, layer, centroids, n_requests, n_pages, max_tokens, device)
        self.pages = moin.KV8Pages.empty(n_pages, layer.n_kv, layer.head_dim, device=device)

    def step(self, x, new_lens):
        """x: the new tokens of all requests, one request after the other; new_lens: how many each brings (a list)."""
        before, T = self.lens, x.shape[0]
        new = torch.tensor(new_lens, dtype=I32, device=x.device)
        offsets, self.lens, slots, self.n_free = self.kv_plan.build(
            before, new, T, self.table, self.free, self.n_free, n_pages=self.pages.n_pages, page_tokens=64,
            n_heads=self.layer.n_heads, n_kv=self.layer.n_kv, max_new=max(new_lens))
        positions = torch.arange(T, dtype=I32, device=x.device) + torch.repeat_interleave(before - offsets[:-1], new, output_size=T)
        self.plan.build(offsets, self.experts, T, self.layer.n_experts)
        return self.layer(self.plan, self.kv_plan, self.pages, self.table, offsets, slots, positions, x), offsets


def main(n_requests=6, steps=8, d_model=512, n_heads=8, n_kv=2, head_dim=64, rank=64, n_experts=8, prompt=150, seed=0):
    ctx = moin.Context(0)
    g = torch.Generator(device="cuda").manual_seed(seed)
    layer = EightBitAttention(ctx, d_model, n_heads, n_kv, head_dim, rank, n_experts, g)
    centroids = torch.randn((n_experts, 64), generator=g, device="cuda")
    server = Server(ctx, layer, centroids, n_requests, n_pages=n_requests * 8, max_tokens=512)
    topics = torch.arange(n_requests, device="cuda") % n_experts
    server.admit(slice(None), centroids[topics] + 0.1 * torch.randn((n_requests, 64), generator=g, device="cuda"))
    lens = [max(1, prompt - 37 * i % prompt) for i in range(n_requests)]
    for step in range(steps):
        if step == steps // 2:    # every other request ends half way and a new one takes its place
            done = [i % 2 for i in range(n_requests)]
            server.finish(done)
            places = torch.tensor(done, device="cuda").nonzero()[:, 0]
            server.admit(places, centroids[(topics[places] + 3) % n_experts])
            lens = [33 if d else 1 for d in done]
        x = torch.randn((sum(lens), d_model), generator=g, device="cuda").to(BF16)
        y, _ = server.step(x, lens)
        ctx.check()
        print(f"step {step}: {x.shape[0]} tokens, keys {server.lens.tolist()}, pages free {int(server.n_free)}, rms {float(y.float().square().mean().sqrt()):.4f}",
              flush=True)
        lens = [1] * n_requests
    server.finish([1] * n_requests)
    ctx.check()
    assert int(server.n_free) == server.pages.n_pages
    ctx.close()


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--requests", type=int, default=6)
    a.add_argument("--steps", type=int, default=8)
    args = a.parse_args()
    main(args.requests, args.steps)
