"""What attention keeps of the context's workspace: 32 rows of partial results a part where a tile has no more, 128 a part of the other tiles."""
import pytest
import torch

from paper_2410_09687_amd import moin

pytestmark = pytest.mark.gpu
BF16, I32 = torch.bfloat16, torch.int32


@pytest.mark.parametrize("new,heads,H,D,most", [
    ([1] * 4, 32, 4, 64, 2 * 512 * 32),                        # parts of tiles, rows
    ([2, 1, 3], 64, 8, 128, 2 * 512 * 32),
    ([200, 200], 32, 4, 64, 2 * 512 * (32 + 128)),             # smaller steps may have both kinds
    ([200, 1], 32, 4, 64, 2 * 512 * (32 + 128)),
    ([50, 3], 64, 1, 64, 2 * 512 * 128)])                      # 64 rows and more a token
def test_no_more_than_the_parts_there_can_be(new, heads, H, D, most):
    ctx = moin.Context(0)
    dev = lambda x: torch.tensor(x, dtype=I32).cuda()   # noqa: E731
    try:
        S, T, plan = len(new), sum(new), moin.KVPlan(ctx)
        table = torch.full((S, 4), -1, dtype=I32, device="cuda")
        _, _, slots, _ = plan.build(dev([0] * S), dev(new), T, table, dev(list(range(4 * S))), dev([4 * S]), n_pages=4 * S, page_tokens=64,
                                    n_heads=heads, n_kv=H, max_new=max(new))
        pages = moin.KVPages.empty(4 * S, H, D)
        k = torch.randn((T, H, D), device="cuda").to(BF16)
        moin.moin_kv_append(ctx, pages, k, k, slots)
        moin.moin_kv_attention(ctx, plan, pages, torch.randn((T, heads, D), device="cuda").to(BF16), table)
        ctx.check()
        floats = most * (D + 2)   # (the parts are counted for all kv heads)
        assert ctx.workspace_bytes() <= floats * 4 * 5 // 4 + (1 << 20)   # room to grow, whole megabytes
        plan.close()
    finally:
        torch.cuda.synchronize()
        ctx.close()
