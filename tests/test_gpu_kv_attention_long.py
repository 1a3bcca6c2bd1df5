"""Attention at the far ends of its range: tiles in as many parts as there are, and caches whose records lie beyond 32 bits of offset."""
import numpy as np
import pytest
import torch

from paper_2410_09687_amd import moin
from tests.gpu_common import ctx
from tests.test_gpu_kv_attention import BF16, F32, I32, Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,new", [(2, 1), (4, 5), (2, 20)])
def test_as_many_parts_as_a_tile_may_have(heads, new):
    """Parts of eight records and more would be 137 and 150; 128 it is, joined in groups."""
    for kv in (70000, 76800):
        s = Step(kv + new, [kv], [new], heads, 1, 64, page=256)
        s.check(F32)


def one_request(pages, table, x, q, heads, H, n, new):
    """Attention of a request with n keys, the last `new` of which the step adds, in the pages that the table names."""
    i32 = lambda *v: torch.tensor(v, dtype=I32, device="cuda")   # noqa: E731
    plan = moin.KVPlan(ctx())
    held = -(-(n - new) // 256)
    given = table.clone()
    given[0, held:] = -1
    stack = table[0, held:].flip(0).contiguous()
    _, _, slots, _ = plan.build(i32(n - new), i32(new), new, given, stack, i32(stack.numel()), n_pages=pages.n_pages, page_tokens=256, n_heads=heads,
                                n_kv=H)
    assert torch.equal(given, table)
    pos = torch.arange(n, device="cuda")
    every = (table[0][pos // 256].long() * 256 + pos % 256).to(I32)
    assert torch.equal(every[n - new:], slots)
    moin.moin_kv_append(ctx(), pages, x[:, 0], x[:, 1], every)
    y, lse = moin.moin_kv_attention(ctx(), plan, pages, q, table, y_dtype=F32, want_lse=True)
    ctx().check()
    return y, lse


@pytest.mark.parametrize("new", [1, 40])
def test_a_cache_beyond_four_gigabytes(new):
    """The same bits as in a small cache."""
    H, D, heads, n = 4, 128, 8, 1000
    n_pages = (9 << 29) // (4 * 8704 * 4)
    big, small = moin.KVPages.empty(n_pages, H, D, 256), moin.KVPages.empty(4, H, D, 256)
    assert big.data.numel() > 2 ** 32
    big.data.fill_(255)
    g = torch.Generator(device="cuda").manual_seed(new)
    x = torch.randn((n, 2, H, D), device="cuda", generator=g).to(BF16)
    q = torch.randn((new, heads, D), device="cuda", generator=g).to(BF16)
    far = torch.tensor([[n_pages - 1, 0, n_pages // 2, n_pages - 2]], dtype=I32, device="cuda")
    near = torch.tensor([[3, 1, 0, 2]], dtype=I32, device="cuda")
    y, lse = one_request(big, far, x, q, heads, H, n, new)
    z, l2 = one_request(small, near, x, q, heads, H, n, new)
    assert torch.equal(y, z) and torch.equal(lse, l2) and np.isfinite(y.cpu().numpy()).all()
