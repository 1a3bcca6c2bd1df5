"""Appends of more requests and heads than a launch of workgroups takes: blocks that lie in the second and later launches."""
import numpy as np
import pytest
import torch

from paper_2410_09687_amd import moin
from tests.gpu_common import ctx

pytestmark = pytest.mark.gpu
BF16, I32 = torch.bfloat16, torch.int32
H, D = 64, 64


def dev(x):
    return torch.tensor(np.asarray(x), dtype=I32).cuda()


# 2^23 workgroups a launch, two for each place and head: 65536 places, of which the requests' first blocks take one each.
@pytest.mark.parametrize("S,new", [(65536 + 3, {0: 1, 7: 200, 65535: 70, 65536: 3, 65537: 130, 65538: 1}), (65536, {3: 300, 65535: 129}), (131072 + 1, {131072: 400})])
def test_blocks_beyond_the_first_launch(S, new):
    lens = np.zeros(S, dtype=np.int64)
    for s, n in new.items():
        lens[s] = n
    T, pages = int(lens.sum()), sum(-(-n // 64) + 1 for n in new.values())
    g = torch.Generator(device="cuda").manual_seed(S)
    k, v = (torch.randn((T, H, D), generator=g, device="cuda").to(BF16) for _ in range(2))
    order, slots, at = np.random.default_rng(S).permutation(pages), [], 0
    for s, n in sorted(new.items()):        # each from place 50 of a page on
        page = order[at:at + (50 + n + 63) // 64]
        at += len(page)
        pos = 50 + np.arange(n)
        slots += (page[pos // 64] * 64 + pos % 64).tolist()
    big, small = (moin.KV8Pages.empty(pages, H, D) for _ in range(2))
    for pages8 in (big, small):             # (the places before them hold tokens of zeros, of the smallest scale)
        pages8.data.zero_()
    moin.moin_kv8_append(ctx(), big, k, v, dev(np.concatenate([[0], np.cumsum(lens)])), dev(slots))
    off = dev(np.concatenate([[0], np.cumsum([n for _, n in sorted(new.items())])]))
    moin.moin_kv8_append(ctx(), small, k, v, off, dev(slots))
    ctx().check()
    assert torch.equal(big.data, small.data)
    # (a code is off by at most 2^-4 of its value, less below the normal ones)
    for got, x in zip(moin.moin_kv8_gather(ctx(), big, dev(slots)), (k, v)):
        assert float((got - x).float().abs().max()) <= 2.0 ** -4 * float(x.float().abs().max())
