"""Tiles of many rows listed by the keys that they see, beside requests whose lengths are at the ends of int32: those get nothing, the others keep
every bit."""
import numpy as np
import pytest
import torch

from paper_2410_09687_amd import moin
from tests import test_gpu_kv8_attention as eight
from tests import test_gpu_kv_attention as four
from tests.gpu_common import ctx

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
TOP = 2 ** 31 - 1


def dev(x):
    return torch.tensor(np.asarray(x), dtype=I32).cuda()


def attention(s, attend, lens, y_dtype):
    """y, lse and offsets of the step with `lens` {request: length} in place of its own, for requests that are then not served."""
    table, every, dealt, kv = s.table.clone(), -(-(s.kv + s.new) // s.page), [], s.kv.copy()
    for r in range(len(s.kv)):
        have = -(-int(s.kv[r]) // s.page)
        if r not in lens:
            dealt += table[r, have:int(every[r])].tolist()
        table[r, have:] = -1
    for r, n in lens.items():
        kv[r] = n
    plan = moin.KVPlan(ctx())
    off, after, slots, left = plan.build(dev(kv), dev(s.new), s.T, table, dev(dealt[::-1] + [0]), dev([len(dealt)]), n_pages=s.n_pages,
                                         page_tokens=s.page, n_heads=s.heads, n_kv=s.H, max_new=int(s.new.max()))
    with pytest.raises(moin.MoinError):
        ctx().check()
    assert left.item() == 0 and after.tolist() == [max(int(kv[r]), 0) if r in lens else int(kv[r] + s.new[r]) for r in range(len(kv))]
    y = torch.full((s.T, s.heads, s.D), 7.0, dtype=y_dtype, device="cuda")
    _, lse = attend(ctx(), plan, s.pages, s.q, table, y_dtype=y_dtype, out=y, want_lse=True)
    ctx().check()
    plan.close()
    return y, lse, off.tolist(), slots


@pytest.mark.parametrize("y_dtype", [BF16, F32])
@pytest.mark.parametrize("module,attend", [(four, moin.moin_kv_attention), (eight, moin.moin_kv8_attention)])
@pytest.mark.parametrize("kv,new,heads,H,D,bad", [
    ([0, 0], [100, 100], 8, 1, 64, [0]),                                  # the first of two
    ([0, 0], [100, 100], 8, 1, 64, [1]),                                  # the last
    ([0, 130, 64, 700, 1], [150, 300, 9, 40, 257], 16, 2, 128, [2, 4]),   # among prompts and chunks
    ([5, 0, 300], [90, 20, 130], 3, 1, 256, [1]),
    ([(37 * s) % 500 for s in range(64)], [9 + s % 50 for s in range(64)], 8, 2, 64, [0, 31, 63])])
def test_lengths_near_the_largest(kv, new, heads, H, D, bad, module, attend, y_dtype):
    s = module.Step(len(kv) + D, kv, new, heads, H, D)
    first = np.concatenate([[0], np.cumsum(s.new)])
    rows = np.concatenate([np.arange(first[r], first[r + 1]) for r in range(len(kv)) if r not in bad])
    at = torch.tensor(rows, device="cuda")
    want_y, want_lse, off, slots = attention(s, attend, {r: -1 for r in bad}, y_dtype)
    assert off == first.tolist()
    four.compare(want_y[at], want_lse[at], [w[rows] for w in s.want()])
    for r in bad:
        assert not want_y[first[r]:first[r + 1]].any() and torch.isneginf(want_lse[first[r]:first[r + 1]]).all()
    for lens in ([TOP] * len(bad), [TOP - int(s.new[r]) // 2 for r in bad], [-TOP - 1] * len(bad), [TOP - 7 * i for i in range(len(bad))]):
        print(f"[gpu] lengths {lens} of requests {bad}", flush=True)
        y, lse, _, z = attention(s, attend, dict(zip(bad, lens)), y_dtype)
        assert torch.equal(y, want_y) and torch.equal(lse, want_lse) and torch.equal(z, slots)
