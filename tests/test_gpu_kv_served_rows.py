"""Lengths with faults among them: the requests that are served all the same have their attention, whichever tiles the others' rows take."""
import numpy as np
import pytest
import torch

from paper_2410_09687_amd import moin
from tests.gpu_common import ctx
from tests.test_gpu_kv_attention import BF16, F32, I32, Step, compare

pytestmark = pytest.mark.gpu


def planned(s, T, max_new, served):
    """A plan of the step's lengths, but of T tokens and at most max_new a request; `served`: the requests that it serves."""
    table, every = s.table.clone(), -(-(s.kv + s.new) // s.page)
    dealt = []
    for r in range(len(s.kv)):
        have = -(-int(s.kv[r]) // s.page)
        if r in served:
            dealt += table[r, have:int(every[r])].tolist()
        table[r, have:] = -1
    dev = lambda x: torch.tensor(np.asarray(x), dtype=I32).cuda()   # noqa: E731
    plan = moin.KVPlan(ctx())
    off, lens, _, left = plan.build(dev(s.kv), dev(s.new), T, table, dev(dealt[::-1] + [0]), dev([len(dealt)]), n_pages=s.n_pages,
                                    page_tokens=s.page, n_heads=s.heads, n_kv=s.H, max_new=max_new)
    with pytest.raises(moin.MoinError):
        ctx().check()
    assert left.item() == 0
    for r in served:
        assert lens[r].item() == s.kv[r] + s.new[r]
    return plan, table, off


@pytest.mark.parametrize("y_dtype", [BF16, F32])
@pytest.mark.parametrize("heads,H,D", [(8, 1, 64), (16, 2, 128), (3, 1, 256), (40, 1, 64)])
@pytest.mark.parametrize("kv,new,T,max_new,served", [
    ([0, 130], [50, 2], 100, 50, [0, 1]),                 # tokens of no request
    ([0, 130], [98, 2], 100, 50, [1]),                    # a request above the most
    ([700, 3000, 5], [1, 90, 1], 300, 95, [0, 1, 2]),     # keys in parts beside it
    ([200], [1], 100, 1, [0]),                            # no request may have many tokens
    ([64, 0, 9], [1, 1, 1], 60, 1, [0, 1, 2]),
    ([30, 40], [20, 1], 20, 20, [0])])                    # tokens beyond T
def test_requests_beside_a_fault(kv, new, T, max_new, served, heads, H, D, y_dtype):
    s = Step(T + D, kv, new, heads, H, D)
    plan, table, off = planned(s, T, max_new, served)
    q = torch.randn((T, heads, D), device="cuda").to(BF16)
    n = min(T, s.T)
    q[:n] = s.q[:n]
    y = torch.full((T, heads, D), 7.0, dtype=y_dtype, device="cuda")
    _, lse = moin.moin_kv_attention(ctx(), plan, s.pages, q, table, y_dtype=y_dtype, out=y, want_lse=True)
    ctx().check()
    want, first = s.want(), np.concatenate([[0], np.cumsum(s.new)])
    rows = np.concatenate([np.arange(first[r], first[r + 1]) for r in served])
    at = torch.tensor(rows, device="cuda")
    compare(y[at], lse[at], [w[rows] for w in want])
    assert (y[s.T:] == 7.0).all()   # tokens of no request: left as they are
