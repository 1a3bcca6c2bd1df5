"""Pages given back by a table that names pages which do not exist: those raise the fault and are not dealt again, the others are."""
import numpy as np
import pytest
import torch

from paper_2410_09687_amd import moin
from tests.gpu_common import ctx

pytestmark = pytest.mark.gpu
I32 = torch.int32


def dev(x):
    return torch.as_tensor(np.asarray(x), dtype=I32).cuda()


def plain(done, kv, table, stack, n, n_pages, page):
    """(kv, table, stack, n) afterwards, request by request."""
    kv, table, stack = list(kv), [list(r) for r in table], list(stack)
    for s, d in enumerate(done):
        if not d:
            continue
        for j in range(min(-(-max(kv[s], 0) // page), len(table[s]))):
            p, table[s][j] = table[s][j], -1
            if 0 <= p < n_pages and n < len(stack):
                stack[n] = p
                n += 1
        kv[s] = 0
    return kv, table, stack, n


def check(done, kv, table, stack, n, n_pages, page=64):
    k, t, f, nf = dev(kv), dev(table), dev(stack), dev([n])
    moin.moin_kv_release(ctx(), dev(done), k, t, f, nf, n_pages=n_pages, page_tokens=page)
    with pytest.raises(moin.MoinError):
        ctx().check()
    got_kv, got_table, got, left = k.cpu().tolist(), t.cpu().tolist(), f.cpu().tolist(), nf.item()
    want_kv, want_table, want, want_left = plain(done, kv, table, stack, n, n_pages, page)
    assert got_kv == want_kv and got_table == want_table and left == want_left and got[:left] == want[:left]
    # above the stack, where pages would lie if all of them existed, may stand anything
    most = n + sum(min(-(-max(x, 0) // page), len(table[0])) for x, d in zip(kv, done) if d)
    assert got[most:] == want[most:]
    return got_kv, got_table, got[:left], left


def test_by_hand():
    # request 0's second page was never there, request 2's last is beyond the cache; request 1 stays
    kv, table, stack, n = check([1, 0, 1], [150, 64, 190], [[4, -1, 7], [5, -1, -1], [0, 1, 12]], [9, 8, -7, -7, -7, -7, -7, -7], 2, 10)
    assert stack == [9, 8, 4, 7, 0, 1] and n == 6 and kv == [0, 64, 0] and table == [[-1] * 3, [5, -1, -1], [-1] * 3]


def test_a_page_that_does_not_exist_takes_no_place_of_one_that_does():
    _, _, stack, n = check([1, 1], [128, 64], [[-1, 3], [2, -1]], [1, -7, -7], 1, 4)
    assert stack == [1, 3, 2] and n == 3


@pytest.mark.parametrize("S,max_pages", [(3, 200), (40, 70), (1500, 9)])
@pytest.mark.parametrize("room", [1.0, 0.5])
def test_many(S, max_pages, room):
    rng = np.random.default_rng(S)
    page, n_pages = 128, 10 ** 6
    kv = rng.integers(0, max_pages * page + 1, S)
    table = rng.integers(0, n_pages, (S, max_pages))
    bad = rng.random((S, max_pages)) < 0.2
    table[bad] = rng.choice([-1, -5, n_pages, 2 ** 31 - 1], size=int(bad.sum()))
    done = rng.integers(0, 2, S)
    done[0], kv[0], table[0, 0] = 1, page, -1
    held = int((-(-kv // page) * done).sum())
    check(done.tolist(), kv.tolist(), table.tolist(), [-7] * (3 + int(held * room)), 3, n_pages, page)
