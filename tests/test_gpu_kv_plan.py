"""Block tables, slot maps and offsets of a step, and pages given back, against a plain walk over the requests."""
import numpy as np
import pytest
import torch

import tests.four_bit as fb
from paper_2410_09687_amd import moin
from tests.gpu_common import ctx

pytestmark = pytest.mark.gpu
I32 = torch.int32


def dev(x):
    return torch.as_tensor(np.asarray(x), dtype=I32).cuda()


def random_step(rng, S, page, max_pages, kv_hi, new_lo, new_hi, spare):
    kv = rng.integers(0, kv_hi + 1, S)
    new = rng.integers(new_lo, new_hi + 1, S)
    have, every = -(-kv // page), -(-(kv + new) // page)
    n_pages = int(every.sum()) + 5
    order = rng.permutation(n_pages)
    table = np.full((S, max_pages), -1)
    at = 0
    for s in range(S):
        table[s, :have[s]] = order[at:at + have[s]]
        at += have[s]
    free = order[at:]
    n_free = max(0, min(len(free), int((every - have).sum()) + spare))
    return kv, new, table, free, n_free, n_pages


def run(kv, new, T, max_new, page, table, free, n_free, n_pages, in_place=False, heads=8, n_kv=2):
    plan = moin.KVPlan(ctx())
    t, k, nf = dev(table), dev(kv), dev([n_free])
    S = len(kv)
    out = None
    if in_place:
        out = (torch.empty(S + 1, dtype=I32, device="cuda"), k, torch.empty(T, dtype=I32, device="cuda"), nf)
    off, lens, slots, left = plan.build(k, dev(new), T, t, dev(free), nf, n_pages=n_pages, page_tokens=page, n_heads=heads, n_kv=n_kv,
                                        max_new=max_new, out=out)
    return plan, [x.cpu().tolist() for x in (t, lens, off, slots, left)]


def check(got, want):
    table, lens, off, slots, n_free, fault = want
    assert got[1] == lens and got[2] == off and got[3] == slots and got[4] == [n_free]
    assert got[0] == table
    if fault:
        with pytest.raises(moin.MoinError):
            ctx().check()
    else:
        ctx().check()


@pytest.mark.parametrize("page", [64, 128, 256])
@pytest.mark.parametrize("S,kv_hi,new_lo,new_hi", [(1, 0, 1, 1), (1, 500, 0, 0), (5, 200, 1, 1), (64, 700, 0, 8), (64, 700, 0, 9), (3, 0, 2049, 6000),
                                                   (1023, 300, 1, 1), (1025, 200, 0, 3), (2500, 130, 0, 60)])
def test_steps(page, S, kv_hi, new_lo, new_hi):
    rng = np.random.default_rng(S * 7 + page)
    kv, new, table, free, n_free, n_pages = random_step(rng, S, page, (kv_hi + new_hi) // page + 2, kv_hi, new_lo, new_hi, 2)
    T = int(new.sum())
    want = fb.plan(kv, new, T, max(new_hi, 1), page, table, free, n_free)
    for in_place in (False, True):
        check(run(kv, new, T, max(new_hi, 1), page, table, free, n_free, n_pages, in_place)[1], want)


@pytest.mark.parametrize("new_hi", [1, 300])
@pytest.mark.parametrize("S", [7, 1500])
def test_too_few_pages_serve_a_prefix_and_those_that_need_none(S, new_hi):
    rng = np.random.default_rng(S + new_hi)
    kv, new, table, free, n_free, n_pages = random_step(rng, S, 64, 12, 380, 0, new_hi, 0)
    new[0] = max(new[0], 1)
    lack = int((-(-(kv + new) // 64) - -(-kv // 64)).sum())
    want = fb.plan(kv, new, int(new.sum()), new_hi, 64, table, free, lack // 2)
    got = run(kv, new, int(new.sum()), new_hi, 64, table, free, lack // 2, n_pages)[1]
    check(got, want)


@pytest.mark.parametrize("case", ["negative length", "negative new", "row too short", "above max_new", "sum above T", "sum below T", "n_free above"])
def test_faults_in_the_data_serve_the_others(case):
    kv, new, page = [100, 70, 5, 0], [3, 1, 60, 2], 64
    table = [[0, 1, -1], [2, 3, -1], [4, -1, -1], [-1, -1, -1]]
    free, n_free, T, max_new = [5, 6, 7, 8], 4, 66, 100
    if case == "negative length":
        kv[1] = -3
    elif case == "negative new":
        new[2], T = -60, 6
    elif case == "row too short":
        new[0], T = 100, 163
    elif case == "above max_new":
        max_new = 50
    elif case == "sum above T":
        T = 60
    elif case == "sum below T":
        T = 70
    elif case == "n_free above":
        n_free = 9
    want = fb.plan(kv, new, T, max_new, page, table, free, n_free)
    assert want[5]
    check(run(kv, new, T, max_new, page, table, free, n_free, 9)[1], want)


def test_pages_that_do_not_exist_give_no_slots():
    plan, got = run([0, 64], [2, 1], 3, 2, 64, [[-1, -1], [50, -1]], [3, 99], 2, 10)
    assert got[3][2] == 3 * 64 and got[3][:2] == [-1, -1]     # the first page dealt is 99
    with pytest.raises(moin.MoinError):
        ctx().check()


@pytest.mark.parametrize("S", [1, 9, 1300])
def test_release(S):
    rng = np.random.default_rng(S)
    kv, new, table, free, _, n_pages = random_step(rng, S, 128, 9, 1000, 0, 0, 0)
    done = rng.integers(0, 2, S)
    done[0] = 1
    stack = np.full(n_pages, -7)
    n = min(3, len(free))
    stack[:n] = free[:n]
    k, t, f, nf = dev(kv), dev(table), dev(stack), dev([n])
    moin.moin_kv_release(ctx(), dev(done), k, t, f, nf, n_pages=n_pages, page_tokens=128)
    ctx().check()
    want = list(stack)
    for s in range(S):
        if done[s]:
            for j in range(-(-kv[s] // 128)):
                want[n] = table[s][j]
                table[s][j] = -1
                n += 1
            kv[s] = 0
    assert f.cpu().tolist() == want and nf.item() == n and k.cpu().tolist() == kv.tolist() and t.cpu().tolist() == table.tolist()


def test_release_beyond_the_stack_is_a_fault():
    k, t, f, nf = dev([100, 10]), dev([[1, 2], [3, -1]]), dev([9, -1]), dev([1])
    moin.moin_kv_release(ctx(), dev([1, 1]), k, t, f, nf, n_pages=10, page_tokens=64)
    with pytest.raises(moin.MoinError):
        ctx().check()
    assert nf.item() == 2 and f.cpu().tolist() == [9, 1]


def test_a_captured_step_replays():
    rng = np.random.default_rng(4)
    kv, new, table, free, n_free, n_pages = random_step(rng, 40, 64, 40, 600, 1, 1, 40)
    k, n, t, f, nf = dev(kv), dev(new), dev(table), dev(free), dev([n_free])
    off, slots = torch.empty(41, dtype=I32, device="cuda"), torch.empty(40, dtype=I32, device="cuda")
    plan = moin.KVPlan(ctx())

    def step():
        plan.build(k, n, 40, t, f, nf, n_pages=n_pages, page_tokens=64, n_heads=8, n_kv=2, max_new=1, out=(off, k, slots, nf))

    fresh = moin.KVPlan(ctx())
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            with pytest.raises(moin.MoinError) as e:   # its buffer would have to grow
                fresh.build(k, n, 40, t, f, nf, n_pages=n_pages, page_tokens=64, n_heads=8, n_kv=2, max_new=1, out=(off, k, slots, nf))
            assert e.value.code == -6
            torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    step()
    want = fb.plan(kv, new, 40, 1, 64, table, free, n_free)
    assert k.cpu().tolist() == want[1] and slots.cpu().tolist() == want[3]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(5):   # lengths and free pages move on by themselves
        prev = want
        want = fb.plan(prev[1], new, 40, 1, 64, prev[0], free, prev[4])
        g.replay()
        torch.cuda.synchronize()
        assert k.cpu().tolist() == want[1] and slots.cpu().tolist() == want[3] and nf.item() == want[4] and t.cpu().tolist() == want[0]
    ctx().check()


def test_refusals():
    plan = moin.KVPlan(ctx())
    ok = dict(n_pages=8, page_tokens=64, n_heads=8, n_kv=2, max_new=1)

    def build(S=2, T=2, kv=None, new=None, table=None, free=None, nf=None, **kw):
        return plan.build(dev([0] * S) if kv is None else kv, dev([1] * S) if new is None else new, T,
                          dev([[-1]] * S) if table is None else table, dev([0, 1]) if free is None else free,
                          dev([2]) if nf is None else nf, **{**ok, **kw})

    build()
    ctx().check()
    for kw in (dict(page_tokens=32), dict(page_tokens=96), dict(n_heads=7), dict(n_heads=0), dict(n_kv=0), dict(n_pages=0), dict(max_new=-1),
               dict(n_pages=1 << 30)):
        with pytest.raises(moin.MoinError) as e:
            build(**kw)
        assert e.value.code == -1
    for kw in (dict(new=dev([1])), dict(table=dev([[-1]])), dict(nf=dev([1, 2])), dict(kv=torch.zeros(2, dtype=I32)), dict(T=-1)):
        with pytest.raises(ValueError):
            build(**kw)
    with pytest.raises(TypeError):
        build(kv=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        build(table=torch.zeros((2, 4), dtype=I32, device="cuda")[:, ::2])
    empty = torch.empty(0, dtype=I32, device="cuda")
    plan.build(empty, empty, 0, torch.empty((0, 3), dtype=I32, device="cuda"), empty, dev([0]), **ok)
    with pytest.raises(moin.MoinError):
        plan.build(empty, empty, 1, torch.empty((0, 3), dtype=I32, device="cuda"), empty, dev([0]), **ok)
    ctx().check()
