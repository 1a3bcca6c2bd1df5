"""A step without requests: its outputs are those of a step that changes nothing."""
import pytest
import torch

from paper_2410_09687_amd import moin
from tests.gpu_common import ctx

pytestmark = pytest.mark.gpu
I32 = torch.int32


def dev(*x):
    return torch.tensor(x, dtype=I32, device="cuda")


def build(plan, free, n_free, out=None):
    empty = torch.empty(0, dtype=I32, device="cuda")
    return plan.build(empty, empty, 0, torch.empty((0, 3), dtype=I32, device="cuda"), free, n_free, n_pages=8, page_tokens=64, n_heads=8, n_kv=2,
                      out=out)


def test_the_free_pages_and_the_offsets_are_written():
    plan, free = moin.KVPlan(ctx()), dev(4, 5, 6)
    empty = torch.empty(0, dtype=I32, device="cuda")
    for _ in range(3):
        out = (dev(-7), empty, empty, dev(-7))
        off, lens, slots, n_free = build(plan, free, dev(2), out)
        ctx().check()
        assert off.tolist() == [0] and n_free.tolist() == [2] and lens.numel() == slots.numel() == 0
        off, _, _, n_free = build(plan, free, dev(2))   # outputs of its own
        ctx().check()
        assert off.tolist() == [0] and n_free.tolist() == [2]
    same = dev(3)   # in place
    build(plan, free, same, (dev(-7), empty, empty, same))
    ctx().check()
    assert same.item() == 3


@pytest.mark.parametrize("n_free,want", [(-2, 0), (9, 3)])
def test_a_stack_of_another_height_than_its_room_is_a_fault(n_free, want):
    off, _, _, left = build(moin.KVPlan(ctx()), dev(4, 5, 6), dev(n_free))
    with pytest.raises(moin.MoinError):
        ctx().check()
    assert off.tolist() == [0] and left.tolist() == [want]


def test_captured():
    plan, free, n_free = moin.KVPlan(ctx()), dev(4, 5, 6), dev(1)
    empty = torch.empty(0, dtype=I32, device="cuda")
    out = (dev(-7), empty, empty, dev(-7))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        build(plan, free, n_free, out)
    for i in range(3):
        out[0].fill_(-7)
        n_free.fill_(i)
        g.replay()
        torch.cuda.synchronize()
        assert out[0].tolist() == [0] and out[3].tolist() == [i]
    ctx().check()


def test_an_idle_step_between_others_deals_the_same_pages():
    plan = moin.KVPlan(ctx())
    free, n_free = dev(4, 5, 6), dev(3)
    _, _, _, n_free = build(plan, free, n_free)
    table = torch.full((1, 2), -1, dtype=I32, device="cuda")
    _, lens, slots, left = plan.build(dev(0), dev(2), 2, table, free, n_free, n_pages=8, page_tokens=64, n_heads=8, n_kv=2)
    ctx().check()
    assert table.tolist() == [[6, -1]] and slots.tolist() == [384, 385] and lens.tolist() == [2] and left.tolist() == [2]
