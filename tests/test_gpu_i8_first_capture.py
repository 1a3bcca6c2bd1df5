"""Few tokens that the integer product quantises itself take no memory from the workspace: a first call may be a captured one, and the workspace stays
free to grow."""
import pytest
import torch

from paper_2410_09687_amd import moin
from tests.gpu_common import ctx
from tests.test_gpu_i8 import BF16, I32, Product

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("planned", [False, True])
@pytest.mark.parametrize("T,d_in,d_out", [(1, 2048, 264), (16, 264, 72), (5, 2048, 5632)])
def test_a_first_call_is_captured(T, d_in, d_out, planned):
    own = moin.Context(0)
    try:
        p = Product(T, T, d_in, d_out)
        want, other = moin.moin_i8_linear(ctx(), p.x, p.w8), p.x.flip(0).contiguous()
        plan = moin.Plan(own).build(torch.tensor([0, T], dtype=I32, device="cuda"), torch.full((1,), -1, dtype=I32, device="cuda"), T, 0)
        y, before = torch.empty((T, d_out), dtype=BF16, device="cuda"), moin.load().moin_workspace_bytes(own._h)

        def call():
            if planned:
                moin.moin_lora_linear_i8_planned(own, plan, p.x, p.w8, None, None, 1.0, out=y)
            else:
                moin.moin_i8_linear(own, p.x, p.w8, out=y)

        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        assert moin.load().moin_workspace_bytes(own._h) == before
        for _ in range(3):
            y.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want)
            assert torch.equal(moin.moin_i8_linear(own, other, p.w8), want.flip(0))
        big = Product(3, 300, d_in, d_out)      # (the workspace grows beside the graph)
        assert torch.equal(moin.moin_i8_linear(own, big.x, big.w8), moin.moin_i8_linear(ctx(), big.x, big.w8))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        del graph
        plan.close()
    finally:
        torch.cuda.synchronize()
        own.close()
