"""On a 4-bit base as on a bf16 one, an eager call with the largest batch prepares captured calls of batches of no more sequences and tokens,
also where those take row tiles, for which the weight is turned into bf16 in the workspace."""
import pytest
import torch

from paper_2410_09687_amd import moin
from tests.gpu_common import ctx as common
from tests.test_gpu_both_groupings import E, _batch

pytestmark = pytest.mark.gpu


def run(ctx, plan, inp, W4, out=None):
    return moin.moin_lora_linear_mx4_planned(ctx, plan, inp.x, W4, inp.A_stack, inp.B_stack, 2.0, out=out)


@pytest.mark.parametrize("first,then,d_in,d_out,r", [
    ([1] * 700, [325, 325], 8192, 8192, 128),      # gathered / row tiles
    ([10] * 100, [450, 450], 4096, 8192, 64),
    ([64] * 300, [16000], 2048, 264, 8),
    ([100] * 12, [1100], 5632, 2048, 136),
    ([450, 450], [1] * 800, 2048, 8192, 64),       # row tiles / gathered
    ([1100, 900], [700, 500], 2048, 264, 64),      # row tiles both
    ([1] * 300, [1] * 128, 2048, 2048, 128)])      # gathered both
def test_captured_after_the_largest_eager_call(first, then, d_in, d_out, r):
    ctx, other = moin.Context(0), common()
    try:
        for lens in (first, then):
            inp, _, _ = _batch(lens, d_in, d_out, r, False)
            W4 = moin.moin_mx4_quantize(ctx, inp.W)
            plan = moin.Plan(ctx).build(inp.seq_offsets, inp.expert_ids, sum(lens), E)
            if lens is first:
                run(ctx, plan, inp, W4)
                ctx.check()
                size = ctx.workspace_bytes()
                plan.close()
        other_plan = moin.Plan(other).build(inp.seq_offsets, inp.expert_ids, sum(then), E)
        want = run(other, other_plan, inp, W4)
        other.check()
        y = torch.empty_like(want)
        torch.cuda.synchronize()
        print(f"[gpu] captured {len(then)} sequences, {sum(then)} tokens after {sum(first)}, {d_in}->{d_out} r={r}", flush=True)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(ctx, plan, inp, W4, y)
        for _ in range(3):
            y.fill_(float("nan"))
            graph.replay()
            ctx.check()
            assert torch.equal(y.view(torch.int16), want.view(torch.int16))
        assert ctx.workspace_bytes() == size
        del graph
        other_plan.close()
        plan.close()
    finally:
        torch.cuda.synchronize()
        ctx.close()


def test_decode_batches_keep_nothing_for_a_weight():
    """No batch of up to 256 tokens takes row tiles."""
    ctx = moin.Context(0)
    try:
        inp, _, _ = _batch([1] * 256, 2048, 5632, 128, False)
        W4 = moin.moin_mx4_quantize(ctx, inp.W)
        plan = moin.Plan(ctx).build(inp.seq_offsets, inp.expert_ids, 256, E)
        run(ctx, plan, inp, W4)
        ctx.check()
        assert ctx.workspace_bytes() < 2048 * 5632 * 2
        plan.close()
    finally:
        torch.cuda.synchronize()
        ctx.close()
