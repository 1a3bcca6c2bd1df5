"""One of a layer's two stacks of adapters without the other is refused, by every call that takes both: its result would be the base's alone."""
import pytest
import torch

from paper_2410_09687_amd import moin
from tests.gpu_common import ctx

pytestmark = pytest.mark.gpu
BF16, I32 = torch.bfloat16, torch.int32
T, D_IN, D_OUT, R, E = 12, 512, 64, 64, 3


@pytest.mark.parametrize("name", ["linear", "planned", "shared", "mx", "mx_planned", "mx4_planned", "i8_planned"])
def test_both_or_none(name):
    g = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda *s: torch.randn(s, generator=g, device="cuda").to(BF16)   # noqa: E731
    x, W, A, B = draw(T, D_IN), draw(D_OUT, D_IN), draw(E, R, D_IN), draw(E, D_OUT, R)
    off, ids = torch.arange(T + 1, dtype=I32, device="cuda"), torch.arange(T, dtype=I32, device="cuda") % E
    plan = moin.Plan(ctx()).build(off, ids, T, E)
    of = lambda A: ids if A is not None else torch.full_like(ids, -1)   # noqa: E731   (without stacks there is no expert to name)
    call = {
        "linear": lambda A, B: moin.moin_lora_linear(ctx(), x, off, of(A), W, A, B, 2.0),
        "planned": lambda A, B: moin.moin_lora_linear_planned(ctx(), plan, x, W, A, B, 2.0),
        "shared": lambda A, B: moin.moin_lora_linear_planned_shared(ctx(), plan, x, [W], [A], [B], 2.0)[0],
        "mx": lambda A, B: moin.moin_lora_linear_mx(ctx(), x, off, of(A), *moin.moin_mx_quantize(ctx(), W, blocked=True), A, B, 2.0),
        "mx_planned": lambda A, B: moin.moin_lora_linear_mx_planned(ctx(), plan, x, *moin.moin_mx_quantize(ctx(), W, blocked=True), A, B, 2.0),
        "mx4_planned": lambda A, B: moin.moin_lora_linear_mx4_planned(ctx(), plan, x, moin.moin_mx4_quantize(ctx(), W), A, B, 2.0),
        "i8_planned": lambda A, B: moin.moin_lora_linear_i8_planned(ctx(), plan, x, moin.moin_i8_quantize(ctx(), W), A, B, 2.0),
    }[name]
    both, none = call(A, B), call(None, None)
    assert not torch.equal(both, none)
    for pair in ((A, None), (None, B)):
        with pytest.raises(ValueError):
            call(*pair)
    assert torch.equal(call(A, B), both)
    ctx().check()
    plan.close()
