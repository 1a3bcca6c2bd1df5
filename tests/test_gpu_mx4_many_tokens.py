"""Products with 4-bit weights of more tokens than a launch's second dimension counts tiles."""
import pytest
import torch

from paper_2410_09687_amd import moin
from tests.gpu_common import ctx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [65535 * 64, 65536 * 64 + 1, 2 * 65536 * 64 + 77])
def test_millions_of_tokens(T):
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn((T, 8), device="cuda", generator=g).to(torch.bfloat16)
    W4 = moin.moin_mx4_quantize(ctx(), torch.randn((8, 8), device="cuda", generator=g).to(torch.bfloat16))
    held = moin.moin_mx4_dequantize(ctx(), W4).double()
    y = moin.moin_mx4_linear(ctx(), x, W4, y_dtype=torch.float32)
    ctx().check()
    # eight exact products in fp32 sums
    for lo in range(0, T, 1 << 20):
        part = x[lo:lo + (1 << 20)].double()
        want, spread = part @ held.t().contiguous(), part.abs() @ held.abs().t().contiguous()
        assert ((y[lo:lo + (1 << 20)].double() - want).abs() <= 8 * 2.0 ** -24 * spread).all(), lo
