"""Few tokens through integer weights of many outputs: each grouping of outputs and tokens that the launch chooses from, with outputs that end inside
a group.  Sums are exact; they and the two products with the scales are rounded to fp32 (2^-22 in all), a bf16 result by 2^-8 of itself."""
import pytest
import torch

from paper_2410_09687_amd import moin
from tests.gpu_common import ctx
from tests.test_gpu_i8 import BF16, F32, Product

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d_in", [264, 1000])
@pytest.mark.parametrize("d_out", [5128, 6152, 16392, 16448])
def test_groups_of_outputs(d_in, d_out):
    p = Product(d_in, 128, d_in, d_out)
    x = p.x
    for T in (1, 8, 16, 17, 24, 32, 33, 64, 65, 100, 128):
        p.x = x[128 - T:].contiguous()      # (of each count other tokens)
        for y_dtype in (BF16, F32):
            print(f"[gpu] {T} tokens {d_in} -> {d_out}", flush=True)
            guard = torch.full((T + 1, d_out), 3.0, dtype=y_dtype, device="cuda")
            p.check(moin.moin_i8_linear(ctx(), p.x, p.w8, y_dtype=y_dtype, out=guard[:T]))
            assert bool((guard[T] == 3.0).all())


@pytest.mark.parametrize("T,d_in,d_out", [(16, 2056, 16392), (13, 4104, 5128), (3, 20000, 16392), (24, 8200, 16392), (16, 3000, 40)])
def test_deep_ones_quantised_ahead(T, d_in, d_out):
    p = Product(T, T, d_in, d_out)
    for y_dtype in (BF16, F32):
        p.check(moin.moin_i8_linear(ctx(), p.x, p.w8, y_dtype=y_dtype))


@pytest.mark.parametrize("T,d_in,d_out", [(129, 1000, 264), (1000, 1024, 256), (300, 264, 1000)])
def test_groups_of_tokens(T, d_in, d_out):
    p = Product(T, T, d_in, d_out)
    for y_dtype in (BF16, F32):
        p.check(moin.moin_i8_linear(ctx(), p.x, p.w8, y_dtype=y_dtype))
