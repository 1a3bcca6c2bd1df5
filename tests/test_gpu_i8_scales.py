"""Integer products of rows and channels of any magnitude: a scale of a token times one of a channel may leave fp32's range on either side where the
result does not, and so may a sum times one of them.

The result is the sum rounded to fp32 and two products rounded: 2^-22 of it, and 2^-8 for bf16.  Results of less than 2^-120 come near the subnormal
numbers, where bits are lost: held to be that small.  Beyond the largest number a result is infinite."""
import numpy as np
import pytest
import torch

import tests.eight_bit as eb
from paper_2410_09687_amd import moin
from tests.gpu_common import ctx

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def f64(t):
    return t.detach().cpu().double().numpy()


def rows(rng, n, cols, powers, half):
    """Rows of magnitudes 2^powers in turn; every third one has zeros in its first (half = 0) or second half of the columns."""
    x = rng.normal(size=(n, cols)) * np.ldexp(1.0, np.resize(powers, n))[:, None]
    x[::3, half * (cols // 2):(half + 1) * (cols // 2)] = 0
    return torch.tensor(x).to(BF16).cuda()


# Few tokens that the product quantises itself, that a launch ahead does; tiles of 128 x 128, in parts of the contraction, of 256 x 256; the planned call on
# tiles of either size (no sequence has an adapter).
@pytest.mark.parametrize("T,d_in,d_out,planned", [(7, 264, 264, 0), (40, 520, 264, 0), (300, 520, 4104, 0), (100, 4096, 72, 0), (9000, 384, 8200, 0), (60, 512, 264, 1), (900, 512, 264, 1),
                                                  (16000, 256, 4104, 16)])
@pytest.mark.parametrize("y_dtype", [BF16, F32])
def test_any_magnitudes(T, d_in, d_out, planned, y_dtype):
    rng = np.random.default_rng(T)
    x = rows(rng, T, d_in, [0, -112, 118, 60, -60, 100, 97], 1)
    W = rows(rng, d_out, d_in, [0, -115, 118, -70, 40], 0)
    w8 = moin.moin_i8_quantize(ctx(), W)
    if planned:
        off = torch.linspace(0, T, planned + 1).to(I32).cuda()
        plan = moin.Plan(ctx()).build(off, torch.full((planned,), -1, dtype=I32, device="cuda"), T, 2)
        A, B = torch.zeros((2, 64, d_in), dtype=BF16, device="cuda"), torch.zeros((2, d_out, 64), dtype=BF16, device="cuda")
        y = moin.moin_lora_linear_i8_planned(ctx(), plan, x, w8, A, B, 2.0, y_dtype=y_dtype)
        plan.close()
    else:
        y = moin.moin_i8_linear(ctx(), x, w8, y_dtype=y_dtype)
    ctx().check()
    q, s = eb.integers(f64(x))
    sums = q.astype(np.float64) @ w8.codes.cpu().numpy()[:, :d_in].astype(np.float64).T       # (below 2^53: exact)
    want, got = sums * s[:, None] * f64(w8.scales), f64(y)
    assert not np.isnan(got).any() and not got[sums == 0].any() and (sums == 0).sum() > 0
    size, largest = np.abs(want), float(torch.finfo(y_dtype).max)
    tiny, huge = size < 2.0 ** -120, size > largest * (1 - 2.0 ** -7)
    assert (np.abs(got[tiny]) <= 2.0 ** -119).all()
    assert (np.abs(got[huge]) >= largest * (1 - 2.0 ** -6)).all() and (np.sign(got[huge]) == np.sign(want[huge])).all()
    assert np.isinf(got[size > largest * (1 + 2.0 ** -7)]).all()
    bound = size * (2.0 ** -22 + (2.0 ** -8 * (1 + 2.0 ** -20) if y_dtype == BF16 else 0.0))
    with np.errstate(invalid="ignore"):
        over = ~(tiny | huge) & ~(np.abs(got - want) <= bound)
    assert not over.any(), f"{int(over.sum())} of {over.size} beyond the bound, first {np.argwhere(over)[:3].tolist()}"
