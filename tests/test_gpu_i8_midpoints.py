"""Codes of rows with the smallest steps, where half a step may not be a number of fp32: every value and every midpoint of rows whose scale lies
between 2^-126 and 2^-124, and of rows below."""
import numpy as np
import pytest
import torch

import tests.eight_bit as eb
from paper_2410_09687_amd import moin
from tests.gpu_common import ctx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [-133, -128, -127, -126, -125, -124, 0])
def test_every_row_of_eight_bits(power):
    rows = []
    for top in range(128, 256):
        x = np.arange(0, 2 * top + 1) / 2.0                      # halves of the largest value's last place
        x = x[np.array([v == 0 or float(np.frexp(v)[0] * 256).is_integer() for v in x])]
        rows.append(np.concatenate([x, -x, np.full(512, top)])[:512])
        rows[-1][-1] = top
    x = np.array(rows) * 2.0 ** power
    x[np.abs(np.rint(x * 2.0 ** 133) - x * 2.0 ** 133) > 0] = 0  # (bf16 has no smaller place)
    t = torch.tensor(x).to(torch.bfloat16).cuda()
    assert np.array_equal(t.cpu().double().numpy(), x)
    w = moin.moin_i8_quantize(ctx(), t)
    q, s = eb.integers(x)
    assert np.array_equal(w.scales.cpu().double().numpy(), s) and np.array_equal(w.codes.cpu().numpy(), q)
    # the same codes where the product makes them: one token against the unit rows
    eye = moin.moin_i8_quantize(ctx(), torch.eye(512, dtype=torch.bfloat16, device="cuda") * 127)
    for r in (0, 94, 127):
        y = moin.moin_i8_linear(ctx(), t[r:r + 1] * 2.0 ** 60, eye, y_dtype=torch.float32)
        q, s = eb.integers(x[r:r + 1] * 2.0 ** 60)
        assert np.array_equal(np.rint(y.cpu().double().numpy() / (127 * s)), q)
    ctx().check()
