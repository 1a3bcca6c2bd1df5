"""Integer products with adapters on each of the tile kernels, and without on several tiles a workgroup: which kernel a call takes goes by its tiles
of 128 x 128 (up to 2.6 of them a compute unit and round of those of 256 x 256), so the shapes lie well beyond the line for 256 compute units.

The magnitudes of tokens and channels change by up to 2^12 from tile to tile, so that a scale of another tile would show.  Bounds as in test_gpu_i8:
the sum is exact and rounded once, the scales' products are rounded twice; u is carried as two bf16 (2^-16 of it), its sum of d_in products and that of r terms
beside the base are fp32; a bf16 result is rounded by 2^-8 of itself."""
import numpy as np
import pytest
import torch

import tests.eight_bit as eb
from paper_2410_09687_amd import moin
from tests.gpu_common import ctx

pytestmark = pytest.mark.gpu
BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32


def normal(g, *shape, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(BF16)


class Case:
    def __init__(self, lens, d_in, d_out, r, E=5, seed=0):
        g, rng = torch.Generator(device="cuda").manual_seed(seed + d_in + r), np.random.default_rng(seed)
        self.lens, self.T, self.d_in, self.d_out, self.r, self.E = lens, int(sum(lens)), d_in, d_out, r, E
        self.off = np.concatenate([[0], np.cumsum(lens)])
        power = lambda n: torch.tensor(np.exp2(rng.integers(-6, 7, n // 128 + 1))[np.arange(n) // 128], device="cuda")[:, None]   # noqa: E731
        self.x = (normal(g, self.T, d_in) * power(self.T)).to(BF16)
        self.W = (normal(g, d_out, d_in, std=d_in ** -0.5) * power(d_out)).to(BF16)
        self.w8 = moin.moin_i8_quantize(ctx(), self.W)
        self.ids = [(3 * s) % (E + 1) - 1 for s in range(len(lens))]      # (-1 among them)
        self.ids = [0 if e == 2 else e for e in self.ids]                 # (and an expert that no sequence has)
        if r:
            self.A, self.B = normal(g, E, r, d_in, std=d_in ** -0.5), normal(g, E, d_out, r, std=r ** -0.5)

    def run(self, y_dtype, context=None, **kw):
        c = context or ctx()
        if not self.r:
            return moin.moin_i8_linear(c, self.x, self.w8, y_dtype=y_dtype, **kw)
        dev = lambda v: torch.tensor(np.asarray(v), dtype=I32).cuda()   # noqa: E731
        plan = moin.Plan(c).build(dev(self.off), dev(self.ids), self.T, self.E)
        y = moin.moin_lora_linear_i8_planned(c, plan, self.x, self.w8, self.A, self.B, 2.0, y_dtype=y_dtype, **kw)
        c.check()
        torch.cuda.synchronize()
        plan.close()
        return y

    def want(self, act=False):
        """Result and bound but for the last rounding, float64 on the device."""
        q, s = eb.integers(self.x.cpu().double().numpy())
        q, s = torch.tensor(q, dtype=F64, device="cuda"), torch.tensor(s, device="cuda")[:, None]
        w = self.w8.codes[:, :self.d_in].to(F64)
        base = q @ w.t().contiguous() * s * self.w8.scales.to(F64)       # (sums below 2^53: exact)
        add, lose = torch.zeros_like(base), base.abs() * 2.0 ** -22
        if self.r:
            for e, a, b in zip(self.ids, self.off[:-1], self.off[1:]):
                if e < 0 or a == b:
                    continue
                x, A, B = self.x[a:b].to(F64), self.A[e].to(F64), self.B[e].to(F64)
                u = x @ A.t().contiguous()
                if act:
                    u = u.clamp(min=0)
                add[a:b] = 2.0 * (u @ B.t().contiguous())
                most = x.abs() @ A.abs().t().contiguous()
                lose[a:b] += 2.0 * (u.abs() @ B.abs().t().contiguous()) * 2.0 ** -16
                lose[a:b] += 2.0 * (most @ B.abs().t().contiguous()) * (self.d_in + self.r + 8) * 2.0 ** -24
            lose += (base.abs() + add.abs()) * (2 * self.r + 16) * 2.0 ** -24
        return base + add, lose

    def check(self, y, want, lose):
        bound = lose + (want.abs() + lose) * (2.0 ** -8 if y.dtype == BF16 else 0)
        over = ~((y.to(F64) - want).abs() <= bound)
        assert not bool(over.any()), f"{int(over.sum())} of {over.numel()} beyond the bound, first {over.nonzero()[:3].tolist()}"


def ragged(n, lo, hi, seed):
    return np.random.default_rng(seed).integers(lo, hi + 1, n).tolist()


MANY = ragged(16, 100, 1900, 1)          # four tiles of 256 x 256 and more a workgroup
HALF = ragged(12, 200, 380, 2)           # 432 tiles of 128 x 128 and more, more than one a compute unit
FEW = ragged(5, 150, 250, 3)             # fewer than compute units


@pytest.mark.parametrize("y_dtype", [BF16, F32])
@pytest.mark.parametrize("lens,d_in,d_out,r", [
    (MANY, 1000, 4104, 64), (MANY, 1000, 4104, 128), (MANY, 256, 4104, 64), (MANY, 200, 4104, 128), (MANY + [0, 1, 257], 512, 4096, 64),
    (ragged(40, 100, 700, 4), 1000, 4104, 64), (HALF, 1000, 1416, 64), (HALF, 256, 1416, 128), (HALF, 8, 2056, 64), (FEW, 1000, 1416, 64),
    ([9000], 512, 8200, 0), ([9000], 136, 8200, 0), ([5000], 1024, 2056, 0)])
def test_tiles(lens, d_in, d_out, r, y_dtype):
    c = Case(lens, d_in, d_out, r)
    y = c.run(y_dtype)
    c.check(y, *c.want())
    for _ in range(2):
        assert torch.equal(c.run(y_dtype), y)


@pytest.mark.parametrize("lens,d_out", [(MANY, 4104), (HALF, 1416)])
def test_activation(lens, d_out):
    own = moin.Context(0)
    try:
        own.set_adapter_activation("relu")
        c = Case(lens, 512, d_out, 64)
        c.check(c.run(F32, own), *c.want(act=True))
    finally:
        torch.cuda.synchronize()
        own.close()


@pytest.mark.parametrize("lens,d_out", [(MANY, 4104), (HALF, 1416), ([1] * 200, 1416)])
def test_what_is_not_finite_stays_with_its_own(lens, d_out):
    """An infinite adapter reaches the rows of its expert alone, a token's NaN its row, a channel's its column."""
    c = Case(lens, 1000, d_out, 64)
    before = c.run(BF16)
    c.B[1, 7, 3], c.A[3, 5, 9] = float("inf"), float("nan")
    c.x[11, 0] = float("nan")
    c.w8.scales[40] = float("nan")
    got = c.run(BF16)
    keep = torch.tensor(np.repeat([e not in (1, 3) for e in c.ids], c.lens), device="cuda")[:, None].expand_as(got).clone()
    keep[11], keep[:, 40] = False, False
    ones = torch.tensor(np.repeat([e == 1 for e in c.ids], c.lens), device="cuda")
    ones[11] = False
    sound = torch.ones(d_out, dtype=torch.bool, device="cuda")
    sound[7], sound[40] = False, False
    assert torch.equal(got[keep], before[keep]) and torch.equal(got[ones][:, sound], before[ones][:, sound])
    assert bool(torch.isnan(got[11]).all()) and bool(torch.isnan(got[:, 40]).all()) and not bool(torch.isfinite(got[ones][:, 7]).any())
