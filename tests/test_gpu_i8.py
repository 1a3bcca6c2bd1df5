"""Products in 8-bit integers with a scale for each token and channel, with adapters and without.

Codes and scales are compared exactly.  The sum of a product is exact; it is rounded to fp32 and so are two products with the scales: 2^-22
of the result.  A bf16 result is rounded by at most 2^-8 of itself.  Adapters add what the framework's adapters' products may lose (`adapters`)."""
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


def normal(seed, *shape, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(BF16)


def same_codes(w, x):
    q, s = eb.integers(f64(x))
    assert np.array_equal(f64(w.scales), s, equal_nan=True)
    fine = np.isfinite(s)
    codes = w.codes.cpu().numpy()
    assert np.array_equal(codes[fine, :x.shape[1]], q[fine]) and not codes[:, x.shape[1]:].any()


@pytest.mark.parametrize("rows,cols", [(1, 8), (3, 128), (5, 264), (2, 1000), (70, 2048), (3, 2056), (2, 8192), (1, 131072), (1100, 136), (1025, 4104)])
def test_codes(rows, cols):
    x = normal(rows + cols, rows, cols) * torch.exp(normal(rows, rows, 1)).to(BF16)
    same_codes(moin.moin_i8_quantize(ctx(), x), x)


def test_codes_of_ties_small_values_zeros_and_nans():
    rng = np.random.default_rng(0)
    rows = []
    for top in (127.0, 254.0, 63.5, 95.25, 190.5, 1.0, 3.0, 2.0 ** -119, 2.0 ** -126, 2.0 ** -133, 3.3e38, 0.0):
        x = rng.integers(-254, 255, 512) / 254.0 * top      # halves of a step among them
        x[0] = top
        rows.append(x)
    bad = rng.normal(size=(3, 512))
    bad[0, 5], bad[1, 511], bad[2, 0] = np.nan, np.inf, -np.inf
    x = torch.tensor(np.concatenate([rows, bad])).to(BF16).cuda()
    same_codes(moin.moin_i8_quantize(ctx(), x), x)
    same_codes(moin.moin_i8_quantize(ctx(), x[:, :8].contiguous()), x[:, :8])


class Product:
    def __init__(self, seed, T, d_in, d_out):
        self.x = normal(seed, T, d_in) * torch.exp(normal(seed + 1, T, 1)).to(BF16)
        self.W = normal(seed + 2, d_out, d_in, std=d_in ** -0.5) * torch.exp(normal(seed + 3, d_out, 1)).to(BF16)
        self.w8 = moin.moin_i8_quantize(ctx(), self.W)

    def base(self):
        q, s = eb.integers(f64(self.x))
        w, t = self.w8.codes.cpu().numpy()[:, :self.x.shape[1]].astype(np.float64), f64(self.w8.scales)
        return (q.astype(np.float64) @ w.T) * s[:, None] * t       # (sums below 2^53: exact)

    def check(self, y):
        ctx().check()
        want = self.base()
        bound = np.abs(want) * (2.0 ** -22 + (2.0 ** -8 * (1 + 2.0 ** -20) if y.dtype == BF16 else 0.0)) + 2.0 ** -140
        over = np.abs(f64(y) - want) > bound
        assert not over.any(), f"{int(over.sum())} of {over.size} beyond the bound, first {np.argwhere(over)[:3].tolist()}"


@pytest.mark.parametrize("y", [BF16, F32])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 33, 64, 65, 130, 300])
@pytest.mark.parametrize("d_in,d_out", [(8, 8), (256, 24), (1000, 264), (2048, 256), (2056, 2000)])
def test_products(d_in, d_out, T, y):
    p = Product(d_in + T, T, d_in, d_out)
    p.check(moin.moin_i8_linear(ctx(), p.x, p.w8, y_dtype=y))


@pytest.mark.parametrize("T,d_in,d_out", [(2000, 384, 5632), (4100, 264, 4104), (9000, 512, 2048), (1, 131072, 8), (5, 20000, 40), (70, 40000, 264)])
def test_larger_products(T, d_in, d_out):
    p = Product(T, T, d_in, d_out)
    for y in (BF16, F32):
        p.check(moin.moin_i8_linear(ctx(), p.x, p.w8, y_dtype=y))


def test_the_largest_sums_do_not_wrap():
    for T in (1, 65, 300):
        x = torch.full((T, 131072), 3.0, dtype=BF16, device="cuda")
        w8 = moin.moin_i8_quantize(ctx(), torch.full((8, 131072), -2.0, dtype=BF16, device="cuda"))
        y = moin.moin_i8_linear(ctx(), x, w8, y_dtype=F32)
        assert np.allclose(f64(y), -6.0 * 131072, rtol=2.0 ** -21)
    ctx().check()


def test_more_rows_than_a_launch_takes():
    rows, far = 2 ** 23 + 3, 2 ** 23 - 2
    x = torch.zeros((rows, 8), dtype=BF16, device="cuda")
    x[:5], x[far:] = normal(9, 5, 8), normal(10, 5, 8)
    got = moin.moin_i8_quantize(ctx(), x)
    for at in (0, far):
        want = moin.moin_i8_quantize(ctx(), x[at:at + 5].clone())
        assert torch.equal(got.codes[at:at + 5], want.codes) and torch.equal(got.scales[at:at + 5], want.scales)
    assert not got.codes[5:far].any() and (got.scales[5:far] == 2.0 ** -126).all()


def test_rows_and_channels_with_nans_stay_alone():
    for T in (4, 40, 100):
        p = Product(T, T, 512, 72)
        p.x[1, 7], p.x[3, 0] = float("nan"), float("inf")
        p.W[5, 3] = float("nan")
        w8 = moin.moin_i8_quantize(ctx(), p.W)
        y = moin.moin_i8_linear(ctx(), p.x, w8)
        nan = torch.zeros_like(y, dtype=torch.bool)
        nan[1], nan[3], nan[:, 5] = True, True, True
        assert torch.equal(torch.isnan(y), nan)


@pytest.mark.parametrize("T,d_in,d_out", [(25, 16384, 40), (100, 4096, 72), (128, 5632, 264), (129, 2120, 2056)])
def test_tiles_over_parts_of_the_contraction(T, d_in, d_out):
    """Few tiles: each in parts, whose sums are added; eager and captured, without and with the plan of no adapters, and beside NaNs."""
    own = moin.Context(0)
    try:
        p = Product(T, T, d_in, d_out)
        for y in (BF16, F32):
            p.check(moin.moin_i8_linear(own, p.x, p.w8, y_dtype=y))
        plan = moin.Plan(own).build(torch.tensor([0, T], dtype=I32, device="cuda"), torch.zeros(1, dtype=I32, device="cuda"), T, 3)
        want, y = moin.moin_i8_linear(own, p.x, p.w8), torch.empty((T, d_out), dtype=BF16, device="cuda")
        assert torch.equal(moin.moin_lora_linear_i8_planned(own, plan, p.x, p.w8, None, None, 1.0), want)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            moin.moin_i8_linear(own, p.x, p.w8, out=y)
        other = p.x.flip(0).contiguous()
        for _ in range(3):
            y.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want)
            assert torch.equal(moin.moin_i8_linear(own, other, p.w8), want.flip(0))
        del graph
        plan.close()
        p.x[3, 5] = float("nan")
        got = moin.moin_i8_linear(own, p.x, p.w8)
        assert torch.isnan(got[3]).all() and torch.equal(got[4:], want[4:]) and torch.equal(got[:3], want[:3])
    finally:
        torch.cuda.synchronize()
        own.close()


def adapters(p, off, ids, A, B, scale, act=None):
    """Result and bound.  u is carried as two bf16 (2^-16 of it), its sum of d_in products and that of r terms beside the base are fp32."""
    x, base = f64(p.x), p.base()
    add, lose = np.zeros_like(base), np.zeros_like(base)
    d_in, r = x.shape[1], A.shape[1]
    for s, e in enumerate(ids):
        if e < 0 or off[s] == off[s + 1]:
            continue
        a, b, xs = f64(A[e]), f64(B[e]), x[off[s]:off[s + 1]]
        u = xs @ a.T
        if act:
            u = np.maximum(u, 0)
        add[off[s]:off[s + 1]] = scale * (u @ b.T)
        lose[off[s]:off[s + 1]] = scale * (np.abs(u) @ np.abs(b.T)) * 2.0 ** -16 + scale * (np.abs(xs) @ np.abs(a.T) @ np.abs(b.T)) * (d_in + r + 8) * 2.0 ** -24
    lose += (np.abs(base) + np.abs(add)) * (2 * r + 16) * 2.0 ** -24
    q = np.abs(eb.integers(x)[0]).astype(np.float64) @ np.abs(p.w8.codes.cpu().numpy()[:, :d_in].astype(np.float64)).T
    lose += q * eb.integers(x)[1][:, None] * f64(p.w8.scales) * 4 * 2.0 ** -24      # (up to four parts of the sum, each rounded)
    return base + add, lose


@pytest.mark.parametrize("y_dtype", [BF16, F32])
@pytest.mark.parametrize("r", [64, 128, 192])
@pytest.mark.parametrize("d_in,d_out,lens", [(512, 264, [1] * 5), (2048, 2000, [1] * 40), (1000, 256, [1] * 90), (2048, 512, [3, 0, 1, 60, 9]), (512, 264, [300, 7, 0, 513]),
                                             (1000, 2048, [200, 900, 64]), (2048, 2048, [128] * 12)])
def test_adapters(d_in, d_out, lens, r, y_dtype):
    T, S, E = sum(lens), len(lens), 5
    p = Product(T + r, T, d_in, d_out)
    ids = [(3 * s) % (E + 1) - 1 for s in range(S)]
    A, B = normal(1, E, r, d_in, std=d_in ** -0.5), normal(2, E, d_out, r, std=r ** -0.5)
    off = np.concatenate([[0], np.cumsum(lens)])
    plan = moin.Plan(ctx()).build(torch.tensor(off, dtype=I32).cuda(), torch.tensor(ids, dtype=I32).cuda(), T, E)
    y = moin.moin_lora_linear_i8_planned(ctx(), plan, p.x, p.w8, A, B, 2.0, y_dtype=y_dtype)
    ctx().check()
    want, lose = adapters(p, off, ids, A, B, 2.0)
    bound = lose + (np.abs(want) + lose) * (2.0 ** -8 if y_dtype == BF16 else 0)
    over = np.abs(f64(y) - want) > bound
    assert not over.any(), f"{int(over.sum())} of {over.size} beyond the bound"
    z = moin.moin_lora_linear_i8_planned(ctx(), plan, p.x, p.w8, A, B, 2.0, y_dtype=y_dtype)
    assert torch.equal(y, z)


@pytest.mark.parametrize("lens", [[1] * 9, [400, 300]])
def test_activations_ranks_and_no_adapters(lens):
    T, S, E, r, d_in, d_out = sum(lens), len(lens), 3, 64, 512, 256
    p = Product(7, T, d_in, d_out)
    ids = [s % E for s in range(S)]
    A, B = normal(3, E, r, d_in, std=d_in ** -0.5), normal(4, E, d_out, r, std=r ** -0.5)
    off = np.concatenate([[0], np.cumsum(lens)])
    o, i = torch.tensor(off, dtype=I32).cuda(), torch.tensor(ids, dtype=I32).cuda()
    own = moin.Context(0)
    try:
        own.set_adapter_activation("relu")
        plan = moin.Plan(own).build(o, i, T, E)
        y = moin.moin_lora_linear_i8_planned(own, plan, p.x, p.w8, A, B, 2.0, y_dtype=F32)
        own.check()
        want, lose = adapters(p, off, ids, A, B, 2.0, act="relu")
        assert (np.abs(f64(y) - want) <= lose).all()
        plan.close()
    finally:
        torch.cuda.synchronize()
        own.close()
    ranks = torch.tensor([0, 24, 64], dtype=I32).cuda()
    plan = moin.Plan(ctx()).build(o, i, T, E, rank_of_expert=ranks)
    y = moin.moin_lora_linear_i8_planned(ctx(), plan, p.x, p.w8, A, B, 2.0, y_dtype=F32)
    A2, B2 = A.clone(), B.clone()
    for e, n in enumerate((0, 24, 64)):
        A2[e, n:], B2[e, :, n:] = 0, 0
    want, lose = adapters(p, off, ids, A2, B2, 2.0)
    assert (np.abs(f64(y) - want) <= lose).all()
    plain = moin.Plan(ctx()).build(o, torch.full_like(i, -1), T, 0)
    a = moin.moin_lora_linear_i8_planned(ctx(), plain, p.x, p.w8, None, None, 2.0, y_dtype=F32)
    assert torch.equal(a, moin.moin_i8_linear(ctx(), p.x, p.w8, y_dtype=F32))
    ctx().check()


@pytest.mark.parametrize("first,then", [(900, 3), (300, 70), (300, 64), (64, 16), (16, 300)])
def test_captured_calls_after_a_larger_eager_one(first, then):
    """Up to the eager call's tokens a captured one needs no more memory; beyond it is refused and nothing is recorded."""
    d_in, d_out, E, r = 2048, 264, 3, 64
    own = moin.Context(0)
    try:
        big, p = Product(1, first, d_in, d_out), Product(2, then, d_in, d_out)
        A, B = normal(5, E, r, d_in, std=d_in ** -0.5), normal(6, E, d_out, r, std=r ** -0.5)

        def planned(T):
            return moin.Plan(own).build(torch.arange(T + 1, dtype=I32, device="cuda"), torch.arange(T, dtype=I32, device="cuda") % E, T, E)

        pa, pb = planned(first), planned(then)
        moin.moin_lora_linear_i8_planned(own, pa, big.x, p.w8, A, B, 2.0)
        want = moin.moin_lora_linear_i8_planned(ctx(), pb, p.x, p.w8, A, B, 2.0)
        alone = moin.moin_i8_linear(ctx(), p.x, p.w8)
        y, z = torch.empty_like(want), torch.empty_like(want)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        refused = then > first
        with torch.cuda.graph(graph):
            if refused:
                with pytest.raises(moin.MoinError) as e:
                    moin.moin_lora_linear_i8_planned(own, pb, p.x, p.w8, A, B, 2.0, out=y)
                assert e.value.code == -6
            else:
                moin.moin_lora_linear_i8_planned(own, pb, p.x, p.w8, A, B, 2.0, out=y)
                moin.moin_i8_linear(own, p.x, p.w8, out=z)
        for _ in range(0 if refused else 3):
            y.zero_()
            z.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want) and torch.equal(z, alone)
            moin.moin_i8_linear(ctx(), big.x, p.w8)
        del graph
        for q in (pa, pb):
            q.close()
    finally:
        torch.cuda.synchronize()
        own.close()
    ctx().check()


def test_no_tokens_given_outputs_other_streams():
    p = Product(11, 30, 512, 64)
    assert moin.moin_i8_linear(ctx(), p.x[:0], p.w8).shape == (0, 64)
    y = moin.moin_i8_linear(ctx(), p.x, p.w8)
    guard = torch.full((32, 64), 5.0, dtype=BF16, device="cuda")
    z = moin.moin_i8_linear(ctx(), p.x, p.w8, out=guard[1:31])
    assert torch.equal(y, z) and (guard[0] == 5).all() and (guard[31] == 5).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z = moin.moin_i8_linear(ctx(), p.x, p.w8)
    side.synchronize()
    assert torch.equal(y, z)


def test_refusals():
    p = Product(12, 4, 512, 64)
    with pytest.raises(ValueError):
        moin.moin_i8_quantize(ctx(), p.W[:, :12].contiguous())
    with pytest.raises(ValueError):
        moin.moin_i8_quantize(ctx(), p.W[:0])
    with pytest.raises(TypeError):
        moin.moin_i8_quantize(ctx(), p.W.float())
    run = lambda x=p.x, w=p.w8, **kw: moin.moin_i8_linear(ctx(), x, w, **kw)   # noqa: E731
    for kw in (dict(x=p.x[:, :504]), dict(x=p.x[0]), dict(x=p.x.cpu()), dict(x=p.x.t()), dict(out=torch.empty((3, 64), dtype=BF16, device="cuda"))):
        with pytest.raises(ValueError):
            run(**kw)
    for kw in (dict(x=p.x.float()), dict(y_dtype=torch.float16)):
        with pytest.raises(TypeError):
            run(**kw)
    odd = moin.moin_i8_quantize(ctx(), p.W[:60])
    with pytest.raises(moin.MoinError) as e:        # outputs not a multiple of 8
        run(w=odd)
    assert e.value.code == -1
    plan = moin.Plan(ctx())
    call = lambda A, B, plan=plan, x=p.x: moin.moin_lora_linear_i8_planned(ctx(), plan, x, p.w8, A, B, 2.0)   # noqa: E731
    A, B = normal(1, 2, 64, 512), normal(2, 2, 64, 64)
    with pytest.raises(ValueError):                 # a plan that is not built has no tokens
        call(A, B)
    with pytest.raises(moin.MoinError):
        call(None, None, x=p.x[:0])
    plan.build(torch.arange(5, dtype=I32, device="cuda"), torch.zeros(4, dtype=I32, device="cuda"), 4, 2)
    call(A, B)
    with pytest.raises(ValueError):
        call(A[:1], B[:1])
    with pytest.raises(ValueError):
        call(A, B[:, :56])
    with pytest.raises(moin.MoinError):             # a rank that is not a multiple of 64
        call(A[:, :40].contiguous(), B[:, :, :40].contiguous())
    ctx().check()
