"""Weights in MXFP4 and products with them, against their definition in 64 bits."""
import numpy as np
import pytest
import torch

import tests.four_bit as fb
from paper_2410_09687_amd import moin
from tests.gpu_common import ctx

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def f64(t):
    return t.detach().cpu().double().numpy()


def same(a, b):
    differ = int((~((a == b) | (np.isnan(a) & np.isnan(b)))).sum())
    assert differ == 0


def weight(seed, d_out, d_in):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((d_out, d_in), generator=g) * d_in ** -0.5).to(BF16).cuda()


def inputs(seed, T, d_in):
    return torch.randn((T, d_in), generator=torch.Generator().manual_seed(seed)).to(BF16).cuda()


def padded(x):
    return np.pad(x, [(0, 0), (0, -x.shape[1] % 32)])


@pytest.mark.parametrize("d_out,d_in", [(8, 8), (16, 512), (17, 520), (40, 1000), (5, 136)])
def test_quantise_and_back(d_out, d_in):
    W = weight(d_out + d_in, d_out, d_in)
    W[0, :4] = torch.tensor([0.0, 1e-30, -3e38, 5.0])
    if d_out > 8:
        W[8] = 0
        W[9, -1] = float("nan")
    W4 = moin.moin_mx4_quantize(ctx(), W)
    want = fb.held(padded(f64(W)))[:, :d_in]
    same(fb.decode_weight(W4.data.cpu().numpy(), d_out, d_in), want)
    same(f64(moin.moin_mx4_dequantize(ctx(), W4)), want)


def check(y, x, W, extra=None):
    """fp32 sums over d_in products that are exact: each off by at most d_in 2^-24 of the sum of magnitudes; then the rounding to bf16, by at most
    2^-8 of the result (half a unit in the last of eight bits)."""
    want, spread = x @ W.T, np.abs(x) @ np.abs(W).T
    bound = x.shape[1] * 2.0 ** -24 * spread + 1e-30
    if extra is not None:
        want = want + extra[0]
        bound = bound + extra[1]
    if y.dtype == BF16:
        bound = bound * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    worst = float((np.abs(f64(y) - want) / bound).max())
    assert worst <= 1, f"worst ratio {worst:.2f}"


@pytest.mark.parametrize("y_dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1, 2, 4, 5, 15, 16, 17, 32, 33, 64, 65, 200, 256, 300, 1100])
@pytest.mark.parametrize("d_out,d_in", [(8, 8), (256, 256), (136, 1000), (1416, 520), (24, 5632)])
def test_linear(T, d_out, d_in, y_dtype):
    W, x = weight(d_in, d_out, d_in), inputs(T, T, d_in)
    W4 = moin.moin_mx4_quantize(ctx(), W)
    y = moin.moin_mx4_linear(ctx(), x, W4, y_dtype=y_dtype)
    ctx().check()
    check(y, f64(x), fb.held(padded(f64(W)))[:, :d_in])
    assert torch.equal(y, moin.moin_mx4_linear(ctx(), x, W4, y_dtype=y_dtype))


@pytest.mark.parametrize("T", [1, 16, 24, 70])
@pytest.mark.parametrize("d_out,d_in", [(4112, 264), (16400, 136), (16400, 1032)])
def test_wide_weights(T, d_out, d_in):
    """More rows than the shapes for few tiles take, and rows of codes that are not whole records."""
    W, x = weight(d_in, d_out, d_in), inputs(T, T, d_in)
    W4 = moin.moin_mx4_quantize(ctx(), W)
    held = moin.moin_mx4_dequantize(ctx(), W4)
    y = moin.moin_mx4_linear(ctx(), x, W4, y_dtype=F32)
    want = x.double() @ held.double().t().contiguous()
    spread = x.double().abs() @ held.double().abs().t().contiguous()
    assert ((y.double() - want).abs() <= d_in * 2.0 ** -24 * spread).all()


def batch(T, S, E, seed):
    rng = np.random.default_rng(seed)
    cut = np.sort(rng.integers(0, T + 1, S - 1))
    off = np.concatenate([[0], cut, [T]])
    ids = rng.integers(-1, E, S)
    return torch.tensor(off, dtype=I32).cuda(), torch.tensor(ids, dtype=I32).cuda(), off, ids


@pytest.mark.parametrize("y_dtype", [BF16, F32])
@pytest.mark.parametrize("T,S", [(1, 1), (8, 8), (40, 7), (200, 3), (256, 256), (300, 2), (700, 3), (1500, 900), (2000, 4)])
@pytest.mark.parametrize("d_out,d_in,r", [(256, 512, 16), (136, 1000, 24), (512, 256, 128)])
def test_with_adapters(T, S, d_out, d_in, r, y_dtype):
    E = 6
    W, x = weight(1, d_out, d_in), inputs(T + 1, T, d_in)
    A = inputs(3, E * r, d_in).view(E, r, d_in) * d_in ** -0.5
    B = inputs(4, E * d_out, r).view(E, d_out, r) * r ** -0.5
    off, ids, h_off, h_ids = batch(T, S, E, T)
    plan = moin.Plan(ctx()).build(off, ids, T, E)
    W4 = moin.moin_mx4_quantize(ctx(), W)
    y = moin.moin_lora_linear_mx4_planned(ctx(), plan, x, W4, A, B, 2.0, y_dtype=y_dtype)
    ctx().check()
    term, off_by = np.zeros((T, d_out)), np.zeros((T, d_out))
    fx, fA, fB = f64(x), f64(A), f64(B)
    for s, e in enumerate(h_ids):
        if e < 0:
            continue
        rows = slice(h_off[s], h_off[s + 1])
        u = fx[rows] @ fA[e].T
        term[rows] = 2 * u @ fB[e].T
        # u is kept to 16 bits or more; sums of d_in and of r products (and of the parts) in fp32
        wide = 2 * (np.abs(fx[rows]) @ np.abs(fA[e]).T) @ np.abs(fB[e]).T
        off_by[rows] = 2 * 2.0 ** -16 * np.abs(u) @ np.abs(fB[e]).T + (d_in + 2 * r + 8) * 2.0 ** -24 * wide
    check(y, fx, fb.held(padded(f64(W)))[:, :d_in], (term, off_by))
    # on the prefill path, the bits of a bf16 weight with these values
    if T > 1024 and T > 128 * S:
        full = moin.moin_mx4_dequantize(ctx(), W4)
        assert torch.equal(y, moin.moin_lora_linear_planned(ctx(), plan, x, full, A, B, 2.0, y_dtype=y_dtype))
    # no adapters at all
    y = moin.moin_lora_linear_mx4_planned(ctx(), plan, x, W4, None, None, 2.0, y_dtype=y_dtype)
    check(y, fx, fb.held(padded(f64(W)))[:, :d_in])


def test_activation_and_ranks():
    T, E, d_out, d_in, r = 50, 4, 128, 256, 32
    W, x = weight(5, d_out, d_in), inputs(6, T, d_in)
    A, B = inputs(7, E * r, d_in).view(E, r, d_in) * d_in ** -0.5, inputs(8, E * d_out, r).view(E, d_out, r) * r ** -0.5
    off, ids, _, _ = batch(T, 9, E, 2)
    ranks = torch.tensor([8, 32, 0, 16], dtype=I32).cuda()
    own = moin.Context(0)
    own.set_adapter_activation("silu")
    plan = moin.Plan(own).build(off, ids, T, E, rank_of_expert=ranks)
    W4 = moin.moin_mx4_quantize(own, W)
    y = moin.moin_lora_linear_mx4_planned(own, plan, x, W4, A, B, 1.5, y_dtype=F32)
    z = moin.moin_lora_linear_planned(own, plan, x, moin.moin_mx4_dequantize(own, W4), A, B, 1.5, y_dtype=F32)
    own.check()
    # the same adapter kernels; the base's fp32 sums in another order
    bound = 2 * d_in * 2.0 ** -24 * (x.abs().float() @ moin.moin_mx4_dequantize(own, W4).abs().float().t()) + 2.0 ** -22 * z.abs()
    assert ((y - z).abs() <= bound).all()
    own.close()


def test_graph_and_stream():
    W4, x = moin.moin_mx4_quantize(ctx(), weight(9, 256, 640)), inputs(9, 20, 640)
    y = torch.empty((20, 256), dtype=BF16, device="cuda")
    want = moin.moin_mx4_linear(ctx(), x, W4)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        moin.moin_mx4_linear(ctx(), x, W4, out=y)
    for _ in range(3):
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z = moin.moin_mx4_linear(ctx(), x, W4)
    side.synchronize()
    assert torch.equal(z, want)


def test_a_first_call_that_needs_the_weight_in_bf16_is_refused_under_capture():
    own = moin.Context(0)
    W4, x = moin.moin_mx4_quantize(own, weight(10, 256, 256)), inputs(10, 2000, 256)
    A, B = inputs(11, 16, 256).view(2, 8, 256), inputs(12, 512, 8).view(2, 256, 8)
    plan = moin.Plan(own).build(torch.tensor([0, 700, 2000], dtype=I32).cuda(), torch.tensor([1, 0], dtype=I32).cuda(), 2000, 2)
    run = lambda: moin.moin_lora_linear_mx4_planned(own, plan, x, W4, A, B, 1.0, out=y)   # noqa: E731
    y = torch.empty((2000, 256), dtype=BF16, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            with pytest.raises(moin.MoinError) as e:
                run()
            assert e.value.code == -6
            torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    want = run().clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for _ in range(3):
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
    del g
    plan.close()
    own.close()


def test_infinities_stay_where_they_are():
    """An infinite activation makes infinities and, where the weight is 0, NaN, also in the last columns of rows that are not whole blocks."""
    for T in (1, 10, 40):
        W = weight(13, 64, 520)
        W[3, 519] = 0
        W[4, 519] = 0.25
        x = inputs(13, T, 520)
        x[0, 519] = float("inf")
        W4 = moin.moin_mx4_quantize(ctx(), W)
        y = moin.moin_mx4_linear(ctx(), x, W4, y_dtype=F32)
        held = moin.moin_mx4_dequantize(ctx(), W4)[:, 519]
        assert torch.equal(torch.isnan(y[0]), held == 0)
        assert (y[0][held > 0] == float("inf")).all() and (y[0][held < 0] == -float("inf")).all() and torch.isfinite(y[1:]).all()


def test_refusals():
    W4, x = moin.moin_mx4_quantize(ctx(), weight(11, 64, 256)), inputs(11, 4, 256)
    assert moin.moin_mx4_linear(ctx(), x[:0], W4).shape == (0, 64)
    for bad in (x[:, :128], x[0], x.cpu(), torch.zeros((512, 4), dtype=BF16, device="cuda").t()):
        with pytest.raises(ValueError):
            moin.moin_mx4_linear(ctx(), bad, W4)
    with pytest.raises(TypeError):
        moin.moin_mx4_linear(ctx(), x.float(), W4)
    with pytest.raises(TypeError):
        moin.moin_mx4_linear(ctx(), x, W4, y_dtype=torch.float16)
    with pytest.raises(ValueError):
        moin.moin_mx4_linear(ctx(), x, W4, out=torch.empty((4, 60), dtype=BF16, device="cuda"))
    with pytest.raises(ValueError):
        moin.MX4Weight(W4.data[:-1], 64, 256)
    for shape in ((4, 12), (0, 8), (4, 0), (4,)):
        with pytest.raises(ValueError):
            moin.moin_mx4_quantize(ctx(), torch.zeros(shape, dtype=BF16, device="cuda"))
    with pytest.raises(TypeError):
        moin.moin_mx4_quantize(ctx(), torch.zeros((8, 8), device="cuda"))
    odd = moin.moin_mx4_quantize(ctx(), weight(12, 12, 64))   # y's rows would not be whole groups of eight
    with pytest.raises(moin.MoinError) as e:
        moin.moin_mx4_linear(ctx(), inputs(12, 3, 64), odd)
    assert e.value.code == -1
    plan = moin.Plan(ctx()).build(torch.tensor([0, 4], dtype=I32).cuda(), torch.tensor([0], dtype=I32).cuda(), 4, 2)
    A, B = inputs(13, 16, 256).view(2, 8, 256), inputs(14, 128, 8).view(2, 64, 8)
    moin.moin_lora_linear_mx4_planned(ctx(), plan, x, W4, A, B, 1.0)
    for kw in (dict(A=A[:, :, :128]), dict(A=A[:1], B=B[:1]), dict(x=x[:3]), dict(B=B[:, :32])):
        with pytest.raises(ValueError):
            moin.moin_lora_linear_mx4_planned(ctx(), plan, kw.get("x", x), W4, kw.get("A", A), kw.get("B", B), 1.0)
    ctx().check()
