"""Norms of queries and keys for each head with the rotation by position, against the definition in 64 bits and more.

Bounds, element by element: the result is rounded to bf16 once (2^-8 of itself).  Before that: the norm's sum of D squares, its
square root and two products, (D / 2 + 8) 2^-24 of the value at most; a sine or cosine is off by 2^-21 (its angle as a fraction of a
turn in fp32, 2^-24 of it, and the function's last places), and by what 64 bits lose of p f, |p f| 2^-51."""
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


def inputs(seed, T, heads, H, D, dtype=BF16, far=5000):
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = torch.randn((T, heads + 2 * H, D), generator=g, device="cuda") * torch.exp(torch.randn((T, 1, 1), generator=g, device="cuda"))
    pos = torch.randint(0, far, (T,), generator=g, device="cuda", dtype=I32)
    gains = [(1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(BF16) for _ in range(2)]
    return qkv.to(dtype), pos, gains


def compare(got, x, pos, freqs, gain, eps, norm, neighbours):
    want, size = eb.norm_rope(f64(x), None if pos is None else f64(pos), None if pos is None else f64(freqs), None if gain is None else f64(gain), eps,
                              norm, neighbours)
    D = want.shape[-1]
    slack = (D / 2 + 8) * 2.0 ** -24 * size
    if pos is not None:
        n = freqs.numel()
        turn = 2.0 ** -21 + np.abs(f64(pos)[:, None] * f64(freqs)) * 2.0 ** -51
        at = np.arange(2 * n) // 2 if neighbours else np.arange(2 * n) % n
        slack[..., :2 * n] += (size[..., :2 * n] * turn[:, None, at])
    got = f64(got)
    fine = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fine)
    over = np.abs(got - want) > 2.0 ** -8 * np.abs(want) + slack * (1 + 2.0 ** -7) + 2.0 ** -133
    assert not over[fine].any(), f"{int(over[fine].sum())} beyond the bound"


def check(qkv, pos, gains, heads, H, freqs, norm=True, eps=1e-6, neighbours=False):
    q, k = moin.moin_qk_norm_rope(ctx(), qkv[:, :heads], qkv[:, heads:heads + H] if H else None, positions=pos, freqs=freqs,
                                  q_gain=gains[0] if norm else None, k_gain=gains[1] if norm and H else None, norm=norm, eps=eps, neighbours=neighbours)
    ctx().check()
    assert q.dtype == BF16 and q.shape == qkv[:, :heads].shape
    compare(q, qkv[:, :heads], pos, freqs, gains[0] if norm else None, eps, norm, neighbours)
    if H:
        compare(k, qkv[:, heads:heads + H], pos, freqs, gains[1] if norm else None, eps, norm, neighbours)
    else:
        assert k is None
    return q, k


HEADS = [(32, 4, 64), (7, 1, 64), (1, 0, 64), (16, 16, 128), (5, 5, 128), (8, 2, 256), (3, 1, 256)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("T", [1, 2, 65])
@pytest.mark.parametrize("heads,H,D", HEADS)
def test_heads_and_tokens(heads, H, D, T, neighbours, dtype):
    qkv, pos, gains = inputs(D + heads + T, T, heads, H, D, dtype)
    check(qkv, pos, gains, heads, H, moin.rope_frequencies(D), neighbours=neighbours)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("rot,D", [(16, 64), (32, 64), (48, 64), (16, 128), (64, 128), (112, 128), (16, 256), (240, 256)])
def test_rotations_of_some_channels(rot, D, neighbours, norm):
    qkv, pos, gains = inputs(rot + D, 37, 6, 2, D)
    check(qkv, pos, gains, 6, 2, moin.rope_frequencies(rot, 500.0), norm=norm, neighbours=neighbours, eps=0.3)


def test_many_tokens_take_all_heads_of_a_token_to_a_wave():
    qkv, pos, gains = inputs(3, 3000, 9, 3, 128)
    check(qkv, pos, gains, 9, 3, moin.rope_frequencies(128))


def test_norms_alone_and_gains_left_out():
    qkv, pos, gains = inputs(4, 70, 9, 3, 64)
    q, k = moin.moin_qk_norm_rope(ctx(), qkv[:, :9], qkv[:, 9:12])
    compare(q, qkv[:, :9], None, None, None, 1e-6, True, False)
    compare(k, qkv[:, 9:12], None, None, None, 1e-6, True, False)
    q, k = moin.moin_qk_norm_rope(ctx(), qkv[:, :9], qkv[:, 9:12], k_gain=gains[1])
    compare(q, qkv[:, :9], None, None, None, 1e-6, True, False)
    compare(k, qkv[:, 9:12], None, None, gains[1], 1e-6, True, False)


def test_far_and_negative_positions():
    qkv, pos, gains = inputs(5, 12, 4, 2, 128)
    pos.copy_(torch.tensor([0, 1, -1, -7, 10 ** 5, 10 ** 6, 2 ** 24 + 1, 2 ** 30, 2 ** 31 - 1, -2 ** 31, 131071, 3], dtype=I32))
    check(qkv, pos, gains, 4, 2, moin.rope_frequencies(128))
    check(qkv, pos, gains, 4, 2, moin.rope_frequencies(128, 1e6), neighbours=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size,eps", [(1e30, 1e-6), (2e38, 1e-6), (1e-18, 1e-30), (1e-25, 1e-38), (1e19, 1.0)])
def test_magnitudes_whose_squares_fp32_does_not_hold(size, eps, dtype):
    qkv, pos, gains = inputs(11, 9, 6, 2, 64)
    x = (qkv.float() / qkv.float().abs().amax() * size)
    x[0] = qkv[0]
    check(x.to(dtype), pos, gains, 6, 2, moin.rope_frequencies(64), eps=eps)


def test_heads_do_not_depend_on_others_magnitudes():
    qkv, pos, gains = inputs(12, 600, 30, 2, 64)
    kw = dict(positions=pos, freqs=moin.rope_frequencies(64), q_gain=gains[0], k_gain=gains[1])
    want, _ = moin.moin_qk_norm_rope(ctx(), qkv[:, :30], qkv[:, 30:32], **kw)
    qkv[:, 0] *= 1e30
    got, _ = moin.moin_qk_norm_rope(ctx(), qkv[:, :30], qkv[:, 30:32], **kw)
    assert torch.equal(got[:, 1:], want[:, 1:])


def test_more_tokens_than_a_launch_takes():
    T, far = 2 ** 24 + 3, 2 ** 24 - 2
    q = torch.zeros((T, 1, 64), dtype=BF16, device="cuda")
    pos = torch.arange(T, dtype=I32, device="cuda")
    qkv, _, gains = inputs(13, 5, 1, 0, 64)
    q[:5], q[far:] = qkv[:, :1], qkv[:, :1]
    kw = dict(freqs=moin.rope_frequencies(64), q_gain=gains[0])
    got, _ = moin.moin_qk_norm_rope(ctx(), q, None, positions=pos, **kw)
    for at in (0, far):
        want, _ = moin.moin_qk_norm_rope(ctx(), qkv[:, :1], None, positions=pos[at:at + 5].clone(), **kw)
        assert torch.equal(got[at:at + 5], want)
    assert not got[5:far].any()


def test_position_zero_passes_everything():
    qkv, pos, gains = inputs(6, 5, 4, 2, 64)
    pos.zero_()
    q, k = moin.moin_qk_norm_rope(ctx(), qkv[:, :4], qkv[:, 4:6], positions=pos, freqs=moin.rope_frequencies(64), norm=False)
    assert torch.equal(q, qkv[:, :4]) and torch.equal(k, qkv[:, 4:6])


def test_in_place_leaves_the_values_alone():
    qkv, pos, gains = inputs(7, 90, 8, 2, 64)
    kw = dict(positions=pos, freqs=moin.rope_frequencies(64), q_gain=gains[0], k_gain=gains[1])
    q, k = moin.moin_qk_norm_rope(ctx(), qkv[:, :8], qkv[:, 8:10], **kw)
    own = qkv.clone()
    a, b = own[:, :8], own[:, 8:10]
    ra, rb = moin.moin_qk_norm_rope(ctx(), a, b, out=(a, b), **kw)
    assert ra is a and rb is b and torch.equal(a, q) and torch.equal(b, k) and torch.equal(own[:, 10:], qkv[:, 10:])


def test_zeros_infinities_and_nans_stay_in_their_heads():
    qkv, pos, gains = inputs(8, 4, 6, 2, 64)
    qkv[0, 0] = 0
    qkv[1, 2, 5] = float("nan")
    qkv[2, 7, 63] = float("inf")
    q, k = moin.moin_qk_norm_rope(ctx(), qkv[:, :6], qkv[:, 6:8], positions=pos, freqs=moin.rope_frequencies(64))
    assert (q[0, 0] == 0).all() and torch.isnan(q[1, 2]).all() and not torch.isfinite(k[2, 1]).all()
    q[1, 2], k[2, 1] = 0, 0
    assert torch.isfinite(q).all() and torch.isfinite(k).all()


def test_no_tokens_other_streams_and_graphs():
    qkv, pos, gains = inputs(9, 20, 8, 2, 128)
    f = moin.rope_frequencies(128)
    kw = dict(freqs=f, q_gain=gains[0], k_gain=gains[1])
    q, k = moin.moin_qk_norm_rope(ctx(), qkv[:0, :8], qkv[:0, 8:10], positions=pos[:0], **kw)
    assert q.shape == (0, 8, 128) and k.shape == (0, 2, 128)
    q, k = moin.moin_qk_norm_rope(ctx(), qkv[:, :8], qkv[:, 8:10], positions=pos, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a, b = moin.moin_qk_norm_rope(ctx(), qkv[:, :8], qkv[:, 8:10], positions=pos, **kw)
    side.synchronize()
    assert torch.equal(a, q) and torch.equal(b, k)
    out = (torch.empty_like(q), torch.empty_like(k))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        moin.moin_qk_norm_rope(ctx(), qkv[:, :8], qkv[:, 8:10], positions=pos, out=out, **kw)
    for i in range(3):
        qkv.copy_(torch.randn(qkv.shape, device="cuda"))
        pos.add_(17)
        graph.replay()
        want = moin.moin_qk_norm_rope(ctx(), qkv[:, :8], qkv[:, 8:10], positions=pos, **kw)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_refusals():
    qkv, pos, gains = inputs(10, 4, 8, 2, 64)
    f = moin.rope_frequencies(64)
    q, k = qkv[:, :8], qkv[:, 8:10]

    def run(q=q, k=k, **kw):
        return moin.moin_qk_norm_rope(ctx(), q, k, **kw)

    for kw in (dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(norm=False, q_gain=gains[0]),
               dict(positions=pos, freqs=moin.rope_frequencies(24)), dict(positions=pos, freqs=moin.rope_frequencies(128)),
               dict(q=qkv[:, :8, :32].contiguous(), k=None)):
        with pytest.raises(moin.MoinError) as e:
            run(**kw)
        assert e.value.code == -1
    lib, st = moin.load(), moin._stream_ptr()
    for dt, ostride in ((0, 640), (1, 768)):      # in place: fp32 over itself, other strides
        assert lib.moin_qk_norm_rope(ctx()._h, qkv.data_ptr(), None, dt, 640, 0, 2, 8, 0, 64, None, None, 0, 0, None, None, 1.0, qkv.data_ptr(), None,
                                     ostride, 0, st) == -1
    for kw in (dict(positions=pos), dict(freqs=f), dict(positions=pos[:3], freqs=f), dict(q=q[:3]), dict(q=q[0]), dict(q=qkv[:, 0:8:2]),
               dict(q_gain=gains[0][:32]), dict(out=(q,)), dict(out=(q[:, :4], k)), dict(q=q.cpu())):
        with pytest.raises(ValueError):
            run(**kw)
    for kw in (dict(q=q.half()), dict(q=q.float()), dict(positions=pos.long(), freqs=f), dict(out=(q.float(), k)), dict(q_gain=gains[0].float())):
        with pytest.raises(TypeError):
            run(**kw)
    with pytest.raises(TypeError):
        run(positions=pos, freqs=f.float())
    ctx().check()
