"""Tokens into the paged MXFP4 cache and back: the format against its definition in 64 bits, the layout byte by byte."""
import numpy as np
import pytest
import torch

import tests.four_bit as fb
from paper_2410_09687_amd import moin
from tests.gpu_common import ctx

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def values(rng, shape):
    """bf16 values over many magnitudes, with blocks of zeros, ties and subnormal ones among them."""
    x = rng.normal(size=shape) * 2.0 ** rng.integers(-20, 20, size=shape[:-1] + (1,))
    flat = x.reshape(-1, 32)
    flat[::11] = 0
    flat[3::13] = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, -0.25, -1.75, -5, 7], size=flat[3::13].shape)
    flat[5::17] *= 2.0 ** -128
    flat[6::19] = flat[6::19] / np.abs(flat[6::19]).max() * 3.3e38 if len(flat) > 6 else 0
    return torch.tensor(flat.reshape(shape), dtype=torch.float32).to(BF16)


def same(a, b):
    differ = int((~((a == b) | (np.isnan(a) & np.isnan(b)))).sum())
    assert differ == 0


def f64(t):
    return t.detach().cpu().double().numpy()


@pytest.mark.parametrize("page", [64, 128, 256])
@pytest.mark.parametrize("H,D,T", [(1, 64, 1), (4, 64, 130), (3, 128, 77), (2, 256, 65)])
def test_append_holds_the_definition_and_nothing_else_moves(H, D, T, page):
    rng = np.random.default_rng(D + T + page)
    n_pages = T // page + 3
    k, v = values(rng, (T, H, D)), values(rng, (T, H, D))
    slots = rng.permutation(n_pages * page)[:T].astype(np.int32)
    pages = moin.KVPages.empty(n_pages, H, D, page)
    start = torch.tensor(rng.integers(0, 256, pages.data.shape), dtype=torch.uint8)
    pages.data.copy_(start)
    moin.moin_kv_append(ctx(), pages, k.cuda(), v.cuda(), torch.tensor(slots).cuda())
    ctx().check()
    gk, gv = fb.decode_pages(pages.data.cpu().numpy(), n_pages, H, D, page)
    wk, wv = fb.held(f64(k)), fb.held(f64(v))
    same(gk[slots], wk)
    same(gv[slots], wv)
    ok, ov = fb.decode_pages(start.numpy(), n_pages, H, D, page)
    rest = np.setdiff1d(np.arange(n_pages * page), slots)
    same(gk[rest], ok[rest])
    same(gv[rest], ov[rest])
    bk, bv = moin.moin_kv_gather(ctx(), pages, torch.tensor(slots).cuda())
    same(f64(bk), wk)
    same(f64(bv), wv)


def test_blocks_with_nan_or_infinity_become_nan_and_neighbours_do_not():
    k = torch.ones((3, 2, 128), dtype=BF16)
    v = torch.ones((3, 2, 128), dtype=BF16)
    k[0, 1, 40], v[2, 0, 3], v[1, 1, 127] = float("nan"), float("inf"), float("-inf")
    pages = moin.KVPages.empty(1, 2, 128)
    slots = torch.tensor([5, 6, 63], dtype=torch.int32, device="cuda")
    moin.moin_kv_append(ctx(), pages, k.cuda(), v.cuda(), slots)
    bk, bv = (x.cpu() for x in moin.moin_kv_gather(ctx(), pages, slots))
    want_k, want_v = torch.ones_like(k), torch.ones_like(v)
    want_k[0, 1, 32:64] = want_v[2, 0, :32] = want_v[1, 1, 96:] = float("nan")
    assert torch.equal(torch.isnan(bk), torch.isnan(want_k)) and torch.equal(torch.isnan(bv), torch.isnan(want_v))
    assert (bk[~torch.isnan(bk)] == 1).all() and (bv[~torch.isnan(bv)] == 1).all()


def test_columns_of_one_projections_output():
    T, H, D = 50, 4, 64
    rng = np.random.default_rng(1)
    qkv = values(rng, (T, 3 * H, D)).cuda()
    slots = torch.arange(T, dtype=torch.int32, device="cuda") + 9
    pages = moin.KVPages.empty(1, H, D)
    moin.moin_kv_append(ctx(), pages, qkv[:, H:2 * H], qkv[:, 2 * H:], slots)
    k, v = moin.moin_kv_gather(ctx(), pages, slots)
    same(f64(k), fb.held(f64(qkv[:, H:2 * H])))
    same(f64(v), fb.held(f64(qkv[:, 2 * H:])))


def test_slots_of_none_and_outside():
    pages = moin.KVPages.empty(2, 1, 64)
    pages.data.zero_()
    x = torch.ones((4, 1, 64), dtype=BF16, device="cuda")
    slots = torch.tensor([-1, 3, -1, 127], dtype=torch.int32, device="cuda")
    moin.moin_kv_append(ctx(), pages, x, x, slots)
    ctx().check()
    k, _ = moin.moin_kv_gather(ctx(), pages, slots)
    assert f64(k)[:, 0, 0].tolist() == [0, 1, 0, 1]
    ctx().check()
    before = pages.data.clone()
    for bad in (128, -2, 2 ** 31 - 1, -2 ** 31):
        slots = torch.tensor([bad], dtype=torch.int32, device="cuda")
        moin.moin_kv_append(ctx(), pages, x[:1], x[:1], slots)
        with pytest.raises(moin.MoinError):
            ctx().check()
        k, v = moin.moin_kv_gather(ctx(), pages, slots)
        with pytest.raises(moin.MoinError):
            ctx().check()
        assert (k == 0).all() and (v == 0).all()
    assert torch.equal(before, pages.data)


def test_an_empty_call_and_another_stream():
    pages = moin.KVPages.empty(4, 2, 64)
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    none = torch.empty((0, 2, 64), dtype=BF16, device="cuda")
    moin.moin_kv_append(ctx(), pages, none, none, empty)
    assert moin.moin_kv_gather(ctx(), pages, empty)[0].shape == (0, 2, 64)
    side = torch.cuda.Stream()
    x = torch.randn((200, 2, 64), device="cuda").to(BF16)
    slots = torch.randperm(256, device="cuda")[:200].to(torch.int32)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        moin.moin_kv_append(ctx(), pages, x, x, slots)
        k, v = moin.moin_kv_gather(ctx(), pages, slots)
    side.synchronize()
    same(f64(k), fb.held(f64(x)))
    assert torch.equal(k, v)


def test_a_cache_beyond_four_gigabytes():
    """Offsets of records that do not fit 32 bits."""
    n_pages = (5 << 30) // (4 * 8704 * 4)
    pages = moin.KVPages.empty(n_pages, 4, 128, 256)
    assert pages.data.numel() > 2 ** 32
    T = 70
    x = torch.randn((T, 4, 128), device="cuda").to(BF16)
    slots = torch.arange(T, dtype=torch.int32, device="cuda") + (n_pages * 256 - T)
    low = torch.arange(T, dtype=torch.int32, device="cuda")
    moin.moin_kv_append(ctx(), pages, -x, x, low)
    moin.moin_kv_append(ctx(), pages, x, -x, slots)
    ctx().check()
    want = fb.held(f64(x))
    for at, sign in ((slots, 1), (low, -1)):
        k, v = moin.moin_kv_gather(ctx(), pages, at)
        same(f64(k), sign * want)
        same(f64(v), -sign * want)


def test_refusals():
    pages = moin.KVPages.empty(1, 2, 64)
    x = torch.zeros((3, 2, 64), dtype=BF16, device="cuda")
    slots = torch.arange(3, dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        moin.moin_kv_append(ctx(), pages, x.float(), x, slots)
    with pytest.raises(TypeError):
        moin.moin_kv_append(ctx(), pages, x, x, slots.long())
    with pytest.raises(ValueError):
        moin.moin_kv_append(ctx(), pages, x[:, :1], x, slots)
    with pytest.raises(ValueError):
        moin.moin_kv_append(ctx(), pages, x[:2], x[:2], slots)
    with pytest.raises(ValueError):
        moin.moin_kv_append(ctx(), pages, x.cpu(), x, slots)
    with pytest.raises(ValueError):   # channels that are not contiguous
        moin.moin_kv_append(ctx(), pages, torch.zeros((3, 64, 2), dtype=BF16, device="cuda").transpose(1, 2), x, slots)
    wide = torch.zeros((3, 132), dtype=BF16, device="cuda")
    for odd in (wide[:, 2:130], wide[:, :128]):   # a start that is not 16-byte aligned, rows that are not
        with pytest.raises(moin.MoinError) as e:
            moin.moin_kv_append(ctx(), pages, odd.view(3, 2, 64) if odd.is_contiguous() else odd.unflatten(1, (2, 64)), x, slots)
        assert e.value.code == -1
    for args in ((1, 2, 96), (1, 0, 64), (1, 2, 64, 32)):
        with pytest.raises(ValueError):
            moin.KVPages.empty(*args)
    with pytest.raises(ValueError):
        moin.KVPages(torch.zeros(100, dtype=torch.uint8, device="cuda"), 2, 64)
