"""Attention over the paged E4M3 cache against its definition in 64 bits, on the values that the cache's bytes stand for.

Bounds as for the 4-bit cache: a weight's relative error is at most `rel` (what fp32 scores and sums may cause, four_bit.attention),
twice that after the division by their sum; a bf16 result's weights are rounded too and so is the result, each by at most 2^-8 of itself."""
import numpy as np
import pytest
import torch

import tests.eight_bit as eb
import tests.four_bit as fb
from paper_2410_09687_amd import moin
from tests.gpu_common import ctx
from tests.test_gpu_kv_attention import compare

pytestmark = pytest.mark.gpu
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def dev(x):
    return torch.tensor(np.asarray(x), dtype=I32).cuda()


class Step:
    """Requests with keys in a cache whose other bytes are garbage, and the plan of a step that adds their last tokens."""

    def __init__(self, seed, kv, new, heads, H, D, page=64, loud=1.0):
        rng = np.random.default_rng(seed)
        self.kv, self.new, self.heads, self.H, self.D, self.page = np.array(kv), np.array(new), heads, H, D, page
        S, self.T = len(kv), int(np.sum(new))
        end = self.kv + self.new
        have, every = -(-self.kv // page), -(-end // page)
        self.n_pages = int(every.sum()) + 4
        order = rng.permutation(self.n_pages)
        table = np.full((S, int(every.max()) + 1), -1)
        at = 0
        for s in range(S):
            table[s, :have[s]] = order[at:at + have[s]]
            at += have[s]
        self.table = dev(table)
        self.pages = moin.KV8Pages.empty(self.n_pages, H, D, page)
        self.pages.data.copy_(torch.tensor(rng.integers(0, 256, self.pages.data.shape), dtype=torch.uint8))
        self.plan = moin.KVPlan(ctx())
        self.off, self.lens, self.slots, _ = self.plan.build(dev(self.kv), dev(self.new), self.T, self.table, dev(order[at:]),
                                                             dev([len(order) - at]), n_pages=self.n_pages, page_tokens=page,
                                                             n_heads=heads, n_kv=H, max_new=int(self.new.max()))
        ctx().check()
        t = self.table.cpu().numpy()
        self.all_slots = [t[s][np.arange(end[s]) // page] * page + np.arange(end[s]) % page for s in range(S)]
        self.every_slot, self.every_off = dev(np.concatenate(self.all_slots)), dev(np.concatenate([[0], np.cumsum(end)]))
        n = self.every_slot.numel()
        # (from block to block of other magnitudes, so that their scales differ)
        size = np.exp(rng.normal(size=(n, H, 1)) * 0.2) * np.exp2(rng.integers(-2, 3, (n // 64 + 1, H, 1)))[np.arange(n) // 64]
        self.k = torch.tensor(rng.normal(size=(n, H, D)) * loud * np.minimum(size, 2)).to(BF16).cuda()
        self.v = torch.tensor((rng.normal(size=(n, H, D)) + 0.3) * size).to(BF16).cuda()
        self.fill()
        self.q = torch.tensor(rng.normal(size=(self.T, heads, D))).to(BF16).cuda()

    def fill(self):
        moin.moin_kv8_append(ctx(), self.pages, self.k, self.v, self.every_off, self.every_slot)

    def run(self, **kw):
        return moin.moin_kv8_attention(ctx(), self.plan, self.pages, self.q, self.table, want_lse=True, **kw)

    def want(self, scale=None, window=0):
        k, v = eb.Cache(self.pages.data.cpu().numpy(), self.n_pages, self.H, self.D, self.page).values()
        q = self.q.cpu().double().numpy()
        off = self.off.cpu().numpy()
        scale = self.D ** -0.5 if scale is None else scale
        parts = [fb.attention(q[off[s]:off[s + 1]], k[sl], v[sl], int(self.kv[s]), scale, window) for s, sl in enumerate(self.all_slots)]
        return [np.concatenate(x) for x in zip(*parts)]

    def check(self, y_dtype=BF16, scale=None, window=0, **kw):
        y, lse = self.run(y_dtype=y_dtype, scale=scale, window=window, **kw)
        ctx().check()
        compare(y, lse, self.want(scale, window))
        return y, lse


HEADS = [(32, 4, 64), (8, 8, 64), (7, 1, 64), (16, 2, 128), (5, 5, 128), (48, 1, 128), (8, 2, 256), (3, 1, 256)]


@pytest.mark.parametrize("y", [BF16, F32])
@pytest.mark.parametrize("heads,H,D", HEADS)
def test_single_tokens(heads, H, D, y):
    Step(D + heads, [0, 1, 62, 63, 64, 65, 300, 1000], [1] * 8, heads, H, D).check(y)


@pytest.mark.parametrize("y", [BF16, F32])
@pytest.mark.parametrize("heads,H,D", HEADS)
def test_several_tokens_and_prompts(heads, H, D, y):
    Step(D * 2 + heads, [0, 100, 0, 7, 130, 63], [5, 4, 70, 0, 1, 66], heads, H, D, page=128).check(y)


@pytest.mark.parametrize("page", [64, 128, 256])
@pytest.mark.parametrize("window", [1, 2, 64, 65, 200, 5000])
def test_windows(window, page):
    Step(window + page, [0, 1, 150, 700, 64, 400], [1, 3, 2, 1, 90, 40], 8, 2, 64, page).check(window=window)


@pytest.mark.parametrize("heads,H,D", [(8, 1, 64), (16, 1, 128), (4, 2, 256), (40, 1, 64)])
@pytest.mark.parametrize("new", [1, 2, 3, 40])
def test_long_axes_are_walked_in_parts(heads, H, D, new):
    s = Step(new + D, [5000, 300, 2047], [new, new, new], heads, H, D)
    a = s.check(F32)
    b = s.run(y_dtype=F32)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    s.check(window=1000)


def test_many_requests():
    rng = np.random.default_rng(8)
    Step(9, rng.integers(0, 300, 700), rng.integers(0, 2, 700), 4, 2, 64).check()


@pytest.mark.parametrize("heads,H,D", [(8, 2, 64), (3, 3, 128), (200, 1, 64), (130, 2, 64)])
@pytest.mark.parametrize("S", [2, 7, 64, 65])
def test_tiles_of_several_requests_are_all_taken(S, heads, H, D):
    """Lists of tiles that go by the keys that they see (up to 64 requests), ties and requests without tokens among them: no row is left out."""
    rng = np.random.default_rng(S + heads)
    new = rng.choice([0, 9, 9, 40, 64, 65, 70], S)
    new[0] = 70
    kv = rng.choice([0, 0, 31, 64, 300], S)
    s = Step(S, kv if S < 64 else kv % 65, new if S < 64 else new % 41 + (np.arange(S) == 1) * 9, heads, H, D)
    out = torch.full((s.T, heads, D), float("nan"), dtype=BF16, device="cuda")
    s.check(out=out)


def test_loud_scores_and_other_scales():
    s = Step(11, [200, 50, 1000], [1, 60, 3], 8, 2, 64, loud=30.0)
    s.check(F32)
    s.check(scale=2.0)
    s.check(scale=1e-6, y_dtype=F32)


def test_equal_scores_give_the_mean():
    s = Step(12, [999], [1], 4, 1, 64)
    s.q.zero_()
    y, lse = s.check(F32)
    assert np.allclose(lse.cpu(), np.log(1000.0), rtol=1e-6)


@pytest.mark.parametrize("heads,H,D", [(8, 2, 64), (4, 2, 128), (4, 1, 256)])
@pytest.mark.parametrize("window", [0, 30])
def test_a_block_of_nans_reaches_the_rows_that_see_a_key_of_it_and_no_others(heads, H, D, window):
    s = Step(13 + D, [100, 0, 64, 400, 200], [40, 90, 1, 1, 3], heads, H, D)
    first = np.cumsum([0] + [len(x) for x in s.all_slots])
    s.v[first[0] + 130, 0, 33] = float("nan")       # values: for the request's last tokens
    s.k[first[1] + 70, H - 1, 2] = float("inf")     # a key: all channels of its rows
    s.v[first[2] + 64, 0, D - 1] = float("inf")     # a request's last token, seen by itself alone
    s.v[first[3] + 5, 0, 0] = float("nan")
    s.k[first[4] + 201, 0, 0] = float("nan")        # between the step's own tokens
    s.fill()
    for y in (BF16, F32):
        got, _ = s.check(y, window=window)
    assert torch.isnan(got).any() and not torch.isnan(got).all()


def test_rows_that_see_nothing_are_zeros():
    """More new tokens than keys: what a table says of a request that was not served."""
    plan = moin.KVPlan(ctx())
    table = dev([[0, -1], [1, -1], [2, -1]])
    off, lens, slots, left = plan.build(dev([10, 60, 3]), dev([1, 30, 70]), 101, table, dev([3]), dev([1]), n_pages=4, page_tokens=64,
                                        n_heads=2, n_kv=1, max_new=70)
    with pytest.raises(moin.MoinError):
        ctx().check()
    assert lens.cpu().tolist() == [11, 90, 3]
    pages = moin.KV8Pages.empty(4, 1, 64)
    pages.data.fill_(255)
    x = torch.ones((101, 1, 64), dtype=BF16, device="cuda")
    moin.moin_kv8_append(ctx(), pages, x[:70], x[:70], dev([0, 10, 70]), dev(list(range(10)) + list(range(64, 124))))
    moin.moin_kv8_append(ctx(), pages, x, x, off, slots)
    q = torch.randn((101, 2, 64), device="cuda").to(BF16)
    y = torch.full((101, 2, 64), 7.0, dtype=BF16, device="cuda")
    y, lse = moin.moin_kv8_attention(ctx(), plan, pages, q, table, out=y, want_lse=True)
    ctx().check()
    assert (y[31:] == 0).all() and torch.isneginf(lse[31:]).all() and (y[:31] == 1).all()
    assert torch.isfinite(lse[:31]).all()


@pytest.mark.parametrize("new", [1, 40])
def test_pages_that_do_not_exist_count_as_unseen(new):
    s = Step(15, [200], [new], 4, 1, 64)
    whole = s.want()
    s.table[0, 1] = 10 ** 6
    y, lse = s.run()
    with pytest.raises(moin.MoinError):
        ctx().check()
    assert torch.isfinite(y).all()
    s.table[0, 1] = -1
    z, _ = s.run()
    with pytest.raises(moin.MoinError):
        ctx().check()
    assert torch.equal(y, z)
    assert np.abs(y.cpu().double().numpy() - whole[0]).max() > 1e-3


def test_strided_queries_given_outputs_other_streams():
    s = Step(16, [100, 30], [1, 33], 8, 2, 64)
    y, lse = s.run()
    wide = torch.zeros((s.T, 12, 64), dtype=BF16, device="cuda")
    wide[:, :8] = s.q
    out = torch.empty_like(y)
    z, _ = moin.moin_kv8_attention(ctx(), s.plan, s.pages, wide[:, :8], s.table, out=out)
    assert z is out and torch.equal(y, z)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z, l2 = s.run()
    side.synchronize()
    assert torch.equal(y, z) and torch.equal(lse, l2)


def test_a_captured_call_replays():
    s = Step(17, [3000, 500, 64], [1, 1, 1], 8, 1, 64)
    y = torch.empty((3, 8, 64), dtype=BF16, device="cuda")
    lib = lambda: moin.moin_kv8_attention(ctx(), s.plan, s.pages, s.q, s.table, out=y)   # noqa: E731
    lib()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lib()
    for i in range(4):
        s.q.copy_(torch.randn(s.q.shape, device="cuda"))
        y.zero_()
        g.replay()
        got = y.clone()
        lib()
        torch.cuda.synchronize()
        assert torch.equal(got, y)


def test_a_page_beyond_4_gb():
    """Offsets that pass 32 bits: pages of 8 heads of 256 channels at the end of a large pool."""
    page = moin.KV8Pages.page_bytes(8, 256, 256)
    n = (5 << 30) // page
    pages = moin.KV8Pages.empty(n, 8, 256, 256)
    table, plan = dev([[n - 1, -1]]), moin.KVPlan(ctx())
    off, lens, slots, _ = plan.build(dev([0]), dev([300]), 300, table, dev([1, n - 2]), dev([2]), n_pages=n, page_tokens=256, n_heads=8, n_kv=8)
    assert slots.cpu()[0] == (n - 2) * 256
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((300, 24, 256), device="cuda", generator=g).to(BF16)
    moin.moin_kv8_append(ctx(), pages, x[:, :8], x[:, 8:16], off, slots)
    y, lse = moin.moin_kv8_attention(ctx(), plan, pages, x[:, 16:], table, want_lse=True)
    ctx().check()
    k, v = (t.cpu().double().numpy() for t in moin.moin_kv8_gather(ctx(), pages, slots))
    compare(y, lse, fb.attention(x[:, 16:].cpu().double().numpy(), k, v, 0, 1 / 16, 0))


def test_refusals():
    s = Step(18, [10], [2], 8, 2, 64)
    run = lambda **kw: moin.moin_kv8_attention(ctx(), kw.pop("plan", s.plan), kw.pop("pages", s.pages), kw.pop("q", s.q),   # noqa: E731
                                               kw.pop("table", s.table), **kw)
    run()
    for kw in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1),
               dict(q=s.q[:, :4]), dict(plan=moin.KVPlan(ctx()), q=s.q[:0], table=s.table[:0]), dict(pages=moin.KV8Pages.empty(4, 2, 64, 128)),
               dict(pages=moin.KV8Pages.empty(4, 1, 64)), dict(table=torch.zeros((1, 9), dtype=I32, device="cuda"))):
        with pytest.raises(moin.MoinError) as e:
            run(**kw)
        assert e.value.code == -1
    for kw in (dict(q=s.q[:1]), dict(q=s.q[..., :32]), dict(table=s.table[:0]), dict(out=torch.empty((2, 8, 64), device="cuda")),
               dict(q=s.q.cpu())):
        with pytest.raises(ValueError):
            run(**kw)
    for kw in (dict(q=s.q.float()), dict(y_dtype=torch.float16), dict(table=s.table.long()), dict(pages=moin.KVPages.empty(4, 2, 64))):
        with pytest.raises(TypeError):
            run(**kw)
    with pytest.raises(TypeError):
        moin.moin_kv_attention(ctx(), s.plan, s.pages, s.q, s.table)
    ctx().check()
