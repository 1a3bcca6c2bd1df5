"""Attention over the paged MXFP4 cache where requests add many tokens at once (tiles of 128 rows, in parts where the keys are long), and
scores that rise, fall and jump along the keys, against the definition in 64 bits; bounds as in test_gpu_kv_attention."""
import numpy as np
import pytest
import torch

from paper_2410_09687_amd import moin
from tests.gpu_common import ctx
from tests.test_gpu_kv_attention import BF16, F32, Step

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 64), (2, 2, 128), (4, 1, 256)]


@pytest.mark.parametrize("heads,H,D", HEADS)
@pytest.mark.parametrize("kv,new", [([2500], [40]), ([0, 1900, 300], [130, 37, 64]), ([700, 5, 3000, 64], [33, 1, 50, 17])])
def test_tiles_in_parts(heads, H, D, kv, new):
    s = Step(D + len(kv), kv, new, heads, H, D, page=128)
    a = s.check(F32)
    b = s.run(y_dtype=F32)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    s.check(BF16)
    s.check(F32, window=500)


def ramp(kind, n, rng):
    t = np.arange(n) / max(n - 1, 1)
    return {"up": 120 * t - 60, "down": 60 - 120 * t, "steps": 8.0 * (np.arange(n) // 64), "spikes": np.where(rng.random(n) < 0.01, 50.0, -3.0),
            "far down": np.full(n, -700.0) + 5 * t}[kind]


@pytest.mark.parametrize("y", [BF16, F32])
@pytest.mark.parametrize("kind", ["up", "down", "steps", "spikes", "far down"])
@pytest.mark.parametrize("heads,H,D", HEADS)
def test_scores_that_move_along_the_keys(heads, H, D, kind, y):
    rng = np.random.default_rng(D)
    s = Step(D + 7, [600, 900, 130], [1, 40, 3], heads, H, D)
    # the first channel carries the score: q there is 8, the others are quiet
    s.q.mul_(0.1)
    s.q[..., 0] = 8.0
    at = 0
    for slots in s.all_slots:
        n = len(slots)
        s.k[at:at + n, :, 0] = torch.tensor(ramp(kind, n, rng) * D ** 0.5 / 8).to(BF16).cuda()[:, None]
        at += n
    s.fill()
    s.check(y)


@pytest.mark.parametrize("heads,H,D", HEADS)
def test_blocks_of_nans_inside_a_prompt(heads, H, D):
    s = Step(D + 1, [0, 1000], [200, 60], heads, H, D)
    s.v[70, 0, 5] = float("nan")             # the first request's: rows 0 .. 69 do not see it
    s.k[199, H - 1, 3] = float("inf")        # its last token, which nobody but itself sees
    s.v[200 + 10, H - 1, D - 1] = float("inf")   # early in the second's: all rows without a window, none with one
    s.fill()
    for window in (0, 64):
        y, _ = s.check(F32, window=window)
        assert torch.isnan(y).any() and not torch.isnan(y).all()


@pytest.mark.parametrize("heads,H,D", HEADS)
@pytest.mark.parametrize("entry", [0, 2, 3])
def test_a_page_that_does_not_exist_counts_as_unseen_by_a_prompt(heads, H, D, entry):
    """The same as a window or a shorter prefix would leave: what stands in other pages reaches nobody."""
    s = Step(D + 2, [210], [40], heads, H, D)
    pages = s.pages.data.view(s.n_pages, -1)
    spare = [i for i in range(s.n_pages) if i not in s.table[0].tolist()]
    pages[spare] = 255                       # NaN everywhere
    if s.table[0].tolist().count(0):         # page 0 is one of the unused ones
        other = spare[0]
        pages[other], pages[0] = pages[0].clone(), torch.full_like(pages[0], 255)
        s.table[s.table == 0] = other
    s.table[0, entry] = -1
    y, lse = s.run(y_dtype=F32)
    with pytest.raises(moin.MoinError):
        ctx().check()
    assert torch.isfinite(y).all() and torch.isfinite(lse).all()
    s.table[0, entry] = s.n_pages
    z, l2 = s.run(y_dtype=F32)
    with pytest.raises(moin.MoinError):
        ctx().check()
    assert torch.equal(y, z) and torch.equal(lse, l2)


def test_long_and_short_prompts_together():
    rng = np.random.default_rng(3)
    kv, new = rng.integers(0, 200, 40), rng.integers(1, 50, 40)
    kv[7], new[7] = 4000, 129
    s = Step(4, kv, new, 4, 2, 64)
    s.check(BF16)
    s.check(F32, window=333)
