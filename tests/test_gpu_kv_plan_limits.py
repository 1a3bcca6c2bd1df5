"""Sizes of a step that the library does not plan are refused before anything is launched, those whose products pass 64 bits among them."""
import pytest
import torch

from paper_2410_09687_amd import moin
from tests.gpu_common import ctx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,max_new,heads,S,max_pages,page", [
    (1 << 61, 1, 8, 2, 4, 64), ((1 << 61) + 1, 8, 8, 2, 4, 64), (1 << 62, 1, 4, 2, 4, 64), ((1 << 63) - 1, 1, 2, 2, 4, 64),
    (1 << 31, 1, 1, 2, 4, 64), ((1 << 31) - 1, 1, 8, 2, 4, 64), (2, 1, 1 << 17, 2, 4, 64),
    (2, 1, 8, (1 << 31) - 1, (1 << 31) - 1, 256), (2, 1, 8, (1 << 31) - 1, 2, 64), (2, 1, 8, 1, 1 << 25, 64)])
def test_sizes_beyond_the_limits(T, max_new, heads, S, max_pages, page):
    lib, plan = moin.load(), moin.KVPlan(ctx())
    some = torch.zeros(64, dtype=torch.int32, device="cuda").data_ptr()
    assert lib.moin_kv_plan_build(ctx()._h, plan._h, some, some, S, T, max_new, heads, 1, page, 8, some, max_pages, some, 8, some, some, some, some,
                                  some, None) == -1
    ctx().check()
