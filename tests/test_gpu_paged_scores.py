"""spec_paged_attention at the ends of the numbers' ranges: scores beyond fp32, the smallest scales."""
import pytest
import torch

import paged_reference as ref
from test_gpu_paged import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROWS = [([1], [40]), ([5, 2], [3000, 60]), ([100], [2300]), ([300, 100], [300, 2300])]  # few rows and many, cut tiles and whole ones


def attend(c, q, **kw):
    from paper_2310_18813_amd import binding as B
    cache, batch = c.on_gpu(B)
    return B.spec_paged_attention(cache, batch, q.to(DEV), **kw).cpu().double()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,lens", ROWS)
def test_scores_beyond_fp32_are_not_taken_for_nothing_seen(dtype, rows, lens):
    """scale * q.k is infinite in fp32, so a softmax of it is NaN; rows at negative positions still see nothing."""
    c = Case(dtype, 4, 1, 64, 16, rows + [3], lens + [1], seed=1, extra_rows=0)
    c.k.copy_(torch.where(torch.isnan(c.k), c.k, torch.full_like(c.k, 1e5)))
    got = attend(c, torch.full((c.T, 4, 64), 1e5, dtype=c.td), scale=1e30)
    n = sum(rows)
    assert bool(torch.isnan(got[:n]).all()) and not bool(got[n:n + 2].any()) and bool(torch.isnan(got[n + 2]).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,lens", ROWS)
@pytest.mark.parametrize("scale", [1e-30, 1.2e-38, 1e-40])
def test_the_smallest_scales_give_every_position_the_same_weight(dtype, rows, lens, scale):
    c = Case(dtype, 4, 1, 64, 16, rows, lens, seed=2, extra_rows=0)
    q = c.rows_of(4)
    want, bound = ref.attention(c.k, c.v, c.table, c.batch, q, scale, 0)
    got = attend(c, q, scale=scale)
    assert bool(((got - want).abs() <= bound).all())
