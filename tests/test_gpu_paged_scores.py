"""spec_paged_attention at the ends of the numbers' ranges: scores beyond fp32, the smallest scales, weights far below the largest."""
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


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows", [1, 9, 40, 130])
@pytest.mark.parametrize("at", [0, 2500])
def test_many_small_weights_beside_a_large_one(dtype, hd, rows, at):
    """One position has a score 18 above all others (2^26 times their weight) and values of zero: what comes out is the others' 1e-5 of the
    weight.  fp16 weights are held with the largest at 2^7 or more, so a rounding is 2^-25 / 2^7 of the largest weight at most where that is more
    than 2^-11 of the weight itself."""
    n, heads = 4000, 2
    c = Case(dtype, heads, 1, hd, 64, [rows], [n + rows], seed=rows, extra_rows=0)
    page, at_page = int(c.table[0, at // 64]), at % 64
    c.k.zero_()
    c.v.copy_((torch.rand(c.v.shape, generator=c.g) * 100 + 50).to(c.td))
    c.k[page, at_page, 0, 0] = 18 * hd ** 0.5
    c.v[page, at_page] = 0
    q = c.rows_of(heads)
    q[:, :, 0] = 1
    want, bound = ref.attention(c.k, c.v, c.table, c.batch, q, hd ** -0.5, 0)
    if dtype == "fp16":
        bound = bound + 2.0 ** -32 * c.v.double().sum((0, 1, 2))
    got = attend(c, q)
    assert float((bound / want.abs()).max()) < 0.03
    assert bool(((got - want).abs() <= bound).all())
