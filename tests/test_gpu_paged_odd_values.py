"""spec_paged_attention beside infinities and NaN in the cache: what a row does not see never reaches it, what it sees shows, in whichever tile, step or
chunk of the work it lies."""
import math

import pytest
import torch

import paged_reference as ref
from test_gpu_paged import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ODD = (math.nan, math.inf, -math.inf)


def attend(c, q, window=0, **kw):
    from paper_2310_18813_amd import binding as B
    cache, batch = c.on_gpu(B)
    out = torch.full(q.shape, 7.0, dtype=c.td, device=DEV)
    return B.spec_paged_attention(cache, batch, q.to(DEV), window=window, out=out, **kw).cpu().double()


def check_odd(got, want, bound):
    """the same infinities and NaN, the rest within the bound"""
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.nan_to_num(got[odd], nan=5.0, posinf=1.0, neginf=-1.0), torch.nan_to_num(want[odd], nan=5.0, posinf=1.0, neginf=-1.0))
    assert bool(torch.isfinite(got[~odd]).all())
    assert bool(((got - want).abs()[~odd] <= bound[~odd]).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads,kv_heads,rows", [(2, 2, 1), (16, 1, 1), (64, 2, 1), (128, 1, 2)])
@pytest.mark.parametrize("window,lens", [(40, [100, 95, 72, 73, 1987]), (13, [100]), (1700, [5000, 1733, 4001])])
def test_what_lies_in_front_of_the_window_never_reaches_a_tile_of_one_position(dtype, hd, heads, kv_heads, rows, window, lens):
    """Plain decoding with a window: every place in front of it is odd, as where a slid-out page went to another owner."""
    c = Case(dtype, heads, kv_heads, hd, 16, [rows] * len(lens), lens, seed=window, ragged=False)
    for b, n in enumerate(lens):
        for p in range(0, n - rows - window + 1):
            c.v[c.table[b, p // 16], p % 16] = ODD[p % 3]
            c.k[c.table[b, p // 16], p % 16] = ODD[(p + 1) % 3]
    q = c.rows_of(heads)
    want, bound = ref.attention(c.k, c.v, c.table, c.batch, q, hd ** -0.5, window)
    assert bool(torch.isfinite(want).all())
    check_odd(attend(c, q, window), want, bound)
