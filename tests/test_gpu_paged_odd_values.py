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


def plant(c, b, positions):
    """one odd value at each position, in an element of its own -> [(position, element, value)]"""
    planted = [(p, i % c.hd, ODD[i % 3]) for i, p in enumerate(positions)]
    assert len(planted) <= c.hd
    for p, d, x in planted:
        page = int(c.table[b, p // c.page])
        assert 0 <= page < c.n_pages
        c.v[page, p % c.page, :, d] = x
    return planted


def borders(rows, kv, G, window):
    """positions on both sides of what all rows of a tile see, for tiles of 16 to 256 query rows, and early ones"""
    at, p0 = {0, 25, kv - 1}, kv - rows
    for R in (16, 32, 64, 128, 256):
        for t in range(3):
            i0, i1 = t * R // G, min(rows - 1, (t * R + R - 1) // G)
            at |= {p0 + i0, p0 + i0 + 1} | ({p0 + i1 - window + 1, p0 + i1 - window, p0 + i0 - window + 1} if window else set())
    return sorted(p for p in at if 0 <= p < kv)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("shape", [(4, 2, 128, 150, 210), (4, 2, 64, 150, 210), (4, 2, 128, 150, 150), (2, 2, 128, 150, 1100), (8, 2, 64, 6, 300),
                                   (16, 1, 128, 3, 3000)], ids=lambda s: "h%dk%dd%d_%drows_%d" % s)
@pytest.mark.parametrize("window", [0, 40, 100])
def test_what_a_row_sees_shows(dtype, shape, window):
    """Also where other rows of the same tile do not see it."""
    heads, kv_heads, hd, rows, kv = shape
    c = Case(dtype, heads, kv_heads, hd, 16, [rows, 1], [kv, 50], seed=kv + window)
    plant(c, 0, borders(rows, kv, heads // kv_heads, window)[:hd])
    q = c.rows_of(heads)
    want, bound = ref.attention(c.k, c.v, c.table, c.batch, q, hd ** -0.5, window)
    got = attend(c, q, window)
    assert not bool(torch.isfinite(want[:rows]).all())
    check_odd(got[:rows + 1], want[:rows + 1], bound[:rows + 1])


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("fp16", 64)])
@pytest.mark.parametrize("window", [0, 100])
def test_what_a_row_sees_shows_in_tiles_of_256_rows(dtype, hd, window):
    heads, kv_heads, rows, lens = 64, 16, [900, 1, 1300], [1000, 700, 1500]
    c = Case(dtype, heads, kv_heads, hd, 32, rows, lens, seed=12)
    seen = torch.zeros((c.T, hd), dtype=torch.bool)
    for b, r0, n, kv in c.batch:
        pos = torch.arange(kv - n, kv)
        for p, d, x in plant(c, b, borders(n, kv, heads // kv_heads, window)[:hd]):
            seen[r0:r0 + n, d] |= (pos >= p) & ((pos - p < window) if window else True)
    got = attend(c, c.rows_of(heads), window)[:sum(rows)]
    assert bool(seen.any()) and torch.equal(~torch.isfinite(got), seen[:sum(rows), None].expand_as(got))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows", [6, 150])
@pytest.mark.parametrize("page,absent,at", [(16, (0, 2, 9), (16, 20, 31, 50, 63, 135, 145)), (8, (1, 6, 7), (0, 3, 17, 40, 63))])
def test_what_a_row_sees_shows_beside_an_absent_page(dtype, rows, page, absent, at):
    """the odd values lie among the 32 positions that the absent page is one of"""
    c = Case(dtype, 4, 2, 128, page, [rows], [rows + 180], seed=page, absent=[(0, j) for j in absent])
    plant(c, 0, [p for p in at if p // page not in absent])
    q = c.rows_of(4)
    want, bound = ref.attention(c.k, c.v, c.table, c.batch, q, 128 ** -0.5, 0)
    assert not bool(torch.isfinite(want[:rows]).all())
    check_odd(attend(c, q)[:rows], want[:rows], bound[:rows])
