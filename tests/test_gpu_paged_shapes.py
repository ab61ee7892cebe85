"""spec_paged_attention in the launch shapes that the tests of its definition do not reach: 17 to 64 query rows of 16 bits, cut tiles of 64 and
256 rows and their joins, many rows over other layouts and absent pages, the largest tile's first call inside a capture."""
import os
import subprocess
import sys

import pytest
import torch

import paged_reference as ref
from test_gpu_paged import Case, check, owned_rows, to_gpu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows,kv_heads", [([4, 1, 3], 2), ([7, 5, 8], 2), ([3, 2, 2], 1)])  # 32, 64 and 48 query rows of a key head at most
@pytest.mark.parametrize("lens", [[700, 1, 30], [5000, 2600, 33]], ids=["whole", "cut"])
@pytest.mark.parametrize("window", [0, 600])
def test_17_to_64_query_rows(dtype, hd, rows, kv_heads, lens, window):
    c = Case(dtype, 16, kv_heads, hd, 16, rows, lens, seed=hd + rows[0])
    q = c.rows_of(16)
    from paper_2310_18813_amd import binding as B
    cache, batch = c.on_gpu(B, max_rows=max(rows), max_len=max(lens))
    out = torch.full(q.shape, 7.0, dtype=c.td, device=DEV)
    B.spec_paged_attention(cache, batch, q.to(DEV), window=window, out=out)
    want, bound = ref.attention(c.k, c.v, c.table, c.batch, q, hd ** -0.5, window)
    check(out, want, bound, owned_rows(c), 7.0)


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("fp16", 64), ("fp16", 128), ("bf16", 64)])
@pytest.mark.parametrize("window", [0, 15000])
def test_cut_tiles_of_256_rows(dtype, hd, window):
    """A few rows over a long context, which are cut, beside a prompt's many tiles."""
    from paper_2310_18813_amd import binding as B
    c = Case(dtype, 64, 4, hd, 64, [2090, 13], [2090, 20000], seed=hd)
    q = c.rows_of(64)
    cache, batch = c.on_gpu(B)
    out = torch.full(q.shape, 7.0, dtype=c.td, device=DEV)
    B.spec_paged_attention(cache, batch, q.to(DEV), window=window, out=out)
    got = out.cpu().double()
    assert bool((got[2103:] == 7.0).all()) and bool(torch.isfinite(got[:2103]).all())
    for b, r0, n, kv in c.batch:
        for i in (0, n // 2, n - 1) if b == 0 else (0, n - 1):
            want, bound = ref.attention(c.k, c.v, c.table, [(b, 0, 1, kv - n + i + 1)], q[r0 + i:r0 + i + 1], hd ** -0.5, window)
            assert bool(((got[r0 + i] - want[0]).abs() <= bound[0]).all()), (b, i)


@pytest.mark.parametrize("layout", ["hnd", "pair"])
@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("fp16", 128), ("fp32", 64)])
@pytest.mark.parametrize("window", [0, 70])
def test_many_rows_over_other_layouts_wide_rows_and_absent_pages(layout, dtype, hd, window):
    from paper_2310_18813_amd import binding as B
    c = Case(dtype, 8, 4, hd, 16, [100, 100, 100], [200, 16, 2600], layout=layout, seed=5, extra_rows=0, ragged=False,
             absent=[(0, 0), (0, 3), (0, 8), (0, 12), (1, 0), (2, 31), (2, 32), (2, 33), (2, 5), (2, 158)])
    q = c.rows_of(8, wide=4)
    cache, batch = c.on_gpu(B)
    wide = torch.full((c.T, 13, hd), 7.0, dtype=c.td, device=DEV)
    B.spec_paged_attention(cache, batch, to_gpu(q), scale=0.31, window=window, out=wide[:, 2:10])
    want, bound = ref.attention(c.k, c.v, c.table, c.batch, q, 0.31, window)
    assert bool((want[100:200] == 0).all())  # the second sequence's only page is absent
    check(wide[:, 2:10], want, bound, owned_rows(c), 7.0)
    assert bool((wide[:, :2] == 7.0).all()) and bool((wide[:, 10:] == 7.0).all())


FIRST_CALL = """
import sys, torch
sys.path[:0] = sys.argv[1:3]
from test_gpu_paged import Case, DEV
from paper_2310_18813_amd import binding as B
c = Case("bf16", 64, 16, 128, 32, [700, 1300], [700, 1300], seed=3, extra_rows=0)
cache, batch = c.on_gpu(B)
q = c.rows_of(64).to(DEV)
out, graph = torch.zeros_like(q), torch.cuda.CUDAGraph()
space = torch.empty(B.spec_paged_attention_workspace_bytes(cache, batch, 64), dtype=torch.uint8, device=DEV)
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    B.spec_paged_attention(cache, batch, q, out=out, workspace=space)
for lens in ([700, 1300], [650, 1290], [700, 1300]):
    batch.lengths.copy_(torch.tensor(lens, dtype=torch.int32))
    q.normal_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, B.spec_paged_attention(cache, batch, q)), lens
    assert bool(torch.isfinite(out).all())
print("replays agree")
"""


def test_the_largest_tiles_first_call_may_be_captured():
    """in a process of its own, so that what is set up once has not been"""
    tests = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL, os.path.dirname(tests), tests], capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "replays agree" in r.stdout, r.stderr[-3000:]
