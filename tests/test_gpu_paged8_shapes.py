"""spec_paged8_attention in launch shapes that the tests of its definition do not reach, each with the kernels that it launches: tiles of 256 query rows with every
wave at work, with windows, absent pages and NaN, cut and joined, their first call inside a capture; 33 to 64 query rows, cut and joined."""
import os
import subprocess
import sys
from types import SimpleNamespace

import pytest
import torch

import paged8_reference as ref
from launches import launched_kernels, template_ints
from test_gpu_paged8_attention import Cache
from test_gpu_paged8_attention import close as within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def B():
    from paper_2310_18813_amd import binding
    return binding


def close(got, want, err, td):
    # The bound's rounding of a result is u of it, which holds from the type's least normal number on.  Below fp16's, 2^-14, the numbers lie 2^-24 apart, so that a
    # result is rounded by up to 2^-25 whatever its size: a row whose weight is on one position with an element of 7e-6 is off by 0.7 * 2^-25.
    within(got, want, err + (2.0 ** -25 if td == torch.float16 else 0.0), td)


def attend(B, b, c, q, window, kernels, max_len=None):
    """-> the call's rows; kernels: what it launches, as (part of the name, its whole numbers)."""
    cache, batch, on = c.on_gpu(B), b.on_gpu(B, max_rows=max(b.rows), max_len=max_len), q.to(DEV)
    out = torch.full(q.shape, 77.0, dtype=q.dtype, device=DEV)
    space = torch.empty(B.spec_paged8_attention_workspace_bytes(cache, batch, q.shape[1]), dtype=torch.uint8, device=DEV)
    call = lambda: B.spec_paged8_attention(cache, batch, on, window=window, out=out, workspace=space)
    call()
    got = out.cpu()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        names = [n for n, _, _ in launched_kernels(B.lib, stream, call)]
    assert len(names) == len(kernels) and all(part in n and template_ints(n) == ints for n, (part, ints) in zip(names, kernels)), names
    assert (got[b.row_start[-1]:] == 77.0).all()
    return got


def some_heads(c, b, q, got, window, heads):
    """The rows of a few key heads against the definition."""
    k, v = c.numbers()
    G = q.shape[1] // k.shape[2]
    for h in heads:
        mine = slice(h * G, h * G + G)
        want, err = ref.attention(k[:, :, h:h + 1], v[:, :, h:h + 1], b, q[:, mine], q.shape[2] ** -0.5, window)
        n = b.row_start[-1]
        close(got[:n, mine], want[:n], err[:n], q.dtype)


def some_rows(c, b, q, got, window, rows):
    """Some rows of all heads against the definition: as a batch of one sequence that ends there."""
    k, v = c.numbers()
    for s, i in rows:
        at = b.row_start[s] + i
        one = SimpleNamespace(B=1, rows=[1], lens=[b.lens[s] - b.rows[s] + i + 1], row_start=[0, 1], table=b.table[s:s + 1], page=b.page, n_pages=b.n_pages)
        want, err = ref.attention(k, v, one, q[at:at + 1], q.shape[2] ** -0.5, window)
        close(got[at:at + 1], want, err, q.dtype)


@pytest.mark.parametrize("td", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("Hq,Hk,rows,lens,window,layout", [
    (64, 16, [900, 1, 1130], [1000, 1400, 1130], 0, "nhd"), (64, 16, [700, 33, 1301], [1500, 33, 1301], 300, "pair"), (48, 16, [1403, 1500], [1777, 1500], 0, "hnd")])
def test_tiles_of_256_rows(B, td, hd, Hq, Hk, rows, lens, window, layout):
    b = ref.Batch(rows, lens, 16, seed=hd + Hq, absent=((0, 5), (0, 30), (2, 0)) if len(rows) > 2 else ((1, 70),))
    c = Cache(b, Hk, hd, td, layout)
    q = b.heads(Hq, hd, td)
    got = attend(B, b, c, q, window, [("k_paged_chunk", [hd, 8])])
    assert torch.isfinite(got[:b.row_start[-1]]).all()
    some_heads(c, b, q, got, window, (0, 7, 15))


@pytest.mark.parametrize("td", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("window", [0, 15000])
def test_cut_tiles_of_256_rows(B, td, hd, window):
    """A few rows over a long context, which are cut, beside a prompt's many tiles."""
    b = ref.Batch([2090, 13], [2090, 20000], 64, seed=hd)
    c = Cache(b, 4, hd, td)
    q = b.heads(64, hd, td)
    got = attend(B, b, c, q, window, [("k_paged_chunk", [hd, 8]), ("k_paged_join", [hd, 16])])
    assert torch.isfinite(got[:2103]).all()
    some_rows(c, b, q, got, window, [(0, 0), (0, 17), (0, 1045), (0, 2089), (1, 0), (1, 12)])


@pytest.mark.parametrize("td", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
def test_nan_in_tiles_of_256_rows(B, td, hd):
    """A NaN among a position's values shows in the rows that see it, and in no others: at both ends of the window, on the diagonal, where two tiles meet."""
    n, window, Hk, G = 1100, 400, 16, 8
    b = ref.Batch([n], [n], 16, seed=7)
    c = Cache(b, Hk, hd, td)
    for h, p in ((0, 0), (0, 1099), (1, 31), (1, 32), (1, 640), (2, 511)):
        c.codes[1][b.table[0, p // 16], p % 16, h] = 0x7f if p % 2 else 0xff
    c.codes[0][b.table[0, 700 // 16], 700 % 16, 3] = 0xff  # a key
    q = b.heads(Hk * G, hd, td)
    got = attend(B, b, c, q, window, [("k_paged_chunk", [hd, 8])])
    some_heads(c, b, q, got, window, (0, 1, 2, 4))
    odd = torch.isnan(got[:n, 3 * G:4 * G])
    assert not odd[:700].any() and odd[700:1100].all()


@pytest.mark.parametrize("td", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows,lens,window,Hk", [([4], [6000], 0, 1), ([3, 3], [6000, 2000], 0, 1), ([4, 4], [9001, 40], 5000, 2), ([3, 0, 4], [4100, 5, 2300], 1999, 8)])
def test_33_to_64_rows_are_cut_and_joined(B, td, hd, rows, lens, window, Hk):
    b = ref.Batch(rows, lens, 32, seed=sum(lens), ragged=len(set(rows)) > 1, absent=((0, 3), (0, 100)))
    c = Cache(b, Hk, hd, td)
    q = b.heads(16 * Hk, hd, td)
    got = attend(B, b, c, q, window, [("k_paged_attend", [hd, 4]), ("k_paged_join_rows", [hd, 4])])
    n = b.row_start[-1]
    want, err = ref.attention(*c.numbers(), b, q, hd ** -0.5, window)
    close(got[:n], want[:n], err[:n], td)


FIRST_CALL = """
import sys, torch
sys.path[:0] = sys.argv[1:3]
import paged8_reference as ref
from test_gpu_paged8_attention import Cache, DEV
from paper_2310_18813_amd import binding as B
b = ref.Batch([700, 1300], [700, 1300], 32, seed=3, extra_rows=0)
cache, batch, q = Cache(b, 16, 128, torch.float16).on_gpu(B), b.on_gpu(B), b.heads(64, 128, torch.float16).to(DEV)
out, graph = torch.zeros_like(q), torch.cuda.CUDAGraph()
space = torch.empty(B.spec_paged8_attention_workspace_bytes(cache, batch, 64), dtype=torch.uint8, device=DEV)
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    B.spec_paged8_attention(cache, batch, q, out=out, workspace=space)
for lens in ([700, 1300], [650, 1290], [700, 1300]):
    batch.lengths.copy_(torch.tensor(lens, dtype=torch.int32))
    q.normal_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, B.spec_paged8_attention(cache, batch, q)), lens
    assert bool(torch.isfinite(out).all())
print("replays agree")
"""


def test_the_largest_tiles_first_call_may_be_captured():
    """in a process of its own, so that what is set up once has not been"""
    tests = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL, os.path.dirname(tests), tests], capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "replays agree" in r.stdout, r.stderr[-3000:]


@pytest.mark.parametrize("td", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("Hq,Hk,rows,lens,window,kernels", [
    (4, 2, [2, 1, 3], [700, 33, 90], 0, [("k_paged_attend", 1)]), (16, 1, [4, 2], [3001, 70], 1700, [("k_paged_attend", 4), ("k_paged_join_rows", 4)]),
    (8, 2, [70, 33], [333, 1040], 200, [("k_paged_chunk", 4)]), (64, 16, [900, 1101], [1000, 1101], 300, [("k_paged_chunk", 8)])])
def test_any_bytes_where_no_row_looks(B, td, hd, Hq, Hk, rows, lens, window, kernels):
    """Pools as they come: any codes under any scale byte, those of infinity among them, in pages that nothing was written to and in front of the window."""
    b = ref.Batch(rows, lens, 16, seed=hd + Hk, absent=((0, 1),))
    c = Cache(b, Hk, hd, td)
    seen = torch.zeros((b.n_pages, b.page), dtype=torch.bool)
    for s in range(b.B):
        for p in range(max(0, lens[s] - rows[s] - window + 1) if window else 0, lens[s]):
            if 0 <= int(b.table[s, p // 16]) < b.n_pages:
                seen[b.table[s, p // 16], p % 16] = True
    want_k, want_v = c.numbers()
    for part in range(2):
        c.codes[part][~seen] = torch.randint(0, 256, c.codes[part][~seen].shape, generator=b.g).to(torch.uint8)
        scales = c.scales[part].transpose(1, 2)
        scales[~seen] = torch.randint(0, 256, scales[~seen].shape, generator=b.g).to(torch.uint8)
        scales[~seen] = torch.where(torch.rand(scales[~seen].shape, generator=b.g) < 0.2, 255, scales[~seen].int()).to(torch.uint8)
    q = b.heads(Hq, hd, td)
    got = attend(B, b, c, q, window, [(k, [hd, n]) for k, n in kernels], max_len=max(lens))
    n = b.row_start[-1]
    want, err = ref.attention(want_k, want_v, b, q, hd ** -0.5, window)
    close(got[:n], want[:n], err[:n], td)
