"""spec_paged_append and spec_paged_attention against the definition in 64 bits (paged_reference): types, head layouts, lengths from none to
several chunks, pages in any order, rows that see nothing, strides, windows, streams and graphs."""
import math

import pytest
import torch

import paged_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


class Case:
    """Pages in random order in a pool whose every place that no sequence owns is NaN, rows behind the last sequence, and outputs filled with a
    mark.  rows: new rows per sequence; lens: lengths."""

    def __init__(self, dtype, heads, kv_heads, hd, page, rows, lens, seed=0, layout="nhd", extra_rows=3, ragged=True, absent=(), fill=math.nan):
        self.td, self.heads, self.kv_heads, self.hd, self.page = TYPES[dtype], heads, kv_heads, hd, page
        self.B, self.lens, self.ragged = len(rows), list(lens), ragged
        g = torch.Generator().manual_seed(seed + 1)
        per = [(n + page - 1) // page for n in lens]
        self.n_pages = sum(per) + 2
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.table = torch.full((self.B, max(per) + 1), -1, dtype=torch.int32)
        at = 0
        k = torch.full((self.n_pages, page, kv_heads, hd), fill, dtype=self.td)
        v = k.clone()
        for b, n in enumerate(per):
            self.table[b, :n] = order[at:at + n]
            at += n
            for j in range(n):  # positions of the sequence hold numbers, the rest of its last page does not
                m = min(page, lens[b] - j * page)
                k[self.table[b, j], :m] = torch.randn((m, kv_heads, hd), generator=g).to(self.td)
                v[self.table[b, j], :m] = torch.randn((m, kv_heads, hd), generator=g).to(self.td)
        for b, j in absent:
            self.table[b, j] = (-1, self.n_pages, 1 << 30)[j % 3]
        self.row_start = [0]
        for n in rows:
            self.row_start.append(self.row_start[-1] + n)
        self.T = self.row_start[-1] + (extra_rows if ragged else 0)
        if not ragged:
            assert len(set(rows)) == 1
        self.k, self.v, self.g = k, v, g
        self.layout = layout
        self.batch = ref.sequences(self.B, self.T, self.row_start if ragged else None, self.lens)

    def rows_of(self, heads, wide=0):
        """[T][heads][hd]; wide: parts of rows that much wider"""
        x = torch.randn((self.T, heads + wide, self.hd), generator=self.g).to(self.td)
        return x[:, wide:]

    def on_gpu(self, B, max_rows=None, max_len=None):
        def pool(x):
            if self.layout == "hnd":  # heads before positions in memory
                return x.permute(0, 2, 1, 3).contiguous().to(DEV).permute(0, 2, 1, 3)
            return x.to(DEV)
        if self.layout == "pair":  # keys and values of a page side by side
            both = torch.stack([self.k, self.v], 1).to(DEV)
            kd, vd = both[:, 0], both[:, 1]
        else:
            kd, vd = pool(self.k), pool(self.v)
        self.kd, self.vd = kd, vd
        cache = B.PagedCache(kd, vd)
        rs = torch.tensor(self.row_start, dtype=torch.int32, device=DEV) if self.ragged else None
        batch = B.PagedBatch(self.table.to(DEV), torch.tensor(self.lens, dtype=torch.int32, device=DEV), self.T, row_start=rs, max_rows=max_rows,
                             max_len=max_len)
        return cache, batch


def to_gpu(x):
    """the same strides on the device: a part of wider rows stays one"""
    base = x._base if x._base is not None else x
    return torch.as_strided(base.to(DEV), x.shape, x.stride(), x.storage_offset())


def check(got, want, bound, owned, mark):
    got = got.cpu().double()
    assert bool((got[~owned] == mark).all())
    diff = (got[owned] - want[owned]).abs()
    assert bool(torch.isfinite(got[owned]).all())
    worst = float((diff / (bound[owned] + 1e-300)).max()) if diff.numel() else 0.0
    assert bool((diff <= bound[owned]).all()), worst


def owned_rows(c, dead=True):
    m = torch.zeros(c.T, dtype=torch.bool)
    for b, r0, n, kv in c.batch:
        for i in range(n):
            m[r0 + i] = dead or kv - n + i >= 0
    return m


SHAPES = [  # heads, key heads, head_dim, page, rows per sequence, lengths
    (4, 4, 64, 8, [1], [1]),
    (4, 2, 128, 16, [1, 1, 1], [1, 17, 300]),
    (6, 2, 64, 32, [4, 4, 4], [4, 33, 95]),
    (8, 1, 128, 16, [5, 0, 1, 9], [5, 40, 64, 129]),
    (3, 3, 128, 64, [2, 7, 3], [1, 7, 0]),             # more rows than positions: dead rows
    (16, 2, 64, 16, [30, 1, 3], [700, 50, 3]),         # several tiles of one sequence
    (2, 1, 128, 8, [1, 2], [1700, 3]),                 # several chunks of one sequence beside a short one
    (5, 5, 64, 128, [3] * 70, list(range(3, 73))),     # more sequences than a wave has lanes
    (24, 2, 128, 32, [40, 2, 1, 70], [1100, 600, 2, 70]),
    (4, 1, 128, 16, [2] * 65, [5000] + [9] * 30 + [2600] + [2] * 33),      # cut tiles among more sequences than a wave has lanes
    (8, 1, 64, 16, [100, 40], [2300, 2100]),                               # cut tiles of many rows
    (12, 4, 128, 8, [300, 1, 200], [310, 4000, 200]),                      # 256 rows a tile needs more of them: see the next test
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "h%dk%dd%dp%d_%d" % (s[0], s[1], s[2], s[3], len(s[4])))
@pytest.mark.parametrize("window", [0, 13])
def test_attention_matches_the_definition(dtype, shape, window):
    from paper_2310_18813_amd import binding as B
    c = Case(dtype, *shape, seed=sum(shape[4]) + shape[2])
    q = c.rows_of(c.heads)
    cache, batch = c.on_gpu(B)
    out = torch.full(q.shape, 7.0, dtype=c.td, device=DEV)
    B.spec_paged_attention(cache, batch, q.to(DEV), window=window, out=out)
    want, bound = ref.attention(c.k, c.v, c.table, c.batch, q, c.hd ** -0.5, window)
    check(out, want, bound, owned_rows(c), 7.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window", [99, 100, 101, 1 << 30, (1 << 31) - 1])
@pytest.mark.parametrize("rows", [[9, 3, 20], [90, 70, 80]])
def test_windows_as_long_as_the_longest_sequence_and_longer(dtype, window, rows):
    """beside dead rows, whose positions are the lowest numbers that a window is taken from: the first tile begins with some"""
    from paper_2310_18813_amd import binding as B
    c = Case(dtype, 4, 2, 64, 16, rows, [4, 100, 2], seed=17)
    q = c.rows_of(c.heads)
    cache, batch = c.on_gpu(B, max_len=100)
    out = torch.full(q.shape, 7.0, dtype=c.td, device=DEV)
    B.spec_paged_attention(cache, batch, q.to(DEV), window=window, out=out)
    want, bound = ref.attention(c.k, c.v, c.table, c.batch, q, 64 ** -0.5, window)
    check(out, want, bound, owned_rows(c), 7.0)


@pytest.mark.parametrize("layout", ["hnd", "pair"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_over_other_layouts_wide_rows_absent_pages_and_another_scale(layout, dtype):
    from paper_2310_18813_amd import binding as B
    c = Case(dtype, 8, 4, 64, 16, [3, 3, 3], [200, 16, 700], layout=layout, seed=5, extra_rows=0, ragged=False,
             absent=[(0, 0), (0, 7), (1, 0), (2, 31), (2, 32), (2, 5)])
    q = c.rows_of(8, wide=4)
    cache, batch = c.on_gpu(B)
    wide = torch.full((c.T, 13, 64), 7.0, dtype=c.td, device=DEV)
    B.spec_paged_attention(cache, batch, to_gpu(q), scale=0.31, out=wide[:, 2:10])
    want, bound = ref.attention(c.k, c.v, c.table, c.batch, q, 0.31, 0)
    assert bool((want[3:6] == 0).all())  # the second sequence's only page is absent
    check(wide[:, 2:10], want, bound, owned_rows(c), 7.0)
    assert bool((wide[:, :2] == 7.0).all()) and bool((wide[:, 10:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("rows", [6, 150])
def test_what_a_row_does_not_see_never_reaches_it(dtype, bad, window, rows):
    """The last rows' own keys and values are not finite, and neither is an early value: the rows that see none of them get numbers."""
    from paper_2310_18813_amd import binding as B
    c = Case(dtype, 4, 2, 128, 16, [rows, 2], [rows + 60, 90], seed=9, extra_rows=0)
    first_bad, early = rows + 60 - 3, 25
    for p in range(first_bad, rows + 60):
        c.v[c.table[0, p // 16], p % 16, :, ::7] = bad
    c.k[c.table[0, (rows + 59) // 16], (rows + 59) % 16] = bad
    if window:
        c.v[c.table[0, early // 16], early % 16, 0, 3] = bad
    q = c.rows_of(4)
    cache, batch = c.on_gpu(B)
    out = B.spec_paged_attention(cache, batch, q.to(DEV), window=window).cpu()
    want, bound = ref.attention(c.k, c.v, c.table, c.batch, q, 128 ** -0.5, window)
    free = torch.isfinite(want)
    assert bool(free[:rows - 3].all()) or window and bool(free[20:rows - 3].all())
    assert not bool(free[rows - 3:rows].all()) and bool(torch.isfinite(out[free]).all())
    assert bool(((out.double()[free] - want[free]).abs() <= bound[free]).all())
    # rows that see an infinite or NaN value show it
    assert not bool(torch.isfinite(out[rows - 2, :, ::7]).any())


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rot", [0, 16, 64, 128])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[2] == 128][:4] + [(4, 2, 128, 8, [1, 3, 20], [70000, 3, 1000])],
                         ids=lambda s: "h%dk%dd%dp%d_%d" % (s[0], s[1], s[2], s[3], len(s[4])))
def test_append_matches_the_definition(dtype, rot, shape):
    from paper_2310_18813_amd import binding as B
    c = Case(dtype, *shape, seed=3 + rot, fill=0.5)
    q, k, v = c.rows_of(c.heads, wide=1), c.rows_of(c.kv_heads, wide=2), c.rows_of(c.kv_heads, wide=3)
    cache, batch = c.on_gpu(B)
    freq = B.spec_rope_frequencies(10000.0, rot) if rot else None
    out = torch.full(q.shape, 7.0, dtype=c.td, device=DEV)
    B.spec_paged_append(cache, batch, to_gpu(q), to_gpu(k), to_gpu(v), freq, out=out)
    qo, ko, vo, qe, ke = ref.append(c.k, c.v, c.table, c.batch, q, k, v, freq.cpu() if rot else None)
    check(out, qo, qe, owned_rows(c, dead=False), 7.0)
    assert bool(((c.kd.cpu().double() - ko).abs() <= ke).all())
    assert torch.equal(c.vd.cpu().double(), vo)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_in_place_without_queries_and_to_absent_pages(dtype):
    from paper_2310_18813_amd import binding as B
    c = Case(dtype, 4, 2, 64, 16, [4, 4], [40, 17], seed=4, fill=0.5, ragged=False, extra_rows=0, absent=[(0, 2), (1, 0)])
    q, k, v = c.rows_of(4), c.rows_of(2), c.rows_of(2)
    freq = B.spec_rope_frequencies(500000.0, 64)
    want = ref.append(c.k, c.v, c.table, c.batch, q, k, v, freq.cpu())
    for with_q in (True, False):
        cache, batch = c.on_gpu(B)
        x = q.to(DEV)
        B.spec_paged_append(cache, batch, x if with_q else None, k.to(DEV), v.to(DEV), freq, out=x if with_q else None)
        assert bool(((c.kd.cpu().double() - want[1]).abs() <= want[4]).all()) and torch.equal(c.vd.cpu().double(), want[2])
        if with_q:
            assert bool(((x.cpu().double() - want[0]).abs() <= want[3]).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bounds_cut_what_lies_beyond(dtype):
    """max_rows and max_len are the caller's promise; rows and positions beyond them are not touched, whatever the device holds."""
    from paper_2310_18813_amd import binding as B
    c = Case(dtype, 4, 2, 64, 8, [5, 2], [60, 30], seed=6)
    c.batch = ref.sequences(2, c.T, c.row_start, c.lens, max_rows=3, max_len=41)
    q = c.rows_of(4)
    cache, batch = c.on_gpu(B, max_rows=3, max_len=41)
    out = torch.full(q.shape, 7.0, dtype=c.td, device=DEV)
    B.spec_paged_attention(cache, batch, q.to(DEV), out=out)
    want, bound = ref.attention(c.k, c.v, c.table, c.batch, q, 64 ** -0.5, 0)
    check(out, want, bound, owned_rows(c), 7.0)


@pytest.mark.parametrize("rows", [2, 70])
def test_offsets_beyond_32_bits(rows):
    """Four pages whose rows lie 2^31 elements apart and more; of 70 rows the first 40 are dead."""
    from paper_2310_18813_amd import binding as B
    page_stride = (1 << 31) + 4096
    store = torch.empty(3 * page_stride + 8192, dtype=torch.bfloat16, device=DEV)
    view = lambda off: torch.as_strided(store, (4, 8, 1, 64), (page_stride, 64, 64, 1), off)
    kd, vd = view(0), view(2048)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((4, 8, 1, 64), generator=g).to(torch.bfloat16) for _ in range(2))
    kd.copy_(k)
    vd.copy_(v)
    table = torch.tensor([[3, 1, 2, 0]], dtype=torch.int32)
    cache = B.PagedCache(kd, vd)
    batch = B.PagedBatch(table.to(DEV), torch.tensor([30], dtype=torch.int32, device=DEV), rows)
    q, nk, nv = (torch.randn((rows, h, 64), generator=g).to(torch.bfloat16) for h in (3, 1, 1))
    seqs = ref.sequences(1, rows, None, [30])
    out = torch.full_like(q, 7.0).to(DEV)
    B.spec_paged_append(cache, batch, q.to(DEV), nk.to(DEV), nv.to(DEV), None, out=out)
    qo, ko, vo, _, _ = ref.append(k, v, table, seqs, q, nk, nv, None)
    dead = max(0, rows - 30)
    assert torch.equal(kd.cpu().double(), ko) and torch.equal(vd.cpu().double(), vo)
    assert torch.equal(out.cpu().double()[dead:], qo[dead:]) and bool((out[:dead] == 7.0).all())
    got = B.spec_paged_attention(cache, batch, q.to(DEV))
    want, bound = ref.attention(ko.to(torch.bfloat16), vo.to(torch.bfloat16), table, seqs, q, 0.125, 0)
    assert bool(((got.cpu().double() - want).abs() <= bound).all()) and not bool(got[:dead].any())


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("fp16", 64)])
@pytest.mark.parametrize("window", [0, 100])
def test_tiles_of_256_rows(dtype, hd, window):
    """Enough query rows for the largest tile; rows of every tile's start, middle and end are compared."""
    from paper_2310_18813_amd import binding as B
    c = Case(dtype, 64, 16, hd, 32, [900, 1, 1300], [1000, 700, 1500], seed=12)
    q = c.rows_of(64)
    cache, batch = c.on_gpu(B)
    out = torch.full(q.shape, 7.0, dtype=c.td, device=DEV)
    B.spec_paged_attention(cache, batch, q.to(DEV), window=window, out=out)
    got = out.cpu().double()
    assert bool((got[2201:] == 7.0).all()) and bool(torch.isfinite(got[:2201]).all())
    for b, r0, n, kv in c.batch:
        for i in sorted({0, 1, 63, 64, 127, n // 2, n - 65, n - 1} & set(range(n))):
            p = kv - n + i
            want, bound = ref.attention(c.k, c.v, c.table, [(b, 0, 1, p + 1)], q[r0 + i:r0 + i + 1], hd ** -0.5, window)
            assert bool(((got[r0 + i] - want[0]).abs() <= bound[0]).all()), (b, i)


def test_sequences_may_share_pages():
    """A common prefix lies in the pool once; each sequence's own rows follow in pages of its own."""
    from paper_2310_18813_amd import binding as B
    c = Case("bf16", 8, 2, 64, 16, [2, 2, 2], [48, 40, 33], seed=13, extra_rows=0, ragged=False)
    c.table[1, :2] = c.table[0, :2]
    c.table[2, :2] = c.table[0, :2]
    q = c.rows_of(8)
    cache, batch = c.on_gpu(B)
    got = B.spec_paged_attention(cache, batch, q.to(DEV))
    want, bound = ref.attention(c.k, c.v, c.table, c.batch, q, 0.125, 0)
    assert bool(((got.cpu().double() - want).abs() <= bound).all())


@pytest.mark.parametrize("rows,warm", [(3, True), (40, False)])
def test_captured_calls_follow_lengths_pages_and_rows_on_another_stream(rows, warm):
    """Append and attention are captured once and replayed with other contents; eager calls on another stream lie between.  Not
    warm: the capture is the kernels' first use."""
    from paper_2310_18813_amd import binding as B
    c = Case("bf16", 8, 2, 128, 16, [rows, rows], [2500, 700], seed=8, ragged=False, extra_rows=0, fill=0.5)
    cache, batch = c.on_gpu(B)
    freq = B.spec_rope_frequencies(10000.0, 128)
    q, k, v = (c.rows_of(h).to(DEV) for h in (8, 2, 2))
    x, out = torch.empty_like(q), torch.empty_like(q)
    space = torch.empty(B.spec_paged_attention_workspace_bytes(cache, batch, 8), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def both(dst, scratch):
        B.spec_paged_append(cache, batch, q, k, v, freq, out=x)
        return B.spec_paged_attention(cache, batch, x, out=dst, workspace=scratch)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        if warm:
            both(out, space)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            both(out, space)
    for lens in ([2500, 700], [3, 64], [900, 690], [0, 2]):
        batch.lengths.copy_(torch.tensor(lens, dtype=torch.int32))
        q.normal_()
        k.normal_()
        graph.replay()
        torch.cuda.synchronize()
        again = both(torch.empty_like(out), torch.empty_like(space))
        assert torch.equal(out, again), lens
