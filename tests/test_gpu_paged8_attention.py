"""spec_paged8_attention against the definition in 64 bits on the numbers that the cache stands for: types, head layouts, lengths from none to several
chunks, rows from one to many, windows, absent pages, NaN where rows do not look and where some do, strides, streams and graphs; against the attention over
the same numbers in 16 bits; and a caller's verification with all operators together."""
import math

import pytest
import torch

import paged8_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def B():
    from paper_2310_18813_amd import binding
    return binding


class Cache:
    """A pool of codes: numbers where a sequence has positions, NaN codes under any scale everywhere else."""

    def __init__(self, b, Hk, hd, td, layout="nhd", loud=True):
        g, self.td, self.layout, self.b = b.g, td, layout, b
        self.codes, self.scales = [], []
        owned = torch.zeros((b.n_pages, b.page), dtype=torch.bool)
        for s in range(b.B):
            for p in range(b.lens[s]):
                pg = int(b.table[s, p // b.page])
                if 0 <= pg < b.n_pages:
                    owned[pg, p % b.page] = True
        for part in range(2):
            y = torch.randn((b.n_pages, b.page, Hk, hd), generator=g).double()
            if loud:  # sizes that differ by position, so that scales do
                y = y * torch.exp(torch.randn((b.n_pages, b.page, Hk, 1), generator=g).double())
            codes, e, _ = ref.encode(y.to(td).double(), td)
            codes[~owned] = 0x7f
            e[~owned] = torch.randint(-15, 8, e[~owned].shape, generator=g)
            self.codes.append(codes)
            self.scales.append((e + 127).to(torch.uint8).transpose(1, 2).contiguous())

    def numbers(self):
        return [ref.decode(c) * torch.ldexp(torch.ones((), dtype=torch.float64), s.transpose(1, 2).int() - 127)[..., None] for c, s in zip(self.codes, self.scales)]

    def on_gpu(self, B):
        if self.layout == "pair":  # keys and values of a page side by side
            both = torch.stack(self.codes, 1).to(DEV)
            k, v = both[:, 0], both[:, 1]
        else:
            k, v = (ref.pool(c, self.layout) for c in self.codes)
        return B.PagedCache8(k, v, *(s.to(DEV) for s in self.scales), self.td)


def close(got, want, err, td):
    got = got.double()
    bad = ~((got - want).abs() <= err) & ~(torch.isnan(got) & torch.isnan(want))
    # fp16: weights far below a row's largest are off by 2^-32 of that, which over the positions of a row is far below its result's rounding
    assert not bad.any(), (float(((got - want).abs() / err.clamp(min=1e-30))[bad].max()), int(bad.sum()))


def run(B, td, Hq, Hk, hd, page, rows, lens, window=0, layout="nhd", ragged=True, absent=(), seed=0, scale=None, wide=0, max_len=None, cache=None):
    b = ref.Batch(rows, lens, page, seed=seed, ragged=ragged, absent=absent)
    c = Cache(b, Hk, hd, td, layout)
    if cache:
        cache(b, c)
    q = b.heads(Hq, hd, td)
    big = q.to(DEV) if not wide else torch.cat([torch.zeros((b.T, wide, hd), dtype=td), q], 1).to(DEV)[:, wide:]
    out = torch.full((b.T, Hq, hd), 77.0, dtype=td, device=DEV)
    B.spec_paged8_attention(c.on_gpu(B), b.on_gpu(B, max_len=max_len), big, scale=scale, window=window, out=out)
    want, err = ref.attention(*c.numbers(), b, q, scale or hd ** -0.5, window)
    got = out.cpu()
    nobody = torch.isnan(want).all(-1).all(-1) & (torch.arange(b.T) >= b.row_start[-1])
    assert (got[nobody] == 77.0).all()
    close(got[~nobody], want[~nobody], err[~nobody], td)
    return got


TYPES = [torch.bfloat16, torch.float16]


@pytest.mark.parametrize("td", TYPES)
@pytest.mark.parametrize("Hq,Hk,hd,page,layout", [(4, 4, 128, 16, "nhd"), (8, 2, 128, 8, "hnd"), (3, 1, 64, 16, "pair"), (16, 1, 64, 64, "nhd"), (40, 2, 128, 32, "pair"),
                                                  (5, 5, 64, 8, "hnd")])
@pytest.mark.parametrize("rows,lens", [([1], [1]), ([1, 1], [500, 3]), ([4, 4, 4], [4, 33, 260]), ([2, 0, 5, 1, 3], [1, 9, 3, 700, 0])])
def test_few_rows(B, td, Hq, Hk, hd, page, layout, rows, lens):
    even = len(set(rows)) == 1
    run(B, td, Hq, Hk, hd, page, rows, lens, layout=layout, ragged=not even, wide=1, absent=((3, 2),) if len(rows) > 3 and page >= 16 else ())
    run(B, td, Hq, Hk, hd, page, rows, lens, window=37, layout=layout, ragged=not even, seed=1)


@pytest.mark.parametrize("td", TYPES)
@pytest.mark.parametrize("Hq,Hk,hd,rows,lens,window", [
    (2, 2, 128, [70, 1, 200], [90, 65, 1200], 0), (4, 1, 64, [33, 129], [700, 129], 0), (8, 2, 64, [300], [1100], 100), (4, 2, 128, [150, 40], [150, 2000], 513),
    (8, 1, 128, [17, 9], [2000, 9], 0)])
def test_many_rows(B, td, Hq, Hk, hd, rows, lens, window):
    run(B, td, Hq, Hk, hd, 16, rows, lens, window=window)


def test_the_largest_tiles(B):
    """Tiles of 256 query rows, with heads of both sizes."""
    for hd in (64, 128):
        run(B, torch.bfloat16, 16, 8, hd, 32, [1100, 1, 600], [1100, 300, 900], absent=((2, 5),))


@pytest.mark.parametrize("td", TYPES)
def test_long_contexts_are_cut_and_joined(B, td):
    run(B, td, 8, 2, 128, 64, [1], [9000])
    run(B, td, 4, 1, 64, 16, [3, 1], [5000, 2600], window=3000)
    run(B, td, 16, 1, 128, 64, [9, 1, 30], [6000, 4000, 2000])
    run(B, td, 4, 1, 128, 128, [1, 1], [20001, 17])  # more chunks than lanes
    run(B, td, 4, 1, 64, 64, [4], [9000], absent=((0, 3), (0, 140)))


@pytest.mark.parametrize("Hq,Hk,hd", [(16, 8, 64), (16, 16, 128), (24, 24, 64), (32, 8, 128)])
def test_heads_in_groups_of_eight(B, Hq, Hk, hd):
    """Heads of one unit of work that run side by side: short, of many sequences, and cut into chunks."""
    run(B, torch.bfloat16, Hq, Hk, hd, 16, [1, 3, 0, 2], [1, 70, 5, 300], absent=((3, 2),))
    run(B, torch.float16, Hq, Hk, hd, 16, [1, 1], [3500, 40])


@pytest.mark.parametrize("Hk", [2, 8])
def test_more_than_64_sequences(B, Hk):
    g = torch.Generator().manual_seed(21)
    lens = torch.randint(0, 90, (131,), generator=g).tolist()
    run(B, torch.bfloat16, 2 * Hk, Hk, 64, 16, torch.randint(0, 4, (131,), generator=g).tolist(), lens)
    lens[77] = 2500
    run(B, torch.float16, 2 * Hk, Hk, 64, 16, [1] * 131, lens, ragged=False)


@pytest.mark.parametrize("td", TYPES)
def test_a_pool_beyond_4_gigabytes(B, td):
    """The last pages of pools of 5 GB: what small pools give."""
    Hk, hd, page = 8, 128, 16
    n = 5 * (1 << 30) // (page * Hk * hd)
    b = ref.Batch([2, 2], [50, 20], page, ragged=False)
    freq = B.spec_rope_frequencies(10000.0, hd)
    t = B.HeadTransform(freq)
    q, k, v = (b.heads(h, hd, td).to(DEV) for h in (16, Hk, Hk))
    small, batch = B.PagedCache8.empty(b.n_pages, page, Hk, hd, td), b.on_gpu(B)
    codes = [torch.empty((n, page, Hk, hd), dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.empty((n, Hk, page), dtype=torch.uint8, device=DEV) for _ in range(2)]
    for c, sc in zip(codes, scales):
        c[n - b.n_pages:] = 0
        sc[n - b.n_pages:] = 127
    large = B.PagedCache8(*codes, *scales, td)
    far = B.PagedBatch(torch.where(batch.pages >= 0, batch.pages + (n - b.n_pages), -1).to(torch.int32), batch.lengths, b.T)
    for other, (cache, bt) in enumerate(((small, batch), (large, far))):
        got = B.spec_paged8_append(cache, bt, q, k, v, t)
        back = B.spec_paged8_read(cache, bt)
        o = B.spec_paged8_attention(cache, bt, got)
        if not other:
            want = (got, *back, o)
    assert all(torch.equal(x, y) for x, y in zip((got, *back, o), want)) and want[3].isfinite().all() and want[1].any()


@pytest.mark.parametrize("td", TYPES)
@pytest.mark.parametrize("hd,rows", [(64, 3), (128, 3), (128, 20), (64, 70), (128, 140)])
def test_nan_at_positions_that_some_rows_see(B, td, hd, rows):
    """A NaN among a position's values shows in the rows that see it, and in no others: at both ends of the window and on the diagonal; a NaN key the same."""
    n, window = rows + 200, 150

    def plant(b, c):
        for p in (n - 1, n - rows, n - rows - window + 1, n - window + 1, n - rows + rows // 2):
            c.codes[1][b.table[0, p // 16], p % 16, 0] = 0x7f
        c.codes[0][b.table[0, (n - 2) // 16], (n - 2) % 16, 1] = 0xff

    got = run(B, td, 4, 2, hd, 16, [rows], [n], window=window, cache=plant)
    assert torch.isnan(got[:rows, :2]).any() and not torch.isnan(got[: rows - 2, 2:]).any() and torch.isnan(got[rows - 2:rows, 2:]).all()


def test_other_scales_and_a_bound_above_the_lengths(B):
    run(B, torch.bfloat16, 4, 2, 128, 16, [2, 2], [40, 300], scale=1.7)
    run(B, torch.float16, 4, 2, 128, 16, [2, 2], [40, 300], scale=1e-3, max_len=319)


def test_the_same_numbers_in_16_bits_give_the_same_bits(B):
    """Codes become the numbers they stand for before the products, so a cache of these numbers in 16 bits gives what they give, up to the order in which elements
    of a head are added."""
    for td in TYPES:
        b = ref.Batch([4, 4, 4], [600, 90, 33], 16, ragged=False)
        c = Cache(b, 2, 128, td)
        q, batch = b.heads(8, 128, td).to(DEV), b.on_gpu(B)
        k, v = (torch.nan_to_num(x).to(td).to(DEV) for x in c.numbers())
        a, d = B.spec_paged8_attention(c.on_gpu(B), batch, q).double(), B.spec_paged_attention(B.PagedCache(k, v), batch, q).double()
        # two roundings of weights and two of results apart at most
        assert (a - d).norm() <= 4 * ref.UNIT[td] * d.norm()


def test_two_calls_at_once_and_another_stream(B):
    td, b = torch.bfloat16, ref.Batch([1, 1], [4000, 300], 64, ragged=False)
    c = Cache(b, 2, 128, td)
    q, batch, cache = b.heads(8, 128, td).to(DEV), b.on_gpu(B), c.on_gpu(B)
    want = B.spec_paged8_attention(cache, batch, q)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        with torch.cuda.stream(s):
            outs.append([B.spec_paged8_attention(cache, batch, q) for _ in range(3)])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for out in outs for o in out)


def test_replayed_graph_follows_lengths_pages_and_contents(B):
    td, b = torch.float16, ref.Batch([2, 2], [3000, 700], 16, ragged=False)
    c = Cache(b, 1, 64, td)
    q, batch, cache = b.heads(4, 64, td).to(DEV), b.on_gpu(B, max_len=3008), c.on_gpu(B)
    out = torch.zeros_like(q)
    space = torch.empty(B.spec_paged8_attention_workspace_bytes(cache, batch, 4), dtype=torch.uint8, device=DEV)
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s), torch.cuda.graph(g, stream=s):
        B.spec_paged8_attention(cache, batch, q, out=out, workspace=space)
    for step in range(4):
        q.copy_(torch.randn_like(q))
        batch.lengths.sub_(37 * step)
        batch.pages[0, :2] = batch.pages[0, :2].flip(0)
        want = B.spec_paged8_attention(cache, batch, q)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("td", TYPES)
def test_a_verification_pass_with_all_operators(B, td):
    """Two rounds of a caller's model of two layers over caches of 8 bits: product, normed and rotated append, attention, product, logits' rules, truncation,
    acceptance.  The second round's rows overwrite what the first rejected.  Against the same pass computed in 64 bits from the codes that the appends left."""
    torch.manual_seed(3)
    nB, s, Hq, Hk, hd, V, page = 5, 3, 4, 2, 64, 1000, 16
    d, rows = Hq * hd, nB * (s + 1)
    W = [(torch.randn(((Hq + 2 * Hk) * hd, d), device=DEV) / d ** 0.5).to(td) for _ in range(2)]
    head, norms = (torch.randn((V, d), device=DEV) / d ** 0.25).to(td), [(1 + 0.1 * torch.randn(hd, device=DEV)).to(td) for _ in range(2)]
    freq = B.spec_rope_frequencies(10000.0, hd)
    t = B.HeadTransform(freq, True, *norms, eps=1e-5)
    b = ref.Batch([s + 1] * nB, [s + 1, 20, 40, 90, 200], page, ragged=False)
    caches, batch = [Cache(b, Hk, hd, td).on_gpu(B) for _ in range(2)], b.on_gpu(B)
    rules = B.SamplingRules(temperature=torch.tensor([0.0, 0.8, 1.0, 1.2, 0.0], device=DEV), top_k=torch.full((nB,), 20, dtype=torch.int32, device=DEV),
                            top_p=torch.full((nB,), 0.9, device=DEV))
    x = torch.randn((rows, d), device=DEV).to(td)
    for round_ in range(2):
        h = x
        for layer in range(2):
            qkv = (h @ W[layer].t()).view(rows, Hq + 2 * Hk, hd)
            q, k, v = qkv.split([Hq, Hk, Hk], dim=1)
            q = B.spec_paged8_append(caches[layer], batch, q, k, v, t)
            o = B.spec_paged8_attention(caches[layer], batch, q)
            kp, vp = (ref.decode(p.view(torch.uint8).cpu()) * torch.ldexp(torch.ones((), dtype=torch.float64), sc.cpu().transpose(1, 2).int() - 127)[..., None]
                      for p, sc in ((caches[layer].k, caches[layer].k_scale), (caches[layer].v, caches[layer].v_scale)))
            b.lens = batch.lengths.cpu().tolist()
            want, err = ref.attention(kp, vp, b, q.cpu(), hd ** -0.5, 0)
            close(o.cpu(), want, err, td)
            h = h + o.view(rows, d)
        logits = (h @ head.t()).view(nB, s + 1, V)
        proposals = logits[:, :s].float().argmax(-1).to(torch.int32)
        proposals[1::2, 1] = (proposals[1::2, 1] + 1) % V
        p, _ = B.spec_truncate_logits(B.spec_process_logits(logits, B.LogitRules()), rules)
        u = torch.rand((nB, s + 1, 3), device=DEV)
        chosen, accepted, emitted = B.spec_sample_accept(p, None, proposals, u, 1.0)
        ga, ge = B.spec_greedy_accept(logits.float(), proposals)
        assert torch.equal(accepted[[0, 4]], ga[[0, 4]]) and torch.equal(emitted[[0, 4]], ge[[0, 4]])
        for i in range(nB):
            for j in range(int(accepted[i]) + 1):
                assert p[i, j, emitted[i, j]] > -math.inf
        # the next pass's lengths: what was accepted, and its own rows (at most the pages that there are)
        batch.lengths.add_(accepted - s).add_(1).clamp_(max=200)
        x = torch.randn((rows, d), device=DEV).to(td)
