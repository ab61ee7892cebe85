"""spec_paged_append_normed, spec_paged8_append and spec_paged8_read against their definition in 64 bits: types, head layouts, norms, both ways to
pair elements, rows that do not count, pages in any order or absent, strides, values at the edges of codes and types."""
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


def transform_of(B, hd, rot, interleaved, norm, td, seed=0):
    """-> (HeadTransform, (inv_freq, q weights, k weights) on the CPU)"""
    g = torch.Generator().manual_seed(seed + 9)
    freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot) if rot else None
    qw, kw = ((1 + 0.3 * torch.randn(hd, generator=g)).to(td) if norm else None for _ in range(2))
    on = [None if x is None else x.to(DEV) for x in (freq, qw, kw)]
    return B.HeadTransform(on[0], interleaved, on[1], on[2], 1e-5), (freq, qw, kw)


SHAPES = [
    # dtype heads kv hd page rot interleaved norm layout wide
    ("bf16", 4, 2, 128, 16, 128, False, True, "nhd", 0),
    ("bf16", 3, 1, 64, 8, 64, True, True, "hnd", 2),
    ("fp16", 8, 8, 128, 32, 64, True, False, "nhd", 3),
    ("fp16", 2, 2, 64, 64, 16, False, True, "hnd", 0),
    ("bf16", 40, 8, 128, 16, 96, False, True, "nhd", 1),   # several workgroups a row, a part that passes
    ("fp16", 1, 1, 64, 16, 0, False, True, "nhd", 0),
    ("bf16", 5, 5, 64, 16, 48, True, False, "nhd", 0),
    ("bf16", 4, 4, 128, 128, 0, False, False, "nhd", 0),
]
BATCHES = [
    ([1], [1], False, ()),
    ([3, 3], [7, 40], False, ()),
    ([2, 0, 5, 1], [2, 9, 3, 70], True, ((3, 4),)),       # no rows, dead rows, a row whose page is absent
]


@pytest.mark.parametrize("shape", SHAPES + [("fp32", 4, 2, 128, 16, 128, True, True, "nhd", 0), ("fp32", 3, 3, 64, 8, 32, False, True, "hnd", 1),
                                            ("fp32", 2, 1, 64, 8, 64, True, False, "nhd", 2)])
@pytest.mark.parametrize("rows,lens,ragged,absent", BATCHES)
def test_normed_append(B, shape, rows, lens, ragged, absent):
    dtype, Hq, Hk, hd, page, rot, inter, norm, layout, wide = shape
    td, mark = ref.TYPES[dtype], 77.0
    b = ref.Batch(rows, lens, page, ragged=ragged, absent=absent if page == 16 else ())
    t, (freq, qw, kw) = transform_of(B, hd, rot, inter, norm, td)
    q, k, v = b.heads(Hq, hd, td, wide), b.heads(Hk, hd, td, wide), b.heads(Hk, hd, td)
    start = [torch.full((b.n_pages, page, Hk, hd), mark, dtype=td) for _ in range(2)]
    kp, vp = (ref.pool(x, layout) for x in start)
    out = torch.full((b.T, Hq, hd), mark, dtype=td, device=DEV)
    big = q.to(DEV) if not wide else torch.cat([torch.zeros((b.T, wide, hd), dtype=td), q], 1).to(DEV)[:, wide:]
    got = B.spec_paged_append_normed(B.PagedCache(kp, vp), b.on_gpu(B), big, k.contiguous().to(DEV), v.to(DEV), t, out=out)
    assert got.data_ptr() == out.data_ptr()
    want_q, want_k, want_v = (torch.full(x.shape, mark, dtype=torch.float64) for x in (q, start[0], start[1]))
    eq, ek = torch.zeros_like(want_q), torch.zeros_like(want_k)
    u = ref.UNIT[td]
    changed = bool(rot or norm)
    for _, row, pos, pg, at in b.places():
        want_q[row], e = ref.transform(q[row], pos, qw, 1e-5, freq, inter)
        eq[row] = e + (u * (want_q[row].abs() + e) if changed else 0)
        if pg >= 0:
            want_k[pg, at], e = ref.transform(k[row], pos, kw, 1e-5, freq, inter)
            ek[pg, at] = e + (u * (want_k[pg, at].abs() + e) if changed else 0)
            want_v[pg, at] = v[row].double()
    assert ((out.cpu().double() - want_q).abs() <= eq).all()
    assert ((kp.cpu().double() - want_k).abs() <= ek).all()
    assert torch.equal(vp.cpu().double(), want_v)


def check_codes(codes, scale, want, want_e, gap, where):
    """Codes [heads][hd] and scale bytes [heads] of one position; elsewhere than within 1e-9 of a border of two codes they are the definition's.  (64 bits: some
    thirty roundings of 2^-53, and an angle of up to 1e5 off by 2^-52 of itself: 3e-11.)"""
    assert torch.equal(scale.long(), want_e.long() + 127), where
    off = codes != want
    assert not (off & (gap > 1e-9 * 448)).any(), where


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("rows,lens,ragged,absent", BATCHES)
def test_append_of_8_bits_and_back(B, shape, rows, lens, ragged, absent):
    dtype, Hq, Hk, hd, page, rot, inter, norm, layout, wide = shape
    td, mark = ref.TYPES[dtype], 0x2b
    b = ref.Batch(rows, lens, page, seed=1, ragged=ragged, absent=absent if page == 16 else ())
    t, (freq, qw, kw) = transform_of(B, hd, rot, inter, norm, td)
    q, k, v = b.heads(Hq, hd, td), b.heads(Hk, hd, td, wide, size=30.0), b.heads(Hk, hd, td, wide, size=1e-3)
    kp, vp = (ref.pool(torch.full((b.n_pages, page, Hk, hd), mark, dtype=torch.uint8), layout) for _ in range(2))
    ks, vs = (torch.full((b.n_pages, Hk, page), mark, dtype=torch.uint8, device=DEV) for _ in range(2))
    cache, batch = B.PagedCache8(kp.view(torch.float8_e4m3fn), vp.view(torch.float8_e4m3fn), ks, vs, td), b.on_gpu(B)
    out = torch.full((b.T, Hq, hd), 77.0, dtype=td, device=DEV)

    def wider(x):
        return x.to(DEV) if not wide else torch.cat([torch.zeros((b.T, wide, hd), dtype=td), x], 1).to(DEV)[:, wide:]

    B.spec_paged8_append(cache, batch, q.to(DEV), wider(k), wider(v), t, out=out)
    back = [torch.full((b.T, Hk + 1, hd), 77.0, dtype=td, device=DEV)[:, 1:] for _ in range(2)]
    B.spec_paged8_read(cache, batch, *back)
    kc, vc, ksc, vsc, out, kb, vb = (x.cpu() for x in (kp, vp, ks, vs, out, *back))
    owned, u = torch.zeros((b.n_pages, page), dtype=torch.bool), ref.UNIT[td]
    alive = {row for _, row, *_ in b.places()}
    for _, row, pos, pg, at in b.places():
        want, e = ref.transform(q[row], pos, qw, 1e-5, freq, inter)
        assert ((out[row].double() - want).abs() <= e + (u * (want.abs() + e) if rot or norm else 0)).all()
        if pg < 0:
            assert not kb[row].any() and not vb[row].any()
            continue
        owned[pg, at] = True
        for x, w, codes, scales, read in ((k, kw, kc, ksc, kb), (v, None, vc, vsc, vb)):
            y = ref.transform(x[row], pos, w, 1e-5, freq if x is k else None, inter)[0]
            check_codes(codes[pg, at], scales[pg, :, at], *ref.encode(y, td), (row, pos))
            stands = ref.decode(codes[pg, at]) * torch.ldexp(torch.ones(Hk, dtype=torch.float64), scales[pg, :, at].int() - 127)[:, None]
            assert torch.equal(read[row].double(), stands)  # exactly: every code times its scale is a number of the type
    for row in set(range(b.T)) - alive:
        assert (out[row] == 77.0).all() and (kb[row] == 77.0).all() and (vb[row] == 77.0).all()
    assert (kc[~owned] == mark).all() and (vc[~owned] == mark).all()
    assert (ksc.transpose(1, 2)[~owned] == mark).all() and (vsc.transpose(1, 2)[~owned] == mark).all()


def test_more_than_64_sequences(B):
    g = torch.Generator().manual_seed(22)
    rows, lens = torch.randint(0, 3, (150,), generator=g).tolist(), torch.randint(0, 60, (150,), generator=g).tolist()
    test_append_of_8_bits_and_back(B, SHAPES[1], rows, lens, True, ())
    test_append_of_8_bits_and_back(B, SHAPES[3], [1] * 150, lens, False, ())
    test_normed_append(B, SHAPES[0], rows, lens, True, ())


def one_row(B, td, x, hd):
    """x [heads][hd] as the values of one position of a cache of 8 bits -> (codes, scale bytes, what is read back), on the CPU."""
    Hk = x.shape[0]
    cache = B.PagedCache8.empty(1, 8, Hk, hd, td, DEV)
    batch = B.PagedBatch(torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV), 1)
    B.spec_paged8_append(cache, batch, None, torch.zeros((1, Hk, hd), dtype=td, device=DEV), x[None].to(DEV))
    back = B.spec_paged8_read(cache, batch)[1][0]
    return cache.v.view(torch.uint8)[0, 0].cpu(), cache.v_scale[0, :, 0].cpu(), back.cpu()


@pytest.mark.parametrize("td", [torch.bfloat16, torch.float16])
def test_every_value_of_the_types_becomes_its_code(B, td):
    """All finite magnitudes of a type beside a largest one that fixes the scale: ties, subnormal codes, zeros and signs; and heads whose largest is at the
    border of two scales."""
    bits = torch.arange(0, 0x7f80 if td == torch.bfloat16 else 0x7c00, dtype=torch.int32)
    every = bits.to(torch.int16).view(td)
    for top in (1.0, 448.0, 449.0 if td == torch.float16 else 450.0, 3.0e4):
        x = every[every <= top]
        n = (x.shape[0] + 62) // 63
        x = torch.cat([x, torch.zeros(63 * n - x.shape[0], dtype=td)]).view(n, 63)
        x[:, 1::2] = -x[:, 1::2]
        x = torch.cat([torch.full((n, 1), top, dtype=td), x], 1)
        codes, scale, back = one_row(B, td, x, 64)
        want, e, _ = ref.encode(x.double(), td)
        assert torch.equal(codes, want) and torch.equal(scale.long(), e + 127)
        assert torch.equal(back.double(), ref.decode(codes) * torch.ldexp(torch.ones(n, dtype=torch.float64), e.int())[:, None])


@pytest.mark.parametrize("td", [torch.bfloat16, torch.float16])
def test_every_code_is_read_exactly(B, td):
    """All 256 codes under every scale that an append can write (as far as the type holds the product)."""
    lo, hi = (ref.LEAST[td], 119) if td == torch.bfloat16 else (ref.LEAST[td], 7)
    n = hi - lo + 1
    cache = B.PagedCache8.empty(1, 8, n, 128, td, DEV)
    codes = torch.arange(256, dtype=torch.uint8).view(2, 1, 128).expand(2, n, 128)
    cache.k.view(torch.uint8)[0, :2] = codes.to(DEV)
    cache.k_scale[0] = (torch.arange(lo, hi + 1)[:, None] + 127).to(torch.uint8).to(DEV)
    batch = B.PagedBatch(torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.full((1,), 2, dtype=torch.int32, device=DEV), 2)
    got = B.spec_paged8_read(cache, batch)[0].cpu().double()
    want = ref.decode(codes) * torch.ldexp(torch.ones(n, dtype=torch.float64), torch.arange(lo, hi + 1))[None, :, None]
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


@pytest.mark.parametrize("td", [torch.bfloat16, torch.float16])
def test_heads_that_are_not_finite_and_the_edges_of_the_type(B, td):
    big = torch.finfo(td).max
    x = torch.zeros((8, 64), dtype=td)
    x[:, 5] = torch.tensor([math.nan, math.inf, -math.inf, big, -big, 0.0, torch.finfo(td).tiny, 2.0 ** -24 if td == torch.float16 else 2.0 ** -120])
    x[0, 6] = 1.0
    codes, scale, back = one_row(B, td, x, 64)
    assert (codes[:3] == 0x7f).all() and torch.isnan(back[:3]).all()
    assert torch.isfinite(back[3:]).all()
    want, e, _ = ref.encode(x.double(), td)
    assert torch.equal(codes, want) and torch.equal(scale.long(), e + 127)
    assert float(back[3, 5]) == ref.MOST[td] == -float(back[4, 5])
    assert not back[5].any() and not back[3, :5].any()


def test_keys_that_turn_out_of_fp16(B):
    """Rotation makes 65504 into up to 92636, which fp16 has no number for."""
    x = torch.full((1, 1, 64), 65504.0, dtype=torch.float16)
    cache = B.PagedCache8.empty(1, 8, 1, 64, torch.float16, DEV)
    batch = B.PagedBatch(torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.full((1,), 2, dtype=torch.int32, device=DEV), 1)
    t = B.HeadTransform(torch.full((32,), math.pi / 4, dtype=torch.float64, device=DEV))
    B.spec_paged8_append(cache, batch, None, x.to(DEV), x.to(DEV), t)
    k, v = B.spec_paged8_read(cache, batch)
    assert torch.isnan(k).all() and (v == 61440.0).all()


def test_norms_of_large_and_of_zero_heads(B):
    """Squares beyond fp32, and heads of zeros."""
    td = torch.bfloat16
    x = torch.stack([torch.full((64,), 1e30), torch.zeros(64), torch.full((64,), 1e-25)]).to(td)[:, None]
    w = torch.ones(64, dtype=td, device=DEV)
    b = B.PagedBatch(torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.full((1,), 3, dtype=torch.int32, device=DEV), 3)
    t = B.HeadTransform(q_norm=w, k_norm=w, eps=1e-6)
    pages = torch.zeros((2, 1, 8, 1, 64), dtype=td, device=DEV)
    q = B.spec_paged_append_normed(B.PagedCache(*pages), b, x.to(DEV), x.to(DEV), x.to(DEV), t).cpu()
    want = torch.stack([ref.transform(x[i], 0, w.cpu(), 1e-6, None, False)[0] for i in range(3)])
    for got in (q, pages[0, 0, :3].cpu()):
        assert ((got.double() - want).abs() <= 2.0 ** -8 * 1.001 * want.abs()).all()
    c8 = B.PagedCache8.empty(1, 8, 1, 64, td, DEV)
    B.spec_paged8_append(c8, b, None, x.to(DEV), x.to(DEV), t)
    codes, e, _ = ref.encode(want, td)
    assert torch.equal(c8.k.view(torch.uint8)[0, :3].cpu(), codes) and torch.equal(c8.k_scale[0, :, :3].t().cpu().long(), e + 127)


@pytest.mark.parametrize("td", [torch.float32, torch.bfloat16, torch.float16])
def test_norms_whose_root_is_beyond_fp32(B, td):
    """eps 1e-80 and elements down to 2^-149: one over the root is up to 1e40, and a head of zeros stays zeros."""
    hd = 64
    x = torch.zeros((1, 4, hd), dtype=torch.float64)
    x[0, 1] = torch.linspace(-1, 1, hd, dtype=torch.float64) * 2.0 ** (-12 if td is torch.float16 else -120)
    x[0, 2, 5] = 2.0 ** (-24 if td is torch.float16 else -133 if td is torch.bfloat16 else -149)
    x[0, 3] = 1e-6
    x = x.to(td)
    w = torch.ones(hd, dtype=td)
    t = B.HeadTransform(None, False, w.to(DEV), w.to(DEV), 1e-80)
    pages = [torch.zeros((1, 8, 4, hd), dtype=td, device=DEV) for _ in range(2)]
    batch = B.PagedBatch(torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV), 1)
    d = x.to(DEV)
    q = B.spec_paged_append_normed(B.PagedCache(*pages), batch, d, d, d, t).cpu().double()[0]
    want, e = ref.transform(x[0], 0, w, 1e-80, None, False)
    e = e + ref.UNIT[td] * (want.abs() + e)
    assert ((q - want).abs() <= e).all() and not q[0].any()
    assert ((pages[0][0, 0].cpu().double() - want).abs() <= e).all()


@pytest.mark.parametrize("norm", [False, True])
def test_in_place_and_on_another_stream(B, norm):
    td, b = torch.bfloat16, ref.Batch([4, 4], [60, 33], 16, ragged=False)
    t, _ = transform_of(B, 128, 128, True, norm, td)
    q, k, v = (x.to(DEV) for x in (b.heads(4, 128, td), b.heads(2, 128, td), b.heads(2, 128, td)))
    batch = b.on_gpu(B)
    one, two = (B.PagedCache8.empty(b.n_pages, 16, 2, 128, td, DEV) for _ in range(2))
    want = B.spec_paged8_append(one, batch, q, k, v, t)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        mine = q.clone()
        assert B.spec_paged8_append(two, batch, mine, k, v, t, out=mine) is mine
        B.spec_paged8_append(two, batch, None, k, v, t)
    s.synchronize()
    assert torch.equal(mine, want) and torch.equal(one.k.view(torch.uint8), two.k.view(torch.uint8)) and torch.equal(one.v_scale, two.v_scale)


def test_replayed_graph_follows_lengths_and_pages(B):
    td, b = torch.float16, ref.Batch([2, 2], [20, 9], 8, ragged=False)
    t, _ = transform_of(B, 64, 64, False, True, td)
    q, k, v = (x.to(DEV) for x in (b.heads(3, 64, td), b.heads(1, 64, td), b.heads(1, 64, td)))
    batch, cache = b.on_gpu(B), B.PagedCache8.empty(b.n_pages, 8, 1, 64, td, DEV)
    out, ko, vo = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            B.spec_paged8_append(cache, batch, q, k, v, t, out=out)
            B.spec_paged8_read(cache, batch, ko, vo)
    for step in range(4):
        q.copy_(torch.randn_like(q)); k.copy_(torch.randn_like(k)); v.copy_(torch.randn_like(v))
        batch.lengths.add_(1 if step else 0)
        batch.pages[:, :3] = batch.pages[:, :3].roll(1, 0)
        fresh = B.PagedCache8.empty(b.n_pages, 8, 1, 64, td, DEV)
        want = B.spec_paged8_append(fresh, batch, q, k, v, t)
        wk, wv = B.spec_paged8_read(fresh, batch)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(ko, wk) and torch.equal(vo, wv)


def test_without_a_transform_it_is_the_plain_append(B):
    td, b = torch.float16, ref.Batch([3, 1], [30, 8], 8)
    q, k, v = (x.to(DEV) for x in (b.heads(4, 64, td), b.heads(2, 64, td), b.heads(2, 64, td)))
    batch, freq = b.on_gpu(B), B.spec_rope_frequencies(10000.0, 64)
    a, c = (torch.zeros((2, b.n_pages, 8, 2, 64), dtype=td, device=DEV) for _ in range(2))
    for with_freq in (None, freq):
        want = B.spec_paged_append(B.PagedCache(*a), batch, q, k, v, with_freq)
        got = B.spec_paged_append_normed(B.PagedCache(*c), batch, q, k, v, None if with_freq is None else B.HeadTransform(with_freq))
        assert torch.equal(got[:4], want[:4]) and torch.equal(a, c)
