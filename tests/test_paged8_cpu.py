"""The refusals of the normed append and of the operators over a cache of 8 bits, every one before any device call; and the reference's e4m3."""
import ctypes as C

import pytest
import torch

import paged8_reference as ref

FAKE = 4096  # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def B():
    from paper_2310_18813_amd import binding
    return binding


def cache(lib, **kw):
    d = dict(dtype=lib.DTYPE_BF16, head_dim=128, n_kv_heads=2, page_size=16, n_pages=10, page_stride=16 * 2 * 128, pos_stride=2 * 128, head_stride=128,
             d_k=FAKE, d_v=FAKE)
    d.update(kw)
    return lib.PagedCacheDesc(**d)


def cache8(lib, **kw):
    d = dict(dtype=lib.DTYPE_BF16, head_dim=128, n_kv_heads=2, page_size=16, n_pages=10, page_stride=16 * 2 * 128, pos_stride=2 * 128, head_stride=128,
             d_k=FAKE, d_v=FAKE, d_k_scale=FAKE, d_v_scale=FAKE)
    d.update(kw)
    return lib.PagedCache8Desc(**d)


def batch(lib, **kw):
    d = dict(B=2, rows=6, max_rows=3, max_len=160, d_row_start=None, d_len=FAKE, d_pages=FAKE, pages_stride=10)
    d.update(kw)
    return lib.PagedBatchDesc(**d)


def transform(lib, **kw):
    d = dict(d_inv_freq=FAKE, rope_dim=128, interleaved=0, d_q_norm=FAKE, d_k_norm=FAKE, eps=1e-6)
    d.update(kw)
    return lib.HeadTransformDesc(**d)


def append(B, c, b, t=None, **kw):
    a = dict(nq=4, q=FAKE, qs=512, k=FAKE, ks=256, v=FAKE, vs=256, out=FAKE, outs=512)
    a.update(kw)
    fn = B.lib.spec_paged8_append if isinstance(c, B.PagedCache8Desc) else B.lib.spec_paged_append_normed
    return fn(None, C.byref(c), C.byref(b), None if t is False else C.byref(t if t is not None else transform(B)), *a.values())


def read(B, c, b, k=FAKE, ks=256, v=FAKE, vs=256):
    return B.lib.spec_paged8_read(None, C.byref(c), C.byref(b), k, ks, v, vs)


BAD_CACHE8 = [(dict(dtype=3), "INVALID_ARG"), (dict(dtype=0), "UNSUPPORTED"), (dict(head_dim=96), "UNSUPPORTED"), (dict(page_size=24), "UNSUPPORTED"),
              (dict(page_size=4), "UNSUPPORTED"), (dict(page_size=2048), "UNSUPPORTED"), (dict(n_pages=0), "INVALID_ARG"), (dict(n_kv_heads=0), "INVALID_ARG"),
              (dict(d_k=None), "INVALID_ARG"), (dict(d_v=FAKE + 8), "INVALID_ARG"), (dict(pos_stride=248), "INVALID_ARG"), (dict(pos_stride=64), "INVALID_ARG"),
              (dict(head_stride=64), "INVALID_ARG"), (dict(page_stride=-4096), "INVALID_ARG"), (dict(page_stride=1 << 36), "CAPACITY"),
              (dict(d_k_scale=None), "INVALID_ARG"), (dict(d_v_scale=FAKE + 4), "INVALID_ARG")]
BAD_BATCH = [(dict(B=-1), "INVALID_ARG"), (dict(rows=7), "INVALID_ARG"), (dict(B=65536, rows=65536), "CAPACITY"), (dict(max_rows=2), "INVALID_ARG"),
             (dict(max_len=161), "INVALID_ARG"), (dict(d_len=None), "INVALID_ARG"), (dict(d_pages=None), "INVALID_ARG")]


def test_descriptions_of_the_cache_of_8_bits_and_the_batch(B):
    for call, who in ((append, b"spec_paged8_append"), (read, b"spec_paged8_read")):
        for kw, code in BAD_CACHE8:
            assert call(B, cache8(B, **kw), batch(B)) == getattr(B, "ERR_" + code), kw
            assert who in B.lib.spec_last_error(None)
        for kw, code in BAD_BATCH:
            assert call(B, cache8(B), batch(B, **kw)) == getattr(B, "ERR_" + code), kw
        assert call(B, cache8(B), batch(B, B=0, rows=0)) == B.OK and call(B, cache8(B), batch(B, rows=0)) == B.OK  # nothing to do
    assert B.lib.spec_paged8_append(None, None, C.byref(batch(B)), None, *([0] * 9)) == B.ERR_INVALID_ARG
    assert B.lib.spec_paged8_read(None, C.byref(cache8(B)), None, FAKE, 256, FAKE, 256) == B.ERR_INVALID_ARG
    assert append(B, cache(B, dtype=3), batch(B)) == B.ERR_INVALID_ARG and b"spec_paged_append_normed" in B.lib.spec_last_error(None)


def test_transforms_and_rows(B):
    inf, nan = float("inf"), float("nan")
    for c in (cache(B), cache8(B)):
        for kw in (dict(rope_dim=136), dict(rope_dim=8), dict(rope_dim=-16), dict(d_inv_freq=None), dict(interleaved=2), dict(eps=0.0), dict(eps=-1.0),
                   dict(eps=inf), dict(eps=nan), dict(d_q_norm=FAKE + 8), dict(d_k_norm=FAKE + 2), dict(d_q_norm=None, eps=0.0)):
            assert append(B, c, batch(B), transform(B, **kw)) == B.ERR_INVALID_ARG, kw
        for kw in (dict(nq=-1), dict(nq=65536), dict(q=None), dict(qs=504), dict(qs=516), dict(out=None), dict(outs=1024), dict(k=FAKE + 2), dict(ks=128),
                   dict(v=None), dict(vs=260)):
            for t in (None, False):
                assert append(B, c, batch(B), t, **kw) == B.ERR_INVALID_ARG, kw
        assert append(B, c, batch(B, rows=1 << 29, max_rows=1 << 29, d_row_start=FAKE)) == B.ERR_CAPACITY
    for kw in (dict(k=None, v=None), dict(k=FAKE + 8), dict(ks=248), dict(ks=260), dict(v=FAKE + 2), dict(vs=0)):
        assert read(B, cache8(B), batch(B), **kw) == B.ERR_INVALID_ARG, kw
    assert read(B, cache8(B, n_kv_heads=64, pos_stride=64 * 128), batch(B, rows=1 << 28, max_rows=1 << 28, d_row_start=FAKE), ks=8192, vs=8192) == B.ERR_CAPACITY


def test_tensors_of_the_host_are_refused(B):
    pages, scales = torch.zeros((2, 8, 1, 64), dtype=torch.uint8), torch.zeros((2, 1, 8), dtype=torch.uint8)
    with pytest.raises(AssertionError):
        B.PagedCache8(pages, pages, scales, scales, torch.bfloat16)
    with pytest.raises(AssertionError):
        B.HeadTransform(q_norm=torch.ones(64, dtype=torch.bfloat16))


@pytest.mark.parametrize("td", [torch.bfloat16, torch.float16])
def test_the_reference_agrees_with_torch_about_e4m3(td):
    assert torch.equal(ref.decode(torch.arange(127, dtype=torch.uint8)), torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double())
    x = torch.randn((200, 64), generator=torch.Generator().manual_seed(1)).to(td)
    codes, e, _ = ref.encode(x.double(), td)
    assert torch.equal(codes, torch.ldexp(x.float(), -e[:, None]).to(torch.float8_e4m3fn).view(torch.uint8))
    top = x.double().abs().amax(-1)
    assert (top <= 448 * 2.0 ** e).all() and (top > 224 * 2.0 ** e).all()


def test_truncation_arguments(B):
    def call(rules=True, logits=FAKE, dtype=B.DTYPE_F32, stride=1000, nB=2, s=3, V=1000, u=FAKE, ws=None, wb=0, out=FAKE + 64, tokens=FAKE):
        return B.lib.spec_truncate_logits(None, logits, dtype, stride, nB, s, V, C.byref(B.SamplingRulesDesc()) if rules else None, u, ws, wb, out, tokens)
    for kw in (dict(nB=-1), dict(s=-1), dict(V=0), dict(dtype=7), dict(stride=999), dict(rules=False), dict(logits=None), dict(out=None, tokens=None),
               dict(u=None), dict(logits=FAKE + 2), dict(out=FAKE + 2), dict(dtype=B.DTYPE_BF16, out=FAKE), dict(stride=1004, out=FAKE)):
        assert call(**kw) == B.ERR_INVALID_ARG, kw
        assert b"spec_truncate_logits" in B.lib.spec_last_error(None)
    for kw in (dict(s=16), dict(nB=65536), dict(V=(1 << 28) + 1, stride=1 << 29)):
        assert call(**kw) == B.ERR_CAPACITY, kw
    assert call(nB=0, logits=None, out=None, tokens=None) == B.OK
    n = C.c_size_t(1)
    assert B.lib.spec_truncate_logits_workspace_bytes(2, 3, 1000, C.byref(n)) == B.OK and n.value > 1
    for kw in (dict(), dict(ws=FAKE + 16, wb=n.value), dict(ws=FAKE, wb=n.value - 1)):
        assert call(**kw) == B.ERR_WORKSPACE
    assert B.lib.spec_truncate_logits_workspace_bytes(65535, 15, 1 << 28, C.byref(n)) == B.OK
    assert B.lib.spec_truncate_logits_workspace_bytes(1, 16, 32000, C.byref(n)) == B.ERR_CAPACITY
    assert B.lib.spec_truncate_logits_workspace_bytes(1, 0, 0, C.byref(n)) == B.ERR_INVALID_ARG
    assert B.lib.spec_truncate_logits_workspace_bytes(1, 0, 10, None) == B.ERR_INVALID_ARG
    with pytest.raises(AssertionError):
        B.SamplingRules(top_p=torch.ones(2))


def test_attention_over_8_bits_arguments(B):
    def attend(c, b, **kw):
        a = dict(nq=4, q=FAKE, qs=512, scale=0.1, window=0, ws=None, wb=0, out=FAKE, outs=512)
        a.update(kw)
        return B.lib.spec_paged8_attention(None, C.byref(c) if c else None, C.byref(b) if b else None, *a.values())
    for kw, code in BAD_CACHE8:
        assert attend(cache8(B, **kw), batch(B)) == getattr(B, "ERR_" + code), kw
        assert b"spec_paged8_attention" in B.lib.spec_last_error(None)
    for kw, code in BAD_BATCH:
        assert attend(cache8(B), batch(B, **kw)) == getattr(B, "ERR_" + code), kw
    assert attend(None, batch(B)) == attend(cache8(B), None) == B.ERR_INVALID_ARG
    for kw in (dict(nq=0), dict(nq=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(scale=2.4e38), dict(window=-1),
               dict(q=None), dict(q=FAKE + 8), dict(qs=500), dict(out=None), dict(outs=256)):
        assert attend(cache8(B), batch(B), **kw) == B.ERR_INVALID_ARG, kw
    long, n = batch(B, pages_stride=1000, max_len=16000), C.c_size_t(0)
    assert B.lib.spec_paged8_attention_workspace_bytes(C.byref(cache8(B)), C.byref(long), 4, C.byref(n)) == B.OK and n.value > 0
    for kw in (dict(), dict(ws=FAKE + 16, wb=n.value), dict(ws=FAKE, wb=n.value - 1)):
        assert attend(cache8(B), long, **kw) == B.ERR_WORKSPACE
    assert attend(cache8(B), batch(B, rows=1 << 29, max_rows=1 << 29, d_row_start=FAKE)) == B.ERR_CAPACITY
    assert attend(cache8(B), batch(B, B=0, rows=0)) == B.OK and attend(cache8(B), batch(B, rows=0)) == B.OK
    assert B.lib.spec_paged8_attention_workspace_bytes(C.byref(cache8(B, dtype=0)), C.byref(long), 4, C.byref(n)) == B.ERR_UNSUPPORTED
    assert B.lib.spec_paged8_attention_workspace_bytes(C.byref(cache8(B)), C.byref(long), 4, None) == B.ERR_INVALID_ARG
