"""The refusals of the operators over a paged cache: every one before any device call, so without a GPU."""
import ctypes as C

import pytest
import torch

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


def batch(lib, **kw):
    d = dict(B=2, rows=6, max_rows=3, max_len=160, d_row_start=None, d_len=FAKE, d_pages=FAKE, pages_stride=10)
    d.update(kw)
    return lib.PagedBatchDesc(**d)


def append(B, c, b, **kw):
    a = dict(nq=4, q=FAKE, qs=512, k=FAKE, ks=256, v=FAKE, vs=256, freq=FAKE, rot=128, out=FAKE, outs=512)
    a.update(kw)
    return B.lib.spec_paged_append(None, C.byref(c), C.byref(b), *a.values())


def attend(B, c, b, **kw):
    a = dict(nq=4, q=FAKE, qs=512, scale=0.1, window=0, ws=None, wb=0, out=FAKE, outs=512)
    a.update(kw)
    return B.lib.spec_paged_attention(None, C.byref(c), C.byref(b), *a.values())


def test_cache_and_batch_descriptions(B):
    bad_cache = [(dict(dtype=3), B.ERR_INVALID_ARG), (dict(head_dim=96), B.ERR_UNSUPPORTED), (dict(page_size=24), B.ERR_UNSUPPORTED),
                 (dict(page_size=4), B.ERR_UNSUPPORTED), (dict(page_size=2048), B.ERR_UNSUPPORTED), (dict(n_pages=0), B.ERR_INVALID_ARG),
                 (dict(n_kv_heads=0), B.ERR_INVALID_ARG), (dict(d_k=None), B.ERR_INVALID_ARG), (dict(d_v=FAKE + 8), B.ERR_INVALID_ARG),
                 (dict(pos_stride=252), B.ERR_INVALID_ARG), (dict(pos_stride=64), B.ERR_INVALID_ARG), (dict(head_stride=64), B.ERR_INVALID_ARG),
                 (dict(page_stride=-4096), B.ERR_INVALID_ARG), (dict(page_stride=1 << 35), B.ERR_CAPACITY), (dict(pos_stride=1 << 35), B.ERR_CAPACITY),
                 (dict(head_stride=1 << 35), B.ERR_CAPACITY)]
    bad_batch = [(dict(B=-1), B.ERR_INVALID_ARG), (dict(rows=-1), B.ERR_INVALID_ARG), (dict(B=65536, rows=65536), B.ERR_CAPACITY),
                 (dict(rows=7), B.ERR_INVALID_ARG), (dict(max_rows=2), B.ERR_INVALID_ARG), (dict(max_rows=7), B.ERR_INVALID_ARG),
                 (dict(max_rows=0, d_row_start=FAKE), B.ERR_INVALID_ARG), (dict(max_len=161), B.ERR_INVALID_ARG), (dict(max_len=0), B.ERR_INVALID_ARG),
                 (dict(d_len=None), B.ERR_INVALID_ARG), (dict(d_pages=None), B.ERR_INVALID_ARG),
                 (dict(pages_stride=1 << 28, max_len=(1 << 30) + 1), B.ERR_CAPACITY)]
    n = C.c_size_t(0)
    for call, who in ((append, b"spec_paged_append"), (attend, b"spec_paged_attention")):
        for kw, code in bad_cache:
            assert call(B, cache(B, **kw), batch(B)) == code, kw
            assert who in B.lib.spec_last_error(None)
        for kw, code in bad_batch:
            assert call(B, cache(B), batch(B, **kw)) == code, kw
            assert who in B.lib.spec_last_error(None)
        assert call(B, cache(B), batch(B, B=0, rows=0)) == B.OK and call(B, cache(B), batch(B, rows=0)) == B.OK  # nothing to do
    assert B.lib.spec_paged_attention_workspace_bytes(C.byref(cache(B)), None, 4, C.byref(n)) == B.ERR_INVALID_ARG
    assert B.lib.spec_paged_attention_workspace_bytes(C.byref(cache(B)), C.byref(batch(B)), 4, None) == B.ERR_INVALID_ARG
    assert B.lib.spec_paged_append(None, None, C.byref(batch(B)), *([0] * 11)) == B.ERR_INVALID_ARG


def test_append_arguments(B):
    for kw in (dict(rot=136), dict(rot=8), dict(rot=-16), dict(freq=None), dict(nq=-1), dict(q=None), dict(qs=504), dict(qs=516), dict(out=None),
               dict(outs=1024), dict(k=FAKE + 2), dict(ks=128), dict(v=None), dict(vs=260)):
        assert append(B, cache(B), batch(B), **kw) == B.ERR_INVALID_ARG, kw
    assert append(B, cache(B), batch(B, rows=1 << 29, max_rows=1 << 29, d_row_start=FAKE)) == B.ERR_CAPACITY


def test_attention_arguments(B):
    for kw in (dict(nq=0), dict(nq=3), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(window=-1),
               dict(q=None), dict(q=FAKE + 8), dict(qs=500), dict(out=None), dict(outs=256)):
        assert attend(B, cache(B), batch(B), **kw) == B.ERR_INVALID_ARG, kw
    long = batch(B, pages_stride=1000, max_len=16000)
    n = C.c_size_t(0)
    assert B.lib.spec_paged_attention_workspace_bytes(C.byref(cache(B)), C.byref(long), 4, C.byref(n)) == B.OK and n.value > 0
    assert attend(B, cache(B), long) == B.ERR_WORKSPACE
    assert attend(B, cache(B), long, ws=FAKE + 16, wb=n.value) == B.ERR_WORKSPACE
    assert attend(B, cache(B), long, ws=FAKE, wb=n.value - 1) == B.ERR_WORKSPACE
    many = batch(B, rows=1 << 29, max_rows=1 << 29, d_row_start=FAKE)
    assert attend(B, cache(B), many) == B.ERR_CAPACITY


def test_attention_scales_whose_power_of_two_form_is_infinite(B):
    for scale in (2.4e38, 3.4e38):
        assert attend(B, cache(B), batch(B), scale=scale) == B.ERR_INVALID_ARG
    assert attend(B, cache(B), batch(B, B=0, rows=0), scale=2.3e38) == B.OK


def test_logit_rules_arguments(B):
    def call(rules=None, logits=FAKE, dtype=B.DTYPE_F32, stride=1000, nB=2, s=3, V=1000, t=FAKE, out=FAKE + 64, **kw):
        r = rules if rules is not None else B.LogitRulesDesc(**kw)
        return B.lib.spec_process_logits(None, logits, dtype, stride, nB, s, V, C.byref(r) if r else None, t, out)
    for kw in (dict(nB=-1), dict(s=-1), dict(V=0), dict(dtype=7), dict(stride=999), dict(rules=False), dict(n_bias=-1), dict(n_bias=3),
               dict(n_bias=3, d_bias=FAKE), dict(d_mask=FAKE, mask_rows=2), dict(d_mask=FAKE), dict(d_tokens=FAKE, tokens_stride=9),
               dict(d_tokens=FAKE, d_len=FAKE), dict(logits=None), dict(out=None), dict(logits=FAKE + 2), dict(out=FAKE + 2),
               dict(dtype=B.DTYPE_BF16, out=FAKE), dict(stride=1004, out=FAKE)):
        assert call(**kw) == B.ERR_INVALID_ARG, kw
        assert b"spec_process_logits" in B.lib.spec_last_error(None)
    for kw in (dict(s=16), dict(nB=65536), dict(V=(1 << 28) + 1, stride=1 << 29), dict(n_bias=4097, d_bias=FAKE, d_bias_ids=FAKE),
               dict(d_tokens=FAKE, d_len=FAKE, tokens_stride=1 << 30)):
        assert call(**kw) == B.ERR_CAPACITY, kw
    assert call(nB=0, logits=None, out=None) == B.OK
    assert B.lib.spec_set_logit_rules(None, None, None) == B.ERR_INVALID_ARG


def test_tensors_of_the_host_are_refused(B):
    """a kernel would take their addresses for the device's"""
    i32 = dict(dtype=torch.int32)
    with pytest.raises(AssertionError):
        B.PagedBatch(torch.zeros((2, 4), **i32), torch.ones(2, **i32), 2)
    for kw in (dict(length=torch.zeros(2, **i32)), dict(repetition=torch.ones(2)), dict(mask=torch.zeros((2, 1, 4), **i32))):
        with pytest.raises(AssertionError):
            B.LogitRules(**kw)
    with pytest.raises(AssertionError):
        B.spec_process_logits(torch.zeros((2, 1, 64)), B.LogitRules())
