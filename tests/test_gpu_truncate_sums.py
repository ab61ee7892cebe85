"""spec_truncate_logits over large vocabularies.  Where its sums have most to add up: one likely token before a tail of equal, unlikely ones, whose weights are all off
in the same direction, so that their errors add up.  And every rule and the draw's ends where a piece of the row's maxima is more than 4096 tokens and a
stretch of a draw from the list more than 256, which they are above 262144."""
import math

import numpy as np
import pytest
import torch

from test_gpu_truncate import check, logits_of, rules_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def B():
    from paper_2310_18813_amd import binding
    return binding


def off(V):
    """What a sum of weights may be off by, relative: the exponential's 3e-13; each weight to a number of 62 - bits bits; what lies below 32 octaves, to 2^-(94 - bits)
    of the largest each."""
    bits = max(12, (V - 1).bit_length())
    return 3e-13 + 2.0 ** (bits - 62) + V * 2.0 ** (bits - 94)


def one_peak(B, V, x, p, td, peak, u, stride=0):
    """A row of V tokens: 0 for the token `peak`, x for all others; what is kept with top-p, and the draw with u."""
    big = torch.full((1, 1, V + stride), x, device=DEV).to(td)
    z = big[..., :V]
    z[0, 0, peak] = 0.0
    w, p, u = math.exp(float(z[0, 0, peak - 1])), float(np.float32(p)), float(np.float32(u))
    total = 1 + (V - 1) * w
    rules = B.SamplingRules(top_p=torch.tensor([p], device=DEV))
    out, token = B.spec_truncate_logits(z, rules, uniforms=torch.tensor([[u]], device=DEV))
    kept = out[0, 0] > -math.inf
    n = int(kept.sum())
    # peak, then the others by their ids: the fewest n - 1 of them with 1 + (n - 1) w >= p total
    t = (p * total - 1) / w if p < 1 else V - 1
    room = 2 * off(V) * total / w if p < 1 else 0.0
    assert max(1, 1 + math.ceil(t - room)) <= n <= max(1, 1 + math.ceil(t + room)), (n, t, room)
    last = n - 1 if n - 1 <= peak else n  # ids behind the last that is kept
    assert kept[peak] and bool(kept[:last].all()) and not bool(kept[max(last, peak + 1):].any())
    # the draw among what is kept, by ids: the tokens before the peak, the peak, those behind it
    at, all_ = u * (1 + (n - 1) * w), off(V) * total / w * 2
    token, before = int(token[0, 0]), min(n - 1, peak)
    if at < before * w:
        assert abs(token - math.floor(at / w)) <= math.ceil(all_), (token, at / w, all_)
    elif at < before * w + 1:
        assert token == peak
    else:
        assert abs(token - (before + 1 + math.floor((at - before * w - 1) / w))) <= math.ceil(all_), (token, at, all_)


@pytest.mark.parametrize("td", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,x,p", [(32000, -22.0, 1 - 2.0 ** -20), (50272, -24.0, 1 - 2.0 ** -20), (151936, -25.0, 1 - 2.0 ** -20), (262208, -22.5, 0.9999),
                                   (262208, -22.5, 1 - 2.0 ** -15), (300001, -26.0, 1 - 2.0 ** -19), (300001, -26.0, 1 - 2.0 ** -21), (600000, -24.0, 1 - 2.0 ** -17), (1 << 22, -28.0, 0.999999), ((1 << 22) + 3, -20.0, 0.995)])
def test_one_likely_token_before_a_flat_tail(B, V, x, p, td):
    w = math.exp(x)
    one_peak(B, V, x, p, td, V - 1, 0.5 * V * w)
    one_peak(B, V, x, p, td, V // 2, 0.5, stride=4)
    one_peak(B, V, x, 1.0, td, V // 3, 1 - 2.0 ** -24)


def test_a_vocabulary_of_millions(B):
    one_peak(B, 1 << 24, -26.7, 0.99999, torch.float32, (1 << 24) - 1, 1e-5)
    one_peak(B, 1 << 26, -25.0, 0.9999, torch.bfloat16, 5, 0.9999)
    one_peak(B, 1 << 28, -24.4, 0.999, torch.bfloat16, 1 << 20, 0.9)


@pytest.mark.parametrize("td", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [151936, 300001, 600000, 1000003])
def test_rules_and_draws_over_large_vocabularies(B, V, td):
    z = logits_of(5, 1, V, td, seed=V)
    z[4, 0, V - 3:] = 40.0  # the last tokens, and none else to speak of
    z[4, 0, 300:700] = 12.0
    rules, on = rules_of(B, temperature=[1.0, 0.8, 1.2, 1.0, 1.0], top_k=[50, 5000, 0, 700, 350], top_p=[1.0, 1.0, 0.9, 0.7, 1.0], min_p=[0.0, 0.0, 0.0, 1e-3, 0.0])
    for u in (0.0, 0.3, 0.5, 0.8, 1 - 2.0 ** -24):
        us = torch.full((5, 1), u)
        out, tokens = B.spec_truncate_logits(z, rules, uniforms=us.to(DEV))
        check(z, out, on["temperature"], on["top_k"], on["top_p"], on["min_p"], us, tokens.cpu())
        alone = B.spec_truncate_logits(z, rules, uniforms=us.to(DEV), want_logits=False)[1]
        assert torch.equal(alone, tokens)


@pytest.mark.parametrize("spread", [0.02, 0.05, 0.2, 0.7])
@pytest.mark.parametrize("V", [300, 2000, 9001, 40000])
def test_borders_among_the_likeliest_bins(B, V, spread):
    """The border in one of the first bins of a sixty-fourth of an octave, with tokens in those beside it."""
    g = torch.Generator().manual_seed(V)
    z = -spread * torch.rand((24, 2, V), generator=g)
    rules, on = rules_of(B, top_p=[(i + 1) / 25 for i in range(24)], top_k=[0, V - V // 3] * 12)
    u = torch.rand((24, 2), generator=g)
    out, tokens = B.spec_truncate_logits(z.to(DEV), rules, uniforms=u.to(DEV))
    check(z, out, k=on["top_k"], p=on["top_p"], u=u, tokens=tokens.cpu())


def test_many_tokens_just_behind_the_border_s_bin(B):
    """Large logits, whose differences are uncertain by more than a bin: what lies just behind the border's bin comes to the list with it."""
    g = torch.Generator().manual_seed(31)
    z = torch.full((24, 1, 9001), 1000.0)
    d = torch.cat([0.1191 * torch.rand((24, 1, 80), generator=g), 0.11913 + 0.0009 * torch.rand((24, 1, 3000), generator=g)], -1)
    at = torch.stack([torch.randperm(9001, generator=g)[:3080] for _ in range(24)])[:, None]
    z.scatter_(-1, at, 1024.0 - d)
    rules, on = rules_of(B, top_p=[0.001 + 0.0012 * i for i in range(24)], top_k=[0, 0, 3050] * 8)
    u = torch.rand((24, 1), generator=g)
    out, tokens = B.spec_truncate_logits(z.to(DEV), rules, uniforms=u.to(DEV))
    check(z, out, k=on["top_k"], p=on["top_p"], u=u, tokens=tokens.cpu())
