"""How far a cache of 8 bits is from what was appended: the bounds that the header states, on heads that come near them."""
import pytest
import torch

import paged8_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def heads(td, n, hd, g):
    """Of rows of type td: [n][1][hd], largest magnitudes from the type's largest down to its least, just above a power of two times 224 in every other head, and
    elements from there to 2^-24 of them."""
    lo, hi = (-23, 15) if td == torch.float16 else (-126, 127)
    top = torch.exp2(torch.randint(lo, hi, (n,), generator=g).double()) * (1 + torch.rand(n, generator=g).double())
    top[::2] = 225.0 * torch.exp2(torch.randint(max(lo - 7, -120), hi - 7, ((n + 1) // 2,), generator=g).double())
    top[0] = torch.finfo(td).max
    x = top[:, None] * torch.exp2(-24 * torch.rand((n, hd), generator=g).double()) * torch.where(torch.rand((n, hd), generator=g) < 0.5, -1.0, 1.0)
    x[:, 7] = top
    x[:, 8:24] = top[:, None] / 225.0 * 2.0 ** -10 * torch.tensor([0.99, 0.5, 0.51, 1.49, 1.51, 2.49, 2.51, -0.99, -1.49, 3.49, 5.49, 7.49, 8.49, 14.9, -15.1, 1.0])
    return x.to(td)[:, None]


@pytest.mark.parametrize("td", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hd", [64, 128])
def test_what_is_read_back_is_as_near_as_stated(td, hd):
    from paper_2310_18813_amd import binding as B
    n, page = 512, 16
    g = torch.Generator().manual_seed(hd)
    b = ref.Batch([n], [n], page, ragged=False)
    k, v = heads(td, n, hd, g), heads(td, n, hd, g)
    cache, batch = B.PagedCache8.empty(b.n_pages, page, 1, hd, td), b.on_gpu(B)
    B.spec_paged8_append(cache, batch, None, k.to(DEV), v.to(DEV))
    for back, x in zip(B.spec_paged8_read(cache, batch), (k, v)):
        x, y = x.double(), back.cpu().double()
        top, off = x.abs().amax(-1, keepdim=True), (y - x).abs()
        least = 2.0 ** (ref.LEAST[td] - 10)
        assert torch.isfinite(y).all()
        assert (off <= torch.maximum(x.abs() / 16, torch.clamp(top * 2.0 ** -17.8, min=least))).all()
        # the heads come near it: beyond 2^-18 of the largest, which is no bound
        inner = (top > 2.0 ** (ref.LEAST[td] + 9))[:, 0, 0]
        assert (off > torch.maximum(x.abs() / 16, top * 2.0 ** -18))[inner].any()
