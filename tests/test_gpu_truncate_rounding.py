"""spec_truncate_logits' kept logits: (z - m) / T, rounded once to fp32."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("td", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("V", [5003, 32000])
def test_kept_logits_are_rounded_once(td, V):
    from paper_2310_18813_amd import binding as B
    g = torch.Generator().manual_seed(V)
    T = torch.tensor([1.0, 0.7, 1.3, 0.013, 77.0, 1e-38, 3e38, math.inf, 1e-42, 3.0])
    z = 3 * torch.randn((10, 2, V), generator=g)
    z[5] *= 1e-37 if td == torch.float32 else 1.0
    z[6] *= 1e37 if td != torch.float16 else 1.0
    z[8] *= 1e-42 if td == torch.float32 else 1.0
    z = z.to(td)
    out, _ = B.spec_truncate_logits(z.to(DEV), B.SamplingRules(temperature=T.to(DEV), top_k=torch.full((10,), 3000, dtype=torch.int32, device=DEV)))
    out, z, T = out.double().cpu().numpy(), z.double().numpy(), T.double().numpy()
    want = (z - z.max(-1, keepdims=True)) / T[:, None, None]
    kept = out > -np.inf
    assert kept.any(-1).all()
    off, size = np.abs(out - want)[kept], np.abs(want)[kept]
    # half a step of fp32, and of 64 bits for the difference, the quotient and its factor
    assert (off <= size * (2.0 ** -24 + 2.0 ** -50) + 2.0 ** -150).all(), float((off / np.maximum(size, 1e-300)).max() * 2 ** 24)
