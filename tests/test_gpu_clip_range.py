"""Clipping where the factor, max_norm / norm, is smaller than a float holds in full."""
import math

import pytest
import torch

from ops_common import HALF, TYPES, U, f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("max_norm", [1.0, 2.0 ** -20, 2.0 ** -40])
@pytest.mark.parametrize("n", [5, 4096 * 3])
def test_small_factors(kind, max_norm, n):
    """Gradients of 1e38: the factor lies below float's normal range (2^-126) with the first bound and around or below its smallest value
    (2^-149) with the others; what comes out is of max_norm's size and rounded as ever: factor and product in double, one rounding to float."""
    from paper_2307_07649_amd import tgnn
    g = (torch.rand(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)) + 0.5).mul_(2.0 ** 126).to(TYPES[kind])
    g[1::2] *= -1
    norm = math.sqrt(float((f64(g) ** 2).sum()))
    out = torch.empty_like(g)
    tgnn.tgnn_clip_grads([g], max_norm, out=[out])
    want = f64(g) * (max_norm / norm)
    assert float(want.abs().min()) > 2.0 ** -100
    assert ((f64(out) - want).abs() <= (1.01 * U + (HALF[out.dtype] if out.dtype != torch.float32 else 0.0)) * want.abs()).all()
    own = g.clone()
    tgnn.tgnn_clip_grads([own], max_norm)
    assert torch.equal(own, out)
