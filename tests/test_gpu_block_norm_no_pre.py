"""block_norm_backward without a norm before the next block: x' is no part of the gradients, whatever it holds.

Then h is absent and dx = alpha dx', du = gate dx' by the formulas: equal to
the bit, as each is one product of fp32 values rounded once.
"""

from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module")
def mpm():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2604_05718_gb300 as pkg
    from paper_2604_05718_gb300 import build

    build.build()
    return pkg


@pytest.mark.parametrize("dim", [96, 100, 385, 768, 1024, 2048, 8200])
@pytest.mark.parametrize("stream", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_streams_that_are_not_finite(mpm, norm, stream, dim):
    gen = torch.Generator().manual_seed(dim)
    rows, alpha = 7, 0.5
    y = torch.randn(rows, dim, generator=gen).to(DEV, torch.bfloat16)
    x = torch.randn(rows, dim, generator=gen).to(DEV, stream)
    gate = torch.randn(dim, generator=gen).to(DEV)
    dxo = torch.randn(rows, dim, generator=gen).to(DEV, stream)
    x[1, 3], x[2, 5], x[3, 0], x[3, 1] = float("inf"), float("nan"), float("inf"), float("-inf")
    args = dict(norm=norm, gate=gate, residual_scale=alpha)
    _, _, stats = mpm.block_norm(y, x, with_stats=True, **args)
    got = mpm.block_norm_backward(dxo, None, y, x, stats, **args)
    assert torch.equal(got.d_residual, (alpha * dxo.float()).to(stream))
    assert torch.equal(got.d_y, (gate * dxo.float()).to(y.dtype))
    assert torch.isfinite(got.d_gate).all()


@pytest.mark.parametrize("dim", [100, 768, 2048])
def test_branches_that_are_not_finite(mpm, dim):
    gen = torch.Generator().manual_seed(dim)
    y = torch.randn(6, dim, generator=gen).to(DEV, torch.bfloat16)
    x = torch.randn(6, dim, generator=gen).to(DEV, torch.bfloat16)
    weight = torch.rand(dim, generator=gen).to(DEV) + 0.5
    dxo = torch.randn(6, dim, generator=gen).to(DEV, torch.bfloat16)
    y[4, 2] = float("nan")
    _, _, stats = mpm.block_norm(y, x, norm="layer", post_weight=weight, with_stats=True)
    got = mpm.block_norm_backward(dxo, None, y, x, stats, norm="layer", post_weight=weight)
    assert torch.equal(got.d_residual, dxo)                      # alpha = 1
    keep = [0, 1, 2, 3, 5]
    assert got.d_y[4].isnan().all() and torch.isfinite(got.d_y[keep]).all()
