"""What the 4-bit ViT encoder (vit_insertion/low_bit.py) hands to the block operators."""

from __future__ import annotations

import pytest
import torch
import torch.nn.functional as F

from test_gpu_low_bit import DEV, models, mpm  # noqa: F401

pytestmark = pytest.mark.gpu


class Recorder:
    """A package's functions, each call noted as (name, keyword arguments)."""

    def __init__(self, package):
        self.package, self.calls = package, []

    def __getattr__(self, name):
        what = getattr(self.package, name)
        if not callable(what):
            return what

        def call(*args, **kw):
            self.calls.append((name, kw))
            return what(*args, **kw)

        return call


def run_all(mpm):  # noqa: F811
    """Calls of a merged forward pass and of two tuning steps."""
    cfg, full, low, images = models()
    low.ops = Recorder(mpm)
    with torch.inference_mode():
        logits = low.forward(images, mpm=mpm)
        x, y, _, _ = low.run_blocks(images)
        low.tune_last_gate(images, torch.zeros(x.shape, device=DEV), steps=2, rate=0.0)
    assert torch.isfinite(logits).all()
    return full, low, low.ops.calls


def test_norms_have_the_full_models_eps(mpm):  # noqa: F811
    full, low, calls = run_all(mpm)
    # torch's layer norm as the full model calls it, on rows whose variance eps decides.
    gen = torch.Generator().manual_seed(0)
    x = (1e-3 * torch.randn(40, full.cfg.dim, generator=gen)).to(DEV, torch.bfloat16)
    w, b = low.head_ln_w, low.head_ln_b
    want = F.layer_norm(x, (full.cfg.dim,), w.to(x.dtype), b.to(x.dtype))
    assert torch.equal(low.norm(x, w, b), want)
    norms = [kw for name, kw in calls if name.startswith("block_norm") and "eps" in kw]
    assert len(norms) == sum(name in ("block_norm", "block_norm_backward") for name, _ in calls)
    for kw in norms:
        _, h, _ = mpm.block_norm(torch.zeros_like(x), x, norm="layer", pre_weight=w, pre_bias=b, eps=kw["eps"])
        # One bf16 rounding apart at most: at 1e-3 an eps ten times smaller makes h three times as large.
        torch.testing.assert_close(h, want, rtol=2.0 ** -7, atol=2.0 ** -7)


def test_device_errors_reach_the_caller(mpm):  # noqa: F811
    full, low, calls = run_all(mpm)
    reporting = [(name, kw) for name, kw in calls if name in ("block_norm", "block_norm_backward", "matmul_mxfp4")]
    assert {name for name, _ in reporting} == {"block_norm", "block_norm_backward", "matmul_mxfp4"}
    for name, kw in reporting:
        assert kw.get("device_status") is low.status, name
    low.check_status()
    low.status[0], low.status[1] = 7, 31          # what a kernel writes when a wait ran out
    with pytest.raises(mpm.MPMError) as e:
        low.check_status()
    assert e.value.code == 7
    low.check_status()                            # once told, cleared
    low.status[0] = 7
    _, _, _, images = models()
    with torch.inference_mode(), pytest.raises(mpm.MPMError):
        low.tune_last_gate(images, torch.zeros(3 * (full.cfg.tokens + full.cfg.special), full.cfg.dim, device=DEV), steps=1)
