"""The 4-bit ViT example with the library's attention and rotary positions: it runs, and its attention is the other one's."""

from __future__ import annotations

import pytest
import torch

from test_gpu_low_bit import mpm  # noqa: F401

pytestmark = pytest.mark.gpu

DEV = "cuda"


def model(**kw):
    from vit_insertion import ViTConfig
    from vit_insertion.low_bit import LowBitViT

    cfg = ViTConfig("tiny", depth=4, dim=128, heads=2, mlp=256, patch=8, image=128, special=2, classes=5, insert_at=(1, 2))
    return cfg, LowBitViT(cfg, DEV, seed=3, **kw)


def images(cfg):
    from vit_insertion import synthetic_images

    return synthetic_images(3, cfg.image, cfg.patch, 1, DEV)


@pytest.mark.parametrize("rotary", [False, True])
def test_attention_of_one_block(mpm, rotary):  # noqa: F811
    """The same joint projection through either attention: two roundings of probabilities and outputs to bf16 apart."""
    cfg, low = model(rotary=rotary)
    _, packed = model(attention="packed", rotary=rotary)
    starts = torch.tensor([0, 200, 201, 201, 350], device=DEV)
    qkv = torch.randn(350, 6, 64, generator=torch.Generator(device=DEV).manual_seed(0), device=DEV).to(torch.bfloat16)
    at = 20 * torch.rand(350, 2, device=DEV) if rotary else None
    a, b = low.attend(qkv.clone(), starts, 200, at), packed.attend(qkv.clone(), starts, 200, at)
    packed.check_status()
    # Each is off by 2^-8 of sum p |v| for the probabilities' rounding, and 2^-8 of the output for its own.
    size = qkv[:, 4:].float().abs().amax()
    assert (a.float() - b.float()).abs().max() <= 2 * 2.0 ** -8 * size + 2 * 2.0 ** -8 * a.float().abs().max()


@pytest.mark.parametrize("attention", ["torch", "packed"])
@pytest.mark.parametrize("rotary", [False, True])
def test_forward(mpm, attention, rotary):  # noqa: F811
    cfg, low = model(attention=attention, rotary=rotary)
    x = images(cfg)
    with torch.no_grad():
        whole, merged = low.forward(x), low.forward(x, mpm=mpm)
    low.check_status()
    assert whole.shape == merged.shape == (3 * cfg.tokens, cfg.classes)
    assert torch.isfinite(whole).all() and torch.isfinite(merged).all()


def test_positions_of_merged_tokens(mpm):  # noqa: F811
    """A pair's position is the mean of its two patches'; maps of two merges in turn."""
    cfg, low = model(rotary=True)
    b, n = 2, cfg.tokens
    gen = torch.Generator(device=DEV).manual_seed(4)
    x = torch.randn(b * n, 128, generator=gen, device=DEV).to(torch.bfloat16)
    off = torch.arange(b + 1, device=DEV) * n
    at = low.grid_positions(b)
    assert at[:2].tolist() == [[1, 1], [1, 2]] and at.shape == (b * n, 2)
    _, off1, m = mpm.merge(x, off)
    total = int(off1[-1])
    got = low.merged_positions(at, off, m, off1, total)
    for image in range(b):
        rows = m[image * n:(image + 1) * n]
        for row in (0, 1, int(rows.max())):
            want = at[image * n:(image + 1) * n][rows == row].mean(0)
            assert torch.allclose(got[int(off1[image]) + row], want)


def test_an_unknown_attention(mpm):  # noqa: F811
    with pytest.raises(ValueError, match="attention"):
        model(attention="other")
