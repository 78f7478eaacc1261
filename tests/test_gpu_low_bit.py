"""The 4-bit ViT encoder (vit_insertion/low_bit.py): the block operators as a model uses them."""

from __future__ import annotations

import pytest
import torch
import torch.nn.functional as F

import exact_blocks

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module")
def mpm():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2604_05718_gb300 as pkg
    from paper_2604_05718_gb300 import build

    build.build()
    pkg.library()
    return pkg


def models(insert_at=(1, 2)):
    from vit_insertion import ViT, ViTConfig, synthetic_images
    from vit_insertion.low_bit import LowBitViT

    cfg = ViTConfig("tiny", depth=4, dim=64, heads=2, mlp=128, patch=8, image=128, special=2, classes=5,
                    insert_at=insert_at)
    return cfg, ViT(cfg, DEV, seed=3), LowBitViT(cfg, DEV, seed=3), synthetic_images(3, cfg.image, cfg.patch, 1, DEV)


def plain_blocks(full, images):
    """The low-bit model without merges, in plain torch on values rounded to MXFP4 (fp32 between roundings to bf16)."""
    cfg = full.cfg

    def q(v):
        return exact_blocks.mxfp4_values(v).to(DEV, torch.float32)

    def linear(x, p, name):
        return (q(x) @ q(p[name + "_w"]).t() + p[name + "_b"].float()).to(torch.bfloat16)

    def norm(x, w, b):
        return F.layer_norm(x.float(), (cfg.dim,), w.float(), b.float(), eps=1e-6).to(torch.bfloat16)

    x = full.embed(images)
    n = cfg.tokens + cfg.special
    for p in full.blocks:
        qkv = linear(norm(x, p["ln1_w"], p["ln1_b"]), p, "qkv").view(-1, n, 3, cfg.heads, cfg.dim // cfg.heads).float()
        k, v = qkv[:, :, 1].transpose(1, 2), qkv[:, :, 2].transpose(1, 2)
        s = torch.softmax(qkv[:, :, 0].transpose(1, 2) @ k.transpose(2, 3) / (cfg.dim // cfg.heads) ** 0.5, dim=-1)
        a = (s @ v).transpose(1, 2).reshape(-1, cfg.dim).to(torch.bfloat16)
        x = (x.float() + linear(a, p, "proj").float()).to(torch.bfloat16)
        f = F.gelu(linear(norm(x, p["ln2_w"], p["ln2_b"]), p, "fc1"))
        x = (x.float() + linear(f, p, "fc2").float()).to(torch.bfloat16)
    h = norm(x, full.head_ln_w, full.head_ln_b).view(-1, n, cfg.dim)[:, cfg.special:].reshape(-1, cfg.dim)
    return F.linear(h, full.head_w, full.head_b)


def test_forward_is_the_model_on_rounded_values(mpm):
    """Where a value lies within bf16's rounding of a half-way point, the two round to neighbouring 4-bit levels:
    a step of up to a third of the value in a few features of 64.  The logits are compared as vectors of a row."""
    _, full, low, images = models()
    with torch.inference_mode():
        got, want = low.forward(images).float(), plain_blocks(full, images).float()
    likeness = F.cosine_similarity(got, want, dim=1)
    assert got.shape == want.shape and likeness.mean() > 0.97 and likeness.min() > 0.7


def test_merged_forward(mpm):
    cfg, full, low, images = models()
    with torch.inference_mode():
        got = low.forward(images, mpm=mpm)
        assert got.shape == (3 * cfg.tokens, cfg.classes) and torch.isfinite(got).all()
        assert torch.equal(got, low.forward(images, mpm=mpm))
        # Merges of one insertion or three go the other ways back to the grid.
        for at in ((1,), (0, 1, 3)):
            assert low.forward(images, mpm=mpm, insert_at=at).shape == got.shape
        # 4 bits change the features much less than another image does.
        want = full.forward(images, mpm=mpm)
    same = F.cosine_similarity(got.float(), want.float(), dim=1).mean()
    other = F.cosine_similarity(got.float(), want.float().roll(cfg.tokens, 0), dim=1).mean()
    assert same > 0.8 and same > other


def test_gate_tuning_brings_the_features_nearer(mpm):
    cfg, full, low, images = models()
    with torch.inference_mode():
        x, y, _, _ = low.run_blocks(images)
        # Features that another gate would give: the fit can reach them.
        wanted = torch.linspace(0.2, 1.8, cfg.dim, device=DEV)
        _, target, _ = mpm.block_norm(y, x, gate=wanted, pre_weight=low.head_ln_w, pre_bias=low.head_ln_b)
        before = (low.blocks[-1]["gate2"] - wanted).abs().mean()
        losses = low.tune_last_gate(images, target.float(), steps=60, rate=0.3)
        after = (low.blocks[-1]["gate2"] - wanted).abs().mean()
    assert losses[-1] < 0.1 * losses[0] and after < 0.5 * before
