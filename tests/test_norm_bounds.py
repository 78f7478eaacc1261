"""The comparison that block_norm's gradients go through (norm_bounds.py), on the CPU.

It has to accept the right gradients, taken in 64 bits and rounded once, and
to reject each of the mistakes below, in every type and at every width.
"""

from __future__ import annotations

import itertools

import pytest
import torch

import exact_blocks
import norm_bounds

TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "f32": (torch.float32, torch.float32),
         "mixed": (torch.bfloat16, torch.float32)}
EPS, ALPHA = 1e-6, 0.75
COUNTS = [5, 0, 1, 30]


def inputs(counts, dim, types, *, seed=0, gate="image", post=True, pre=True, bias=True, device="cpu"):
    """(tensors by argument name, offsets, every row's image, gradients of both outputs)."""
    gen = torch.Generator(device=device).manual_seed(seed)
    rows = sum(counts)
    ty, tx = TYPES[types]

    def draw(*shape, around=0.0, spread=1.0):
        return around + spread * torch.randn(*shape, generator=gen, device=device)

    t = {"y": draw(rows, dim).to(ty), "residual": draw(rows, dim, spread=2.0).to(tx)}
    if post:
        t["post_weight"] = draw(dim, around=1.0, spread=0.3)
        if bias:
            t["post_bias"] = draw(dim, spread=0.3)
    if gate == "channel":
        t["gate"] = draw(dim, spread=0.5)
    elif gate == "image":
        t["gate"] = draw(len(counts), dim, spread=0.5)
    if pre:
        t["pre_weight"] = draw(dim, around=1.0, spread=0.3)
        if bias:
            t["pre_bias"] = draw(dim, spread=0.3)
    off = torch.tensor([0] + list(itertools.accumulate(counts)), device=device)
    rows_of = torch.repeat_interleave(torch.arange(len(counts), device=device), torch.tensor(counts, device=device))
    return t, off, rows_of, (draw(rows, dim).to(tx), draw(rows, dim).to(ty) if pre else None)


def rounded(values: dict, types: str) -> dict:
    """What a kernel without errors of its own returns."""
    ty, tx = TYPES[types]
    of = {"residual_out": tx, "h": ty, "d_residual": tx, "d_y": ty}
    return {k: v.to(of.get(k, torch.float32)) for k, (v, _) in values.items()}


def both(dim, types, norm, *, drop=(), seed=0, **kw):
    t, off, rows_of, (dxo, dh) = inputs(COUNTS, dim, types, seed=seed, **kw)
    args = (t, rows_of, norm, EPS, ALPHA, dxo, dh, len(COUNTS))
    return norm_bounds.reference(*args), rounded(norm_bounds.reference(*args, drop=drop), types)


@pytest.mark.parametrize("gate", ["none", "channel", "image"])
@pytest.mark.parametrize("post,pre,bias", [(True, True, True), (True, True, False), (False, True, True), (True, False, True),
                                           (False, False, False)])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_the_formulas_are_autograds(norm, post, pre, bias, gate):
    t, off, rows_of, (dxo, dh) = inputs(COUNTS, 40, "f32", gate=gate, post=post, pre=pre, bias=bias)
    got = norm_bounds.reference(t, rows_of, norm, EPS, ALPHA, dxo, dh, len(COUNTS))
    leaves = {k: v.double().requires_grad_() for k, v in t.items()}
    xo, h = exact_blocks.block_norm(leaves["y"], leaves["residual"], norm=norm, eps=EPS, residual_scale=ALPHA,
                                    rows_of=rows_of, **{k: v for k, v in leaves.items() if k not in ("y", "residual")})
    outs, seeds = ([xo, h], [dxo.double(), dh.double()]) if pre else ([xo], [dxo.double()])
    grads = dict(zip(("d_" + k for k in leaves), torch.autograd.grad(outs, list(leaves.values()), seeds)))
    want = {"residual_out": xo, **({"h": h} if pre else {}), **grads}
    assert set(want) == set(got)
    for k, v in want.items():
        torch.testing.assert_close(got[k][0], v, rtol=1e-10, atol=1e-10)


DIMS = [8, 33, 196, 768, 1024, 2048, 4104, 8200]


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_right_gradients_are_accepted(norm, types, dim):
    want, got = both(dim, types, norm, seed=dim)
    far = norm_bounds.check(got, want)
    assert max(far.values()) <= 1.0


MISTAKES = ["product1", "product2", "stream", "alpha", "gate", "deviation", "gate bias", "gate in sums"]


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("norm,mistake", [(n, m) for n in ("rms", "layer") for m in MISTAKES] +
                         [("layer", "mean1"), ("layer", "mean2")])
def test_a_term_left_out_is_rejected(norm, mistake, types, dim):
    want, got = both(dim, types, norm, drop=(mistake,), seed=dim)
    with pytest.raises(AssertionError, match="parts of the bound"):
        norm_bounds.check(got, want)


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_each_output_alone_is_looked_at(norm, types, dim):
    want, got = both(dim, types, norm, seed=dim)
    for name, v in got.items():
        wrong = {"zeros": torch.zeros_like(v), "rows of others": v.roll(1, 0) if v.dim() == 2 else v.roll(1),
                 "one off": v.clone(), "not a number": v.clone()}
        spot = (v.shape[0] // 2, v.shape[-1] // 3) if v.dim() == 2 else (v.shape[0] // 3,)
        if v.dim() == 2 and name == "d_gate":
            spot = (3, v.shape[-1] // 3)
        wrong["one off"][spot] += 0.01 + 0.05 * wrong["one off"][spot].abs()
        wrong["not a number"][spot] = float("nan")
        for what, w in wrong.items():
            if torch.equal(w, v):
                continue
            assert norm_bounds.worst(w, *want[name]) > 1.0, (name, what)


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_a_row_missing_from_a_sum_or_taken_twice(norm, dim):
    t, off, rows_of, (dxo, dh) = inputs(COUNTS, dim, "f32", seed=dim)
    args = (norm, EPS, ALPHA)
    want = norm_bounds.reference(t, rows_of, *args, dxo, dh, len(COUNTS))
    for rows in (list(range(36))[:-1], [0] + list(range(36)), [r for r in range(36) if r != 17]):
        part = {k: v[rows] if k in ("y", "residual") else v for k, v in t.items()}
        got = rounded(norm_bounds.reference(part, rows_of[rows], *args, dxo[rows], dh[rows], len(COUNTS)), "f32")
        for name in ("d_gate", "d_post_weight", "d_post_bias", "d_pre_weight", "d_pre_bias"):
            assert norm_bounds.worst(got[name], *want[name]) > 1.0, name
