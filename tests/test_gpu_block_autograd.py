"""The block operators and torch's autograd: no gradient is lost in silence, and writes in place are seen.

Outputs are not tied to a graph (block_norm_backward gives the gradients), so
an input that requires grad is refused while grad mode is on.
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


def norm_args():
    gen = torch.Generator().manual_seed(0)
    draw = lambda *s: torch.randn(*s, generator=gen).to(DEV)  # noqa: E731
    t = {"y": draw(6, 32), "residual": draw(6, 32), "pre_weight": draw(32), "pre_bias": draw(32),
         "post_weight": draw(32), "post_bias": draw(32), "gate": draw(2, 32)}
    return t, {"offsets": torch.tensor([0, 2, 6], device=DEV)}


@pytest.mark.parametrize("name", ["y", "residual", "pre_weight", "pre_bias", "post_weight", "post_bias", "gate"])
def test_norm_inputs_that_require_grad(mpm, name):
    t, rest = norm_args()
    want = mpm.block_norm(**t, **rest, with_stats=True)
    grads = mpm.block_norm_backward(want[0], want[1], stats=want[2], **t, **rest)
    t[name].requires_grad_()
    with pytest.raises(ValueError, match=name + ".*grad"):
        mpm.block_norm(**t, **rest)
    with pytest.raises(ValueError, match=name + ".*grad"):
        mpm.block_norm_backward(want[0], want[1], stats=want[2], **t, **rest)
    with torch.no_grad():
        got = mpm.block_norm(**t, **rest, with_stats=True)
        again = mpm.block_norm_backward(want[0], want[1], stats=want[2], **t, **rest)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(torch.equal(a, b) for a, b in zip(again, grads))


def test_gradients_and_outputs_that_require_grad(mpm):
    t, rest = norm_args()
    xo, h, stats = mpm.block_norm(**t, **rest, with_stats=True)
    leaf = lambda: torch.zeros(6, 32, device=DEV, requires_grad=True)  # noqa: E731
    for bad in (dict(residual_out=leaf()), dict(h=leaf())):
        with pytest.raises(ValueError, match="grad"):
            mpm.block_norm(**t, **rest, **bad)
    for left, right in ((leaf(), h), (xo, leaf())):
        with pytest.raises(ValueError, match="grad"):
            mpm.block_norm_backward(left, right, stats=stats, **t, **rest)


def test_linear_inputs_that_require_grad(mpm):
    x = torch.randn(5, 64, device=DEV)
    q, w = mpm.quantize_mxfp4(x), mpm.quantize_mxfp4(torch.randn(8, 64, device=DEV))
    with pytest.raises(ValueError, match="tokens.*grad"):
        mpm.quantize_mxfp4(x.clone().requires_grad_())
    with pytest.raises(ValueError, match="bias.*grad"):
        mpm.matmul_mxfp4(q, w, bias=torch.zeros(8, device=DEV, requires_grad=True))
    with pytest.raises(ValueError, match="out.*grad"):
        mpm.matmul_mxfp4(q, w, out=torch.zeros(5, 8, device=DEV, requires_grad=True))
    with pytest.raises(ValueError, match="out.*grad"):
        mpm.dequantize_mxfp4(q, out=torch.zeros(5, 64, device=DEV, requires_grad=True))
    with torch.no_grad():
        assert torch.equal(mpm.quantize_mxfp4(x.clone().requires_grad_()).codes, q.codes)


def test_within_a_function_of_autograd(mpm):
    """Where a program ties them to a graph: in a Function grad mode is off."""
    t, rest = norm_args()
    args = {k: v for k, v in t.items() if k not in ("y", "residual")}

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, y, x):
            xo, h, stats = mpm.block_norm(y, x, with_stats=True, **args, **rest)
            ctx.save_for_backward(y, x, stats)
            return xo, h

        @staticmethod
        def backward(ctx, dxo, dh):
            y, x, stats = ctx.saved_tensors
            return mpm.block_norm_backward(dxo, dh, y, x, stats, **args, **rest)[:2]

    y, x = t["y"].clone().requires_grad_(), t["residual"].clone().requires_grad_()
    xo, h = Norm.apply(y, x)
    got = torch.autograd.grad([xo, h], [y, x], [torch.ones_like(xo), torch.ones_like(h)])
    _, _, stats = mpm.block_norm(with_stats=True, **t, **rest)
    want = mpm.block_norm_backward(torch.ones_like(xo), torch.ones_like(h), stats=stats, **t, **rest)
    assert torch.equal(got[0], want.d_y) and torch.equal(got[1], want.d_residual)


def test_writes_in_place_are_new_versions(mpm):
    t, rest = norm_args()
    xo, h = torch.zeros(6, 32, device=DEV), torch.zeros(6, 32, device=DEV)
    mpm.block_norm(**t, **rest, residual_out=xo, h=h)
    assert (xo._version, h._version) == (1, 1)
    assert all(v._version == 0 for v in t.values())
    x = t["residual"].clone()
    before = x._version
    mpm.block_norm(**{**t, "residual": x}, **rest, residual_out=x)
    assert x._version == before + 1
    q = mpm.quantize_mxfp4(t["y"])
    into = mpm.MXFP4(torch.zeros_like(q.codes), torch.zeros_like(q.scales), q.dim)
    mpm.quantize_mxfp4(t["y"], out=into)
    assert (into.codes._version, into.scales._version) == (1, 1)
    wide = torch.zeros(6, 64, device=DEV)
    mpm.dequantize_mxfp4(q, out=wide[:, 8:40])
    mpm.matmul_mxfp4(q, q, out=wide[:, 8:14])
    assert wide._version == 2                     # a view and its base share one
    with pytest.raises(mpm.MPMError):             # nothing is written by a call that fails
        mpm.block_norm(**t, **rest, h=h, eps=float("nan"))
    assert h._version == 1


def test_a_saved_tensor_that_is_written_is_noticed(mpm):
    t, rest = norm_args()
    h = torch.ones(6, 32, device=DEV)
    leaf = torch.ones(6, 32, device=DEV, requires_grad=True)
    product = leaf * h                            # keeps h for the gradient
    mpm.block_norm(**t, **rest, h=h)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        product.sum().backward()


def test_outputs_of_inference_mode(mpm):
    t, rest = norm_args()
    with torch.inference_mode():
        h = torch.zeros(6, 32, device=DEV)
        mpm.block_norm(**t, **rest, h=h)
        mpm.block_norm(**t, **rest, h=h)
    assert torch.equal(h, mpm.block_norm(**t, **rest)[1])
