"""block_norm and block_norm_backward element by element against 64 bits (norm_bounds.py has the bounds)."""

from __future__ import annotations

import pytest
import torch

import exact_blocks
import norm_bounds
from test_norm_bounds import COUNTS, DIMS, EPS, TYPES, inputs

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


def run(mpm, t, off, norm, alpha, dxo, dh):
    """Outputs and gradients of the kernels by name."""
    args = {k: v for k, v in t.items() if k not in ("y", "residual")}
    args.update(norm=norm, eps=EPS, residual_scale=alpha, offsets=off)
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    xo, h, stats = mpm.block_norm(t["y"], t["residual"], with_stats=True, device_status=status, **args)
    grads = mpm.block_norm_backward(dxo, dh, t["y"], t["residual"], stats, device_status=status, **args)
    assert status.tolist() == [0, 0]
    out = {"residual_out": xo, "h": h, **grads._asdict()}
    return {k: v for k, v in out.items() if v is not None}


def check(mpm, counts, dim, types, norm, *, alpha=0.75, seed=0, **kw):
    t, off, rows_of, (dxo, dh) = inputs(counts, dim, types, seed=seed, device=DEV, **kw)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    want = norm_bounds.reference(t, rows_of, norm, EPS, alpha, dxo, dh, len(counts), sms)
    return norm_bounds.check(run(mpm, t, off, norm, alpha, dxo, dh), want)


@pytest.mark.parametrize("dim", sorted(DIMS + [1, 7, 256, 257, 385, 512, 1000, 1032, 2049, 6152, 16384]))
@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_every_width(mpm, norm, types, dim):
    check(mpm, COUNTS, dim, types, norm, seed=dim)


@pytest.mark.parametrize("gate", ["none", "channel", "image"])
@pytest.mark.parametrize("post,pre", [(True, True), (False, True), (True, False), (False, False)])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("dim", [192, 1024])
def test_every_part_may_be_absent(mpm, dim, norm, post, pre, gate):
    check(mpm, [17, 3, 0, 64], dim, "bf16", norm, alpha=-0.5, gate=gate, post=post, pre=pre, bias=norm == "layer")


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("dim", [48, 385])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_gradients_against_differences_in_64_bits(mpm, norm, dim, types):
    """<gradient, way> against differences of L = <dx', x'> + <dh, h>, L in 64 bits.

    Three steps, each half of the one before, extrapolated twice: the last
    result is off by less than what the last extrapolation changed.
    """
    counts, alpha = [4, 0, 5], 0.75
    t, off, rows_of, (dxo, dh) = inputs(counts, dim, types, seed=3, device=DEV)
    got = run(mpm, t, off, norm, alpha, dxo, dh)
    bounds = norm_bounds.reference(t, rows_of, norm, EPS, alpha, dxo, dh, len(counts))
    exact = {k: v.double() for k, v in t.items()}
    gen = torch.Generator(device=DEV).manual_seed(9)

    def loss(name, by):
        s = dict(exact)
        s[name] = s[name] + by
        xo, h = exact_blocks.block_norm(s.pop("y"), s.pop("residual"), norm=norm, eps=EPS, residual_scale=alpha,
                                        rows_of=rows_of, **s)
        return ((dxo.double() * xo).sum() + (dh.double() * h).sum()).item()

    for name in t:
        way = torch.randn(t[name].shape, generator=gen, device=DEV, dtype=torch.float64)
        slope = [(loss(name, s * way) - loss(name, -s * way)) / (2 * s) for s in (2.0 ** -8, 2.0 ** -9, 2.0 ** -10)]
        once = [(4 * slope[1] - slope[0]) / 3, (4 * slope[2] - slope[1]) / 3]
        best = (16 * once[1] - once[0]) / 15
        value, bound = bounds["d_" + name]
        bound = bound + norm_bounds.ROUND[got["d_" + name].dtype] * (value.abs() + bound)
        # 64-bit noise of a difference: 2^-53 of L's terms over the step.
        noise = 2.0 ** -50 * ((dxo.double() * exact["residual"]).abs().sum() + dh.double().abs().sum() * 4).item() * 2 ** 10
        assert abs((got["d_" + name].double() * way).sum().item() - best) <= \
            (bound * way.abs()).sum().item() + abs(best - once[1]) + noise, name


@pytest.mark.parametrize("biases", [(), ("post_bias",), ("pre_bias",), ("post_bias", "pre_bias")])
@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("dim", [100, 768, 1024])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_every_set_of_biases(mpm, norm, dim, types, biases):
    """Either norm with either bias: layer norm has them as a rule, root mean square has not."""
    counts, alpha = [9, 0, 31], 0.5
    t, off, rows_of, (dxo, dh) = inputs(counts, dim, types, seed=dim, device=DEV)
    t = {k: v for k, v in t.items() if not k.endswith("bias") or k in biases}
    want = norm_bounds.reference(t, rows_of, norm, EPS, alpha, dxo, dh, len(counts))
    norm_bounds.check(run(mpm, t, off, norm, alpha, dxo, dh), want)
