"""Block operators where positions pass 32 bits, and products of blocks whose scales lie far apart.

The last rows of a matrix of more than 2^31 values (and, in bytes, 2^32) have
to come out as they do alone: rows do not depend on one another.
"""

from __future__ import annotations

import pytest
import torch

import norm_bounds
from test_gpu_mxfp4 import mpm, product_bound  # noqa: F401

pytestmark = pytest.mark.gpu

DEV = "cuda"
TAIL = 300


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def matrix(rows, dim, dtype, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    out = torch.empty(rows, dim, dtype=dtype, device=DEV)
    for lo in range(0, rows, 1 << 18):
        part = out[lo:lo + (1 << 18)]
        part.copy_(torch.randn(part.shape, generator=gen, device=DEV))
    return out


@pytest.mark.parametrize("dim", [1024, 1025])
def test_norms_past_32_bits(mpm, dim):  # noqa: F811
    rows = (1 << 31) // dim + 40000
    y, x = matrix(rows, dim, torch.bfloat16, 0), matrix(rows, dim, torch.bfloat16, 1)
    gen = torch.Generator(device=DEV).manual_seed(2)
    draw = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
    args = dict(pre_weight=draw(dim), pre_bias=draw(dim), post_weight=draw(dim), post_bias=draw(dim))
    gate, off = draw(2, dim), torch.tensor([0, rows - TAIL, rows], device=DEV)
    xo, h, stats = mpm.block_norm(y, x, gate=gate, offsets=off, with_stats=True, **args)
    tail = (y[-TAIL:].contiguous(), x[-TAIL:].contiguous())
    one = torch.tensor([0, TAIL], device=DEV)
    want = mpm.block_norm(*tail, gate=gate[1:], offsets=one, with_stats=True, **args)
    assert torch.equal(xo[-TAIL:], want[0]) and torch.equal(h[-TAIL:], want[1]) and torch.equal(stats[-TAIL:], want[2])
    got = mpm.block_norm_backward(xo, h, y, x, stats, gate=gate, offsets=off, **args)
    part = mpm.block_norm_backward(want[0], want[1], *tail, want[2], gate=gate[1:], offsets=one, **args)
    assert torch.equal(got.d_y[-TAIL:], part.d_y) and torch.equal(got.d_residual[-TAIL:], part.d_residual)
    # The last image's gate has the tail's rows alone, in runs of another length.
    values = norm_bounds.reference({"y": tail[0], "residual": tail[1], "gate": gate[1], **args},
                                   torch.zeros(TAIL, dtype=torch.int64, device=DEV), "layer", 1e-6, 1.0, want[0], want[1])
    value, bound = values["d_gate"]
    assert norm_bounds.worst(got.d_gate[1], value, bound * (1 + TAIL / 64)) <= 1.0


@pytest.mark.parametrize("dim", [1024, 1025])
def test_quantisation_past_32_bits(mpm, dim):  # noqa: F811
    rows = (1 << 31) // dim + 40000
    rows += 128 - rows % 128                       # the tail below starts a tile
    x = matrix(rows, dim, torch.bfloat16, 3)
    q = mpm.quantize_mxfp4(x)
    part = mpm.quantize_mxfp4(x[-256:].contiguous())
    assert torch.equal(q.codes[-256:], part.codes) and torch.equal(q.scales[-2:], part.scales)
    assert torch.equal(mpm.dequantize_mxfp4(q)[-256:], mpm.dequantize_mxfp4(part))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [2304, 2305])
def test_products_past_32_bits(mpm, n, dtype):  # noqa: F811
    m = (1 << 31) // n + 30000
    m += 256 - m % 256
    a = mpm.quantize_mxfp4(matrix(m, 64, torch.bfloat16, 4))
    b = mpm.quantize_mxfp4(matrix(n, 64, torch.bfloat16, 5))
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    out = mpm.matmul_mxfp4(a, b, out_dtype=dtype, device_status=status)
    part = mpm.matmul_mxfp4(mpm.MXFP4(a.codes[-256:].contiguous(), a.scales[-2:].contiguous(), 64), b, out_dtype=dtype)
    assert status.tolist() == [0, 0] and torch.equal(out[-256:], part)
    middle = m // 2 - m // 2 % 256
    part = mpm.matmul_mxfp4(mpm.MXFP4(a.codes[middle:middle + 256].contiguous(),
                                      a.scales[middle // 128:middle // 128 + 2].contiguous(), 64), b, out_dtype=dtype)
    assert torch.equal(out[middle:middle + 256], part)


@pytest.mark.parametrize("ea,eb", [(-110, 110), (110, -110), (-122, 118), (118, -122), (-50, -50), (55, 55), (0, 0)])
@pytest.mark.parametrize("m", [5, 200])
def test_products_of_scales_far_apart(mpm, m, ea, eb):  # noqa: F811
    """Scales near both ends of their range, whose products lie within fp32's."""
    gen = torch.Generator().manual_seed(m)
    k = 160
    x = torch.randn(m, k, generator=gen, dtype=torch.float64) * 2.0 ** ea
    w = torch.randn(90, k, generator=gen, dtype=torch.float64) * 2.0 ** eb
    a, b = mpm.quantize_mxfp4(x.to(DEV, torch.float32)), mpm.quantize_mxfp4(w.to(DEV, torch.float32))
    va, vb = (mpm.dequantize_mxfp4(v, torch.float32).double() for v in (a, b))
    got, want = mpm.matmul_mxfp4(a, b, out_dtype=torch.float32), va @ vb.t()
    assert torch.isfinite(got).all()
    assert ((got.double() - want).abs() <= product_bound(va, vb, want, k, torch.float32)).all()
