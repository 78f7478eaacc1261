"""Refusals of the encoder-block entry points at the C boundary (no GPU needed:
arguments are checked before any CUDA call)."""

from __future__ import annotations

import ctypes

import pytest

P = ctypes.c_void_p
FAKE = 1 << 24      # a stand-in address, 16-byte aligned; never dereferenced
STEP = 1 << 24      # buffers of the sizes below do not reach the next one


@pytest.fixture(scope="module")
def lib():
    from paper_2604_05718_gb300 import build, mpm

    build.build()
    return mpm.library()


def at(i):
    return FAKE + i * STEP


def forward(lib, **kw):
    a = dict(y=at(0), y_stride=64, residual=at(1), residual_stride=64, offsets=at(2), batch=2, rows=100, dim=64, dtype=1,
             stream_dtype=1, norm=1, eps=1e-6, scale=1.0, post_weight=at(3), post_bias=at(4), gate=at(5), per_image=1,
             pre_weight=at(6), pre_bias=at(7), residual_out=at(8), h=at(9), stats=at(10), status=None, stream=None)
    a.update(kw)
    return lib.mpm_block_norm(*a.values())


def backward(lib, **kw):
    a = dict(dxo=at(0), dxo_stride=64, dh=at(1), dh_stride=64, y=at(2), y_stride=64, residual=at(3), residual_stride=64,
             stats=at(4), offsets=at(5), batch=2, rows=100, dim=64, dtype=1, stream_dtype=1, norm=0, scale=1.0,
             post_weight=at(6), post_bias=at(7), gate=at(8), per_image=1, pre_weight=at(9), d_y=at(10),
             d_residual=at(11), d_post_weight=at(12), d_post_bias=at(13), d_gate=at(14), d_pre_weight=at(15),
             d_pre_bias=at(16), workspace=at(17), workspace_bytes=1 << 30, status=None, stream=None)
    a.update(kw)
    return lib.mpm_block_norm_backward(*a.values())


def test_block_norm(lib):
    for bad in (dict(rows=-1), dict(batch=0), dict(dim=0), dict(dtype=7), dict(norm=2), dict(eps=-1.0),
                dict(eps=float("inf")), dict(scale=float("nan")), dict(y=None), dict(residual=None),
                dict(residual_out=None), dict(h=None), dict(pre_weight=None), dict(post_weight=None),
                dict(offsets=None), dict(gate=None), dict(y_stride=63), dict(residual_stride=0),
                dict(pre_weight=None, h=None)):
        assert forward(lib, **bad) == 1, bad
    assert forward(lib, dim=20000, y_stride=20000, residual_stride=20000) == 2
    assert forward(lib, dtype=0) == 2                       # fp32 blocks on a bf16 stream
    for bad in (dict(y=at(0) + 1), dict(residual_out=at(8) + 1), dict(stats=at(10) + 8), dict(gate=at(5) + 2),
                dict(offsets=at(2) + 4), dict(pre_bias=at(7) + 1)):
        assert forward(lib, **bad) == 3, bad
    for bad in (dict(h=at(0)), dict(residual_out=at(0) + 128), dict(residual_out=at(1) + 128), dict(h=at(8) + 256),
                dict(residual_out=at(1), residual_stride=72), dict(stats=at(9) + 64)):
        assert forward(lib, **bad) == 8, bad
    assert forward(lib, rows=0) == 0


def test_block_norm_backward(lib):
    assert lib.mpm_block_norm_workspace_size(0) == 0 and lib.mpm_block_norm_workspace_size(16385) == 0
    assert lib.mpm_block_norm_workspace_size(768) > 0
    for bad in (dict(rows=-1), dict(batch=0), dict(dim=0), dict(norm=-1), dict(y=None), dict(stats=None),
                dict(d_y=None), dict(d_residual=None), dict(pre_weight=None), dict(post_weight=None),
                dict(gate=None, per_image=0), dict(offsets=None), dict(dh_stride=8), dict(dxo_stride=63)):
        assert backward(lib, **bad) == 1, bad
    assert backward(lib, dtype=0) == 2
    for bad in (dict(stats=at(4) + 4), dict(d_y=at(10) + 1), dict(d_gate=at(14) + 2)):
        assert backward(lib, **bad) == 3, bad
    for bad in (dict(workspace=None), dict(workspace=at(17) + 16), dict(workspace_bytes=64)):
        assert backward(lib, **bad) == 4, bad
    for bad in (dict(d_y=at(2)), dict(d_residual=at(0) + 64), dict(d_gate=at(10) + 128), dict(workspace=at(3)),
                dict(d_pre_bias=at(15) + 16)):
        assert backward(lib, **bad) == 8, bad


def test_mxfp4(lib):
    assert lib.mpm_mxfp4_code_bytes(3, 65) == 3 * 64 and lib.mpm_mxfp4_code_bytes(-1, 64) == 0
    assert lib.mpm_mxfp4_scale_bytes(129, 129) == 2 * 2 * 512 and lib.mpm_mxfp4_scale_bytes(4, 0) == 0

    def quantize(tokens=at(0), stride=64, rows=10, dim=64, dtype=1, codes=at(1), scales=at(2)):
        return lib.mpm_mxfp4_quantize(tokens, stride, rows, dim, dtype, codes, scales, None)

    for bad in (dict(rows=-1), dict(dim=0), dict(dtype=3), dict(tokens=None), dict(codes=None), dict(scales=None),
                dict(stride=63)):
        assert quantize(**bad) == 1, bad
    assert quantize(dim=(1 << 20) + 1, stride=1 << 21) == 2
    assert quantize(tokens=at(0) + 1) == 3 and quantize(codes=at(1) + 8) == 3 and quantize(scales=at(2) + 4) == 3
    assert quantize(codes=at(0) + 64) == 8 and quantize(scales=at(1) + 16) == 8
    assert quantize(rows=0) == 0

    def dequantize(codes=at(0), scales=at(1), rows=10, dim=64, dtype=1, out=at(2), stride=64):
        return lib.mpm_mxfp4_dequantize(codes, scales, rows, dim, dtype, out, stride, None)

    for bad in (dict(rows=-1), dict(dim=0), dict(dtype=3), dict(codes=None), dict(out=None), dict(stride=1)):
        assert dequantize(**bad) == 1, bad
    assert dequantize(out=at(2) + 1) == 3 and dequantize(codes=at(0) + 8) == 3
    assert dequantize(out=at(0)) == 8

    def matmul(ac=at(0), asc=at(1), m=10, bc=at(2), bs=at(3), n=20, k=64, bias=at(4), dtype=1, out=at(5), stride=20):
        return lib.mpm_mxfp4_matmul(ac, asc, m, bc, bs, n, k, bias, dtype, out, stride, None, None)

    for bad in (dict(m=-1), dict(n=0), dict(k=0), dict(dtype=9), dict(ac=None), dict(bs=None), dict(out=None),
                dict(stride=19)):
        assert matmul(**bad) == 1, bad
    assert matmul(m=(1 << 30) + 1) == 2 and matmul(k=(1 << 20) + 1) == 2
    assert matmul(m=1 << 30, k=1 << 20) == 2
    assert matmul(ac=at(0) + 8) == 3 and matmul(out=at(5) + 1) == 3 and matmul(bias=at(4) + 2) == 3
    assert matmul(out=at(0)) == 8 and matmul(out=at(4) + 16) == 8
    assert matmul(m=0) == 0


def test_misaligned_status_word(lib):
    """The kernels report by an atomic on the word: off 4 bytes it would be a misaligned address on the device."""
    for off in (1, 2, 3):
        assert forward(lib, status=at(12) + off) == 3
        assert backward(lib, status=at(20) + off) == 3
        assert lib.mpm_mxfp4_matmul(at(0), at(1), 10, at(2), at(3), 20, 64, at(4), 1, at(5), 20, at(6) + off, None) == 3
