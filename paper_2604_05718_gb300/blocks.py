"""Python binding of the encoder-block entry points of libmpm.so.

``block_norm`` is everything elementwise between two blocks of an encoder
(norm after the block, gate, scaled residual stream, norm before the next
block) in one pass over packed tokens, with ``block_norm_backward`` for its
gradients.  ``quantize_mxfp4`` and ``matmul_mxfp4`` are a linear layer on
4-bit operands.  As in ``mpm``, arguments are checked and marshalled only, and
every step runs in the library's kernels on the current torch stream.
"""

from __future__ import annotations

from typing import NamedTuple

import torch

from .mpm import MPM_BF16, MPM_F32, _call, _check, _cuda, _dtype_code, _ptr, _stream, library

NORMS = {"rms": 0, "layer": 1}
_DTYPES = {torch.float32: MPM_F32, torch.bfloat16: MPM_BF16}


class MXFP4(NamedTuple):
    """[rows, dim] values in MXFP4: blocks of 32 along the row that share a power of two.

    codes   uint8 [rows, 32 ceil(dim / 64)], two E2M1 codes a byte, the even feature in the low half
    scales  uint8 [ceil(rows / 128), ceil(dim / 128), 512], tiled as described in include/mpm.h
    """

    codes: torch.Tensor
    scales: torch.Tensor
    dim: int

    @property
    def rows(self) -> int:
        return self.codes.shape[0]


class BlockNormGrads(NamedTuple):
    """Gradients of block_norm's inputs; None where the parameter was not given."""

    d_y: torch.Tensor
    d_residual: torch.Tensor
    d_gate: torch.Tensor | None
    d_post_weight: torch.Tensor | None
    d_post_bias: torch.Tensor | None
    d_pre_weight: torch.Tensor | None
    d_pre_bias: torch.Tensor | None


def _rows(t: torch.Tensor, name: str, dev: torch.device | None = None, shape=None) -> torch.Tensor:
    """A CUDA matrix of bf16 or fp32 rows, each contiguous, any distance apart."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dim() != 2:
        raise ValueError(f"{name} must have 2 dimensions")
    if dev is not None and t.device != dev:
        raise ValueError(f"{name} must be on {dev}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype not in _DTYPES:
        raise TypeError(f"{name} must be bfloat16 or float32, got {t.dtype}")
    if (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return t


def _vector(t: torch.Tensor | None, name: str, dev: torch.device, *shape: int) -> torch.Tensor | None:
    if t is None:
        return None
    _cuda(t, name, torch.float32)
    if t.device != dev:
        raise ValueError(f"{name} must be on {dev}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
    return t


def _status(t: torch.Tensor | None, dev: torch.device) -> torch.Tensor | None:
    if t is not None:
        _cuda(t, "device_status", torch.int32, 1)
        if t.device != dev or t.numel() < 2:
            raise ValueError(f"device_status must be an int32 [2] tensor on {dev}")
    return t


class _Norm(NamedTuple):
    """The checked arguments that both directions share."""

    dev: torch.device
    rows: int
    dim: int
    batch: int
    per_image: int


def _norm_args(y, residual, norm, pre_weight, pre_bias, post_weight, post_bias, gate, offsets) -> _Norm:
    _rows(y, "y")
    dev = y.device
    _rows(residual, "residual", dev, y.shape)
    if norm not in NORMS:
        raise ValueError(f"norm must be one of {sorted(NORMS)}, got {norm!r}")
    rows, dim = y.shape
    batch = 1
    if offsets is not None:
        _cuda(offsets, "offsets", torch.int64, 1)
        if offsets.device != dev or offsets.numel() < 2:
            raise ValueError(f"offsets must be an int64 [B+1] tensor on {dev}")
        batch = offsets.numel() - 1
    _vector(pre_weight, "pre_weight", dev, dim)
    _vector(pre_bias, "pre_bias", dev, dim)
    _vector(post_weight, "post_weight", dev, dim)
    _vector(post_bias, "post_bias", dev, dim)
    if (pre_bias is not None and pre_weight is None) or (post_bias is not None and post_weight is None):
        raise ValueError("a norm's bias needs its weight")
    per_image = int(gate is not None and gate.dim() == 2)
    if per_image:
        if offsets is None:
            raise ValueError("a gate per image needs offsets")
        _vector(gate, "gate", dev, batch, dim)
    else:
        _vector(gate, "gate", dev, dim)
    return _Norm(dev, rows, dim, batch, per_image)


def block_norm(y: torch.Tensor, residual: torch.Tensor, *, norm: str = "layer", pre_weight: torch.Tensor | None = None,
               pre_bias: torch.Tensor | None = None, post_weight: torch.Tensor | None = None,
               post_bias: torch.Tensor | None = None, gate: torch.Tensor | None = None,
               offsets: torch.Tensor | None = None, residual_scale: float = 1.0, eps: float = 1e-6,
               residual_out: torch.Tensor | None = None, h: torch.Tensor | None = None, with_stats: bool = False,
               device_status: torch.Tensor | None = None):
    """Norm after a block, gate, scaled residual stream and norm before the next block.

        u            = N(y) * post_weight + post_bias       (u = y without post_weight)
        residual_out = residual_scale * residual + gate * u
        h            = N(residual_out) * pre_weight + pre_bias

    y [rows, D] bf16 or fp32; residual [rows, D] of y's type or fp32.  norm:
    "layer" or "rms".  Parameters are fp32: [D], and the gate also [B, D], a
    row per image of ``offsets`` (int64 [B+1]).  With offsets, rows from
    offsets[B] on are left alone: the padded outputs of ``merge`` go in as
    they are.  residual_out may be ``residual`` itself (not before a backward
    pass, which needs the old one).

    Returns (residual_out, h, stats): h is None without pre_weight, stats
    (float32 [rows, 4], for ``block_norm_backward``) None unless with_stats.
    """
    a = _norm_args(y, residual, norm, pre_weight, pre_bias, post_weight, post_bias, gate, offsets)
    if residual_out is None:
        residual_out = torch.empty(a.rows, a.dim, dtype=residual.dtype, device=a.dev)
    else:
        _cuda(residual_out, "residual_out", residual.dtype, 2)
        if residual_out.shape != y.shape or residual_out.device != a.dev:
            raise ValueError("residual_out must have y's shape and device")
    if pre_weight is None:
        if h is not None:
            raise ValueError("h needs pre_weight")
    elif h is None:
        h = torch.empty(a.rows, a.dim, dtype=y.dtype, device=a.dev)
    else:
        _cuda(h, "h", y.dtype, 2)
        if h.shape != y.shape or h.device != a.dev:
            raise ValueError("h must have y's shape and device")
    stats = torch.empty(a.rows, 4, dtype=torch.float32, device=a.dev) if with_stats else None
    code = _call("mpm_block_norm", a.dev, _ptr(y), y.stride(0), _ptr(residual), residual.stride(0), _ptr(offsets),
                 a.batch, a.rows, a.dim, _dtype_code(y), _dtype_code(residual), NORMS[norm], eps, residual_scale,
                 _ptr(post_weight), _ptr(post_bias), _ptr(gate), a.per_image, _ptr(pre_weight), _ptr(pre_bias),
                 _ptr(residual_out), _ptr(h), _ptr(stats), _ptr(_status(device_status, a.dev)), _stream(a.dev))
    _check("mpm_block_norm", code)
    return residual_out, h, stats


def block_norm_workspace(dim: int, device) -> torch.Tensor:
    """Device scratch of block_norm_backward for rows of dim features (uint8)."""
    n = library().mpm_block_norm_workspace_size(int(dim))
    if n == 0:
        raise ValueError(f"invalid dim {dim} for block_norm")
    return torch.empty(int(n), dtype=torch.uint8, device=device)


def block_norm_backward(d_residual_out: torch.Tensor | None, d_h: torch.Tensor | None, y: torch.Tensor,
                        residual: torch.Tensor, stats: torch.Tensor, *, norm: str = "layer",
                        pre_weight: torch.Tensor | None = None, pre_bias: torch.Tensor | None = None,
                        post_weight: torch.Tensor | None = None, post_bias: torch.Tensor | None = None,
                        gate: torch.Tensor | None = None, offsets: torch.Tensor | None = None,
                        residual_scale: float = 1.0, eps: float = 1e-6, workspace: torch.Tensor | None = None,
                        device_status: torch.Tensor | None = None) -> BlockNormGrads:
    """Gradients of block_norm from those of its two outputs (None: zero).

    The other arguments are block_norm's own, ``stats`` what it returned.
    Token gradients have the tokens' types, parameter gradients are fp32 and
    summed in a fixed order.  Rows from offsets[B] on are left alone.
    """
    a = _norm_args(y, residual, norm, pre_weight, pre_bias, post_weight, post_bias, gate, offsets)
    if d_h is not None:
        if pre_weight is None:
            raise ValueError("d_h needs pre_weight")
        if _rows(d_h, "d_h", a.dev, y.shape).dtype != y.dtype:
            raise TypeError(f"d_h must be {y.dtype}, got {d_h.dtype}")
    if d_residual_out is not None:
        if _rows(d_residual_out, "d_residual_out", a.dev, y.shape).dtype != residual.dtype:
            raise TypeError(f"d_residual_out must be {residual.dtype}, got {d_residual_out.dtype}")
    _vector(stats, "stats", a.dev, a.rows, 4)
    if workspace is None:
        workspace = block_norm_workspace(a.dim, a.dev)
    d_y = torch.empty(a.rows, a.dim, dtype=y.dtype, device=a.dev)
    d_residual = torch.empty(a.rows, a.dim, dtype=residual.dtype, device=a.dev)
    params = (gate, post_weight, post_bias, pre_weight, pre_bias)
    d_gate, d_wpost, d_bpost, d_wpre, d_bpre = (None if p is None else torch.empty_like(p) for p in params)
    code = _call("mpm_block_norm_backward", a.dev, _ptr(d_residual_out),
                 0 if d_residual_out is None else d_residual_out.stride(0), _ptr(d_h),
                 0 if d_h is None else d_h.stride(0), _ptr(y), y.stride(0), _ptr(residual), residual.stride(0),
                 _ptr(stats), _ptr(offsets), a.batch, a.rows, a.dim, _dtype_code(y), _dtype_code(residual),
                 NORMS[norm], residual_scale, _ptr(post_weight), _ptr(post_bias), _ptr(gate), a.per_image,
                 _ptr(pre_weight), _ptr(d_y), _ptr(d_residual), _ptr(d_wpost), _ptr(d_bpost), _ptr(d_gate),
                 _ptr(d_wpre), _ptr(d_bpre), _ptr(workspace), workspace.numel(),
                 _ptr(_status(device_status, a.dev)), _stream(a.dev))
    _check("mpm_block_norm_backward", code)
    return BlockNormGrads(d_y, d_residual, d_gate, d_wpost, d_bpost, d_wpre, d_bpre)


def _mx_shapes(rows: int, dim: int):
    return (rows, -(-dim // 64) * 32), (-(-rows // 128), -(-dim // 128), 512)


def _mx(t: MXFP4, name: str, dev: torch.device | None = None) -> MXFP4:
    _cuda(t.codes, f"{name}.codes", torch.uint8, 2)
    _cuda(t.scales, f"{name}.scales", torch.uint8, 3)
    codes, scales = _mx_shapes(t.codes.shape[0], int(t.dim))
    if t.codes.shape != codes or t.scales.shape != scales:
        raise ValueError(f"{name}: codes {tuple(t.codes.shape)} and scales {tuple(t.scales.shape)} do not belong to "
                         f"{t.codes.shape[0]} rows of {t.dim} values")
    if t.scales.device != t.codes.device or (dev is not None and t.codes.device != dev):
        raise ValueError(f"{name} must be on one device, with the other operands")
    return t


def quantize_mxfp4(tokens: torch.Tensor, out: MXFP4 | None = None) -> MXFP4:
    """[rows, D] bf16 or fp32 -> MXFP4: per block of 32 the scale 2^(floor(log2 max) - 2), elements to nearest even.

    A block with a NaN or an infinity becomes NaN as a whole.
    """
    _rows(tokens, "tokens")
    rows, dim = tokens.shape
    dev = tokens.device
    if out is None:
        codes, scales = _mx_shapes(rows, dim)
        out = MXFP4(torch.empty(codes, dtype=torch.uint8, device=dev),
                    torch.empty(scales, dtype=torch.uint8, device=dev), dim)
    else:
        _mx(out, "out", dev)
        if out.rows != rows or out.dim != dim:
            raise ValueError("out must have the tokens' shape")
    code = _call("mpm_mxfp4_quantize", dev, _ptr(tokens), tokens.stride(0), rows, dim, _dtype_code(tokens),
                 _ptr(out.codes), _ptr(out.scales), _stream(dev))
    _check("mpm_mxfp4_quantize", code)
    return out


def dequantize_mxfp4(x: MXFP4, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values that x stands for, [rows, D] in bf16 or fp32."""
    _mx(x, "x")
    dev = x.codes.device
    if out is None:
        out = torch.empty(x.rows, x.dim, dtype=dtype, device=dev)
    _rows(out, "out", dev, torch.Size((x.rows, x.dim)))
    code = _call("mpm_mxfp4_dequantize", dev, _ptr(x.codes), _ptr(x.scales), x.rows, x.dim, _dtype_code(out), _ptr(out),
                 out.stride(0), _stream(dev))
    _check("mpm_mxfp4_dequantize", code)
    return out


def matmul_mxfp4(a: MXFP4, b: MXFP4, bias: torch.Tensor | None = None, out_dtype: torch.dtype = torch.bfloat16,
                 out: torch.Tensor | None = None, device_status: torch.Tensor | None = None) -> torch.Tensor:
    """a [M, K] @ b [N, K]^T + bias [N] (fp32), summed in fp32, rounded once to bf16 or fp32: [M, N].

    out may be a matrix with rows further apart, e.g. columns of a wider one.
    """
    _mx(a, "a")
    dev = a.codes.device
    _mx(b, "b", dev)
    if a.dim != b.dim:
        raise ValueError(f"a has {a.dim} features and b {b.dim}")
    _vector(bias, "bias", dev, b.rows)
    if out is None:
        out = torch.empty(a.rows, b.rows, dtype=out_dtype, device=dev)
    _rows(out, "out", dev, torch.Size((a.rows, b.rows)))
    code = _call("mpm_mxfp4_matmul", dev, _ptr(a.codes), _ptr(a.scales), a.rows, _ptr(b.codes), _ptr(b.scales), b.rows,
                 a.dim, _ptr(bias), _dtype_code(out), _ptr(out), out.stride(0), _ptr(_status(device_status, dev)),
                 _stream(dev))
    _check("mpm_mxfp4_matmul", code)
    return out
