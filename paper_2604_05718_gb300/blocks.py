"""Python binding of the encoder-block entry points of libmpm.so.

``block_norm`` is everything elementwise between two blocks of an encoder
(norm after the block, gate, scaled residual stream, norm before the next
block) in one pass over packed tokens, with ``block_norm_backward`` for its
gradients.  ``quantize_mxfp4`` and ``matmul_mxfp4`` are a linear layer on
4-bit operands.  As in ``mpm``, arguments are checked and marshalled only, and
every step runs in the library's kernels on the current torch stream; the
marshalling is the extension module ``_blocks`` (csrc/blocks_binding.cpp).

Nothing is recorded for autograd: ``block_norm_backward`` is called by hand (or
from a ``torch.autograd.Function``), and a tensor that requires grad is refused
while grad mode is on.
"""

from __future__ import annotations

import ctypes
import importlib
from typing import NamedTuple

import torch

from .mpm import _check, library

_ENTRIES = ("mpm_block_norm", "mpm_block_norm_workspace_size", "mpm_block_norm_backward", "mpm_mxfp4_quantize",
            "mpm_mxfp4_dequantize", "mpm_mxfp4_matmul")
_module = None


def load_binding():
    """The extension module, bound to the loaded library's entry points; raises where it has not been built."""
    global _module
    if _module is None:
        lib = library()
        try:
            module = importlib.import_module("._blocks", __package__)
        except ImportError as e:
            raise RuntimeError("the binding of the block operators is missing or does not load; build it with "
                               "paper_2604_05718_gb300.build.build()") from e
        module.bind(tuple(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _ENTRIES), _check)
        _module = module
    return _module


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
    return (_module or load_binding()).block_norm(y, residual, norm, pre_weight, pre_bias, post_weight, post_bias, gate,
                                                  offsets, residual_scale, eps, residual_out, h, with_stats, device_status)


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
    return BlockNormGrads(*(_module or load_binding()).block_norm_backward(
        y, residual, norm, pre_weight, pre_bias, post_weight, post_bias, gate, offsets, residual_scale, eps, d_residual_out,
        d_h, stats, workspace, device_status))


def quantize_mxfp4(tokens: torch.Tensor, out: MXFP4 | None = None) -> MXFP4:
    """[rows, D] bf16 or fp32 -> MXFP4: per block of 32 the scale 2^(floor(log2 max) - 2), elements to nearest even.

    A block with a NaN or an infinity becomes NaN as a whole.
    """
    if out is None:
        codes, scales = (_module or load_binding()).quantize(tokens, None, None)
        return MXFP4(codes, scales, tokens.shape[1])
    if out.dim != tokens.shape[-1]:
        raise ValueError("out must have the tokens' shape")
    (_module or load_binding()).quantize(tokens, out.codes, out.scales)
    return out


def dequantize_mxfp4(x: MXFP4, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values that x stands for, [rows, D] in bf16 or fp32."""
    codes, scales, dim = x
    return (_module or load_binding()).dequantize(codes, scales, dim, dtype, out)


def matmul_mxfp4(a: MXFP4, b: MXFP4, bias: torch.Tensor | None = None, out_dtype: torch.dtype = torch.bfloat16,
                 out: torch.Tensor | None = None, device_status: torch.Tensor | None = None) -> torch.Tensor:
    """a [M, K] @ b [N, K]^T + bias [N] (fp32), summed in fp32, rounded once to bf16 or fp32: [M, N].

    out may be a matrix with rows further apart, e.g. columns of a wider one.
    """
    ac, asc, k = a
    bc, bs, kb = b
    return (_module or load_binding()).matmul(ac, asc, k, bc, bs, kb, bias, out_dtype, out, device_status)
