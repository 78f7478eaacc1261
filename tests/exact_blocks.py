"""64-bit forms of the encoder-block operators, from their definitions.

Test infrastructure: plain torch in float64, no code shared with the library.
"""

from __future__ import annotations

import torch


def normalised(v: torch.Tensor, norm: str, eps: float) -> torch.Tensor:
    if norm == "layer":
        v = v - v.mean(1, keepdim=True)
    return v / ((v * v).mean(1, keepdim=True) + eps).sqrt()


def block_norm(y, residual, *, norm, eps, residual_scale, rows_of=None, post_weight=None, post_bias=None, gate=None,
               pre_weight=None, pre_bias=None):
    """(residual_out, h) in float64; rows_of gives every row's image for a gate per image."""
    u = y
    if post_weight is not None:
        u = normalised(y, norm, eps) * post_weight
        if post_bias is not None:
            u = u + post_bias
    if gate is not None:
        u = u * (gate[rows_of] if gate.dim() == 2 else gate)
    out = residual_scale * residual + u
    if pre_weight is None:
        return out, None
    h = normalised(out, norm, eps) * pre_weight
    return out, h if pre_bias is None else h + pre_bias


LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def mxfp4_values(x: torch.Tensor) -> torch.Tensor:
    """The MXFP4 values nearest to x [rows, dim] (float64, CPU): a search over all levels, block by block."""
    x = x.double().cpu()
    rows, dim = x.shape
    out = torch.empty_like(x)
    levels = torch.tensor(LEVELS, dtype=torch.float64)
    # A tie goes to the even code: tried in this order, the first nearest level wins.
    order = [0, 2, 4, 6, 1, 3, 5, 7]
    for lo in range(0, dim, 32):
        b = x[:, lo:lo + 32]
        bad = ~torch.isfinite(b).all(1, keepdim=True)
        b = torch.where(bad, torch.zeros_like(b), b)
        top = b.abs().amax(1, keepdim=True)
        _, e = torch.frexp(top)                                  # top = m 2^e, 1/2 <= m < 1
        unit = torch.ldexp(torch.ones_like(top), (e - 3).clamp(min=-127))
        unit = torch.where(top > 0, unit, torch.ones_like(unit))
        a = (b / unit).abs()
        far = (a.unsqueeze(2) - levels[order]).abs()
        q = levels[order][far.argmin(2)] * unit
        out[:, lo:lo + 32] = torch.where(bad, torch.full_like(q, float("nan")), torch.where(b < 0, -q, q))
    return out


def mxfp4_unpack(codes: torch.Tensor, scales: torch.Tensor, dim: int):
    """Codes and scale codes as [rows, dim] and [rows, blocks] integers, byte by byte from the documented layout."""
    codes, scales = codes.cpu().long(), scales.cpu().long()
    rows = codes.shape[0]
    k = torch.arange(dim)
    code = (codes[:, k // 2] >> (4 * (k % 2))) & 15
    r = torch.arange(rows)[:, None]
    j = torch.arange(-(-dim // 32))[None, :]
    return code, scales[r // 128, j // 4, 16 * (r % 32) + 4 * (r % 128 // 32) + j % 4]


def mxfp4_decode(codes: torch.Tensor, scales: torch.Tensor, dim: int) -> torch.Tensor:
    """The float64 values of packed codes and tiled scales."""
    code, c = mxfp4_unpack(codes, scales, dim)
    v = torch.tensor(LEVELS, dtype=torch.float64)[code & 7]
    v = torch.where(code >= 8, -v, v)
    unit = torch.ldexp(torch.ones(c.shape, dtype=torch.float64), c - 127)
    unit = torch.where(c == 255, torch.full_like(unit, float("nan")), unit)
    return v * unit.repeat_interleave(32, 1)[:, :dim]
