"""64-bit forms of attention between packed sequences and of rotary positions, with bounds for their errors.

Test infrastructure: plain torch in float64, no code shared with the library.

A bound follows each quantity's error to first order (the tests add a quarter for
what lies beyond).  u is half a step of the tokens' type, w half a step of fp32, and
v half a step of what probabilities are rounded to before they multiply (bf16, or
nothing more than fp32).  A sum of n terms in fp32, in any order, is off by at most
n w times the sum of their sizes.

Where v is bf16's, score gradients multiply as two bf16 values, the second half a step
of bf16 from what the first left: v^2.  Elsewhere factors multiply as two tf32 values
of eleven bits.  The second is at most 2^-11 of the factor, so the dropped product of
both seconds is 2^-22; it has up to twelve bits, of which one is cut, 2^-23 a factor.
Together y = 2^-21 = 8 w a product.
"""

from __future__ import annotations

import math
from typing import NamedTuple

import torch

W = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: W}


class Exact(NamedTuple):
    """Values, and how far a computed one may be."""

    out: torch.Tensor
    lse: torch.Tensor
    d_q: torch.Tensor
    d_k: torch.Tensor
    d_v: torch.Tensor
    out_bound: torch.Tensor
    lse_bound: torch.Tensor
    d_q_bound: torch.Tensor
    d_k_bound: torch.Tensor
    d_v_bound: torch.Tensor


def attention(q, k, v, d_out, q_offsets, k_offsets, mask, scale, probabilities=None) -> Exact:
    """All of it for packed tensors; rows outside the sequences are zeros.  probabilities: the type they are rounded to."""
    u, pu = HALF[q.dtype], HALF[probabilities or q.dtype]
    y, du = (8 * W, W) if pu == W else (0.0, pu * pu)
    q, k, v, g = q.double(), k.double(), v.double(), d_out.double()
    heads, group, dim = q.shape[1], q.shape[1] // k.shape[1], q.shape[2]
    zeros = torch.zeros_like
    r = Exact(zeros(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device), zeros(q), zeros(k), zeros(v),
              zeros(q), torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device), zeros(q), zeros(k), zeros(v))
    for b in range(len(q_offsets) - 1):
        rows = slice(q_offsets[b], q_offsets[b + 1])
        cols = torch.arange(k_offsets[b], k_offsets[b + 1], device=q.device)
        if mask is not None:
            cols = cols[mask[cols] != 0]
        nq, nk = q_offsets[b + 1] - q_offsets[b], cols.numel()
        if nq == 0 or nk == 0:
            continue
        for h in range(heads):
            kv = h // group
            qh, kh, vh, gh = q[rows, h], k[cols, kv], v[cols, kv], g[rows, h]
            s = scale * qh @ kh.t()
            lse = torch.logsumexp(s, 1, keepdim=True)
            p = torch.exp(s - lse)
            o = p @ vh
            # Scores: the product's sum, the factor's rounding, that of score - maximum, and the exponential's few units.
            size = scale * qh.abs() @ kh.abs().t()
            es = ((dim + 4) * W + y) * size + 4 * W * (s.abs() + lse.abs())
            ep = es + (p * es).sum(1, keepdim=True) + (8 + nk) * W
            r.out[rows, h], r.lse[rows, h] = o, lse[:, 0]
            eo = (p * (ep + pu + nk * W + y)) @ vh.abs()
            r.out_bound[rows, h] = eo + u * o.abs()
            r.lse_bound[rows, h] = (p * es).sum(1) + (8 + nk) * W + 4 * W * (lse[:, 0].abs() + s.abs().amax(1))
            # Backward: p from the kept lse, its own error among it.
            el = r.lse_bound[rows, h][:, None]
            ep = es + el + 8 * W
            t = gh @ vh.t()
            delta = (gh * o).sum(1, keepdim=True)
            # delta is taken from the output and what its rounding left.
            ed = (gh.abs() * (eo + u * u * o.abs())).sum(1, keepdim=True) + dim * W * (gh.abs() * o.abs()).sum(1, keepdim=True)
            ds = p * (t - delta)
            eds = p * ((t - delta).abs() * (ep + 2 * W) + ed + ((dim + 2) * W + y) * (gh.abs() @ vh.abs().t())) + du * ds.abs()
            r.d_q[rows, h] = scale * ds @ kh
            r.d_q_bound[rows, h] = scale * (eds + (nk * W + y) * ds.abs()) @ kh.abs() + u * r.d_q[rows, h].abs()
            n = nq * group * W
            r.d_v[cols, kv] += p.t() @ gh
            r.d_v_bound[cols, kv] += (p * (ep + pu + n + y)).t() @ gh.abs()
            r.d_k[cols, kv] += scale * ds.t() @ qh
            r.d_k_bound[cols, kv] += scale * (eds + (n + y) * ds.abs()).t() @ qh.abs()
    r.d_k_bound.add_(u * r.d_k.abs())
    r.d_v_bound.add_(u * r.d_v.abs())
    return r


def check(got: torch.Tensor, want: torch.Tensor, bound: torch.Tensor, what: str) -> None:
    """Every element within 1.25 times its bound (and of what the smallest normal numbers lose)."""
    got = got.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, 0.0, (got - want).abs())
    over = off - (1.25 * bound + 1e-36)
    assert not torch.isnan(over).any(), f"{what}: NaN where there is none, or the other way round"
    worst = int(over.argmax()) if over.numel() else 0
    assert over.numel() == 0 or float(over.max()) <= 0, \
        f"{what}: element {worst} is {got.flatten()[worst]:.9g}, wants {want.flatten()[worst]:.9g} within {1.25 * bound.flatten()[worst]:.3g}"


def rotary(x, positions, frequencies, sections, layout, inverse=False):
    """x in float64, its pairs turned as complex numbers."""
    pairs = sum(sections)
    at = positions.double().reshape(x.shape[0], -1).repeat_interleave(torch.tensor(sections, device=x.device), dim=1)
    angle = at * frequencies.double() * (-1.0 if inverse else 1.0)
    unit = torch.complex(angle.cos(), angle.sin())[:, None, :]
    x = x.double()
    first, second = ((slice(0, pairs), slice(pairs, 2 * pairs)) if layout == "halves"
                     else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)))
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * unit
    out = x.clone()
    out[..., first], out[..., second] = z.real, z.imag
    return out


def rotary_bound(x, want, sections, layout):
    """Sines and cosines off by 2^-22 (angles to 2^-24 turns, and their own rounding), two products, one sum, the output's rounding."""
    pairs = sum(sections)
    first, second = ((slice(0, pairs), slice(pairs, 2 * pairs)) if layout == "halves"
                     else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)))
    size = x.double().abs()
    both = size[..., first] + size[..., second]
    bound = torch.zeros_like(size)
    bound[..., first] = bound[..., second] = both * (2.0 ** -21 + 3 * W)
    # The output is rounded from a value that is that far off itself.
    return bound + HALF[x.dtype] * (want.abs() + bound) * (size >= 0)
