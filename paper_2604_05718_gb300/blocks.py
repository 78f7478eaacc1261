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

from .mpm import MPM_BF16, MPM_F32, _check, _cuda, _ptr, library

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


# Small calls are bound by the host, so what is right is recognised in one
# expression per tensor, and only what is not goes through the checks that say
# why.  (One row through block_norm: 19 us a call when every check was a call of
# its own and every argument looked up again, 14 now: 4 each for the outputs'
# allocation, the marshalling of the arguments and the launch.)
_entries: dict = {}


def _run(name: str, index: int, *args) -> None:
    """library().<name>(*args, stream) on the current stream of CUDA device `index`, made current if need be."""
    fn = _entries.get(name)
    if fn is None:
        fn = _entries[name] = getattr(library(), name)
    if torch._C._cuda_getDevice() == index:
        code = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            code = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    if code != 0:
        _check(name, code)


def _rows(t: torch.Tensor, name: str, index: int | None = None, shape=None) -> int:
    """Checks a CUDA matrix of bf16 or fp32 rows, each contiguous, any distance apart; its type's code."""
    if isinstance(t, torch.Tensor) and t.get_device() == index and t.shape == shape and t.is_contiguous():
        code = _DTYPES.get(t.dtype)
        if code is not None:
            return code
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dim() != 2:
        raise ValueError(f"{name} must have 2 dimensions")
    if index is not None and t.get_device() != index:
        raise ValueError(f"{name} must be on CUDA device {index}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype not in _DTYPES:
        raise TypeError(f"{name} must be bfloat16 or float32, got {t.dtype}")
    if (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return _DTYPES[t.dtype]


def _buffer(t: torch.Tensor, name: str, index: int, dtype: torch.dtype, shape: tuple) -> int | None:
    """Checks a contiguous CUDA tensor of the given type and shape; its address."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == index and t.shape == shape and
            t.is_contiguous()):
        _cuda(t, name, dtype)
        if t.get_device() != index:
            raise ValueError(f"{name} must be on CUDA device {index}")
        if t.shape != shape:
            raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr() or None


def _new_like(t: torch.Tensor) -> torch.Tensor:
    """A new contiguous matrix of t's shape and type (1.3 us; torch.empty 1.7)."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _status(t: torch.Tensor | None, index: int) -> int | None:
    if t is None:
        return None
    _cuda(t, "device_status", torch.int32, 1)
    if t.get_device() != index or t.numel() < 2:
        raise ValueError(f"device_status must be an int32 [2] tensor on CUDA device {index}")
    return t.data_ptr()


def _norm_args(y, residual, norm, pre_weight, pre_bias, post_weight, post_bias, gate, offsets) -> tuple:
    """Checks the arguments that both directions share; (device, rows, dim, types, addresses and counts)."""
    if norm not in NORMS:
        raise ValueError(f"norm must be one of {sorted(NORMS)}, got {norm!r}")
    dtype = _rows(y, "y")
    index, shape = y.get_device(), y.shape
    stream_dtype = _rows(residual, "residual", index, shape)
    rows, dim = shape
    vector = (dim,)
    batch, per_image, poff, pgate = 1, 0, None, None
    if offsets is not None:
        _cuda(offsets, "offsets", torch.int64, 1)
        batch = offsets.numel() - 1
        if offsets.get_device() != index or batch < 1:
            raise ValueError(f"offsets must be an int64 [B+1] tensor on CUDA device {index}")
        poff = offsets.data_ptr()
    pw = qw = pb = qb = None
    if pre_weight is not None:
        qw = _buffer(pre_weight, "pre_weight", index, torch.float32, vector)
    if post_weight is not None:
        pw = _buffer(post_weight, "post_weight", index, torch.float32, vector)
    if pre_bias is not None:
        qb = _buffer(pre_bias, "pre_bias", index, torch.float32, vector)
        if pre_weight is None:
            raise ValueError("pre_bias needs pre_weight")
    if post_bias is not None:
        pb = _buffer(post_bias, "post_bias", index, torch.float32, vector)
        if post_weight is None:
            raise ValueError("post_bias needs post_weight")
    if gate is not None:
        if gate.dim() == 2:
            if offsets is None:
                raise ValueError("a gate per image needs offsets")
            per_image = 1
            vector = (batch, dim)
        pgate = _buffer(gate, "gate", index, torch.float32, vector)
    return index, rows, dim, dtype, stream_dtype, batch, poff, pw, pb, pgate, per_image, qw, qb


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
    index, rows, dim, dtype, stream_dtype, batch, poff, pw, pb, pgate, per_image, qw, qb = _norm_args(
        y, residual, norm, pre_weight, pre_bias, post_weight, post_bias, gate, offsets)
    shape = y.shape
    if residual_out is None:
        residual_out = _new_like(residual)
        out = residual_out.data_ptr() or None
    else:
        out = _buffer(residual_out, "residual_out", index, residual.dtype, shape)
    ph = None
    if pre_weight is None:
        if h is not None:
            raise ValueError("h needs pre_weight")
    elif h is None:
        h = _new_like(y)
        ph = h.data_ptr() or None
    else:
        ph = _buffer(h, "h", index, y.dtype, shape)
    stats = torch.empty((rows, 4), dtype=torch.float32, device=y.device) if with_stats else None
    _run("mpm_block_norm", index, y.data_ptr() or None, y.stride(0), residual.data_ptr() or None, residual.stride(0), poff,
         batch, rows, dim, dtype, stream_dtype, NORMS[norm], eps, residual_scale, pw, pb, pgate, per_image, qw, qb, out, ph,
         _ptr(stats), _status(device_status, index))
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
    index, rows, dim, dtype, stream_dtype, batch, poff, pw, pb, pgate, per_image, qw, qb = _norm_args(
        y, residual, norm, pre_weight, pre_bias, post_weight, post_bias, gate, offsets)
    dev, shape = y.device, y.shape
    if d_h is not None:
        if pre_weight is None:
            raise ValueError("d_h needs pre_weight")
        if _rows(d_h, "d_h", index, shape) != dtype:
            raise TypeError(f"d_h must be {y.dtype}, got {d_h.dtype}")
    if d_residual_out is not None and _rows(d_residual_out, "d_residual_out", index, shape) != stream_dtype:
        raise TypeError(f"d_residual_out must be {residual.dtype}, got {d_residual_out.dtype}")
    pstats = _buffer(stats, "stats", index, torch.float32, (rows, 4))
    if workspace is None:
        workspace = block_norm_workspace(dim, dev)
    d_y, d_residual = _new_like(y), _new_like(residual)
    params = (gate, post_weight, post_bias, pre_weight, pre_bias)
    d_gate, d_wpost, d_bpost, d_wpre, d_bpre = grads = [None if p is None else torch.empty_like(p) for p in params]
    pg, pwp, pbp, pwq, pbq = [None if g is None else g.data_ptr() or None for g in grads]
    _run("mpm_block_norm_backward", index, _ptr(d_residual_out), 0 if d_residual_out is None else d_residual_out.stride(0),
         _ptr(d_h), 0 if d_h is None else d_h.stride(0), y.data_ptr() or None, y.stride(0), residual.data_ptr() or None,
         residual.stride(0), pstats, poff, batch, rows, dim, dtype, stream_dtype, NORMS[norm], residual_scale, pw, pb, pgate,
         per_image, qw, d_y.data_ptr() or None, d_residual.data_ptr() or None, pwp, pbp, pg, pwq, pbq,
         _ptr(workspace), workspace.numel(), _status(device_status, index))
    return BlockNormGrads(d_y, d_residual, d_gate, d_wpost, d_bpost, d_wpre, d_bpre)


def _mx_shapes(rows: int, dim: int):
    return (rows, -(-dim // 64) * 32), (-(-rows // 128), -(-dim // 128), 512)


def _mx(t: MXFP4, name: str, index: int | None = None) -> tuple:
    """Checks an MXFP4 matrix; (device, rows, addresses of codes and scales)."""
    codes, scales, dim = t
    if index is None:
        _cuda(codes, f"{name}.codes", torch.uint8, 2)
        index = codes.get_device()
    rows = codes.shape[0]
    shapes = _mx_shapes(rows, dim)
    if codes.shape != shapes[0] or scales.shape != shapes[1]:
        raise ValueError(f"{name}: codes {tuple(codes.shape)} and scales {tuple(scales.shape)} do not belong to "
                         f"{rows} rows of {dim} values")
    return (index, rows, _buffer(codes, f"{name}.codes", index, torch.uint8, shapes[0]),
            _buffer(scales, f"{name}.scales", index, torch.uint8, shapes[1]))


def quantize_mxfp4(tokens: torch.Tensor, out: MXFP4 | None = None) -> MXFP4:
    """[rows, D] bf16 or fp32 -> MXFP4: per block of 32 the scale 2^(floor(log2 max) - 2), elements to nearest even.

    A block with a NaN or an infinity becomes NaN as a whole.
    """
    dtype = _rows(tokens, "tokens")
    index = tokens.get_device()
    rows, dim = tokens.shape
    if out is None:
        codes, scales = _mx_shapes(rows, dim)
        out = MXFP4(torch.empty(codes, dtype=torch.uint8, device=tokens.device),
                    torch.empty(scales, dtype=torch.uint8, device=tokens.device), dim)
        pc, ps = out[0].data_ptr() or None, out[1].data_ptr() or None
    else:
        _, out_rows, pc, ps = _mx(out, "out", index)
        if out_rows != rows or out.dim != dim:
            raise ValueError("out must have the tokens' shape")
    _run("mpm_mxfp4_quantize", index, tokens.data_ptr() or None, tokens.stride(0), rows, dim, dtype, pc, ps)
    return out


def dequantize_mxfp4(x: MXFP4, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """The values that x stands for, [rows, D] in bf16 or fp32."""
    index, rows, pc, ps = _mx(x, "x")
    if out is None:
        out = torch.empty((rows, x.dim), dtype=dtype, device=x.codes.device)
    code = _rows(out, "out", index, (rows, x.dim))
    _run("mpm_mxfp4_dequantize", index, pc, ps, rows, x.dim, code, out.data_ptr() or None, out.stride(0))
    return out


def matmul_mxfp4(a: MXFP4, b: MXFP4, bias: torch.Tensor | None = None, out_dtype: torch.dtype = torch.bfloat16,
                 out: torch.Tensor | None = None, device_status: torch.Tensor | None = None) -> torch.Tensor:
    """a [M, K] @ b [N, K]^T + bias [N] (fp32), summed in fp32, rounded once to bf16 or fp32: [M, N].

    out may be a matrix with rows further apart, e.g. columns of a wider one.
    """
    index, m, ac, asc = _mx(a, "a")
    _, n, bc, bs = _mx(b, "b", index)
    k = a.dim
    if k != b.dim:
        raise ValueError(f"a has {k} features and b {b.dim}")
    pbias = None if bias is None else _buffer(bias, "bias", index, torch.float32, (n,))
    if out is None:
        out = torch.empty((m, n), dtype=out_dtype, device=a.codes.device)
    code = _rows(out, "out", index, (m, n))
    _run("mpm_mxfp4_matmul", index, ac, asc, m, bc, bs, n, k, pbias, code, out.data_ptr() or None, out.stride(0),
         _status(device_status, index))
    return out
