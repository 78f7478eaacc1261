"""block_norm in 64 bits with a bound on what fp32 arithmetic may be off by, element by element.

Every quantity of the forward and the backward formulas is followed by a first
order bound on its error in units of U = 2^-24, taken from the magnitudes of
that very element and the sums it depends on:

  sum over a row of |v|     at most K roundings of each term: 16 pairs after one
                            another in a thread, 6 steps in a warp, 15 warps, the
                            product, 1 / dim and the scaling by it: K = 48
  mean m                    K mean|v|
  1 / deviation r           (K + 2) / 2 + 4 of itself, and what the row's own
                            error moves it by
  n = (v - m) r             r (error of v and m, one rounding) and r's own
  sums over rows            2 x rows a run + 64 roundings of each term (rows of a
                            run, its images, 16 groups, 152 blocks joined in 16
                            rows); a gate per image that spans many runs a
                            quarter of their number more

An output is then off by its bound and one rounding to its type.  The bound is
some hundred U of the largest term of an element, so that a term left out, a
row in another's place or a sum that misses a row shows (test_norm_bounds.py).
No code shared with the library.
"""

from __future__ import annotations

import torch

U = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
K = 48
SECOND_ORDER = 1.01  # products of errors


def _mean(v):
    return v.mean(1, keepdim=True)


class _Normed:
    """Normalised rows of v, with bounds (in U): n, r and their errors, given v's own."""

    def __init__(self, v, error, norm, eps):
        layer = norm == "layer"
        m = _mean(v) if layer else torch.zeros_like(v[:, :1])
        em = _mean(error) + K * _mean(v.abs()) if layer else torch.zeros_like(m)
        c = v - m
        self.r = 1 / (_mean(c * c) + eps).sqrt()
        self.n = c * self.r
        self.er = (K + 2) / 2 + 4 + self.r * _mean(self.n.abs() * error)      # of r itself
        self.en = self.r * (error + em + c.abs()) + self.n.abs() * (self.er + 1)


def _normed_back(a, ea, nd, norm, drop, which):
    """a - [layer] mean(a) - n mean(a n), and its bound."""
    layer = norm == "layer"
    ma = _mean(a) if layer and f"mean{which}" not in drop else torch.zeros_like(a[:, :1])
    ema = _mean(ea) + K * _mean(a.abs()) if layer else torch.zeros_like(ma)
    man = _mean(a * nd.n)
    eman = K * _mean((a * nd.n).abs()) + _mean(ea * nd.n.abs() + a.abs() * nd.en)
    if f"product{which}" in drop:
        man = torch.zeros_like(man)
    t = a - ma - nd.n * man
    et = ea + ema + (a - ma).abs() + nd.n.abs() * eman + man.abs() * nd.en + t.abs()
    return t, et


def reference(t, rows_of, norm, eps, alpha, d_residual_out=None, d_h=None, images=1, sms=152, drop=()):
    """{name: (value, bound)} in float64 of block_norm's outputs and, given their gradients, of its gradients.

    t: tensors by argument name; rows_of: every row's image.  ``drop`` names
    terms to leave out of the gradients (for tests of the comparison).
    """
    d = {k: v.double() for k, v in t.items()}
    y, x = d["y"], d["residual"]
    zero = torch.zeros_like(y)
    per_image = "gate" in d and d["gate"].dim() == 2
    gate = d["gate"][rows_of] if per_image else d.get("gate", torch.ones_like(y[:1]))
    post, pre = "post_weight" in d, "pre_weight" in d
    w1 = d.get("post_weight", torch.ones_like(y[0]))
    b1 = d.get("post_bias", torch.zeros_like(y[0]))
    A, B = gate * w1, gate * b1
    one = _Normed(y, zero, norm, eps) if post else None
    n1, en1 = (one.n, one.en) if post else (y, zero)
    xo = alpha * x + n1 * A + B
    exo = A.abs() * en1 + (n1 * A).abs() + B.abs() + (alpha * x + B).abs() + xo.abs()
    out = {"residual_out": (xo, exo)}
    if pre:
        w2, b2 = d["pre_weight"], d.get("pre_bias", torch.zeros_like(y[0]))
        two = _Normed(xo, exo, norm, eps)
        h = two.n * w2 + b2
        out["h"] = (h, w2.abs() * two.en + h.abs())
    if d_residual_out is not None or d_h is not None:
        grad = d_residual_out.double() if d_residual_out is not None else zero
        eg = zero
        dh = d_h.double() if d_h is not None else zero
        if "stream" in drop:
            grad = zero
        if pre:
            a = dh * w2
            s, es = _normed_back(a, a.abs(), two, norm, drop, 2)
            grad = grad + two.r * s
            eg = two.r * es + (two.r * s).abs() * two.er + grad.abs()
        scale = 1.0 if "alpha" in drop else alpha
        out["d_residual"] = (scale * grad, abs(alpha) * (eg + grad.abs()))
        c = grad * (w1 if "gate" in drop else A)
        ec = A.abs() * eg + 2 * c.abs()
        if post:
            s, es = _normed_back(c, ec, one, norm, drop, 1)
            dy = (1.0 if "deviation" in drop else one.r) * s
            out["d_y"] = (dy, one.r * es + dy.abs() * (one.er + 1))
        else:
            out["d_y"] = (c, ec)
        runs = -(-y.shape[0] // sms) * 2 + 64
        n1g, en1g = grad * n1, n1.abs() * eg + grad.abs() * en1

        def total(v, e, more=0.0):
            return v.sum(0), e.sum(0) + (runs + more) * v.abs().sum(0)

        def total_per_image(v, e):
            count = torch.zeros(images, dtype=torch.float64, device=v.device).index_add_(
                0, rows_of, torch.ones_like(v[:, 0]))
            into = torch.zeros(images, v.shape[1], dtype=torch.float64, device=v.device)
            parts = runs + count.clamp(max=16.0 * sms)[:, None] / 4
            return into.index_add(0, rows_of, v), into.index_add(0, rows_of, e) + parts * into.index_add(0, rows_of, v.abs())

        if "gate" in d:
            of = total_per_image if per_image else total
            (s1, e1), (s0, e0) = of(n1g, en1g), of(grad, eg)
            value = w1 * s1 + (0 if "gate bias" in drop else b1 * s0)
            out["d_gate"] = (value, w1.abs() * (e1 + s1.abs()) + b1.abs() * (e0 + s0.abs()) + value.abs())
        if post:
            g = torch.ones_like(gate) if "gate in sums" in drop else gate
            out["d_post_weight"] = total(g * n1g, gate.abs() * (en1g + n1g.abs()))
            if "post_bias" in d:
                out["d_post_bias"] = total(g * grad, gate.abs() * (eg + grad.abs()))
        if pre:
            out["d_pre_weight"] = total(dh * two.n, dh.abs() * two.en)
            if "pre_bias" in d:
                out["d_pre_bias"] = total(dh, torch.zeros_like(dh))
    return {k: (v, SECOND_ORDER * U * e) for k, (v, e) in out.items()}


def worst(got: torch.Tensor, want: torch.Tensor, bound: torch.Tensor) -> float:
    """The largest error in parts of what is allowed: the bound and one rounding to got's type."""
    if got.numel() == 0:
        return 0.0
    if not torch.isfinite(got).all():
        return float("inf")
    allowed = bound + ROUND[got.dtype] * (want.abs() + bound)
    return ((got.double() - want).abs() / allowed.clamp(min=1e-300)).max().item()


def check(got: dict, reference: dict) -> dict:
    """Asserts every output of ``got`` against the reference; how near each came to its bound."""
    assert set(got) == set(reference), (sorted(got), sorted(reference))
    far = {k: worst(v, *reference[k]) for k, v in got.items()}
    for k, v in got.items():
        assert v.shape == reference[k][0].shape, k
    bad = {k: round(f, 3) for k, f in far.items() if not f <= 1.0}
    assert not bad, f"parts of the bound: {bad}"
    return far
