"""block_norm and block_norm_backward against 64 bits, at the sizes where they can go wrong.

Bounds.  All arithmetic is fp32 with unit roundoff U = 2^-24, every output is
rounded once to its type.  A value of a row is the result of fewer than 256
roundings (a row's sum: at most 32 values a thread, 5 shuffle steps, 16 warps;
two sums and some ten operations after one another, their errors added), each
of a quantity no larger than the row's magnitudes combined below, so

  |got - want| <= u(type) |want| + 256 U x (magnitude).

Column sums over rows add, per column, at most rows / 100 + 256 such terms
after one another (runs of rows of about 150 groups, then groups and blocks).
"""

from __future__ import annotations

import itertools

import pytest
import torch

import exact_blocks

pytestmark = pytest.mark.gpu

DEV = "cuda"
U = 2.0 ** -24
STEPS = 256
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "f32": (torch.float32, torch.float32),
         "mixed": (torch.bfloat16, torch.float32)}


@pytest.fixture(scope="module")
def mpm():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2604_05718_gb300 as pkg
    from paper_2604_05718_gb300 import build

    build.build()
    pkg.library()
    return pkg


def inputs(counts, dim, types, *, seed=0, layer=True, gate="channel", post=True, pre=True, mean=0.0):
    """(tensors by argument name, offsets, image of every row)."""
    gen = torch.Generator().manual_seed(seed)
    rows = sum(counts)
    ty, tx = TYPES[types]

    def draw(*shape, around=0.0, spread=1.0):
        return (around + spread * torch.randn(*shape, generator=gen, dtype=torch.float64)).to(DEV)

    t = {"y": draw(rows, dim, around=mean).to(ty), "residual": draw(rows, dim, around=mean, spread=2.0).to(tx)}
    if post:
        t["post_weight"] = draw(dim, around=1.0, spread=0.3).float()
        if layer:
            t["post_bias"] = draw(dim, spread=0.3).float()
    if gate == "channel":
        t["gate"] = draw(dim, spread=0.5).float()
    elif gate == "image":
        t["gate"] = draw(len(counts), dim, spread=0.5).float()
    if pre:
        t["pre_weight"] = draw(dim, around=1.0, spread=0.3).float()
        if layer:
            t["pre_bias"] = draw(dim, spread=0.3).float()
    off = torch.tensor([0] + list(itertools.accumulate(counts)), dtype=torch.int64, device=DEV)
    rows_of = torch.repeat_interleave(torch.arange(len(counts), device=DEV), torch.tensor(counts, device=DEV))
    return t, off, rows_of


def params_of(t):
    return {k: v for k, v in t.items() if k not in ("y", "residual")}


def magnitudes(t, rows_of, norm, eps, alpha):
    """Per row: 1 / deviation of both norms and the largest |y| r1 w1 + b1, stream value, and n2."""
    y, x = t["y"].double(), t["residual"].double()

    def rdev(v):
        c = v - v.mean(1, keepdim=True) if norm == "layer" else v
        return 1 / ((c * c).mean(1, keepdim=True) + eps).sqrt()

    zero = torch.zeros(1, dtype=torch.float64, device=DEV)
    top = lambda v: v.abs().amax(-1, keepdim=True)  # noqa: E731
    r1 = rdev(y) if "post_weight" in t else torch.ones_like(y[:, :1])
    w1 = top(t["post_weight"].double()) if "post_weight" in t else zero + 1
    b1 = top(t["post_bias"].double()) if "post_bias" in t else zero
    u = top(y) * r1 * w1 + b1
    g = zero + 1
    if "gate" in t:
        g = top(t["gate"].double())
        g = g[rows_of] if t["gate"].dim() == 2 else g
    xo, _ = exact_blocks.block_norm(y, x, norm=norm, eps=eps, residual_scale=alpha, rows_of=rows_of,
                                    **{k: v.double() for k, v in params_of(t).items()})
    r2 = rdev(xo) if "pre_weight" in t else torch.ones_like(r1)
    s = abs(alpha) * top(x) + g * u
    w2 = top(t["pre_weight"].double()) if "pre_weight" in t else zero
    b2 = top(t["pre_bias"].double()) if "pre_bias" in t else zero
    return {"r1": r1, "w1": w1, "n1": top(y) * r1, "u": u, "g": g, "s": s, "r2": r2, "w2": w2, "b2": b2, "n2": s * r2}


def within(got, want, magnitude, what, steps=STEPS):
    bound = ROUND[got.dtype] * want.abs() + steps * U * magnitude
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all(), what
    worst = (off / bound.clamp(min=1e-300)).max().item() if got.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} of the bound"


def check_forward(mpm, t, off, rows_of, norm, eps=1e-6, alpha=1.0, with_offsets=True):
    xo, h, stats = mpm.block_norm(t["y"], t["residual"], norm=norm, eps=eps, residual_scale=alpha, with_stats=True,
                                  offsets=off if with_offsets else None, **params_of(t))
    want_x, want_h = exact_blocks.block_norm(t["y"].double(), t["residual"].double(), norm=norm, eps=eps,
                                             residual_scale=alpha, rows_of=rows_of,
                                             **{k: v.double() for k, v in params_of(t).items()})
    m = magnitudes(t, rows_of, norm, eps, alpha)
    assert xo.dtype == t["residual"].dtype
    within(xo, want_x, m["s"], "residual_out")
    if "pre_weight" in t:
        assert h.dtype == t["y"].dtype
        within(h, want_h, m["n2"] * m["w2"] + m["b2"], "h")
    else:
        assert h is None
    return xo, h, stats


def check_backward(mpm, t, off, rows_of, norm, eps=1e-6, alpha=1.0, seed=1, strided=False):
    _, _, stats = check_forward(mpm, t, off, rows_of, norm, eps, alpha)
    gen = torch.Generator().manual_seed(seed)
    rows, dim = t["y"].shape

    def draw(dtype):
        wide = torch.randn(rows, dim + 8, generator=gen, dtype=torch.float64).to(DEV, dtype)
        return wide[:, :dim] if strided else wide[:, :dim].contiguous()

    dxo, dh = draw(t["residual"].dtype), draw(t["y"].dtype) if "pre_weight" in t else None
    got = mpm.block_norm_backward(dxo, dh, t["y"], t["residual"], stats, norm=norm, eps=eps, residual_scale=alpha,
                                  offsets=off, **params_of(t))
    leaves = {k: v.double().requires_grad_() for k, v in t.items()}
    xo, h = exact_blocks.block_norm(leaves["y"], leaves["residual"], norm=norm, eps=eps, residual_scale=alpha,
                                    rows_of=rows_of, **{k: v for k, v in leaves.items() if k not in ("y", "residual")})
    outs, seeds = [xo], [dxo.double()]
    if h is not None:
        outs, seeds = [xo, h], [dxo.double(), dh.double()]
    want = dict(zip(leaves, torch.autograd.grad(outs, list(leaves.values()), seeds)))
    m = magnitudes(t, rows_of, norm, eps, alpha)
    top = lambda v: v.abs().amax(1, keepdim=True)  # noqa: E731
    a = top(dh.double()) * m["w2"] if dh is not None else 0.0
    n2, n1 = m["n2"], m["n1"]
    grad = top(dxo.double()) + (m["r2"] * a * (2 + n2 * n2) if dh is not None else 0.0)
    # n2 (or n1) itself is off by so many roundings of its magnitude: it enters the gradients as a factor.
    grad = grad * (1 + n2)
    within(got.d_residual, want["residual"], abs(alpha) * grad, "d_residual")
    c = m["g"] * grad * m["w1"]
    within(got.d_y, want["y"], m["r1"] * c * (2 + n1 * n1) * (1 + n1) if "post_weight" in t else c, "d_y")
    terms = {"gate": m["u"] * grad, "post_weight": m["g"] * grad * n1, "post_bias": m["g"] * grad,
             "pre_weight": top(dh.double()) * n2 if dh is not None else None,
             "pre_bias": top(dh.double()) if dh is not None else None}
    for k, each in terms.items():
        g = getattr(got, "d_" + k)
        if k not in t:
            assert g is None
            continue
        assert g.shape == t[k].shape and g.dtype == torch.float32
        total = each.sum() if t[k].dim() == 1 else torch.zeros(len(off) - 1, 1, dtype=torch.float64, device=DEV) \
            .index_add_(0, rows_of, each.expand(rows, 1))
        within(g, want[k], total, "d_" + k, steps=2 * STEPS + rows / 100)
    return got, (dxo, dh, stats)


DIMS = [1, 7, 8, 33, 196, 256, 257, 385, 512, 768, 1000, 1024, 1032, 2048, 2049, 4104, 8200]


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("types", ["bf16", "f32", "mixed"])
@pytest.mark.parametrize("dim", DIMS)
def test_every_width_both_directions(mpm, dim, types, norm):
    t, off, rows_of = inputs([5, 0, 1, 30], dim, types, seed=dim, layer=norm == "layer", gate="image")
    check_backward(mpm, t, off, rows_of, norm, alpha=0.75)


def test_widest_row(mpm):
    t, off, rows_of = inputs([3, 2], 16384, "bf16", layer=True, gate="image")
    check_backward(mpm, t, off, rows_of, "layer")
    t, off, rows_of = inputs([3], 16383, "f32", layer=False, gate="channel")
    check_backward(mpm, t, off, rows_of, "rms")


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("pre", [False, True])
@pytest.mark.parametrize("gate", ["none", "channel", "image"])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_every_part_may_be_absent(mpm, norm, gate, pre, post):
    t, off, rows_of = inputs([17, 3, 0, 64], 192, "bf16", layer=norm == "layer", gate=gate, post=post, pre=pre)
    check_backward(mpm, t, off, rows_of, norm, alpha=-0.5)


@pytest.mark.parametrize("counts", [[1], [0, 1, 0], [1] * 300, [0] * 40 + [7] + [0] * 40, [4000, 1, 2, 3000],
                                    [13] * 211, [1024] * 9, [2431]])
@pytest.mark.parametrize("gate", ["channel", "image"])
def test_images_of_all_sizes(mpm, counts, gate):
    t, off, rows_of = inputs(counts, 128, "bf16", gate=gate)
    got, _ = check_backward(mpm, t, off, rows_of, "layer")
    if gate == "image":
        for b, n in enumerate(counts):
            if n == 0:
                assert not got.d_gate[b].any()


def test_rows_of_zeros_and_of_one_value(mpm):
    # Without variance the deviation is sqrt(eps): finite, as the formula has it.
    for norm in ("rms", "layer"):
        t, off, rows_of = inputs([6], 96, "f32", layer=norm == "layer")
        t["y"][1:3] = 0.0
        t["y"][3] = 2.0
        t["residual"][2:5] = 0.0
        check_backward(mpm, t, off, rows_of, norm, eps=1e-3)


def test_large_mean_keeps_its_variance(mpm):
    # mean 1000, deviation about 1: E[v^2] - m^2 would lose the variance in fp32.
    t, off, rows_of = inputs([9, 4], 768, "f32", mean=1000.0, gate="none")
    check_forward(mpm, t, off, rows_of, "layer")


def test_infinities_and_nans_stay_in_their_rows(mpm):
    t, off, rows_of = inputs([8], 256, "bf16", gate="channel")
    clean_x, clean_h, stats = mpm.block_norm(t["y"], t["residual"], norm="layer", with_stats=True, **params_of(t))
    t["y"][2, 5] = float("nan")
    t["residual"][4, 7] = float("inf")
    xo, h, stats = mpm.block_norm(t["y"], t["residual"], norm="layer", with_stats=True, **params_of(t))
    keep = [0, 1, 3, 5, 6, 7]
    assert torch.equal(xo[keep], clean_x[keep]) and torch.equal(h[keep], clean_h[keep])
    assert xo[2].isnan().all() and h[2].isnan().all() and h[4].isnan().all()
    assert torch.equal(xo[4, :7], clean_x[4, :7]) and xo[4, 7] == float("inf")
    g = mpm.block_norm_backward(torch.ones_like(xo), torch.ones_like(h), t["y"], t["residual"], stats, norm="layer",
                                **params_of(t))
    assert torch.isfinite(g.d_y[keep]).all() and torch.isfinite(g.d_residual[keep]).all()


@pytest.mark.parametrize("types", ["bf16", "f32", "mixed"])
@pytest.mark.parametrize("pad", [8, 3])
def test_strided_rows(mpm, types, pad):
    t, off, rows_of = inputs([20, 11], 64, types, gate="image")
    for k in ("y", "residual"):
        wide = torch.full((31, 64 + pad), 7.0, dtype=t[k].dtype, device=DEV)
        wide[:, :64] = t[k]
        t[k] = wide[:, :64]
    check_backward(mpm, t, off, rows_of, "layer", strided=True)


def test_unaligned_buffers(mpm):
    t, off, rows_of = inputs([9], 64, "bf16")
    for k in list(t):
        flat = torch.empty(t[k].numel() + 1, dtype=t[k].dtype, device=DEV)
        flat[1:] = t[k].reshape(-1)
        t[k] = flat[1:].view(t[k].shape)
    check_backward(mpm, t, off, rows_of, "layer")


def test_rows_past_the_last_image_are_left_alone(mpm):
    t, off, rows_of = inputs([10, 6], 72, "bf16", gate="image")
    used = {k: v.clone() for k, v in t.items()}
    for k in ("y", "residual"):
        t[k] = torch.cat([used[k], torch.full((5, 72), float("nan"), dtype=used[k].dtype, device=DEV)])
    xo, h = torch.full_like(t["residual"], 3.0), torch.full_like(t["y"], 3.0)
    _, _, stats = mpm.block_norm(t["y"], t["residual"], offsets=off, residual_out=xo, h=h, with_stats=True,
                                 **params_of(t))
    assert (xo[16:] == 3).all() and (h[16:] == 3).all()
    want_x, want_h, want_s = mpm.block_norm(used["y"], used["residual"], offsets=off, with_stats=True, **params_of(t))
    assert torch.equal(xo[:16], want_x) and torch.equal(h[:16], want_h)
    ones = torch.ones_like(t["y"])
    got = mpm.block_norm_backward(ones, ones, t["y"], t["residual"], stats, offsets=off, **params_of(t))
    want = mpm.block_norm_backward(ones[:16], ones[:16], used["y"], used["residual"], want_s, offsets=off,
                                   **params_of(t))
    for a, b in zip(got[2:], want[2:]):
        assert torch.isfinite(a).all()
        torch.testing.assert_close(a, b, rtol=2e-5, atol=2e-5)


def test_in_place_on_the_stream(mpm):
    t, off, rows_of = inputs([50], 1032, "mixed")
    want_x, want_h, _ = mpm.block_norm(t["y"], t["residual"], **params_of(t))
    x = t["residual"].clone()
    got_x, got_h, _ = mpm.block_norm(t["y"], x, residual_out=x, **params_of(t))
    assert got_x is x and torch.equal(x, want_x) and torch.equal(got_h, want_h)


def test_no_rows(mpm):
    t, off, rows_of = inputs([0, 0, 0], 40, "f32", gate="image")
    got, _ = check_backward(mpm, t, off, rows_of, "layer")
    for g in got[2:]:
        assert not g.any()


@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_gradients_against_differences(mpm, norm):
    """Directional derivatives of the forward kernel by central differences.

    L = <dx', x'> + <dh, h>, summed in 64 bits from fp32 outputs.  The error of
    the extrapolated difference is at most the change between the two steps;
    each L is off by at most STEPS U times its terms.
    """
    t, off, rows_of = inputs([4, 0, 5], 48, "f32", layer=norm == "layer", gate="image", seed=3)
    gen = torch.Generator().manual_seed(9)
    draw = lambda v: torch.randn(v.shape, generator=gen).to(DEV)  # noqa: E731
    xo, h, stats = mpm.block_norm(t["y"], t["residual"], norm=norm, offsets=off, residual_scale=0.8, with_stats=True,
                                  **params_of(t))
    dxo, dh = draw(xo), draw(h)
    grads = mpm.block_norm_backward(dxo, dh, t["y"], t["residual"], stats, norm=norm, offsets=off, residual_scale=0.8,
                                    **params_of(t))

    def loss(name, by):
        s = dict(t)
        s[name] = t[name] + by
        a, b, _ = mpm.block_norm(s["y"], s["residual"], norm=norm, offsets=off, residual_scale=0.8, **params_of(s))
        return ((dxo.double() * a.double()).sum() + (dh.double() * b.double()).sum()).item()

    noise = STEPS * U * ((dxo * xo).abs().sum() + (dh * h).abs().sum() + dh.abs().sum() * 4).item()
    for name in t:
        way = draw(t[name])
        step = 2.0 ** -6
        slope = [(loss(name, s * way) - loss(name, -s * way)) / (2 * s) for s in (step, step / 2)]
        best = (4 * slope[1] - slope[0]) / 3
        grad = getattr(grads, "d_" + name)
        got = (grad.double() * way.double()).sum().item()
        assert abs(got - best) <= abs(slope[0] - slope[1]) + 3 * noise / step, name


def test_same_bits_every_time(mpm):
    t, off, rows_of = inputs([700, 123, 0, 900], 384, "bf16", gate="image")
    first, (dxo, dh, stats) = check_backward(mpm, t, off, rows_of, "layer")
    for _ in range(5):
        again = mpm.block_norm_backward(dxo, dh, t["y"], t["residual"], stats, offsets=off, **params_of(t))
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_one_gradient_may_be_absent(mpm):
    t, off, rows_of = inputs([12, 20], 100, "f32", gate="image")
    xo, h, stats = mpm.block_norm(t["y"], t["residual"], offsets=off, with_stats=True, **params_of(t))
    d = torch.randn(h.shape, generator=torch.Generator().manual_seed(2)).to(DEV)
    zero = torch.zeros_like(d)
    for left, right in (((None, d), (zero, d)), ((d, None), (d, zero)), ((None, None), (zero, zero))):
        a = mpm.block_norm_backward(*left, t["y"], t["residual"], stats, offsets=off, **params_of(t))
        b = mpm.block_norm_backward(*right, t["y"], t["residual"], stats, offsets=off, **params_of(t))
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_another_stream(mpm):
    t, off, rows_of = inputs([4000], 768, "bf16")
    want = mpm.block_norm(t["y"], t["residual"], with_stats=True, **params_of(t))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = t["y"] * 0
        for _ in range(20):
            y = y + 0
        y = y + t["y"]
        got = mpm.block_norm(y, t["residual"], with_stats=True, **params_of(t))
        g = mpm.block_norm_backward(got[0], got[1], y, t["residual"], got[2], **params_of(t))
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    again = mpm.block_norm_backward(want[0], want[1], t["y"], t["residual"], want[2], **params_of(t))
    assert all(torch.equal(a, b) for a, b in zip(g, again) if a is not None)


def test_bad_offsets_are_reported_and_stay_inside(mpm):
    t, off, rows_of = inputs([10, 10, 10], 64, "bf16", gate="image")
    for bad in ([0, 20, 10, 30], [0, 10, 20, 31], [1, 10, 20, 30], [0, -5, 20, 30], [0, 10, 20, -3], [0, 2**40, 5, 30]):
        status = torch.zeros(2, dtype=torch.int32, device=DEV)
        o = torch.tensor(bad, dtype=torch.int64, device=DEV)
        _, _, stats = mpm.block_norm(t["y"], t["residual"], offsets=o, device_status=status, with_stats=True,
                                     **params_of(t))
        assert status[0].item() == 6
        status.zero_()
        mpm.block_norm_backward(torch.ones_like(t["residual"]), torch.ones_like(t["y"]), t["y"], t["residual"], stats,
                                offsets=o, device_status=status, **params_of(t))
        assert status[0].item() == 6
    status.zero_()
    mpm.block_norm(t["y"], t["residual"], offsets=off, device_status=status, **params_of(t))
    assert status.tolist() == [0, 0]


def test_refusals(mpm):
    t, off, _ = inputs([8, 8], 64, "bf16", gate="image")
    y, x, p = t["y"], t["residual"], params_of(t)
    with pytest.raises(ValueError):
        mpm.block_norm(y.cpu(), x, **p, offsets=off)
    with pytest.raises(ValueError):
        mpm.block_norm(y, x[:8], **p, offsets=off)
    with pytest.raises(ValueError):
        mpm.block_norm(y.t(), x.t(), **p, offsets=off)
    with pytest.raises(ValueError):
        mpm.block_norm(y, x, **p)                                        # a gate per image without offsets
    with pytest.raises(ValueError):
        mpm.block_norm(y, x, **p, offsets=torch.cat([off, off[-1:]]))    # a gate for each of three images
    with pytest.raises(ValueError):
        mpm.block_norm(y, x, norm="batch", offsets=off, **p)
    with pytest.raises(ValueError):
        mpm.block_norm(y, x, pre_bias=p["pre_bias"])                     # a bias without its weight
    with pytest.raises(TypeError):
        mpm.block_norm(y.half(), x)
    with pytest.raises(TypeError):
        mpm.block_norm(y, x, gate=p["gate"][0].bfloat16())
    with pytest.raises(mpm.MPMError) as e:
        mpm.block_norm(y.float(), x)                                     # fp32 blocks on a bf16 stream
    assert e.value.code == 2
    with pytest.raises(mpm.MPMError) as e:
        mpm.block_norm(y, x, residual_out=y)                             # output over an input
    assert e.value.code == 8
    with pytest.raises(mpm.MPMError) as e:
        mpm.block_norm(y, x, eps=float("nan"))
    assert e.value.code == 1
    xo, h, stats = mpm.block_norm(y, x, offsets=off, with_stats=True, **p)
    with pytest.raises(ValueError):
        mpm.block_norm_backward(xo, h, y, x, stats[:4], offsets=off, **p)
    with pytest.raises(TypeError):
        mpm.block_norm_backward(xo.float(), h, y, x, stats, offsets=off, **p)
    with pytest.raises(mpm.MPMError) as e:
        mpm.block_norm_backward(xo, h, y, x, stats, offsets=off, workspace=stats.new_empty(64, dtype=torch.uint8), **p)
    assert e.value.code == 4
