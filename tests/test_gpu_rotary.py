"""rotary and rotary_backward against the 64-bit form, element by element."""

from __future__ import annotations

import pytest
import torch

import exact_attention as exact

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


def draw(rows, heads, dim, axes, dtype, far=64.0, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(rows, heads, dim, generator=gen, device=DEV).to(dtype)
    at = far * torch.rand(rows, axes, generator=gen, device=DEV)
    return x, torch.where(torch.rand(rows, axes, generator=gen, device=DEV) < 0.5, at.round(), at)


def check(mpm, x, at, sections, layout, frequencies=None, **kw):
    f = mpm.rotary_frequencies(sections) if frequencies is None else frequencies
    for call, inverse in ((mpm.rotary, False), (mpm.rotary_backward, True)):
        got = call(x, at, f, sections, layout=layout, **kw)
        want = exact.rotary(x, at, f, sections, layout, inverse)
        exact.check(got, want, exact.rotary_bound(x, want, sections, layout), call.__name__)
        rest = 2 * sum(sections)
        assert torch.equal(got[..., rest:], x[..., rest:])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layout", ["halves", "interleaved"])
@pytest.mark.parametrize("shape", [(1, 1, 2, (1,)), (1, 40, 128, (16, 24, 24)), (3, 2, 7, (1, 1)), (5, 3, 64, (16, 16)),
                                   (1300, 2, 40, (7, 13)), (257, 12, 64, (8,)), (100, 1, 96, (4, 8, 12, 16)),
                                   (33, 5, 33, (5, 11)), (4, 2, 1024, (512,)), (9, 3, 256, (1, 2, 3, 4, 5, 6, 7, 8)),
                                   (2000, 24, 64, (16, 16))])
def test_shapes(mpm, shape, layout, dtype):
    rows, heads, dim, sections = shape
    x, at = draw(rows, heads, dim, len(sections), dtype)
    check(mpm, x, at, sections, layout)


@pytest.mark.parametrize("far", [1e3, 1e5, 1e7, -3e6])
def test_far_positions(mpm, far):
    """Angles of a million turns are as exact as near ones."""
    x, at = draw(64, 2, 64, 2, torch.float32, far)
    check(mpm, x, at, (16, 16), "halves")
    check(mpm, x, at, (16, 16), "interleaved", frequencies=torch.linspace(0.3, 3.0, 32, dtype=torch.float64, device=DEV))


def test_positions_that_are_no_numbers(mpm):
    x, at = draw(4, 2, 8, 1, torch.float32)
    at[1], at[2] = float("nan"), float("inf")
    got = mpm.rotary(x, at, mpm.rotary_frequencies((2,)), (2,))
    assert torch.isnan(got[1:3, :, :4]).all() and torch.equal(got[..., 4:], x[..., 4:])
    assert torch.isfinite(got[[0, 3]]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layout", ["halves", "interleaved"])
@pytest.mark.parametrize("kind", ["joint", "heads_first", "odd_rows"])
def test_strides_and_in_place(mpm, kind, layout, dtype):
    x, at = draw(50, 4, 64, 2, dtype)
    f, sections = mpm.rotary_frequencies((8, 12)), (8, 12)
    want = mpm.rotary(x, at, f, sections, layout=layout)
    if kind == "joint":                       # queries and keys of a joint projection, values behind them
        base = torch.cat([x.reshape(50, 256), torch.ones(50, 128, dtype=dtype, device=DEV)], 1)
        view = base[:, :256].unflatten(1, (4, 64))
    elif kind == "heads_first":
        base = x.transpose(0, 1).contiguous()
        view = base.transpose(0, 1)
    else:
        base = torch.zeros(50 * 259 + 3, dtype=dtype, device=DEV)
        view = base[3:].as_strided((50, 4, 64), (259, 64, 1), 3)
        view.copy_(x)
    assert torch.equal(mpm.rotary(view, at, f, sections, layout=layout), want)
    before = view._version
    got = mpm.rotary(view, at, f, sections, layout=layout, out=view)
    assert got is view and view._version == before + 1 and torch.equal(view, want)
    if kind == "joint":
        assert (base[:, 256:] == 1).all()
    into = torch.zeros(50, 8, 64, dtype=dtype, device=DEV)
    mpm.rotary(x, at, f, sections, layout=layout, out=into[:, 2:6])
    assert torch.equal(into[:, 2:6], want) and (into[:, :2] == 0).all() and (into[:, 6:] == 0).all()


def test_rows_behind_the_last_sequence(mpm):
    x, at = draw(300, 3, 64, 2, torch.bfloat16)
    f = mpm.rotary_frequencies((16, 16))
    want = mpm.rotary(x, at, f, (16, 16))
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    for live in (0, 1, 170, 300):
        out = torch.full_like(x, 3.0)
        mpm.rotary(x, at, f, (16, 16), offsets=torch.tensor([0, live // 2, live], device=DEV), out=out, device_status=status)
        assert torch.equal(out[:live], want[:live]) and (out[live:] == 3).all()
    assert status.tolist() == [0, 0]
    mpm.rotary(x, at, f, (16, 16), offsets=torch.tensor([0, 9, 400], device=DEV), device_status=status)
    assert status[0] == 6
    assert mpm.rotary(x[:0], at[:0], f, (16, 16)).shape == (0, 3, 64)


def test_there_and_back(mpm):
    """Turning back what was turned gives x: the gradient of an orthogonal map is its inverse."""
    x, at = draw(200, 4, 64, 3, torch.float32, 1e4)
    f, s = mpm.rotary_frequencies((8, 12, 12)), (8, 12, 12)
    y = mpm.rotary(x, at, f, s)
    back = mpm.rotary_backward(y, at, f, s)
    # Each way a pair is off by no more than 2^-20 of its length.
    size = (x[..., :32] ** 2 + x[..., 32:] ** 2).sqrt()
    assert ((back - x)[..., :32].abs() <= 2.0 ** -19 * size).all() and ((back - x)[..., 32:].abs() <= 2.0 ** -19 * size).all()


def test_captured(mpm):
    x, at = draw(100, 4, 64, 2, torch.bfloat16)
    f = mpm.rotary_frequencies((16, 16))
    mpm.rotary(x, at, f, (16, 16))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = mpm.rotary(x, at, f, (16, 16))
        z = mpm.rotary_backward(y, at, f, (16, 16))
    at.add_(5.0)
    graph.replay()
    want = mpm.rotary(x, at, f, (16, 16))
    assert torch.equal(y, want) and torch.equal(z, mpm.rotary_backward(want, at, f, (16, 16)))
