"""Outputs of the norms' entry points that lie over a parameter, the offsets or the status word are refused.

Arguments are checked before any CUDA call, so made-up addresses will do and
no GPU is needed; the test with real buffers packs them next to one another.
"""

from __future__ import annotations

import pytest
import torch

from test_block_args import at, backward, forward, lib  # noqa: F401

ALIASING = 8
ROWS, DIM, BATCH = 100, 64, 2
VECTOR = 4 * DIM
# Addresses that the helpers of test_block_args give to a call's buffers, and the bytes of each.
FORWARD_IN = {"offsets": (2, 8 * (BATCH + 1)), "post_weight": (3, VECTOR), "post_bias": (4, VECTOR),
              "gate": (5, BATCH * VECTOR), "pre_weight": (6, VECTOR), "pre_bias": (7, VECTOR)}
FORWARD_OUT = ("residual_out", "h", "stats")
BACKWARD_IN = {"offsets": (5, 8 * (BATCH + 1)), "post_weight": (6, VECTOR), "post_bias": (7, VECTOR),
               "gate": (8, BATCH * VECTOR), "pre_weight": (9, VECTOR)}
BACKWARD_OUT = ("d_y", "d_residual", "d_post_weight", "d_post_bias", "d_gate", "d_pre_weight", "d_pre_bias")


@pytest.mark.parametrize("out", FORWARD_OUT)
@pytest.mark.parametrize("name", list(FORWARD_IN))
def test_forward_outputs_over_a_parameter(lib, name, out):  # noqa: F811
    place, size = FORWARD_IN[name]
    assert forward(lib, **{out: at(place)}) == ALIASING
    assert forward(lib, **{out: at(place) + (size - 1) // 16 * 16}) == ALIASING      # over its last bytes
    # Or the parameter within the output.
    first = {"residual_out": at(8), "h": at(9), "stats": at(10)}[out]
    assert forward(lib, **{name: first + 64}) == ALIASING


@pytest.mark.parametrize("out", BACKWARD_OUT)
@pytest.mark.parametrize("name", list(BACKWARD_IN))
def test_gradients_over_a_parameter(lib, name, out):  # noqa: F811
    place, size = BACKWARD_IN[name]
    assert backward(lib, **{out: at(place)}) == ALIASING
    assert backward(lib, **{out: at(place) + (size - 1) // 16 * 16}) == ALIASING
    assert backward(lib, **{out: at(20), name: at(20) + 64}) == ALIASING


@pytest.mark.parametrize("name", list(BACKWARD_IN))
def test_workspace_over_a_parameter(lib, name):  # noqa: F811
    assert backward(lib, workspace=at(BACKWARD_IN[name][0])) == ALIASING
    assert backward(lib, **{name: at(17) + 1024}) == ALIASING


def test_status_word_over_an_argument(lib):  # noqa: F811
    for place in (0, 1, 2, 3, 5, 6, 8, 9, 10):
        assert forward(lib, status=at(place)) == ALIASING, place
    for place in (0, 2, 3, 4, 5, 6, 8, 10, 12, 14, 17):
        assert backward(lib, status=at(place)) == ALIASING, place
    one = [at(0), at(1), 10, at(2), at(3), 20, 64, at(4), 1, at(5), 20]
    for place in range(6):
        assert lib.mpm_mxfp4_matmul(*one, at(place), None) == ALIASING, place


@pytest.mark.gpu
@pytest.mark.parametrize("per_image", [False, True])
def test_neighbouring_buffers_are_taken(per_image):
    import paper_2604_05718_gb300 as mpm
    from paper_2604_05718_gb300 import build

    build.build()
    rows, dim, dev = 12, 64, "cuda"
    gen = torch.Generator().manual_seed(4)
    draw = lambda *s: torch.randn(*s, generator=gen).to(dev)  # noqa: E731
    x, y, w, b = draw(rows, dim), draw(rows, dim), draw(dim), draw(dim)
    gate = draw(2, dim) if per_image else draw(dim)
    off = torch.tensor([0, 5, rows], device=dev)
    args = dict(pre_weight=w, pre_bias=b, post_weight=w, post_bias=b, offsets=off)
    want = mpm.block_norm(y, x, gate=gate, **args)
    # gate | residual_out | h in one allocation, without a gap.
    arena = torch.zeros(gate.numel() + 2 * rows * dim, device=dev)
    g, out, h = arena.split([gate.numel(), rows * dim, rows * dim])
    g.copy_(gate.reshape(-1))
    mpm.block_norm(y, x, gate=g.view(gate.shape), residual_out=out.view(rows, dim), h=h.view(rows, dim), **args)
    assert torch.equal(out.view(rows, dim), want[0]) and torch.equal(h.view(rows, dim), want[1])
    with pytest.raises(mpm.MPMError) as e:
        mpm.block_norm(y, x, gate=arena[:gate.numel()].view(gate.shape), h=arena[gate.numel() - 4:][:rows * dim].view(rows, dim),
                       **args)
    assert e.value.code == ALIASING
