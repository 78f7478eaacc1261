"""Refusals of the attention and rotary entry points at the C boundary (no GPU needed: arguments are checked before any
CUDA call), and the workspaces' sizes."""

from __future__ import annotations

import ctypes

import pytest

from test_block_args import at, lib  # noqa: F401

WS = 1 << 24


def attend(lib, **kw):  # noqa: F811
    a = dict(q=at(0), q_row=256, q_head=64, k=at(1), k_row=128, k_head=64, v=at(2), v_row=128, v_head=64, q_offsets=at(3),
             k_offsets=at(4), batch=2, q_rows=100, k_rows=200, q_heads=4, kv_heads=2, dim=64, dtype=1, scale=0.125,
             mask=at(5), out=at(6), rest=at(7), lse=at(8), workspace=at(9), workspace_bytes=WS, status=None, stream=None)
    a.update(kw)
    return lib.mpm_cross_attention(*a.values())


def learn(lib, **kw):  # noqa: F811
    a = dict(g=at(0), g_row=256, g_head=64, q=at(1), q_row=256, q_head=64, k=at(2), k_row=128, k_head=64, v=at(3), v_row=128,
             v_head=64, out=at(4), rest=at(5), lse=at(6), q_offsets=at(7), k_offsets=at(8), batch=2, q_rows=100, k_rows=200,
             q_heads=4, kv_heads=2, dim=64, dtype=1, scale=0.125, mask=at(9), d_q=at(10), d_k=at(11), d_v=at(12),
             workspace=at(13), workspace_bytes=WS, status=None, stream=None)
    a.update(kw)
    return lib.mpm_cross_attention_backward(*a.values())


def turn(lib, sections=(8, 8), **kw):  # noqa: F811
    n = (ctypes.c_int32 * len(sections))(*sections) if sections is not None else None
    a = dict(x=at(0), x_row=256, x_head=64, positions=at(1), frequencies=at(2), sections=n,
             axes=2 if sections is None else len(sections), layout=0, inverse=0, offsets=at(3), batch=2, rows=100, heads=4, dim=64,
             dtype=1, out=at(4), out_row=256, out_head=64, status=None, stream=None)
    a.update(kw)
    return lib.mpm_rotary(*a.values())


SHARED = [(dict(q_rows=-1), 1), (dict(k_rows=-1), 1), (dict(batch=0), 1), (dict(q_heads=0), 1), (dict(kv_heads=0), 1),
          (dict(kv_heads=3), 1), (dict(dim=0), 1), (dict(dtype=7), 1), (dict(scale=0.0), 1), (dict(scale=-1.0), 1),
          (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(q=None), 1), (dict(k=None), 1), (dict(v=None), 1),
          (dict(q_offsets=None), 1), (dict(k_offsets=None), 1), (dict(q_offsets=None, k_offsets=None), 1),
          (dict(q_row=63), 1), (dict(k_head=32), 1), (dict(v_row=64, v_head=64), 1), (dict(q_rows=1 << 31), 1),
          (dict(dim=129, q_row=1024, q_head=129, k_row=1024, k_head=129, v_row=1024, v_head=129), 2),
          (dict(q_heads=8192, kv_heads=2, q_row=8192 * 64), 2), (dict(dtype=0), 2),      # the rest of a rounding that fp32 has not
          (dict(q=at(20) + 1), 3), (dict(k=at(20) + 1), 3), (dict(q_offsets=at(20) + 4), 3), (dict(lse=at(20) + 2), 3),
          (dict(rest=at(20) + 1), 3), (dict(status=at(20) + 2), 3), (dict(workspace=None), 4), (dict(workspace=at(20) + 16), 4),
          (dict(workspace_bytes=16), 4)]


@pytest.mark.parametrize("bad, code", SHARED, ids=[str(b) for b, _ in SHARED])
def test_shared_refusals(lib, bad, code):  # noqa: F811
    assert attend(lib, **bad) == code
    if "dim" in bad and bad["dim"] == 129:
        bad = dict(bad, g_row=1024, g_head=129)
    if "q_heads" in bad and bad["q_heads"] == 8192:
        bad = dict(bad, g_row=8192 * 64)
    assert learn(lib, **bad) == code


def test_attention_outputs(lib):  # noqa: F811
    assert attend(lib, out=None) == 1
    assert attend(lib, out=at(6) + 1) == 3
    inputs = dict(q=0, k=1, v=2, q_offsets=3, k_offsets=4, mask=5)
    for out in ("out", "rest", "lse", "status", "workspace"):
        for name, place in inputs.items():
            assert attend(lib, **{out: at(place)}) == 8, (out, name)
    assert attend(lib, lse=at(6) + 128) == 8 and attend(lib, rest=at(6) + 128) == 8 and attend(lib, status=at(7)) == 8
    # The last of its bytes, with rows far apart.
    assert attend(lib, out=at(0) + (99 * 1000 + 4 * 64) * 2 - 16, q_row=1000) == 8
    assert attend(lib, q_rows=0) == 0


def test_gradients(lib):  # noqa: F811
    for bad in (dict(g=None), dict(out=None), dict(lse=None), dict(d_q=None), dict(d_k=None), dict(d_v=None), dict(g_row=8)):
        assert learn(lib, **bad) == 1, bad
    for bad in (dict(g=at(20) + 1), dict(d_q=at(10) + 1), dict(d_v=at(12) + 1), dict(out=at(20) + 1)):
        assert learn(lib, **bad) == 3, bad
    for out in ("d_q", "d_k", "d_v", "workspace", "status"):
        for place in range(10):
            assert learn(lib, **{out: at(place)}) == 8, (out, place)
    assert learn(lib, d_k=at(10) + 64) == 8 and learn(lib, d_v=at(11)) == 8 and learn(lib, workspace=at(12)) == 8
    assert learn(lib, q_rows=0, k_rows=0) == 0


def test_rotary(lib):  # noqa: F811
    for bad in (dict(rows=-1), dict(heads=0), dict(dim=1), dict(dtype=9), dict(layout=2), dict(batch=0), dict(x=None),
                dict(out=None), dict(positions=None), dict(frequencies=None), dict(sections=None), dict(x_row=100), dict(out_head=8)):
        assert turn(lib, **bad) == 1, bad
    for sections in ((0, 8), (-1, 8), (16, 17), (33,), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert turn(lib, sections) == 1, sections
    assert turn(lib, (), axes=0) == 1
    assert turn(lib, (1,) * 9) == 2
    assert turn(lib, dim=1025, x_head=1025, x_row=5000, out_head=1025, out_row=5000) == 2
    for bad in (dict(x=at(0) + 1), dict(out=at(4) + 1), dict(positions=at(1) + 2), dict(frequencies=at(2) + 4),
                dict(offsets=at(3) + 4), dict(status=at(20) + 1)):
        assert turn(lib, **bad) == 3, bad
    for place in (1, 2, 3):
        assert turn(lib, out=at(place)) == 8 and turn(lib, status=at(place)) == 8
    assert turn(lib, status=at(0)) == 8 and turn(lib, status=at(4)) == 8
    assert turn(lib, out=at(0) + 128) == 8                        # over x, but not x itself
    assert turn(lib, out=at(0), out_row=300) == 8                 # x with other strides
    assert turn(lib, rows=0) == 0


def test_workspace_sizes(lib):  # noqa: F811
    forward, backward = lib.mpm_cross_attention_workspace_size, lib.mpm_cross_attention_backward_workspace_size
    assert forward(2, 100, 200, 4, 3, 64, 1) == 0 and forward(0, 100, 200, 4, 2, 64, 1) == 0 and backward(2, -1, 5, 4, 2, 64, 1) == 0
    assert backward(2, 100, 200, 4, 2, 64, 1) >= 100 * 4 * 4
    # Parts only where there is little to do side by side: a batch of many rows needs none.
    assert forward(64, 65536, 65536, 12, 12, 64, 1) == 0
    assert forward(1, 1, 1 << 20, 8, 8, 64, 1) >= 2 * 8 * 64 * 4
    for rows in (1, 100, 1000, 100000):
        for keys in (1, 77, 5000, 1 << 20):
            for size in (forward, backward):
                assert size(1, rows, keys, 8, 8, 128, 1) % 256 == 0 and size(3, rows, keys, 8, 1, 128, 0) <= 1 << 33
