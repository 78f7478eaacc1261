"""Long runs of rows: ring slots that are filled again, several images a run, and rows over several warps.

A group of warps works on a run of neighbouring rows.  The backward pass has
up to 16 groups a block, one block an SM, and up to 4 rows in a group's ring;
the cases give every group at least three times its ring, so that slots are
filled again, their phase flips, and the halves of the sums' scratch alternate.
"""

from __future__ import annotations

import pytest
import torch

from test_gpu_block_norm_bounds import check, mpm  # noqa: F401
from test_norm_bounds import TYPES

pytestmark = pytest.mark.gpu

RING = 4
# Features and the most groups of a block that they can have: warps of a block (16 for up to
# 256 features a warp, 12 for 512, 8 for 768 or 1024) over those that a row takes.
GROUPS = {96: 16, 256: 16, 384: 12, 512: 12, 768: 8, 1024: 6, 1536: 4, 2048: 3, 4104: 1, 8200: 1,
          257: 12, 770: 6, 1025: 4, 2050: 2}      # the last ones: rows that are not 16-byte aligned in bf16


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def counts_of(rows: int, seed: int) -> list:
    """Images of 0 to 9 rows, now and then a long one: several a run, and some over many runs."""
    gen = torch.Generator().manual_seed(seed)
    out = []
    while sum(out) < rows:
        small = torch.randint(0, 10, (40,), generator=gen).tolist()
        out += small + [int(torch.randint(100, 700, (1,), generator=gen))]
    return out


def test_the_rows_fill_every_ring():
    """The groups above are no fewer than a block can have, from the file's own rule for warps and chunks."""
    for dim, groups in GROUPS.items():
        chunks = -(-dim // 256)
        per_warp = 1 if chunks == 1 else 4 if chunks > 24 else 3 if chunks % 3 == 0 else 2
        warps = {3: 8, 2: 12, 1: 16, 4: 16 if dim > 8192 else 8}[per_warp]
        assert groups >= warps // -(-dim // (256 * per_warp)), dim


@pytest.mark.parametrize("gate", ["channel", "image"])
@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("dim", list(GROUPS))
def test_many_rows_a_group(mpm, dim, types, gate):  # noqa: F811
    rows = 3 * RING * sms() * GROUPS[dim] + 41
    check(mpm, counts_of(rows, dim), dim, types, "layer", seed=dim, gate=gate)


@pytest.mark.parametrize("post,pre", [(False, True), (True, False), (False, False)])
@pytest.mark.parametrize("dim", [384, 768, 1024, 2048, 8200])
def test_many_rows_a_group_with_parts_absent(mpm, dim, post, pre):  # noqa: F811
    rows = 3 * RING * sms() * GROUPS[dim] + 17
    check(mpm, counts_of(rows, dim + 1), dim, "bf16", "layer", seed=dim, post=post, pre=pre)
    check(mpm, counts_of(rows, dim + 2), dim, "mixed", "rms", seed=dim, post=post, pre=pre)


@pytest.mark.parametrize("dim", [768, 1024, 2048])
def test_the_same_bits_from_run_to_run(mpm, dim):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(dim)
    rows = 3 * RING * sms() * GROUPS[dim] + 5
    draw = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    y, x, dxo, dh = (draw(rows, dim).bfloat16() for _ in range(4))
    off = torch.tensor([0] + counts_of(rows, 1), device="cuda").cumsum(0).clamp(max=rows)
    args = dict(pre_weight=draw(dim), pre_bias=draw(dim), post_weight=draw(dim), post_bias=draw(dim),
                gate=draw(len(off) - 1, dim), offsets=off)
    _, _, stats = mpm.block_norm(y, x, with_stats=True, **args)
    first = mpm.block_norm_backward(dxo, dh, y, x, stats, **args)
    for _ in range(4):
        assert all(torch.equal(a, b) for a, b in zip(first, mpm.block_norm_backward(dxo, dh, y, x, stats, **args)))
