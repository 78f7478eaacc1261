"""A pair of CTAs that gives up waits for the copies of both (csrc/pair_ring.cuh), however far each had come.

The kernel of pair_ring_drain.cu loads as the 4-bit product does, into three
slots, and stops each CTA after its own number of loads.  Nothing faults or
hangs: each wait ends by its limit, and none should need it.
"""

from __future__ import annotations

import ctypes
import os
import subprocess
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
SLOTS, ROWS, COLS, LOADS = 3, 8, 32, 12
LIMIT_US = 200000


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_05718_gb300 import build

    lib = str(tmp_path_factory.mktemp("pair") / "pair_ring.so")
    subprocess.run([build.nvcc(), "-shared", os.path.join(HERE, "pair_ring_drain.cu"), "-o", lib, "-cudart", "static"] +
                   build.NVCC_FLAGS, check=True)
    entry = ctypes.CDLL(lib).run_pair_ring
    entry.argtypes = [ctypes.c_void_p] + [ctypes.c_int] * 5 + [ctypes.c_uint32, ctypes.c_void_p, ctypes.c_void_p]
    n, r = torch.arange(LOADS)[:, None, None], torch.arange(2)[None, :, None]
    values = (10000 * n + 1000 * r + torch.arange(ROWS * COLS)).to("cuda", torch.int32).contiguous()

    def call(common, mine, theirs, failed_rank):
        result = torch.full((2 + 2 * SLOTS,), -7, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        assert entry(values.data_ptr(), LOADS, common, mine, theirs, failed_rank, LIMIT_US, result.data_ptr(),
                     torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        return result[:2].tolist(), result[2:].view(2, SLOTS).tolist(), time.perf_counter() - t0

    return call


def last(count):
    return sorted(list(range(max(count - SLOTS, 0), count)) + [-1] * max(SLOTS - count, 0))


@pytest.mark.parametrize("failed_rank", [0, 1])
@pytest.mark.parametrize("theirs", range(SLOTS + 1))
@pytest.mark.parametrize("mine", range(SLOTS + 1))
@pytest.mark.parametrize("common", [0, 1, 4, 8])
def test_every_pair_of_counts(run, common, mine, theirs, failed_rank):
    (drained, in_step), landed, took = run(common, common + mine, common + theirs, failed_rank)
    assert in_step == common
    assert drained == 1 and took < LIMIT_US * 1e-6          # no wait ran to its limit
    assert sorted(landed[0]) == last(common + mine) and sorted(landed[1]) == last(common + theirs)


def test_a_pair_without_a_failure_leaves_at_once(run):
    (drained, in_step), _, _ = run(8, 8, 8, -1)
    assert (drained, in_step) == (-1, 8)
