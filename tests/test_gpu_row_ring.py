"""A ring of rows whose wait runs out (csrc/row_ring.cuh): it asks for no more rows and waits for those under way.

The kernel of row_ring_timeout.cu takes ten rows of 64 numbers through three
slots as the backward pass of block_norm does; one barrier expects bytes that
nobody sends.  Nothing faults or hangs: each wait ends by its limit.
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
SLOTS, WORDS, ROWS = 3, 64, 10


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_05718_gb300 import build

    lib = str(tmp_path_factory.mktemp("ring") / "row_ring.so")
    subprocess.run([build.nvcc(), "-shared", os.path.join(HERE, "row_ring_timeout.cu"), "-o", lib, "-cudart", "static"] +
                   build.NVCC_FLAGS, check=True)
    entry = ctypes.CDLL(lib).run_row_ring
    entry.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_uint32, ctypes.c_void_p, ctypes.c_void_p,
                      ctypes.c_void_p]
    rows = (1000 * torch.arange(ROWS)[:, None] + torch.arange(WORDS)).to("cuda", torch.int32)

    def call(stuck, limit_us=20000):
        sums = torch.zeros(ROWS, 2, dtype=torch.int32, device="cuda")
        result = torch.full((3 + SLOTS,), -7, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        assert entry(rows.data_ptr(), ROWS, stuck, limit_us, sums.data_ptr(), result.data_ptr(),
                     torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        return sums.cpu(), result.tolist(), time.perf_counter() - t0

    call.want = torch.stack([rows[:, :32].sum(1), rows[:, 32:].sum(1)], 1).cpu()
    return call


def test_rows_of_a_whole_run(run):
    sums, (asked, ran_out, drained, *landed), _ = run(-1)
    assert torch.equal(sums.long(), run.want) and (asked, ran_out, drained) == (ROWS, 0, -1)
    assert sorted(landed) == [7, 8, 9]


@pytest.mark.parametrize("stuck", range(ROWS))
def test_after_a_wait_that_ran_out(run, stuck):
    sums, (asked, ran_out, drained, *landed), took = run(stuck)
    assert torch.equal(sums[:stuck].long(), run.want[:stuck])
    assert ran_out > 0 and drained == 0                     # the stuck row's barrier stays open
    # The refill after the stuck row is the first that is not made.
    assert asked == min(stuck + SLOTS, ROWS)
    # All copies that were asked for have landed: the last of each slot.
    assert sorted(landed) == sorted(range(max(asked - SLOTS, 0), asked))
    assert 0.02 <= took < 5.0
