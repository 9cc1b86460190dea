"""What the operators of requests promise beyond their formulas."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2601_12347_b200 import inputs as I
from paper_2601_12347_b200 import ripple, serve

import test_gpu_parity as P
import test_gpu_requests as R

pytestmark = pytest.mark.gpu
env = P.env     # skips without a device, builds the library

U32, F64 = R.U32, R.F64
rnd, gen, runs, near = R.rnd, R.gen, R.runs, R.near


@pytest.fixture(autouse=True)
def _device(env):
    pass


# ---- waits that run out
@pytest.mark.parametrize("dtype,K,N,rows,run", [
    ("bf16", 200, 300, 20_000, 500),        # tiles of 256 columns
    ("fp16", 200, 264, 5003, 16),           # of 128
    ("bf16", 130, 60, 2800, 16),            # of 32, x A row by row
    ("fp32", 200, 264, 5003, 16),           # parts, one unit of K
    ("fp32", 520, 264, 5003, 16),           # several
    ("fp32", 256, 47, 12_000, 300),         # x W and x A in one pass
])
def test_a_wait_that_gives_up_is_reported(monkeypatch, dtype, K, N, rows, run):
    """The diagnostic switch withholds what the epilogues wait for: the call returns, the roles of its kernels leave one after the
    other, the status says so once, and the next call is right."""
    g = gen(30)
    t = R.Tenants(g, K, N, R.DTYPES[dtype], slots=9, max_rank=20)
    x, of = rnd(g, rows, K, dtype=R.DTYPES[dtype]), runs(g, rows, run, 9)
    serve.check_requests()
    monkeypatch.setenv("RIPPLE_DEBUG_TC_WITHHOLD", "1")
    for slots in (None, of):
        serve.project_rows(x, t.proj, t.bank if slots is not None else None, slots)
        with pytest.raises(serve.RippleError, match="gave up") as e:
            serve.check_requests()
        assert e.value.status == ripple.ERR_TIMEOUT
        serve.check_requests()
    monkeypatch.delenv("RIPPLE_DEBUG_TC_WITHHOLD")
    t.check(x, of)
    serve.check_requests()
