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


# ---- gates over an fp32 stream
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("act", [serve.GATE_SIGMOID, serve.GATE_SILU])
@pytest.mark.parametrize("wide", [True, False])
@pytest.mark.parametrize("width", [5, 256, 2050])
def test_gates_of_an_fp32_stream_are_as_exact_as_fp32(dtype, act, wide, width):
    """s = act(gate) y in fp32: an exponential (2 steps: 4 u32), a sum, a reciprocal (1 step: 2 u32), two products (SiLU's, y's):
    9 u32, whatever the type of the gate and however far it lies from zero."""
    g = gen(31)
    T = R.DTYPES[dtype]
    y = rnd(g, 300, width, dtype=T) + 1
    gate = torch.linspace(-40, 40, 300 * (width if wide else 1), device="cuda").view(300, -1).to(T)
    s, _ = serve.norm_rows(y, gate=gate, gate_act=act, residual=torch.zeros(300, width, device="cuda"))
    want = R.ACTS[act](gate.to(F64)) * y.to(F64)
    assert s.dtype == torch.float32
    worst = ((s.to(F64) - want).abs() / want.abs().clamp(min=2.0 ** -100)).max()
    assert float(worst) <= 9 * U32, f"{float(worst) / U32} u32"


# ---- adapters that are refused
@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("rows", [7, 4000])
def test_a_refused_scale_empties_its_slots(scale, rows):
    g = gen(32)
    t = R.Tenants(g, 60, 30, torch.float32, slots=4, max_rank=8)
    x = rnd(g, rows, 60)
    of = (torch.arange(rows, device="cuda") % 4).to(torch.int32)
    with pytest.raises(serve.RippleError, match="not finite"):
        t.bank.set(1, torch.stack([t.A[0][:, :3]] * 2), torch.stack([t.B[0][:3]] * 2), [0.5, scale])
    del t.A[1], t.A[2]                  # both slots of the call hold no adapter any more, the others what they held
    t.check(x, of)
    t.A[2], t.B[2], t.scale[2] = t.A[0][:, :3].contiguous(), t.B[0][:3].contiguous(), 2.0
    t.bank.set(2, t.A[2], t.B[2], 2.0)
    t.check(x, of)
