"""The calls of requests without a device: their argument structures agree with the header, and what they cannot read or write
safely never reaches a kernel."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2601_12347_b200 import build as B
from paper_2601_12347_b200 import ripple, serve

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# (made-up addresses: on a machine with a device a call that is wrongly accepted would use them)
no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses")

NORM = ("rows width type stream_type gate_act y ld_y gate ld_gate residual ld_residual residual_rows ids scale_vector stream ld_stream "
        "normed ld_normed post pre scale gate_width device reserved cuda_stream").split()
PROJECT = ("rows type out_type k n act n_slots max_rank device x ld_x x_rows ids layout bias bank slots y ld_y workspace "
           "workspace_bytes cuda_stream").split()


@pytest.fixture(scope="module")
def lib():
    B.build_library()
    return ripple.load_library()


def _offsets(fmt):
    """Where struct.pack puts each field of a format."""
    import struct
    at, fields = [], []
    for part in fmt.replace("=", "").replace(" ", ""):
        if part.isdigit():
            fields.append(part)
            continue
        n = int(fields.pop()) if fields else 1
        for _ in range(n):
            at.append((part, sum(struct.calcsize("=" + p) for p, _ in at)))
    return [a for _, a in at]


def test_argument_structures_match_the_header(tmp_path):
    def show(struct_name, fields):
        return "".join(f'printf("%zu ", offsetof({struct_name}, {f}));' for f in fields) + f'printf("%zu\\n", sizeof({struct_name}));'
    src = tmp_path / "o.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "ripple.h"\nint main(void){' + show("ripple_norm_rows_args", NORM)
                   + show("ripple_project_rows_args", PROJECT) + show("ripple_norm", ["kind", "eps", "weight", "bias"]) + "return 0;}\n")
    exe = tmp_path / "o"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    norm, project, one = ([int(x) for x in line.split()] for line in subprocess.check_output([str(exe)]).decode().splitlines())
    got = _offsets(serve._NORM_ARGS.format)
    post = norm[NORM.index("post")]
    assert one == [0, 4, 8, 16, 24]
    want = norm[:NORM.index("post")] + [post + o for o in one[:-1]] + [post + 24 + o for o in one[:-1]] + norm[NORM.index("scale"):-1]
    assert got == want and serve._NORM_ARGS.size == norm[-1]
    assert _offsets(serve._PROJECT_ARGS.format) == project[:-1] and serve._PROJECT_ARGS.size == project[-1]


def _norm_args(**kw):
    M, D = kw.get("rows", 4), kw.get("width", 8)
    v = dict(rows=M, width=D, type=0, stream_type=0, gate_act=0, y=1 << 20, ld_y=D, gate=0, ld_gate=0, residual=2 << 20, ld_residual=D,
             residual_rows=M, ids=0, scale_vector=0, stream=3 << 20, ld_stream=D, normed=4 << 20, ld_normed=D, post=(0, 0.0, 0, 0),
             pre=(2, 1e-5, 0, 0), scale=1.0, gate_width=1, device=-1, reserved=0, cuda_stream=0)
    v.update(kw)
    flat = []
    for f in NORM:
        flat += list(v[f]) if isinstance(v[f], tuple) else [v[f]]
    return serve._NORM_ARGS.pack(*flat)


@no_device
@pytest.mark.parametrize("wrong", [
    dict(rows=-1), dict(rows=1 << 31), dict(width=0), dict(width=16385), dict(type=3), dict(type=-1), dict(stream_type=1), dict(stream_type=7),
    dict(type=1, stream_type=2), dict(gate_act=4), dict(gate_act=-1), dict(post=(3, 0.0, 0, 0)), dict(pre=(-1, 0.0, 0, 0)),
    dict(pre=(1, -1.0, 0, 0)), dict(pre=(1, float("nan"), 0, 0)), dict(pre=(1, 0.0, 2, 0)), dict(y=0, residual=0),
    dict(y=0, gate=5 << 20), dict(y=0, post=(1, 0.0, 0, 0)), dict(gate=5 << 20, gate_width=4), dict(gate=5 << 20, gate_width=0),
    dict(ids=6 << 20, residual=0), dict(residual_rows=3), dict(residual_rows=-1, ids=6 << 20), dict(stream=0, normed=0), dict(normed=0),
    dict(pre=(0, 0.0, 0, 0)), dict(ld_y=-1), dict(ld_gate=-1), dict(ld_residual=-8), dict(ld_stream=7), dict(ld_normed=7),
    dict(y=(1 << 20) + 2), dict(stream=(3 << 20) + 1), dict(ids=(6 << 20) + 2), dict(scale_vector=(6 << 20) + 1),
    # overlaps
    dict(stream=4 << 20), dict(stream=(4 << 20) + 32), dict(stream=(1 << 20) + 4), dict(stream=(1 << 20) + 32), dict(normed=(2 << 20) + 64),
    dict(stream=1 << 20, ld_stream=16), dict(stream=2 << 20, ids=6 << 20), dict(ids=3 << 20), dict(scale_vector=(4 << 20) + 16),
    dict(pre=(2, 0.0, 3 << 20, 0)), dict(post=(1, 0.0, 0, (4 << 20) + 4)), dict(y=1 << 20, ld_y=0, stream=1 << 20),
    dict(stream=1 << 20, type=1, stream_type=0, normed=9 << 20), dict(gate=3 << 20, gate_width=1, ld_gate=1),
    dict(ld_y=16, stream=(1 << 20) + 28, ld_stream=16), dict(residual=1 << 20, stream=1 << 20, ids=6 << 20),
], ids=str)
def test_norm_rows_refuses(lib, wrong):
    assert lib.ripple_norm_rows(_norm_args(**wrong)) == ripple.ERR_INVALID_ARG
    assert lib.ripple_last_error(None).startswith(b"norm_rows")


def test_nothing_to_do_is_fine(lib):
    assert lib.ripple_norm_rows(_norm_args(rows=0)) == ripple.OK
    assert lib.ripple_project_rows(_project_args(rows=0)) == ripple.OK
    assert lib.ripple_norm_rows(None) == ripple.ERR_INVALID_ARG
    assert lib.ripple_project_rows(None) == ripple.ERR_INVALID_ARG


def _project_args(**kw):
    M, K, N = kw.get("rows", 4), kw.get("k", 16), kw.get("n", 8)
    v = dict(rows=M, type=0, out_type=0, k=K, n=N, act=0, n_slots=2, max_rank=8, device=-1, x=1 << 24, ld_x=K, x_rows=M, ids=0, layout=2 << 24,
             bias=3 << 24, bank=4 << 24, slots=5 << 24, y=6 << 24, ld_y=N, workspace=7 << 24, workspace_bytes=1 << 24, cuda_stream=0)
    v.update(kw)
    return serve._PROJECT_ARGS.pack(*(v[f] for f in PROJECT))


@no_device
@pytest.mark.parametrize("wrong", [
    dict(rows=-1), dict(rows=1 << 31), dict(type=3), dict(out_type=1), dict(type=1, out_type=2), dict(k=0), dict(k=8193), dict(n=0), dict(n=65537),
    dict(act=2), dict(act=-1), dict(n_slots=0), dict(n_slots=4097), dict(max_rank=0), dict(max_rank=65), dict(x=0), dict(layout=0), dict(y=0),
    dict(x=(1 << 24) + 2), dict(y=(6 << 24) + 2), dict(layout=(2 << 24) + 64), dict(bank=(4 << 24) + 16), dict(bias=(3 << 24) + 1),
    dict(ids=(8 << 24) + 1), dict(slots=(5 << 24) + 2), dict(ld_x=-1), dict(ld_y=7), dict(x_rows=3), dict(x_rows=-1, ids=8 << 24),
    dict(bank=0), dict(slots=0), dict(workspace=0), dict(workspace_bytes=16), dict(workspace=(7 << 24) + 64),
    dict(y=1 << 24), dict(y=(1 << 24) + 128), dict(y=2 << 24), dict(y=(3 << 24) + 4), dict(y=4 << 24), dict(y=5 << 24), dict(y=7 << 24),
    dict(ids=6 << 24), dict(workspace=1 << 24), dict(workspace=4 << 24), dict(workspace=5 << 24),
], ids=str)
def test_project_rows_refuses(lib, wrong):
    assert lib.ripple_project_rows(_project_args(**wrong)) == ripple.ERR_INVALID_ARG
    assert lib.ripple_last_error(None).startswith(b"project_rows")


@no_device
def test_layouts_and_banks_refuse(lib):
    assert lib.ripple_project_layout_bytes(0, 100, 47) == 2 * 3 * 16384 + 18816      # chunks in three parts, and W to 128 bytes
    assert lib.ripple_project_layout_bytes(1, 64, 129) == 2 * 16384 + 16512
    for bad in ((3, 8, 8), (0, 0, 8), (0, 8193, 8), (0, 8, 0), (0, 8, 65537)):
        assert lib.ripple_project_layout_bytes(*bad) == -1
        assert lib.ripple_adapter_bytes(*bad, 4, 8) == -1
        assert lib.ripple_project_layout(*bad, 1 << 20, 1 << 17, 1 << 24, -1, None) == ripple.ERR_INVALID_ARG
    for slots, rank in ((0, 8), (4097, 8), (4, 0), (4, 65)):
        assert lib.ripple_adapter_bytes(0, 8, 8, slots, rank) == -1
    for W, ld, out in ((0, 8, 1 << 20), (1 << 20, 8, 0), (1 << 20, 7, 2 << 20), ((1 << 20) + 2, 8, 2 << 20), (1 << 20, 8, (2 << 20) + 64)):
        assert lib.ripple_project_layout(0, 8, 8, W, ld, out, -1, None) == ripple.ERR_INVALID_ARG
    one = (ctypes.c_float * 2)(1.0, 1.0)
    bad_scale = (ctypes.c_float * 2)(1.0, float("inf"))
    for bank, first, count, rank, A, B_, scale in (
            (0, 0, 1, 4, 1 << 20, 2 << 20, one), ((3 << 20) + 4, 0, 1, 4, 1 << 20, 2 << 20, one), (3 << 20, -1, 1, 4, 1 << 20, 2 << 20, one),
            (3 << 20, 3, 2, 4, 1 << 20, 2 << 20, one), (3 << 20, 0, 5, 4, 1 << 20, 2 << 20, one), (3 << 20, 0, -1, 4, 1 << 20, 2 << 20, one),
            (3 << 20, 0, 1, 9, 1 << 20, 2 << 20, one), (3 << 20, 0, 1, -1, 1 << 20, 2 << 20, one), (3 << 20, 0, 1, 4, 0, 2 << 20, one),
            (3 << 20, 0, 1, 4, 1 << 20, 0, one), (3 << 20, 0, 1, 4, 1 << 20, 2 << 20, None), (3 << 20, 0, 2, 4, 1 << 20, 2 << 20, bad_scale),
            (3 << 20, 0, 1, 4, (1 << 20) + 2, 2 << 20, one)):
        assert lib.ripple_adapter_set(bank, 0, 8, 8, 4, 8, first, count, rank, A, B_, scale, -1, None) == ripple.ERR_INVALID_ARG


def test_host_tensors_are_refused():
    x = torch.zeros(2, 4)
    with pytest.raises(ValueError, match="CUDA tensor"):
        serve.norm_rows(x)
    with pytest.raises(ValueError, match="neither"):
        serve.norm_rows()
    with pytest.raises(TypeError, match="CUDA tensor"):
        serve.norm_rows([1.0])
    with pytest.raises(ValueError):
        serve.Norm(serve.NORM_NONE)
    with pytest.raises(ValueError):
        serve.Norm(serve.NORM_RMS, eps=-1.0)
