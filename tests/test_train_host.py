"""The calls of training without a device: their argument structures agree with the header, and what they cannot read or write safely
never reaches a kernel."""
import os
import subprocess

import pytest
import torch

from paper_2601_12347_b200 import build as B
from paper_2601_12347_b200 import ripple, train

import test_requests_host as H

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
no_device = H.no_device

LOOKUP = "rows width type out_type device table ld_table table_rows ids out ld_out scale reserved cuda_stream".split()
LOOKUP_GRAD = ("rows width type out_type device dy ld_dy ids out ld_out out_rows scale accumulate workspace workspace_bytes cuda_stream").split()
NORM_GRAD = ("rows width type x_type device dn ld_dn x ld_x x_rows ids add ld_add dx ld_dx dweight dbias norm workspace workspace_bytes "
             "cuda_stream").split()
LOSS = "rows type k n device x ld_x W ld_w bias labels loss lse workspace workspace_bytes cuda_stream".split()
LOSS_GRAD = ("rows type k n device x ld_x W ld_w bias labels lse dloss dx ld_dx dW ld_dw dbias scale reserved workspace workspace_bytes "
             "cuda_stream").split()


@pytest.fixture(scope="module")
def lib():
    B.build_library()
    return ripple.load_library()


def test_argument_structures_match_the_header(tmp_path):
    structs = [("ripple_lookup_rows_args", LOOKUP, train._LOOKUP_ARGS), ("ripple_lookup_rows_grad_args", LOOKUP_GRAD, train._LOOKUP_GRAD_ARGS),
               ("ripple_norm_rows_grad_args", NORM_GRAD, train._NORM_GRAD_ARGS), ("ripple_loss_rows_args", LOSS, train._LOSS_ARGS),
               ("ripple_loss_rows_grad_args", LOSS_GRAD, train._LOSS_GRAD_ARGS)]
    lines = "".join("".join(f'printf("%zu ", offsetof({name}, {f}));' for f in fields) + f'printf("%zu\\n", sizeof({name}));'
                    for name, fields, _ in structs)
    src = tmp_path / "o.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "ripple.h"\nint main(void){' + lines + "return 0;}\n")
    exe = tmp_path / "o"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    for line, (name, fields, packed) in zip(subprocess.check_output([str(exe)]).decode().splitlines(), structs):
        want = [int(x) for x in line.split()]
        if "norm" in fields:         # kind, eps, weight, bias
            at = fields.index("norm")
            want = want[:at] + [want[at] + o for o in (0, 4, 8, 16)] + want[at + 1:]
        assert H._offsets(packed.format) == want[:-1] and packed.size == want[-1], name


def _pack(packed, fields, values, kw):
    v = {**values, **kw}
    flat = []
    for f in fields:
        flat += list(v[f]) if isinstance(v[f], tuple) else [v[f]]
    return packed.pack(*flat)


A = 1 << 24          # made-up addresses, far apart


def lookup_args(**kw):
    M, D = kw.get("rows", 4), kw.get("width", 8)
    return _pack(train._LOOKUP_ARGS, LOOKUP, dict(rows=M, width=D, type=0, out_type=0, device=-1, table=A, ld_table=D, table_rows=9, ids=2 * A, out=3 * A,
                                                  ld_out=D, scale=1.0, reserved=0, cuda_stream=0), kw)


def lookup_grad_args(**kw):
    M, D = kw.get("rows", 300), kw.get("width", 8)
    return _pack(train._LOOKUP_GRAD_ARGS, LOOKUP_GRAD, dict(
        rows=M, width=D, type=0, out_type=0, device=-1, dy=A, ld_dy=D, ids=2 * A, out=3 * A, ld_out=D, out_rows=9, scale=1.0, accumulate=0,
        workspace=4 * A, workspace_bytes=1 << 22, cuda_stream=0), kw)


def norm_grad_args(**kw):
    M, D = kw.get("rows", 40), kw.get("width", 8)
    return _pack(train._NORM_GRAD_ARGS, NORM_GRAD, dict(
        rows=M, width=D, type=0, x_type=0, device=-1, dn=A, ld_dn=D, x=2 * A, ld_x=D, x_rows=M, ids=0, add=0, ld_add=0, dx=3 * A, ld_dx=D,
        dweight=4 * A, dbias=5 * A, norm=(1, 1e-5, 6 * A, 0), workspace=7 * A, workspace_bytes=1 << 22, cuda_stream=0), kw)


def loss_args(**kw):
    M, K, N = kw.get("rows", 4000), kw.get("k", 16), kw.get("n", 8)
    return _pack(train._LOSS_ARGS, LOSS, dict(rows=M, type=0, k=K, n=N, device=-1, x=A, ld_x=K, W=2 * A, ld_w=N, bias=3 * A, labels=4 * A, loss=5 * A,
                                              lse=6 * A, workspace=7 * A, workspace_bytes=1 << 23, cuda_stream=0), kw)


def loss_grad_args(**kw):
    M, K, N = kw.get("rows", 4000), kw.get("k", 16), kw.get("n", 8)
    return _pack(train._LOSS_GRAD_ARGS, LOSS_GRAD, dict(
        rows=M, type=0, k=K, n=N, device=-1, x=A, ld_x=K, W=2 * A, ld_w=N, bias=3 * A, labels=4 * A, lse=5 * A, dloss=6 * A, dx=7 * A, ld_dx=K,
        dW=8 * A, ld_dw=N, dbias=9 * A, scale=1.0, reserved=0, workspace=10 * A, workspace_bytes=1 << 23, cuda_stream=0), kw)


def refused(lib, call, packed):
    assert getattr(lib, "ripple_" + call)(packed) == ripple.ERR_INVALID_ARG
    assert lib.ripple_last_error(None).startswith(call.encode() + b":")


@no_device
@pytest.mark.parametrize("wrong", [
    dict(rows=-1), dict(rows=1 << 31), dict(width=0), dict(width=16385), dict(type=3), dict(type=-1), dict(type=1), dict(out_type=3),
    dict(type=1, out_type=2), dict(type=1, out_type=0), dict(table_rows=-1), dict(table=0), dict(ids=0), dict(out=0), dict(ld_table=-1),
    dict(ld_out=7), dict(table=A + 2), dict(ids=2 * A + 1), dict(out=3 * A + 2), dict(out=A), dict(out=A + 32), dict(out=2 * A), dict(ids=3 * A + 4),
], ids=str)
def test_lookup_rows_refuses(lib, wrong):
    refused(lib, "lookup_rows", lookup_args(**wrong))


@no_device
@pytest.mark.parametrize("wrong", [
    dict(rows=-1), dict(rows=1 << 31), dict(width=0), dict(width=16385), dict(type=3), dict(out_type=1), dict(type=1, out_type=2), dict(out_rows=-1),
    dict(rows=(1 << 31) - 1), dict(out_rows=(1 << 31) - 1), dict(accumulate=2), dict(accumulate=-1), dict(dy=0), dict(ids=0), dict(out=0), dict(ld_dy=-1), dict(ld_out=7),
    dict(dy=A + 1), dict(ids=2 * A + 2), dict(out=3 * A + 2), dict(workspace=0), dict(workspace_bytes=64), dict(workspace=4 * A + 64), dict(out=A),
    dict(out=2 * A + 4), dict(out=4 * A), dict(workspace=A), dict(workspace=2 * A - 128),
], ids=str)
def test_lookup_rows_grad_refuses(lib, wrong):
    refused(lib, "lookup_rows_grad", lookup_grad_args(**wrong))


@no_device
@pytest.mark.parametrize("wrong", [
    dict(rows=-1), dict(rows=1 << 31), dict(width=0), dict(width=16385), dict(type=3), dict(x_type=1), dict(type=1, x_type=2), dict(norm=(0, 1e-5, 0, 0)),
    dict(norm=(3, 1e-5, 0, 0)), dict(norm=(1, -1.0, 0, 0)), dict(norm=(1, float("nan"), 0, 0)), dict(norm=(1, 1e-5, 2, 0)), dict(dx=0, dweight=0, dbias=0),
    dict(add=8 * A, ld_add=8, dx=0), dict(x_rows=3), dict(x_rows=-1, ids=8 * A), dict(dn=0), dict(x=0), dict(ld_dn=-1), dict(ld_x=-1), dict(ld_add=-1),
    dict(ld_dx=7), dict(dn=A + 2), dict(x=2 * A + 1), dict(dx=3 * A + 2), dict(dweight=4 * A + 2), dict(ids=8 * A + 1), dict(workspace=0),
    dict(workspace_bytes=4), dict(workspace=7 * A + 4), dict(dx=A + 4), dict(dx=A, ld_dx=16), dict(dx=2 * A, ids=8 * A), dict(dx=6 * A), dict(dweight=A),
    dict(dweight=5 * A), dict(dbias=3 * A + 8), dict(dbias=6 * A), dict(workspace=A), dict(workspace=4 * A), dict(ids=3 * A), dict(dx=A, type=1, x_type=0),
], ids=str)
def test_norm_rows_grad_refuses(lib, wrong):
    refused(lib, "norm_rows_grad", norm_grad_args(**wrong))


@no_device
@pytest.mark.parametrize("wrong", [
    dict(rows=-1), dict(rows=(1 << 31) - 1), dict(type=3), dict(k=0), dict(k=8193), dict(n=0), dict(n=(1 << 24) + 1), dict(ld_x=-1), dict(ld_w=-1),
    dict(x=0), dict(W=0), dict(labels=0), dict(lse=0), dict(x=A + 2), dict(W=2 * A + 1), dict(bias=3 * A + 2), dict(labels=4 * A + 1), dict(lse=6 * A + 2),
    dict(workspace=0), dict(workspace_bytes=128), dict(workspace=7 * A + 64), dict(lse=A), dict(lse=5 * A + 4), dict(loss=2 * A + 4), dict(loss=4 * A),
    dict(loss=3 * A), dict(workspace=A), dict(workspace=2 * A), dict(workspace=5 * A), dict(lse=7 * A),
], ids=str)
def test_loss_rows_refuses(lib, wrong):
    refused(lib, "loss_rows", loss_args(**wrong))


@no_device
@pytest.mark.parametrize("wrong", [
    dict(rows=-1), dict(rows=(1 << 31) - 1), dict(type=3), dict(k=0), dict(k=8193), dict(n=0), dict(n=(1 << 24) + 1), dict(ld_x=-1), dict(ld_w=-1),
    dict(ld_dx=15), dict(ld_dw=7), dict(dx=0, dW=0, dbias=0), dict(x=0), dict(W=0), dict(labels=0), dict(lse=0), dict(x=A + 2), dict(dx=7 * A + 2),
    dict(dW=8 * A + 1), dict(dbias=9 * A + 2), dict(dloss=6 * A + 1), dict(lse=5 * A + 1), dict(workspace=0), dict(workspace_bytes=128),
    dict(workspace=10 * A + 64), dict(dx=A), dict(dx=8 * A), dict(dW=2 * A + 64), dict(dW=9 * A), dict(dbias=3 * A + 4), dict(dbias=5 * A), dict(dx=6 * A),
    dict(workspace=A), dict(workspace=7 * A), dict(workspace=8 * A), dict(dx=4 * A),
], ids=str)
def test_loss_rows_grad_refuses(lib, wrong):
    refused(lib, "loss_rows_grad", loss_grad_args(**wrong))


def test_nothing_to_do_is_fine(lib):
    assert lib.ripple_lookup_rows(lookup_args(rows=0)) == ripple.OK
    assert lib.ripple_lookup_rows_grad(lookup_grad_args(out_rows=0, out=0)) == ripple.OK
    assert lib.ripple_loss_rows(loss_args(rows=0)) == ripple.OK
    for call in ("lookup_rows", "lookup_rows_grad", "norm_rows_grad", "loss_rows", "loss_rows_grad"):
        assert getattr(lib, "ripple_" + call)(None) == ripple.ERR_INVALID_ARG


def test_workspaces_of_sizes_out_of_range(lib):
    for call, args in (("lookup_rows_grad", lookup_grad_args(width=0)), ("norm_rows_grad", norm_grad_args(rows=-1)), ("loss_rows", loss_args(k=9000)),
                       ("loss_rows_grad", loss_grad_args(type=5)), ("lookup_rows_grad", None), ("norm_rows_grad", None), ("loss_rows", None),
                       ("loss_rows_grad", None)):
        assert getattr(lib, f"ripple_{call}_workspace_bytes")(args) == -1


def test_workspaces_stay_below_the_logits(lib):
    """What a call of many rows and classes keeps is a piece of them."""
    rows, k, n = 65_536, 512, 500_000
    for call, args in (("loss_rows", loss_args(rows=rows, k=k, n=n, type=1)), ("loss_rows_grad", loss_grad_args(rows=rows, k=k, n=n, type=1))):
        got = getattr(lib, f"ripple_{call}_workspace_bytes")(args)
        assert 0 < got < rows * n * 2 / 20


def test_what_is_no_cuda_tensor_is_refused():
    x, ids, v = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    for call in (lambda: train.lookup_rows(x, ids), lambda: train.lookup_rows_grad(x, ids, 3), lambda: train.loss_rows(x, x.T, ids),
                 lambda: train.loss_rows_grad(x, x.T, ids, v)):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
    with pytest.raises(TypeError):
        train.norm_rows_grad(x, x, None)
    with pytest.raises(TypeError):
        train.lookup_rows(None, ids)


def test_rules_of_the_device_code():
    """As for the kernels of requests: lanes of a warp give up together, and what the kernel before may write is read by ordinary loads."""
    import re

    import test_device_rules as D
    D.test_lanes_of_a_warp_give_up_together("row_loss.cu")
    for name in ("row_loss.cu", "row_lookup.cu", "row_norms_grad.cu", "row_vectors.cuh"):
        text = open(os.path.join(D.CSRC, name)).read()
        assert not re.search(r"__restrict__|ld\.global\.nc|__ldg", text), name
        # every kernel waits for the one before it
        for m in re.finditer(r"\b__global__\b[^;{]*\{(.{0,4000}?)\n\}", text, flags=re.S):
            assert "pdl_enter();" in m.group(1) or len(m.group(1)) >= 3990, text[m.start():m.start() + 200]
