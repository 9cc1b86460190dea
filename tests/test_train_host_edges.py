"""The calls of training without a device, beside what test_train_host.py asks of them."""
import os
import subprocess

import pytest

from paper_2601_12347_b200 import ripple, train

import test_requests_host as H
import test_train_host as T

no_device, lib = H.no_device, T.lib
A = T.A

LIVE = "rows classes device ids table_rows labels live_ids live_rows live_labels cuda_stream".split()


def live_args(**kw):
    return T._pack(train._LIVE_ARGS, LIVE, dict(rows=40, classes=7, device=-1, ids=A, table_rows=9, labels=2 * A, live_ids=3 * A, live_rows=4 * A, live_labels=5 * A,
                                                cuda_stream=0), kw)


def test_arguments_of_live_rows_match_the_header(tmp_path):
    src, exe = tmp_path / "o.c", tmp_path / "o"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "ripple.h"\nint main(void){'
                   + "".join(f'printf("%zu ", offsetof(ripple_live_rows_args, {f}));' for f in LIVE) + 'printf("%zu", sizeof(ripple_live_rows_args));return 0;}\n')
    subprocess.check_call(["gcc", "-I", os.path.join(T.ROOT, "include"), str(src), "-o", str(exe)])
    want = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert H._offsets(train._LIVE_ARGS.format) == want[:-1] and train._LIVE_ARGS.size == want[-1]


@no_device
@pytest.mark.parametrize("wrong", [
    dict(rows=-1), dict(rows=1 << 31), dict(table_rows=-1), dict(classes=0), dict(classes=(1 << 24) + 1), dict(ids=0), dict(labels=0), dict(ids=A + 1),
    dict(live_rows=4 * A + 2), dict(live_ids=0, live_rows=0, live_labels=0), dict(live_ids=A), dict(live_rows=2 * A + 4), dict(live_labels=3 * A), dict(live_rows=3 * A + 156),
], ids=str)
def test_live_rows_refuses(lib, wrong):
    T.refused(lib, "live_rows", live_args(**wrong))


def test_no_rows_are_fine(lib):
    assert lib.ripple_live_rows(live_args(rows=0, ids=0, labels=0)) == ripple.OK
    assert lib.ripple_live_rows(None) == ripple.ERR_INVALID_ARG
