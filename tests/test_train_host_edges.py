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


def kernels_of(text):
    """(name, body) of every kernel of a source, whatever its length."""
    import re
    for m in re.finditer(r"\b__global__\b", text):
        name = re.compile(r"\b(k_\w+)\s*\(").search(text, m.end())
        at = text.index("{", text.index(")", name.end()))
        depth, end = 1, at + 1
        while depth:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
        yield name.group(1), text[at + 1:end - 1]


@pytest.mark.parametrize("name", ["row_lookup.cu", "row_norms_grad.cu", "row_loss.cu", "row_norms.cu"])
def test_every_kernel_waits_for_the_one_before(name):
    """Launches may overlap with the kernel before: nothing is read before pdl_enter, the first statement.  Products of the losses set up barriers and tensor memory
    first, and read nothing of the caller's until then."""
    import re

    import test_device_rules as D
    text = D.source(name)
    found = dict(kernels_of(text))
    assert len(found) == len(re.findall(r"\b__global__\b", text)) > 0
    for kernel, body in found.items():
        if kernel != "k_product":
            assert re.match(r"\s*pdl_enter\(\);", body), kernel
            continue
        outer = [m.start() for m in re.finditer(r"\bpdl_enter\(\);", body) if body[:m.start()].count("{") == body[:m.start()].count("}")]
        assert len(outer) == 1
        inner = re.search(r"if \(p\.by_row\) \{\s*pdl_enter\(\);\s*if \(!p\.control->differ\) return;\s*\}", body)
        before = body[:inner.start()] + body[inner.end():outer[0]]
        assert not re.search(r"\bp\.(control|raw|raw_labels|bias|labels|sums|at_label|lse|dloss|g|g_sums|out|dead_rows|a|a_clean|b)\b", before)
