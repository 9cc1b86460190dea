"""What the calls of requests promise that needs no device to be seen."""
import copy
import pickle

import pytest

from paper_2601_12347_b200 import ripple, serve

import test_requests_host as H

lib = H.lib


@H.no_device
@pytest.mark.parametrize("clear", [-1, 2, 1 << 20])
def test_unknown_treatments_of_padding_rows_are_refused(lib, clear):
    assert lib.ripple_norm_rows(H._norm_args(reserved=clear)) == ripple.ERR_INVALID_ARG
    assert b"clear_padding" in lib.ripple_last_error(None)


@H.no_device
@pytest.mark.parametrize("x", [0, 1 << 24])
@pytest.mark.parametrize("adapters", [True, False])
def test_a_table_without_rows_has_no_address(lib, x, adapters):
    """Every id lies outside: the call is fine and launches nothing, whatever the address of nothing is."""
    kw = {} if adapters else dict(bank=0, slots=0)
    assert lib.ripple_project_rows(H._project_args(x=x, x_rows=0, ids=8 << 24, **kw)) == ripple.OK
    assert lib.ripple_project_rows(H._project_args(x=x, x_rows=0, **kw)) == ripple.ERR_INVALID_ARG      # rows without ids
    assert lib.ripple_project_rows(H._project_args(x=0, x_rows=4, ids=8 << 24, **kw)) == ripple.ERR_INVALID_ARG


def test_operators_are_not_copied_with_the_addresses_of_another():
    """Their arguments are packed once, addresses included: a deep copy read the first one's memory, kept or not."""
    n = serve.Norm(serve.NORM_RMS, eps=1e-3)
    for make in (copy.deepcopy, pickle.dumps, lambda x: copy.deepcopy([x])):
        with pytest.raises(TypeError, match="device memory"):
            make(n)
    m = copy.copy(n)                   # shares the memory, and keeps it
    assert type(m) is serve.Norm and m.eps == 1e-3 and m._args is n._args
