"""The delta rule's entries refuse what needs more threads than a launch takes (fewer than 2^32), and nothing below that, on the host.  Made-up addresses: these run
only where nothing can be launched, and a call that gets as far as its launch ends there as LA_ERR_RUNTIME."""
import pytest
import torch

import paper_1710_08717_amd as la

F32, BF16, F16 = 0, 2, 3
UNSUPPORTED, RUNTIME = 2, 3


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.device_count() > 0:
        pytest.skip("made-up addresses: only where nothing can be launched")
    return la.load()


def at(i):
    return (1 << 50) + (i << 42)


@pytest.mark.parametrize("batch,hv,dv,refused", [((1 << 24) - 1, 1, 32, False), (1 << 24, 1, 1, True), (1 << 19, 1, 1024, True), ((1 << 19) - 1, 1, 1024, False),
                                                 (1 << 20, 16, 3, True), ((1 << 20) - 1, 16, 32, False)])
def test_step(lib, batch, hv, dv, refused):
    """256 threads for 32 columns of a state"""
    got = lib.la_delta_rule_step(F32, batch, 1, hv, 1, dv, at(1), 1, at(2), 1, at(3), hv * dv, at(4), at(5), 1.0, at(6), batch, None, at(7), None)
    assert got == (UNSUPPORTED if refused else RUNTIME)


@pytest.mark.parametrize("dt,dk", [(F16, 1), (F32, 1), (BF16, 1), (BF16, 128)])
@pytest.mark.parametrize("batch,refused", [((1 << 19) - 1, False), (1 << 19, True)])
def test_walks(lib, dt, dk, batch, refused):
    """8192 threads for the 1024 columns of a sequence"""
    size = (dt, batch, 1, 1, 1, dk, 1024)
    operands = (at(1), dk, at(2), dk, at(3), 1024, at(4), at(5), 1.0, None)
    want = UNSUPPORTED if refused else RUNTIME
    need = lib.la_delta_rule_workspace_bytes(*size, 0)
    assert lib.la_delta_rule(*size, None, *operands, at(6), None, None, 0, at(7), need, None) == want
    kept = lib.la_delta_rule_saved_bytes(*size, 0)
    assert lib.la_delta_rule(*size, None, *operands, at(6), None, at(7), kept, None, 0, None) == want
    need = lib.la_delta_rule_backward_workspace_bytes(*size, 0, 1)
    assert lib.la_delta_rule_backward(*size, None, *operands, at(6), None, at(7), kept, *[at(i) for i in range(8, 13)], None, at(14), need, None) == want
