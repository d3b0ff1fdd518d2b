"""The gated delta rule where few sequences and heads meet many tokens: the walk in segments, on its own and under the gradient, against the recurrence
in 64 bits."""
import pytest
import torch

import test_gpu_delta_rule as t
from test_gpu_delta_rule import _announce, la  # noqa: F401

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("dtype,T", [(BF16, 1536), (BF16, 1900), (F32, 769), (F16, 1000)])
@pytest.mark.parametrize("batch,hk,hv,dk,dv", [(1, 1, 2, 64, 40), (2, 1, 1, 100, 130)])
def test_long_sequences_of_few_heads(la, dtype, T, batch, hk, hv, dk, dv):  # noqa: F811
    w = t.make(dtype, batch, T, hk, hv, dk, dv, seed=T, decay=0.02)
    o_ref, S_ref = t.reference(w)
    c = t.cuda(w)
    x = [c[n] for n in t.ARGS]
    o, S, _ = la.delta_rule(*x, initial_state=c["S0"], want_state=True)
    t.check(("o", "state"), (o, S), (o_ref, S_ref), (dtype, F32))
    ref = t.reference_bars(w)
    o2, S2, saved = la.delta_rule(*x, initial_state=c["S0"], want_state=True, keep=True)
    assert torch.equal(o, o2) and torch.equal(S, S2)
    bars = la.delta_rule_backward(*x, c["ob"], initial_state=c["S0"], state_bar=c["Sb"], saved=saved)
    t.check(t.ARGS + ("S0",), bars, ref, (dtype,) * 3 + (F32,) * 3)
    again = la.delta_rule_backward(*x, c["ob"], initial_state=c["S0"], state_bar=c["Sb"])
    assert all(torch.equal(a, b) for a, b in zip(bars, again))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("ends", [[0, 5, 5, 2500, 2501, 4700], [0, 3300, 3300], [0, 1700, 4800]])
def test_packed_sequences_of_few_heads(la, dtype, ends):  # noqa: F811
    w = t.make(dtype, len(ends) - 1, 0, 1, 1, 64, 64, seed=len(ends), lead=(1, ends[-1]), decay=0.02)
    o_ref, S_ref = t.reference(w, ends)
    c = t.cuda(w)
    at = torch.tensor(ends, dtype=torch.int32, device="cuda")
    o, S, _ = la.delta_rule(*[c[n] for n in t.ARGS], initial_state=c["S0"], offsets=at, want_state=True)
    t.check(("o", "state"), (o, S), (o_ref, S_ref), (dtype, F32))
    # in place of the initial states, on a workspace full of NaN
    state = c["S0"].clone()
    ws = torch.full((96 << 20,), 255, dtype=torch.uint8, device="cuda")
    o3, _, _ = la.delta_rule(*[c[n] for n in t.ARGS], initial_state=state, offsets=at, workspace=ws)
    assert torch.equal(o, o3)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_final_states_in_place_of_the_initial_ones(la, dtype):  # noqa: F811
    """the first segment is walked from the state that it had, whenever the last one writes"""
    w = t.make(dtype, 3, 2100, 1, 1, 48, 80, seed=8, decay=0.02)
    c = t.cuda(w)
    o, S, _ = la.delta_rule(*[c[n] for n in t.ARGS], initial_state=c["S0"], want_state=True)
    lib, state, again = la.load(), c["S0"].clone(), torch.empty_like(o)
    code = 2 if dtype == BF16 else 0
    size = (code, 3, 2100, 1, 1, 48, 80)
    ws = torch.empty(int(lib.la_delta_rule_workspace_bytes(*size, 0)), dtype=torch.uint8, device="cuda")
    q, k, v, g, beta = (c[n] for n in t.ARGS)
    rc = lib.la_delta_rule(*size, None, q.data_ptr(), 48, k.data_ptr(), 48, v.data_ptr(), 80, g.data_ptr(), beta.data_ptr(), 48 ** -0.5, state.data_ptr(),
                           again.data_ptr(), state.data_ptr(), None, 0, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    assert torch.equal(o, again) and torch.equal(S, state)
