"""The gated delta rule walked in segments, for key sizes that fill the padded width of a segment's matrix and for those that do not: what the workspace or the
kept buffer held before does not matter, to the last bit, and the results are the recurrence's in 64 bits."""
import pytest
import torch

import test_gpu_delta_rule as t
from test_gpu_delta_rule import _announce, la  # noqa: F401

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
CODE = {F32: 0, BF16: 2, F16: 3}
# 25 chunks (of 64 tokens in bf16, else 32): segments of 8 chunks, four of them, two of which the joining pass forms
TOKENS = {BF16: 24 * 64 + 5, F16: 24 * 32 + 5, F32: 24 * 32 + 5}


def entry(lib, w, dtype, o, state, saved=None, workspace=None):
    """la_delta_rule itself, on buffers of the caller's; `w` with one length for all sequences"""
    q, k, v, g, beta = (w[n] for n in t.ARGS)
    b, T, hk, dk = q.shape
    hv, dv = v.shape[2:]
    at = lambda x: (None, 0) if x is None else (x.data_ptr(), x.numel())  # noqa: E731
    rc = lib.la_delta_rule(CODE[dtype], b, T, hk, hv, dk, dv, None, q.data_ptr(), hk * dk, k.data_ptr(), hk * dk, v.data_ptr(), hv * dv, g.data_ptr(),
                           beta.data_ptr(), w["scale"], w["S0"].data_ptr(), o.data_ptr(), state.data_ptr(), *at(saved), *at(workspace),
                           torch.cuda.current_stream().cuda_stream)
    assert rc == 0


def bytes_of(lib, which, w, dtype):
    q, v = w["q"], w["v"]
    b, T, hk, dk = q.shape
    return int(getattr(lib, "la_delta_rule_%s_bytes" % which)(CODE[dtype], b, T, hk, *v.shape[2:3], dk, v.shape[3], 0))


# (the last case walks four column groups a block, the others two)
CASES = [(1, 1, 2, dk, 40) for dk in (1, 8, 24, 32, 33, 64, 65, 72, 96, 97, 128)] + [(2, 1, 1, 90, 100), (1, 12, 48, 24, 16)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("batch,hk,hv,dk,dv", CASES)
def test_segments_on_a_workspace_of_anything(la, dtype, batch, hk, hv, dk, dv):  # noqa: F811
    w = t.make(dtype, batch, TOKENS[dtype], hk, hv, dk, dv, seed=dk + dv, decay=0.02)
    o_ref, S_ref = t.reference(w)
    c, lib = t.cuda(w), la.load()
    for which in ("workspace", "saved"):
        got = []
        for byte in (0, 255):  # zeros, and NaN in every type
            buffer = torch.full((bytes_of(lib, which, c, dtype),), byte, dtype=torch.uint8, device="cuda")
            o, S = torch.empty_like(c["v"]), torch.empty_like(c["S0"])
            entry(lib, c, dtype, o, S, **{which: buffer})
            t.check(("o", "state"), (o, S), (o_ref, S_ref), (dtype, F32))
            got.append((o, S))
        assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("dk", [24, 72, 96])
def test_gradient_of_segments_kept_in_anything(la, dtype, dk):  # noqa: F811
    w = t.make(dtype, 1, TOKENS[dtype], 1, 2, dk, 40, seed=dk, decay=0.02)
    ref = t.reference_bars(w)
    c, lib = t.cuda(w), la.load()
    x, got = [c[n] for n in t.ARGS], []
    for byte in (0, 255):
        saved = torch.full((bytes_of(lib, "saved", c, dtype),), byte, dtype=torch.uint8, device="cuda")
        entry(lib, c, dtype, torch.empty_like(c["v"]), torch.empty_like(c["S0"]), saved=saved)
        work = torch.full((256 << 20,), byte, dtype=torch.uint8, device="cuda")
        bars = la.delta_rule_backward(*x, c["ob"], initial_state=c["S0"], state_bar=c["Sb"], saved=saved, workspace=work)
        t.check(t.ARGS + ("S0",), bars, ref, (dtype,) * 3 + (F32,) * 3)
        work.fill_(byte)
        again = la.delta_rule_backward(*x, c["ob"], initial_state=c["S0"], state_bar=c["Sb"], workspace=work)  # (the forward pass in its workspace)
        assert all(torch.equal(a, b) for a, b in zip(bars, again))
        got.append(bars)
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_packed_segments_on_a_workspace_of_anything(la):  # noqa: F811
    """one sequence of many segments among short ones"""
    ends = [0, 3, 1700, 1701, 3400]
    w = t.make(F16, 4, 0, 1, 2, 72, 40, seed=3, lead=(1, ends[-1]), decay=0.02)
    o_ref, S_ref = t.reference(w, ends)
    c = t.cuda(w)
    at, got = torch.tensor(ends, dtype=torch.int32, device="cuda"), []
    for byte in (0, 255):
        ws = torch.full((256 << 20,), byte, dtype=torch.uint8, device="cuda")
        o, S, _ = la.delta_rule(*[c[n] for n in t.ARGS], initial_state=c["S0"], offsets=at, want_state=True, workspace=ws)
        t.check(("o", "state"), (o, S), (o_ref, S_ref), (F16, F32))
        got.append((o, S))
    assert all(torch.equal(a, b) for a, b in zip(*got))
