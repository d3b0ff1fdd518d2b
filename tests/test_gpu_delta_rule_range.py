"""The gated delta rule where a token takes as much out of the state as the recurrence allows without growing: beta |k|^2 up to 2, keys of any length, states that hardly
decay, keys that are nearly the same."""
import pytest
import torch

import layer_formulas as f
import test_gpu_delta_rule as t
from test_gpu_delta_rule import _announce, la  # noqa: F401

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
NAMES = t.ARGS + ("S0",)


def inputs(dtype, T, dk, kind):
    w = t.make(dtype, 1, T, 1, 2, dk, 40, seed=dk + T, decay=0.002)
    r = torch.Generator().manual_seed(T)
    if kind == "reflections":  # unit keys, beta of 2: every token turns the state over along its key
        w["beta"].fill_(2.0)
    elif kind == "long keys":  # |k| of 4, beta |k|^2 between 0 and 2
        w["k"] = (4.0 * w["k"].float()).to(dtype)
        w["beta"] = 2.0 / 16.0 * torch.rand(w["beta"].shape, generator=r)
    elif kind == "short keys":  # |k| of 1/8, beta |k|^2 up to 2
        w["k"] = (0.125 * w["k"].float()).to(dtype)
        w["beta"] = 2.0 * 64.0 * torch.rand(w["beta"].shape, generator=r)
    else:  # "one key": all within a tenth of one direction, beta up to 2
        k = torch.randn(dk, generator=r) + 0.1 * w["k"].float() * dk ** 0.5
        w["k"] = (k / k.norm(dim=-1, keepdim=True)).to(dtype)
        w["beta"] = 2.0 * torch.rand(w["beta"].shape, generator=r)
    # (16-bit keys are rounded: what is taken out stays within 2)
    w["beta"] = torch.minimum(w["beta"], 2.0 / w["k"].double().square().sum(-1).repeat_interleave(2, -1).float() * (1 - 2e-7))
    return w


def tolerance(w, dtype, chunk):
    """What the chunked form may add to f.tolerance.  Its T = (I + A)^-1 is formed in 32 bits: relative to U = T Z an error of up to cond(I + A) 2^-24, in every chunk, and the
    state, which does not shrink, hands it on; the gradient has a second product with T beside the first."""
    T, cond = w["k"].shape[1], 1.0
    for a in range(0, T, chunk):
        z = slice(a, min(a + chunk, T))
        k = w["k"][0, z, 0].double()
        for h in range(2):
            b = w["g"][0, z, h].double().cumsum(0)
            A = (w["beta"][0, z, h].double()[:, None] * torch.exp(b[:, None] - b) * (k @ k.T)).tril(-1)
            cond = max(cond, float(torch.linalg.cond(torch.eye(len(k), dtype=torch.float64) + A)))
    return f.tolerance(dtype) + 2 * -(-T // chunk) * cond * 2.0 ** -24


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("kind", ["reflections", "long keys", "short keys", "one key"])
@pytest.mark.parametrize("T,dk", [(70, 8), (150, 64), (200, 128)])
def test_up_to_what_does_not_grow(la, dtype, kind, T, dk):  # noqa: F811
    w = inputs(dtype, T, dk, kind)
    chunk = 64 if dtype == BF16 else 32
    extra = tolerance(w, dtype, chunk) - f.tolerance(dtype)
    assert extra < 0.01  # (the bound says something)
    o_ref, S_ref = t.reference(w)
    ref = t.reference_bars(w)
    c = t.cuda(w)
    x = [c[n] for n in t.ARGS]
    o, S, _ = la.delta_rule(*x, initial_state=c["S0"], want_state=True)
    bars = la.delta_rule_backward(*x, c["ob"], initial_state=c["S0"], state_bar=c["Sb"])
    worst = {}
    for n, a, b in zip(("o", "state") + NAMES, (o, S, *bars), (o_ref, S_ref, *ref)):
        off, tol = f.rel(a, b), f.tolerance(a.dtype) + extra
        worst[n] = (off, tol)
    assert all(off <= tol for off, tol in worst.values()), worst
