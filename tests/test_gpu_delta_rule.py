"""The gated delta rule on the GPU against the recurrence in 64 bits: whole sequences, packed ones, the gradient, single tokens, and what is refused."""
import sys

import pytest
import torch

import layer_formulas as f

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def la():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1710_08717_amd as la_mod

    la_mod.load()
    return la_mod


@pytest.fixture(autouse=True)
def _announce(request):
    sys.stderr.write(f"\n[gpu-case] {request.node.nodeid}\n")
    sys.stderr.flush()
    yield


def make(dtype, batch, T, hk, hv, dk, dv, seed, decay=0.3, lead=None):
    """Inputs on the CPU in the operator's types: unit keys, decays of many sizes, beta in (0, 1)."""
    r = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=r)  # noqa: E731
    lead = (batch, T) if lead is None else lead
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    return {"q": unit(n(*lead, hk, dk)).to(dtype), "k": unit(n(*lead, hk, dk)).to(dtype), "v": n(*lead, hv, dv).to(dtype),
            "g": -decay * n(*lead, hv).abs(), "beta": torch.sigmoid(n(*lead, hv)), "S0": 0.3 * n(batch, hv, dk, dv),
            "ob": n(*lead, hv, dv).to(dtype), "Sb": 0.3 * n(batch, hv, dk, dv), "scale": dk ** -0.5}


ARGS = ("q", "k", "v", "g", "beta")


def reference(w, ends=None):
    """(o, final states) of every sequence; `ends` for packed ones."""
    if ends is None:
        parts = [f.delta_rule(*[w[n][b].double() for n in ARGS], w["scale"], w["S0"][b].double()) for b in range(w["q"].shape[0])]
        return torch.stack([p[0] for p in parts]), torch.stack([p[1] for p in parts])
    o = torch.zeros_like(w["v"], dtype=torch.float64)
    S = []
    for b, (a, z) in enumerate(zip(ends[:-1], ends[1:])):
        x, s = f.delta_rule(*[w[n][0, a:z].double() for n in ARGS], w["scale"], w["S0"][b].double())
        o[0, a:z] = x
        S.append(s)
    return o, torch.stack(S)


def reference_bars(w, ends=None):
    pieces = [(b, slice(None), b) for b in range(w["q"].shape[0])] if ends is None else \
        [(0, slice(a, z), n) for n, (a, z) in enumerate(zip(ends[:-1], ends[1:]))]
    out = [torch.zeros_like(w[n], dtype=torch.float64) for n in ARGS + ("S0",)]
    for row, at, n in pieces:
        bars = f.delta_rule_bars(*[w[x][row, at].double() for x in ARGS], w["scale"], w["S0"][n].double(), w["ob"][row, at].double(),
                                 w["Sb"][n].double())
        for y, x in zip(out[:5], bars):
            y[row, at] = x
        out[5][n] = bars[5]
    return out


def cuda(w):
    return {k: x.cuda() if torch.is_tensor(x) else x for k, x in w.items()}


def check(names, got, want, dtypes):
    for n, x, y, dt in zip(names, got, want, dtypes):
        assert x.dtype == dt
        off, tol = f.rel(x, y), f.tolerance(dt)
        assert off <= tol, (n, off, tol)


SHAPES = [(1, 1, 1, 1, 1, 1), (2, 3, 1, 1, 8, 8), (1, 31, 1, 2, 16, 17), (1, 32, 2, 2, 64, 64), (1, 33, 1, 1, 65, 33), (2, 63, 1, 3, 40, 48),
          (1, 64, 1, 1, 128, 128), (1, 65, 2, 4, 128, 96), (2, 130, 2, 2, 72, 100), (1, 257, 1, 2, 127, 129), (3, 100, 3, 3, 12, 20)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("batch,T,hk,hv,dk,dv", SHAPES)
def test_forward(la, dtype, batch, T, hk, hv, dk, dv):
    w = make(dtype, batch, T, hk, hv, dk, dv, seed=T + dk)
    o_ref, S_ref = reference(w)
    c = cuda(w)
    o, S, saved = la.delta_rule(*[c[n] for n in ARGS], initial_state=c["S0"], want_state=True)
    assert saved is None
    check(("o", "state"), (o, S), (o_ref, S_ref), (dtype, F32))
    # the same answers with the intermediate results kept, and again
    o2, S2, saved = la.delta_rule(*[c[n] for n in ARGS], initial_state=c["S0"], want_state=True, keep=True)
    assert saved.dtype == torch.uint8 and torch.equal(o, o2) and torch.equal(S, S2)
    # no initial state is one of zeros
    o3, S3, _ = la.delta_rule(*[c[n] for n in ARGS], want_state=True)
    o4, S4, _ = la.delta_rule(*[c[n] for n in ARGS], initial_state=torch.zeros_like(c["S0"]), want_state=True)
    assert torch.equal(o3, o4) and torch.equal(S3, S4)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("batch,T,hk,hv,dk,dv", SHAPES)
def test_gradient(la, dtype, batch, T, hk, hv, dk, dv):
    w = make(dtype, batch, T, hk, hv, dk, dv, seed=T + dk + 1)
    ref = reference_bars(w)
    c = cuda(w)
    x = [c[n] for n in ARGS]
    bars = la.delta_rule_backward(*x, c["ob"], initial_state=c["S0"], state_bar=c["Sb"])
    check(ARGS + ("S0",), bars, ref, (dtype,) * 3 + (F32,) * 3)
    _, _, saved = la.delta_rule(*x, initial_state=c["S0"], keep=True)
    again = la.delta_rule_backward(*x, c["ob"], initial_state=c["S0"], state_bar=c["Sb"], saved=saved)
    for a, b in zip(bars, again):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradient_without_states(la, dtype):
    w = make(dtype, 2, 70, 1, 2, 24, 40, seed=5)
    w["S0"].zero_()
    w["Sb"].zero_()
    ref = reference_bars(w)
    c = cuda(w)
    bars = la.delta_rule_backward(*[c[n] for n in ARGS], c["ob"])
    assert bars[5] is None
    check(ARGS, bars[:5], ref[:5], (dtype,) * 3 + (F32,) * 2)


def test_gradient_against_differences(la):
    """Along random directions, central differences of the recurrence in 64 bits."""
    w = make(F32, 1, 45, 1, 2, 20, 24, seed=77)
    c = cuda(w)
    bars = la.delta_rule_backward(*[c[n] for n in ARGS], c["ob"], initial_state=c["S0"], state_bar=c["Sb"])
    names = ARGS + ("S0",)
    r = torch.Generator().manual_seed(3)
    for n, bar in zip(names, bars):
        d = torch.randn(w[n].shape, generator=r, dtype=torch.float64)
        h, value = 1e-5, []
        for sign in (1, -1):
            x = {m: w[m].double() for m in names}
            x[n] = x[n] + sign * h * d
            o, S = f.delta_rule(*[x[m][0] for m in ARGS], w["scale"], x["S0"][0])
            value.append(float((o * w["ob"][0].double()).sum() + (S * w["Sb"][0].double()).sum()))
        want, got = (value[0] - value[1]) / (2 * h), float((bar.double().cpu() * d).sum())
        # the difference's own error is h^2; the gradient's that of its type, against the size of the summed terms
        assert abs(got - want) <= 1e-5 * float(bar.double().norm().cpu()) * float(d.norm()), n


PACKED = [[0, 1], [0, 5, 5, 6], [0, 64, 128], [0, 1, 66, 130, 131, 300], [0, 0, 31, 64, 97, 97], [0, 200]]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("ends", PACKED)
def test_packed(la, dtype, ends):
    w = make(dtype, len(ends) - 1, 0, 2, 4, 48, 72, seed=len(ends), lead=(1, ends[-1]))
    o_ref, S_ref = reference(w, ends)
    ref = reference_bars(w, ends)
    c = cuda(w)
    x, at = [c[n] for n in ARGS], torch.tensor(ends, dtype=torch.int32, device="cuda")
    o, S, _ = la.delta_rule(*x, initial_state=c["S0"], offsets=at, want_state=True)
    check(("o", "state"), (o, S), (o_ref, S_ref), (dtype, F32))
    bars = la.delta_rule_backward(*x, c["ob"], initial_state=c["S0"], state_bar=c["Sb"], offsets=at)
    check(ARGS + ("S0",), bars, ref, (dtype,) * 3 + (F32,) * 3)


def test_packed_tokens_of_no_sequence_are_zero(la):
    ends, total = [7, 90, 150], 240
    w = make(BF16, 2, 0, 1, 2, 32, 40, seed=9, lead=(1, total))
    o_ref, S_ref = reference(w, ends)
    ref = reference_bars(w, ends)
    c = cuda(w)
    x, at = [c[n] for n in ARGS], torch.tensor(ends, dtype=torch.int32, device="cuda")
    out = torch.full_like(c["v"], float("nan"))
    o, S, _ = la.delta_rule(*x, initial_state=c["S0"], offsets=at, want_state=True, out=out)
    assert not o[:, :7].any() and not o[:, 150:].any()
    check(("o", "state"), (o, S), (o_ref, S_ref), (BF16, F32))
    bars = la.delta_rule_backward(*x, c["ob"], initial_state=c["S0"], state_bar=c["Sb"], offsets=at)
    check(ARGS + ("S0",), bars, ref, (BF16,) * 3 + (F32,) * 3)
    for b in bars[:5]:
        assert not b[:, :7].any() and not b[:, 150:].any()


def test_no_tokens_pass_the_state_on(la):
    w = make(F32, 2, 0, 1, 2, 8, 12, seed=1)
    c = cuda(w)
    o, S, _ = la.delta_rule(*[c[n] for n in ARGS], initial_state=c["S0"], want_state=True)
    assert o.shape == (2, 0, 2, 12) and torch.equal(S, c["S0"])
    bars = la.delta_rule_backward(*[c[n] for n in ARGS], c["ob"], initial_state=c["S0"], state_bar=c["Sb"])
    assert torch.equal(bars[5], c["Sb"])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_extreme_decays_and_gates(la, dtype):
    """Decays that clear the state at once (minus infinity among them), none at all, beta of exactly zero and one, and keys of zero."""
    w = make(dtype, 1, 150, 1, 3, 64, 64, seed=21)
    w["g"][0, 10, 0] = float("-inf")
    w["g"][0, 11, 0] = -3.0e38
    w["g"][0, 70:80, 0] = -200.0
    w["g"][0, :, 1] = 0.0
    w["beta"][0, :, 2] = 0.0
    w["beta"][0, ::2, 1] = 1.0
    w["k"][0, 5] = 0.0
    w["q"][0, 6] = 0.0
    o_ref, S_ref = reference(w)
    ref = reference_bars(w)
    c = cuda(w)
    o, S, _ = la.delta_rule(*[c[n] for n in ARGS], initial_state=c["S0"], want_state=True)
    check(("o", "state"), (o, S), (o_ref, S_ref), (dtype, F32))
    bars = la.delta_rule_backward(*[c[n] for n in ARGS], c["ob"], initial_state=c["S0"], state_bar=c["Sb"])
    ref[3][0, 10:12, 0] = 0.0  # exp(g) and its derivative are zero
    check(ARGS + ("S0",), bars, ref, (dtype,) * 3 + (F32,) * 3)


def test_nan_stays_in_its_sequence_and_head(la):
    w = make(BF16, 2, 100, 2, 2, 32, 32, seed=8)
    w["v"][0, 70, 1, 3] = float("nan")
    c = cuda(w)
    o, S, _ = la.delta_rule(*[c[n] for n in ARGS], initial_state=c["S0"], want_state=True)
    assert torch.isnan(o[0, 70, 1, 3]) and torch.isnan(S[0, 1, :, 3]).all()
    assert torch.isfinite(o[1]).all() and torch.isfinite(o[0, :, 0]).all() and torch.isfinite(o[0, :64]).all()
    assert torch.isfinite(o[0, :, 1, :3]).all() and torch.isfinite(S[1]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_views_of_a_wider_projection(la, dtype):
    """q, k and v as slices of one tensor, off every alignment."""
    hk, hv, dk, dv, T = 2, 4, 24, 20, 75
    w = make(dtype, 2, T, hk, hv, dk, dv, seed=31)
    wide = torch.randn(2, T, 1 + 2 * hk * dk + hv * dv + 3).to(dtype)
    parts, at = {}, 1
    for n, h, d in (("q", hk, dk), ("k", hk, dk), ("v", hv, dv)):
        wide[..., at:at + h * d] = w[n].flatten(2)
        parts[n] = (at, h, d)
        at += h * d
    gpu, c = wide.cuda(), cuda(w)
    x = [gpu[..., a:a + h * d].unflatten(-1, (h, d)) for a, h, d in parts.values()] + [c["g"], c["beta"]]
    o, S, _ = la.delta_rule(*x, initial_state=c["S0"], want_state=True)
    o2, S2, _ = la.delta_rule(*[c[n] for n in ARGS], initial_state=c["S0"], want_state=True)
    assert torch.equal(o, o2) and torch.equal(S, S2)
    b1 = la.delta_rule_backward(*x, c["ob"], initial_state=c["S0"])
    b2 = la.delta_rule_backward(*[c[n] for n in ARGS], c["ob"], initial_state=c["S0"])
    for a, b in zip(b1, b2):
        assert torch.equal(a, b)
    state = [c["S0"].clone(), c["S0"].clone()]
    s1 = la.delta_rule_step(*[t[:, 5] if i < 3 else t[:, 5].contiguous() for i, t in enumerate(x)], state[0])
    s2 = la.delta_rule_step(*[c[n][:, 5].contiguous() for n in ARGS], state[1])
    assert torch.equal(s1, s2) and torch.equal(state[0], state[1])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("batch,hk,hv,dk,dv", [(1, 1, 1, 1, 1), (3, 2, 4, 64, 64), (5, 1, 3, 128, 128), (2, 2, 2, 33, 35), (4, 1, 1, 127, 66), (70, 2, 4, 16, 130)])
def test_step(la, dtype, batch, hk, hv, dk, dv):
    """Single tokens one after another are the sequence; slots in any order, one without a state."""
    T = 3
    w = make(dtype, batch, T, hk, hv, dk, dv, seed=batch + dv)
    o_ref, S_ref = reference(w)
    c = cuda(w)
    slots = torch.randperm(batch + 4, generator=torch.Generator().manual_seed(1))[:batch].to(torch.int32)
    cache = torch.randn(batch + 4, hv, dk, dv, generator=torch.Generator().manual_seed(2)).cuda()
    cache[slots.long().cuda()] = c["S0"]
    before, at = cache.clone(), slots.cuda()
    for t in range(T):
        o = la.delta_rule_step(*[c[n][:, t].contiguous() for n in ARGS], cache, slots=at)
        check(("o",), (o,), (o_ref[:, t],), (dtype,))
    check(("state",), (cache[slots.long().cuda()],), (S_ref,), (F32,))
    rest = [i for i in range(batch + 4) if i not in slots.tolist()]
    assert torch.equal(cache[rest], before[rest])
    at = slots.clone()
    at[0] = -1 if batch % 2 else batch + 4
    before = cache.clone()
    o = la.delta_rule_step(*[c[n][:, 0].contiguous() for n in ARGS], cache, slots=at.cuda())
    assert not o[0].any() and torch.equal(cache[int(slots[0])], before[int(slots[0])])
    direct = c["S0"].clone()
    o1 = la.delta_rule_step(*[c[n][:, 0].contiguous() for n in ARGS], direct)
    check(("o",), (o1,), (o_ref[:, 0],), (dtype,))


def test_many_chunks_and_blocks(la):
    """More heads, chunks and columns than one wave of blocks."""
    w = make(BF16, 3, 700, 4, 8, 128, 128, seed=4, decay=0.05)
    o_ref, S_ref = reference(w)
    c = cuda(w)
    o, S, _ = la.delta_rule(*[c[n] for n in ARGS], initial_state=c["S0"], want_state=True)
    check(("o", "state"), (o, S), (o_ref, S_ref), (BF16, F32))
    ref = reference_bars(w)
    bars = la.delta_rule_backward(*[c[n] for n in ARGS], c["ob"], initial_state=c["S0"], state_bar=c["Sb"])
    check(ARGS + ("S0",), bars, ref, (BF16,) * 3 + (F32,) * 3)


def test_on_another_stream_and_in_a_graph(la):
    w = make(BF16, 2, 90, 1, 2, 64, 64, seed=12)
    c = cuda(w)
    x = [c[n] for n in ARGS]
    o_ref, _, _ = la.delta_rule(*x, initial_state=c["S0"])
    b_ref = la.delta_rule_backward(*x, c["ob"], initial_state=c["S0"])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        o, _, _ = la.delta_rule(*x, initial_state=c["S0"])
    s.synchronize()
    assert torch.equal(o, o_ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, _, _ = la.delta_rule(*x, initial_state=c["S0"])
        bars = la.delta_rule_backward(*x, c["ob"], initial_state=c["S0"])
    for _ in range(3):
        o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, o_ref)
        for a, b in zip(bars, b_ref):
            assert torch.equal(a, b)
        torch.randn(1000, device="cuda").sum()


def test_workspace_of_garbage(la):
    """What a workspace held before does not matter."""
    w = make(F16, 2, 70, 1, 2, 40, 40, seed=6)
    c = cuda(w)
    x = [c[n] for n in ARGS]
    o_ref, _, _ = la.delta_rule(*x)
    ws = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")  # every float in it is NaN
    o, _, _ = la.delta_rule(*x, workspace=ws)
    assert torch.equal(o, o_ref)
    b_ref = la.delta_rule_backward(*x, c["ob"])
    ws.fill_(255)
    for a, b in zip(b_ref, la.delta_rule_backward(*x, c["ob"], workspace=ws)):
        assert a is b is None or torch.equal(a, b)


def test_refusals(la):
    w = cuda(make(F32, 2, 6, 2, 4, 16, 16, seed=1))
    x = {n: w[n] for n in ARGS}

    def refused(**change):
        with pytest.raises(la.LaError):
            la.delta_rule(**{**x, **change})

    refused(q=x["q"].double(), k=x["k"].double(), v=x["v"].double())
    refused(q=x["q"].to(BF16))
    refused(k=x["k"][:, :5])
    refused(v=x["v"][:, :, :3].contiguous(), g=x["g"][..., :3].contiguous(), beta=x["beta"][..., :3].contiguous())
    refused(g=x["g"].to(BF16))
    refused(beta=x["beta"].transpose(0, 1).contiguous())
    refused(q=x["q"].transpose(2, 3).contiguous().transpose(2, 3))
    refused(q=x["q"].cpu())
    refused(initial_state=w["S0"][:1].contiguous())
    refused(initial_state=w["S0"].to(BF16))
    refused(offsets=torch.tensor([0, 6], dtype=torch.int32, device="cuda"))  # two rows of tokens
    refused(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    refused(out=x["v"])
    big = cuda(make(F32, 1, 2, 1, 1, 129, 4, seed=1))
    with pytest.raises(la.LaError, match="UNSUPPORTED"):
        la.delta_rule(*[big[n] for n in ARGS])
    one = {n: x[n][:, 0].contiguous() for n in ARGS}
    with pytest.raises(la.LaError):
        la.delta_rule_step(**one, state=w["S0"].to(BF16))
    with pytest.raises(la.LaError):
        la.delta_rule_step(**one, state=w["S0"][:1].contiguous())  # fewer states than sequences
    with pytest.raises(la.LaError):
        la.delta_rule_step(**one, state=w["S0"], slots=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(la.LaError):
        la.delta_rule_backward(**x, o_bar=w["ob"], saved=torch.empty(256, dtype=torch.uint8, device="cuda"))
