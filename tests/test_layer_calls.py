"""The sequence layer's operators at their C entries and through the binding's two ways: what is refused is refused on the host, before anything is launched
(the operands' addresses are made up: these tests run only where there is no GPU, and a call that gets as far as a launch fails them), and plain calls through csrc/host_call.cpp give what the ctypes calls give, bit for bit."""
import ctypes

import pytest
import torch

import paper_1710_08717_amd as la
from paper_1710_08717_amd import binding

F32, F64, BF16, F16 = 0, 1, 2, 3
AT = 1 << 40  # operands at addresses far apart, that nothing may read
NAN = float("nan")


def at(i):
    return AT + (i << 32)


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.device_count() > 0:
        pytest.skip("made-up addresses: only where nothing can be launched")
    return la.load()


@pytest.fixture(scope="module")
def codes():
    """the header's values of the statuses"""
    import os
    import re

    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "la.h")) as f:
        text = f.read()
    return {k: int(v) for k, v in re.findall(r"\b(LA_(?:OK|ERR_\w+))\s*=\s*(\d+)", text)}


def rule(lib, dt=F32, batch=2, tokens=5, hk=2, hv=4, dk=16, dv=24, offsets=None, ldq=32, ldk=32, ldv=96, q=at(1), o=at(6), state0=None, state=None, saved=None,
         saved_bytes=0, workspace=at(9), workspace_bytes=1 << 30):
    return lib.la_delta_rule(dt, batch, tokens, hk, hv, dk, dv, offsets, q, ldq, at(2), ldk, at(3), ldv, at(4), at(5), 1.0, state0, o, state, saved,
                             saved_bytes, workspace, workspace_bytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(dt=F64), "LA_ERR_UNSUPPORTED"), (dict(dk=129, ldq=258, ldk=258), "LA_ERR_UNSUPPORTED"), (dict(dv=1025, ldv=4100), "LA_ERR_UNSUPPORTED"),
    (dict(ldv=(1 << 24) + 8), "LA_ERR_UNSUPPORTED"), (dict(hv=1 << 15, dv=1024, ldv=1 << 25), "LA_ERR_UNSUPPORTED"), (dict(dt=7), "LA_ERR_INVALID_ARG"),
    (dict(hv=3), "LA_ERR_INVALID_ARG"), (dict(hk=0), "LA_ERR_INVALID_ARG"), (dict(batch=-1), "LA_ERR_INVALID_ARG"), (dict(tokens=-1), "LA_ERR_INVALID_ARG"),
    (dict(dk=0), "LA_ERR_INVALID_ARG"), (dict(ldq=31), "LA_ERR_INVALID_ARG"), (dict(ldv=95), "LA_ERR_INVALID_ARG"), (dict(q=None), "LA_ERR_INVALID_ARG"),
    (dict(o=at(1) + 64), "LA_ERR_INVALID_ARG"), (dict(state=at(4)), "LA_ERR_INVALID_ARG"), (dict(state0=at(8), state=at(8) + 256), "LA_ERR_INVALID_ARG"),
    (dict(workspace=at(3)), "LA_ERR_INVALID_ARG"), (dict(workspace_bytes=100), "LA_ERR_WORKSPACE"), (dict(workspace=None), "LA_ERR_WORKSPACE"),
    (dict(saved=at(9), saved_bytes=100), "LA_ERR_WORKSPACE"), (dict(batch=0, offsets=at(11)), "LA_ERR_INVALID_ARG"), (dict(batch=0), "LA_OK")])
def test_delta_rule_refusals(lib, codes, change, status):
    assert rule(lib, **change) == codes[status]


def test_delta_rule_sizes_grow_with_what_is_kept(lib):
    size = (BF16, 2, 300, 2, 4, 64, 64)
    plain, kept = (getattr(lib, "la_delta_rule_%s_bytes" % x)(*size, 0) for x in ("workspace", "saved"))
    assert 0 < plain < kept
    assert lib.la_delta_rule_backward_workspace_bytes(*size, 0, 0) > lib.la_delta_rule_backward_workspace_bytes(*size, 0, 1) > 0
    assert lib.la_delta_rule_workspace_bytes(F64, *size[1:], 0) == 0  # not taken


def test_delta_rule_step_refusals(lib, codes):
    def step(dt=F16, batch=3, hk=1, hv=2, dk=16, dv=24, ldq=16, ldv=48, state=at(6), slots=3, slot=None, o=at(8)):
        return lib.la_delta_rule_step(dt, batch, hk, hv, dk, dv, at(1), ldq, at(2), 16, at(3), ldv, at(4), at(5), 1.0, state, slots, slot, o, None)

    assert step(batch=0) == codes["LA_OK"]
    assert step(dt=F64) == codes["LA_ERR_UNSUPPORTED"] == step(dk=200, ldq=200)
    for change in (dict(slots=-1), dict(slots=2), dict(state=None), dict(ldq=15), dict(ldv=47), dict(o=at(6)), dict(o=at(4)), dict(state=at(4)), dict(hv=0)):
        assert step(**change) == codes["LA_ERR_INVALID_ARG"], change


def test_layer_norm_refusals(lib, codes):
    def forward(dt=F32, wdt=F32, rows=4, n=10, ldx=10, x=at(1), eps=1e-5, y=at(2), mean=None, rstd=None):
        return lib.la_layer_norm(dt, wdt, rows, n, ldx, x, None, None, eps, y, mean, rstd, None)

    def backward(dt=F32, wdt=F32, rows=4, n=10, ldx=10, mean=at(3), x_bar=at(5), w_bar=at(6), workspace=at(8), size=1 << 20):
        return lib.la_layer_norm_backward(dt, wdt, rows, n, ldx, at(1), at(2), mean, at(4), None, x_bar, w_bar, at(7), workspace, size, None)

    assert forward(rows=0) == forward(n=0) == codes["LA_OK"]
    for change in (dict(dt=9), dict(wdt=F64), dict(dt=BF16, wdt=F16), dict(rows=-1), dict(n=-1), dict(ldx=9), dict(x=None), dict(y=None), dict(y=at(1) + 8),
                   dict(ldx=12, y=at(1)), dict(mean=at(3)), dict(mean=at(3), rstd=at(1) + 4), dict(mean=at(3), rstd=at(3) + 8), dict(eps=NAN), dict(eps=-1.0)):
        assert forward(**change) == codes["LA_ERR_INVALID_ARG"], change
    for change in (dict(dt=9), dict(wdt=F64), dict(n=-1), dict(ldx=9), dict(mean=None), dict(x_bar=None), dict(x_bar=at(1) + 4), dict(w_bar=at(1)),
                   dict(w_bar=at(3)), dict(w_bar=at(2) + 8), dict(w_bar=at(7) + 4), dict(workspace=at(6)), dict(workspace=at(4)), dict(workspace=at(8) + 8)):
        assert backward(**change) == codes["LA_ERR_INVALID_ARG"], change
    assert backward(size=0) == backward(workspace=None) == codes["LA_ERR_WORKSPACE"]


def test_clip_refusals(lib, codes):
    def clip(count=2, types=(F32, BF16), sizes=(100, 50), src=(at(1), at(2)), out=(at(3), at(4)), max_norm=1.0, norm_type=F32, norm=at(5), workspace=at(6),
             size=1 << 20):
        def array(kind, values):
            return None if values is None else (kind * len(values))(*values)

        return lib.la_clip_gradients(count, array(ctypes.c_int, types), array(ctypes.c_int64, sizes), array(ctypes.c_void_p, src),
                                     array(ctypes.c_void_p, out), max_norm, norm_type, norm, workspace, size, None)

    for change in (dict(count=-1), dict(types=(F32, 9)), dict(sizes=(100, -1)), dict(src=(at(1), None)), dict(out=(at(3), None)), dict(out=(at(1) + 4, at(4))),
                   dict(max_norm=-1.0), dict(max_norm=NAN), dict(norm_type=BF16), dict(norm=None), dict(types=None), dict(norm=at(3)), dict(norm=at(2) + 8),
                   dict(workspace=at(1)), dict(workspace=at(4)), dict(norm=at(6))):
        assert clip(**change) == codes["LA_ERR_INVALID_ARG"], change
    assert clip(size=0) == clip(workspace=None) == codes["LA_ERR_WORKSPACE"]


def calls(dt):
    torch.manual_seed(3)
    x, y_bar = (torch.randn(7, 3, 130, dtype=dt, device="cuda") for _ in range(2))
    w, b = (torch.randn(130, device="cuda", dtype=torch.float64 if dt == torch.float64 else torch.float32) for _ in range(2))
    _, mean, rstd = la.layer_norm(x, want_stats=True)
    grads = [torch.randn(n, dtype=dt, device="cuda") for n in (5, 0, 4097)] + [torch.randn(33, device="cuda")]
    out = {
        "norm": lambda: la.layer_norm(x, w, b), "norm_stats": lambda: la.layer_norm(x[:, 1], None, b, 1e-3, True), "norm_plain": lambda: la.layer_norm(x, w),
        "norm_back": lambda: la.layer_norm_backward(x, y_bar, mean, rstd, w), "norm_back_x": lambda: la.layer_norm_backward(x, y_bar, mean, rstd, None, False),
        "clip": lambda: (lambda g: (la.clip_gradients(g, 0.5), *g))([t.clone() for t in grads]),
        "clip_out": lambda: (lambda g: (la.clip_gradients(grads, 1e9, out=g), *g))([torch.empty_like(t) for t in grads]),
    }
    if dt != torch.float64:
        q, k = (torch.randn(6, 2, 40, dtype=dt, device="cuda") for _ in range(2))
        v = torch.randn(6, 9, 24, dtype=dt, device="cuda")[:, :4]
        g, beta, state = -torch.rand(6, 4, device="cuda"), torch.rand(6, 4, device="cuda"), torch.randn(8, 4, 40, 24, device="cuda")
        slots = torch.tensor([3, 1, -1, 7, 0, 9], dtype=torch.int32, device="cuda")
        out["step"] = lambda: (lambda s: (la.delta_rule_step(q, 0.1 * k, v, g, beta, s), s))(state.clone())
        out["step_slots"] = lambda: (lambda s: (la.delta_rule_step(q, 0.1 * k, v, g, beta, s, slots, 0.3), s))(state.clone())
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [torch.float32, torch.float64, torch.bfloat16, torch.float16])
def test_both_ways_agree(dt, monkeypatch):
    work = calls(dt)
    fast = {k: f() for k, f in work.items()}
    monkeypatch.setattr(binding, "_host", None)
    for k, f in work.items():
        many = [t if isinstance(t, tuple) else (t,) for t in (fast[k], f())]
        assert len(many[0]) == len(many[1]), k
        for x, z in zip(*many):
            assert (x is None) == (z is None), k
            if x is not None:
                assert x.shape == z.shape and x.dtype == z.dtype and torch.equal(x, z), k
