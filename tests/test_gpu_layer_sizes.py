"""Sizes past the C entries' integers are refused by the binding, in both its ways, and not taken modulo 2^32; states of the wrong number of axes as well."""
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(params=[True, False])
def la(request, monkeypatch):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1710_08717_amd as la_mod
    from paper_1710_08717_amd import binding

    la_mod.load()
    if not request.param:
        monkeypatch.setattr(binding, "_host", None)
    return la_mod


@pytest.fixture(autouse=True)
def _announce(request):
    sys.stderr.write(f"\n[gpu-case] {request.node.nodeid}\n")
    sys.stderr.flush()
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [(1 << 32) + 8, 1 << 31])
def test_rows_of_layer_norm(la, n):
    x = torch.empty(1, n, dtype=BF16, device="cuda")
    x[:, :8] = 1.0
    with pytest.raises(la.LaError):
        la.layer_norm(x)
    stat = torch.ones(1, device="cuda")
    with pytest.raises(la.LaError):
        la.layer_norm_backward(x, x, stat, stat, want_weights=False, out=x)


@pytest.mark.parametrize("which", ["dk", "dv", "hv"])
def test_heads_of_the_delta_rule(la, which):
    big = (1 << 32) + 2
    hk, hv, dk, dv = 1, big if which == "hv" else 1, big if which == "dk" else 2, big if which == "dv" else 1
    q = torch.zeros(1, hk, dk, dtype=BF16, device="cuda")
    v = torch.zeros(1, hv, dv, dtype=BF16, device="cuda")
    g = torch.zeros(1, hv, device="cuda")
    state = torch.empty(0, hv, dk, dv, device="cuda")
    for call in (lambda: la.delta_rule(q[None], q[None], v[None], g[None], g[None]),
                 lambda: la.delta_rule_backward(q[None], q[None], v[None], g[None], g[None], v[None]),
                 lambda: la.delta_rule_step(q, q, v, g, g, state, slots=torch.zeros(1, dtype=torch.int32, device="cuda"))):
        with pytest.raises(la.LaError):
            call()


@pytest.mark.parametrize("shape", [(), (3,), (3, 2, 4), (3, 2, 4, 5, 1), (3, 2, 5, 4)])
def test_states_of_the_wrong_shape(la, shape):
    q, v, g = torch.zeros(3, 1, 4, device="cuda"), torch.zeros(3, 2, 5, device="cuda"), torch.zeros(3, 2, device="cuda")
    with pytest.raises(la.LaError):
        la.delta_rule_step(q, q, v, g, g, torch.zeros(shape, device="cuda"))
