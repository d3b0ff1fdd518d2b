"""Layer norm of more rows than the threads of one launch serve: the same to the last bit as of the rows in parts."""
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu


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


PART = 1 << 24


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,ld", [(3, 3), (4, 5)])
@pytest.mark.parametrize("rows", [4 * (1 << 24) - 4, 4 * (1 << 24) + 101])  # four rows a block of 256 threads: as many as fit, and more
def test_rows_past_one_launch(la, dtype, n, ld, rows):
    some = torch.randn((1 << 20) + 7, ld, device="cuda").to(dtype)  # (a period that divides nothing)
    x = some.repeat(-(-rows // some.shape[0]), 1)[:rows, :n]
    w, c = torch.randn(n, device="cuda").to(dtype), torch.randn(n, device="cuda").to(dtype)
    y, mean, rstd = la.layer_norm(x, w, c, want_stats=True)
    x_bar, w_bar, c_bar = la.layer_norm_backward(x, y, mean, rstd, w)
    for a in range(0, rows, PART):
        z = slice(a, min(a + PART, rows))
        part = la.layer_norm(x[z], w, c, want_stats=True)
        assert all(torch.equal(p, q[z]) for p, q in zip(part, (y, mean, rstd))), a
        assert torch.equal(la.layer_norm_backward(x[z], part[0], *part[1:], w, want_weights=False)[0], x_bar[z]), a
    assert torch.isfinite(w_bar).all() and torch.isfinite(c_bar).all()
