"""The norm over all gradients and their clipping on the GPU against 64 bits."""
import math
import sys

import pytest
import torch

import layer_formulas as f

pytestmark = pytest.mark.gpu
BF16, F16, F32, F64 = torch.bfloat16, torch.float16, torch.float32, torch.float64


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


def make(sizes, dtypes, seed, spread=1.0):
    r = torch.Generator().manual_seed(seed)
    return [(spread * torch.randn(n, generator=r)).to(dtypes[i % len(dtypes)]).cuda() for i, n in enumerate(sizes)]


def norm_of(grads):
    return math.sqrt(sum(float(x.double().square().sum()) for x in grads))


SIZES = [[1], [5, 0, 3], [8192], [8193, 1, 24577], [100] * 300, [0, 0], [200001, 7], list(range(1, 120)), [70000] * 130]


@pytest.mark.parametrize("dtypes", [[F32], [F64], [BF16], [F16], [BF16, F32], [F64, F32, F16, BF16]])
@pytest.mark.parametrize("sizes", SIZES)
def test_clip(la, sizes, dtypes):
    grads = make(sizes, dtypes, seed=len(sizes))
    norm = norm_of(grads)
    kind = F64 if any(x.dtype == F64 for x in grads) else F32
    for limit in (0.5 * norm, 2.0 * norm + 1.0):
        want = [x.double() * min(1.0, limit / norm if norm else 1.0) for x in grads]
        out = [torch.full_like(x, float("nan")) for x in grads]
        got = la.clip_gradients(grads, limit, out=out)
        assert got.dtype == kind and got.shape == ()
        assert abs(float(got) - norm) <= (1e-12 if kind == F64 else 1e-7) * norm
        for x, y in zip(out, want):
            assert f.rel(x, y) <= f.tolerance(x.dtype)
        again = [torch.empty_like(x) for x in grads]
        assert torch.equal(la.clip_gradients(grads, limit, out=again), got) and all(torch.equal(a, b) for a, b in zip(out, again))
        mine = [x.clone() for x in grads]
        assert torch.equal(la.clip_gradients(mine, limit), got)
        assert all(torch.equal(a, b) for a, b in zip(mine, out))
    if norm and limit > norm:
        assert all(torch.equal(a, b) for a, b in zip(out, grads))


def test_views_off_every_alignment(la):
    flat = torch.randn(100000, device="cuda").to(BF16)
    spans = [(1, 9), (10, 3), (13, 8300), (8313, 1), (8314, 50001)]
    grads = [flat[a:a + n] for a, n in spans]
    want = [x.double() * min(1.0, 1.0 / norm_of(grads)) for x in grads]
    for shift in (0, 1):
        space = torch.empty(100000, device="cuda", dtype=BF16)
        out = [space[a + shift:a + shift + n] for a, n in spans]
        la.clip_gradients(grads, 1.0, out=out)
        for x, y in zip(out, want):
            assert f.rel(x, y) <= f.tolerance(BF16)
    outside = torch.ones(100000, dtype=torch.bool)
    for a, n in spans:
        outside[a:a + n] = False
    before = flat.clone()
    la.clip_gradients(grads, 1.0)
    assert torch.equal(flat[outside.cuda()], before[outside.cuda()])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_norm_that_is_not_finite_changes_nothing(la, bad):
    grads = make([1000, 20], [F32], seed=1)
    grads[1][3] = bad
    before = [x.clone() for x in grads]
    norm = la.clip_gradients(grads, 1.0)
    assert not math.isfinite(float(norm))
    for x, y in zip(grads, before):
        assert torch.equal(x.view(torch.int32), y.view(torch.int32))


def test_squares_that_32_bits_do_not_hold(la):
    for size in (1e30, 1e-30):
        x = torch.full((1000,), size, device="cuda")
        norm = la.clip_gradients([x], 0.5 * size)
        assert abs(float(norm) / (size * math.sqrt(1000.0)) - 1) < 1e-6
        assert torch.allclose(x, torch.full_like(x, 0.5 * size / math.sqrt(1000.0)), rtol=1e-6, atol=0.0)


def test_limits_of_zero_and_infinity(la):
    x = torch.randn(100, device="cuda")
    y = x.clone()
    la.clip_gradients([y], float("inf"))
    assert torch.equal(x, y)
    la.clip_gradients([y], 0.0)
    assert not y.any()
    assert float(la.clip_gradients([torch.zeros(5, device="cuda")], 1.0)) == 0.0


def test_refusals(la):
    x = torch.randn(10, device="cuda")
    for call in (lambda: la.clip_gradients([], 1.0), lambda: la.clip_gradients([x.cpu()], 1.0), lambda: la.clip_gradients([x[::2]], 1.0),
                 lambda: la.clip_gradients([x.int()], 1.0), lambda: la.clip_gradients([x], -1.0), lambda: la.clip_gradients([x], float("nan")),
                 lambda: la.clip_gradients([x], 1.0, out=[]), lambda: la.clip_gradients([x], 1.0, out=[x[:5]]),
                 lambda: la.clip_gradients([x[:8]], 1.0, out=[x[2:]]), lambda: la.clip_gradients([x], 1.0, out=[torch.empty(10, device="cuda", dtype=BF16)]),
                 lambda: la.clip_gradients([x], 1.0, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(la.LaError):
            call()
