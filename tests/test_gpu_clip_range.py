"""Clipping at the ends of the types' ranges, against sums scaled on the CPU: norms that the type of the norm does not hold, squares that 64 bits do not
hold, factors below the smallest normal number."""
import ctypes
import math
import sys

import pytest
import torch

import layer_formulas as f

pytestmark = pytest.mark.gpu
BF16, F16, F32, F64 = torch.bfloat16, torch.float16, torch.float32, torch.float64
CODE = {F32: 0, F64: 1, BF16: 2, F16: 3}


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


def norm_of(grads):
    """in 64 bits, the largest element taken out: as a fraction and a power of two, since the norm itself may be past the range"""
    top = max(float(x.double().abs().max()) for x in grads if x.numel())
    e = math.frexp(top)[1]
    half = e // 2  # (two steps: 2^-e alone may be past the range)
    return math.sqrt(sum(float((x.double() * 2.0 ** -half * 2.0 ** (half - e)).square().sum()) for x in grads)), e


def value(norm):
    try:
        return math.ldexp(*norm)
    except OverflowError:
        return math.inf


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def make(n, size, dtype, seed=1):
    x = 0.5 + 0.5 * torch.rand(n, generator=torch.Generator().manual_seed(seed), dtype=F64)
    return (x * size * torch.where(torch.arange(n) % 3 == 0, -1.0, 1.0)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_norm_past_its_type_counts_as_infinite(la, dtype):
    """norm and gradients agree: where the norm is written as infinity, nothing is scaled"""
    grads = [make(1000, 3e38, dtype), make(7, 1.0, dtype)]
    norm = norm_of(grads)
    assert 3.5e38 < value(norm) < 1e41
    out = [torch.empty_like(x) for x in grads]
    assert float(la.clip_gradients(grads, 1.0, out=out)) == math.inf
    assert all(same(a, b) for a, b in zip(out, grads))
    # a norm in 64 bits holds it: the gradients are scaled by 2
    lib = la.load()
    got, ws = torch.empty((), dtype=F64, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    rc = lib.la_clip_gradients(2, (ctypes.c_int * 2)(*[CODE[dtype]] * 2), (ctypes.c_int64 * 2)(1000, 7), (ctypes.c_void_p * 2)(*[x.data_ptr() for x in grads]),
                               (ctypes.c_void_p * 2)(*[x.data_ptr() for x in out]), value(norm) / 2, 1, got.data_ptr(), ws.data_ptr(), ws.numel(),
                               torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and abs(float(got) / value(norm) - 1) <= 1e-12
    for x, y in zip(out, grads):
        assert f.rel(x, 0.5 * y.double()) <= f.tolerance(dtype)


def test_the_largest_norm_that_32_bits_hold_is_clipped(la):
    x = make(4, 1e38, F32)
    want = x.double() * (2.0 / value(norm_of([x])))
    norm = la.clip_gradients([x], 2.0)
    assert math.isfinite(float(norm)) and f.rel(x, want) <= f.tolerance(F32)
