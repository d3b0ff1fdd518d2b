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


@pytest.mark.parametrize("sizes", [(1e200,), (1e-200,), (1e306, 1e300, 1.0), (1e200, 1.0, 1e-200), (1.0, 1e-200), (1e145, 1e146), (1e-146, 1e-144), (1e-308,), (4e-320,)])
def test_squares_that_64_bits_do_not_hold(la, sizes):
    grads = [make(9001 + 100 * i, s, F64, seed=i) for i, s in enumerate(sizes)]
    norm = norm_of(grads)
    for limit in (0.25 * value(norm), 4.0 * value(norm)):
        out = [torch.empty_like(x) for x in grads]
        got = la.clip_gradients(grads, limit, out=out)
        # (numbers below 2^-1022 are rounded to a multiple of 2^-1074)
        assert abs(float(got) - value(norm)) <= 1e-12 * value(norm) + 2.0 ** -1074
        if limit > value(norm):
            assert all(same(a, b) for a, b in zip(out, grads))
        else:
            for a, b in zip(out, grads):
                assert bool(((a - 0.25 * b).abs() <= 1e-12 * b.abs() + 2.0 ** -1073).all())
    assert value(norm_of(out)) > 0


def test_many_large_squares(la):
    """what is just below the limit between two sums does not overflow by its number"""
    grads = [make(3_000_000, s, F64) for s in (2.0 ** 479, 2.0 ** -479, 2.0 ** 481)]
    for x in grads:
        assert abs(float(la.clip_gradients([x.clone()], math.inf)) / value(norm_of([x])) - 1) <= 1e-12


def test_large_doubles_beside_other_types(la):
    grads = [make(500, 1e250, F64), make(300, 3e38, F32), make(20, 1e-40, BF16), make(99, 60000.0, F16)]
    norm = value(norm_of(grads))
    want = [x.double() * (1e245 / norm) for x in grads]
    out = [torch.empty_like(x) for x in grads]
    assert abs(float(la.clip_gradients(grads, 1e245, out=out)) / norm - 1) <= 1e-12
    for x, y in zip(out[:2] + out[3:], want[:2] + want[3:]):  # (the third is below the smallest number of its type)
        assert f.rel(x, y) <= f.tolerance(x.dtype)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("rest", [1e300, 1.0, 1e-300, 0.0])
def test_doubles_that_are_not_finite_change_nothing(la, bad, rest):
    grads = [make(4000, rest, F64), make(5, rest, F64)]
    grads[1][2] = bad
    before = [x.clone() for x in grads]
    norm = float(la.clip_gradients(grads, 1e-3))
    assert math.isnan(norm) if math.isnan(bad) else norm == math.inf
    assert all(same(a, b) for a, b in zip(grads, before))


def test_a_double_norm_past_its_range_changes_nothing(la):
    x = make(1000, 1.7e308, F64)
    y = x.clone()
    assert float(la.clip_gradients([x], 1.0)) == math.inf and same(x, y)


@pytest.mark.parametrize("dtype,size,limit", [(F32, 1e37, 1e-5), (F32, 1e37, 1e-2), (BF16, 1e37, 1e-5), (F32, 1e37, 1e-20), (F64, 1e306, 1e-3), (F64, 1e300, 1e-250)])
@pytest.mark.parametrize("shift", [0, 1])
def test_factors_below_the_smallest_normal_number(la, dtype, size, limit, shift):
    """the factor is rounded as a number of its type only where that costs nothing"""
    grads = [make(700, size, dtype), make(33, size, dtype, seed=2)]
    norm = value(norm_of(grads))
    assert limit / norm < (2.0 ** -1022 if dtype == F64 else 2.0 ** -126)
    want = [x.double() * 1e-200 * (limit / (norm * 1e-200)) for x in grads]
    space = [torch.empty(x.numel() + 1, dtype=dtype, device="cuda") for x in grads]
    out = [s[shift:shift + x.numel()] for s, x in zip(space, grads)]
    la.clip_gradients(grads, limit, out=out)
    for x, y in zip(out, want):
        assert f.rel(x, y) <= f.tolerance(dtype)
    mine = [x.clone() for x in grads]
    la.clip_gradients(mine, limit)
    for x, y in zip(mine, want):
        assert f.rel(x, y) <= f.tolerance(dtype)


def test_a_limit_of_zero_clears_the_largest_numbers(la):
    for x in (make(100, 1e37, F32), make(100, 1e300, F64), make(100, 1e37, BF16)):
        la.clip_gradients([x], 0.0)
        assert not x.any()
