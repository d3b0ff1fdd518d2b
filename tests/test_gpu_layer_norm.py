"""Layer norm and its gradient on the GPU against the formulas in 64 bits."""
import sys

import pytest
import torch

import layer_formulas as f

pytestmark = pytest.mark.gpu
BF16, F16, F32, F64 = torch.bfloat16, torch.float16, torch.float32, torch.float64
TYPES = [(F32, F32), (F64, F64), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)]


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


def make(dtype, wdtype, rows, n, seed):
    r = torch.Generator().manual_seed(seed)
    g = lambda *s: torch.randn(*s, generator=r, dtype=F64)  # noqa: E731
    return (g(rows, n) * torch.exp(0.5 * g(n)) + 0.4 * g(rows, 1)).to(dtype), (1 + 0.1 * g(n)).to(wdtype), (0.1 * g(n)).to(wdtype), g(rows, n).to(dtype)


def check(pairs):
    for name, x, y, dt in pairs:
        assert x.dtype == dt, name
        off = f.rel(x, y)
        assert off <= f.tolerance(dt), (name, off, f.tolerance(dt))


SHAPES = [(1, 1), (3, 2), (5, 7), (4, 64), (9, 65), (70, 128), (1300, 129), (2, 256), (17, 300), (6, 511), (1100, 1024), (33, 1023), (3, 2048), (2, 2049),
          (7, 4096), (2, 4100), (3, 8192), (2, 8195), (2, 16384), (3, 16389), (2, 32768), (2, 40000), (700, 96)]


@pytest.mark.parametrize("dtype,wdtype", TYPES)
@pytest.mark.parametrize("rows,n", SHAPES)
def test_layer_norm_and_gradient(la, dtype, wdtype, rows, n):
    x, w, c, yb = make(dtype, wdtype, rows, n, seed=rows + n)
    D = [t.double() for t in (x, w, c, yb)]
    y_ref, mean_ref, rstd_ref = f.layer_norm(D[0], D[1], D[2], 1e-5)
    stat = F64 if dtype == F64 else F32
    gx, gw, gc, gyb = (t.cuda() for t in (x, w, c, yb))
    y, mean, rstd = la.layer_norm(gx, gw, gc, want_stats=True)
    if n > 1:  # (one element is its own mean: y is the bias, and a mean's rounding decides the rest)
        check([("y", y, y_ref, dtype), ("rstd", rstd, rstd_ref, stat)])
        assert torch.all((mean.double().cpu() - mean_ref).abs() <= f.SUMS[stat] * D[0].abs().mean(-1))
    else:
        assert torch.equal(y, gc.to(dtype).expand(rows, 1))
    assert torch.equal(la.layer_norm(gx, gw, gc)[0], y) and la.layer_norm(gx, gw, gc)[1] is None
    xb, wb, cb = la.layer_norm_backward(gx, gyb, mean, rstd, gw)
    if n > 2:  # (of two elements the gradient is what cancellation leaves: eps over the square of their difference)
        xb_ref, wb_ref, cb_ref = f.layer_norm_bars(D[0], D[1], 1e-5, D[3])
        check([("x_bar", xb, xb_ref, dtype), ("weight_bar", wb, wb_ref, wdtype), ("bias_bar", cb, cb_ref, wdtype)])
    again = la.layer_norm_backward(gx, gyb, mean, rstd, gw)
    assert all(torch.equal(a, b) for a, b in zip((xb, wb, cb), again))
    # in place
    buf = gyb.clone()
    xb2, wb2, cb2 = la.layer_norm_backward(gx, buf, mean, rstd, gw, out=buf)
    assert xb2 is buf and torch.equal(xb2, xb) and torch.equal(wb2, wb) and torch.equal(cb2, cb)
    buf = gx.clone()
    assert torch.equal(la.layer_norm(buf, gw, gc, out=buf)[0], y)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [40, 100, 2048, 2051])
def test_without_weights_and_on_strided_rows(la, dtype, n):
    x, _, _, yb = make(dtype, dtype, 12, n, seed=n)
    wide = torch.randn(12, n + 5).to(dtype)
    wide[:, 3:3 + n] = x
    view = wide.cuda()[:, 3:3 + n]
    y, mean, rstd = la.layer_norm(x.cuda(), want_stats=True)
    y2, mean2, rstd2 = la.layer_norm(view, want_stats=True)
    y_ref, _, _ = f.layer_norm(x.double(), 1.0, 0.0, 1e-5)
    check([("y", y, y_ref, dtype), ("y of a view", y2, y_ref, dtype)])
    xb_ref, _, _ = f.layer_norm_bars(x.double(), 1.0, 1e-5, yb.double())
    xb, wb, cb = la.layer_norm_backward(view, yb.cuda(), mean2, rstd2, want_weights=False)
    assert wb is None and cb is None
    check([("x_bar", xb, xb_ref, dtype)])
    # three axes are rows too
    assert torch.equal(la.layer_norm(x.cuda().view(3, 4, n))[0].view(12, n), y)


def test_gradient_against_differences(la):
    x, w, c, yb = make(F64, F64, 4, 37, seed=3)
    _, mean, rstd = la.layer_norm(x.cuda(), w.cuda(), c.cuda(), want_stats=True)
    bars = la.layer_norm_backward(x.cuda(), yb.cuda(), mean, rstd, w.cuda())
    r = torch.Generator().manual_seed(1)
    for i, bar in enumerate(bars):
        d = torch.randn([x, w, c][i].shape, generator=r, dtype=F64)
        value = []
        for h in (1e-6, -1e-6):
            a = [x, w, c]
            a[i] = a[i] + h * d
            value.append(float((f.layer_norm(*a, 1e-5)[0] * yb).sum()))
        want = (value[0] - value[1]) / 2e-6
        assert abs(float((bar.cpu() * d).sum()) - want) <= 1e-7 * float(bar.norm().cpu()) * float(d.norm())


def test_rows_far_from_zero_and_constant_rows(la):
    """A mean of thousands of standard deviations costs no more than the input's own rounding; equal elements give the bias."""
    x = (1000.0 + torch.randn(8, 512, generator=torch.Generator().manual_seed(1))).cuda()
    y_ref, _, _ = f.layer_norm(x.double().cpu(), 1.0, 0.0, 1e-5)
    # the mean in 32 bits is off by up to 2^-24 of 1000, against a standard deviation of 1
    assert f.rel(la.layer_norm(x)[0], y_ref) <= 2e-4
    bias = torch.randn(512, generator=torch.Generator().manual_seed(2)).cuda()
    assert torch.equal(la.layer_norm(torch.full((3, 512), 2.5, device="cuda"), None, bias)[0], bias.expand(3, 512))


def test_nan_and_infinity_stay_in_their_row(la):
    x = torch.randn(6, 300, generator=torch.Generator().manual_seed(1))
    x[1, 5], x[3, 7] = float("nan"), float("inf")
    y = la.layer_norm(x.cuda())[0].cpu()
    for r in range(6):
        assert torch.isnan(y[r]).any() if r in (1, 3) else torch.isfinite(y[r]).all()


def test_empty(la):
    w = torch.ones(5, device="cuda")
    x = torch.empty(0, 5, device="cuda")
    y, mean, rstd = la.layer_norm(x, w, w, want_stats=True)
    assert y.shape == (0, 5)
    xb, wb, cb = la.layer_norm_backward(x, x, mean, rstd, w)
    assert xb.shape == (0, 5) and not wb.any() and not cb.any()
    assert la.layer_norm(torch.empty(4, 0, device="cuda"))[0].shape == (4, 0)


def test_refusals(la):
    x = torch.randn(4, 6, device="cuda")
    w = torch.ones(6, device="cuda")
    _, mean, rstd = la.layer_norm(x, want_stats=True)
    for call in (lambda: la.layer_norm(x.cpu()), lambda: la.layer_norm(x.int()), lambda: la.layer_norm(x, w[:5].contiguous()),
                 lambda: la.layer_norm(x, w.to(BF16)), lambda: la.layer_norm(x.double(), w), lambda: la.layer_norm(x.t()),
                 lambda: la.layer_norm(x, eps=-1.0), lambda: la.layer_norm(x, w, w, out=x[:, :5]), lambda: la.layer_norm(x.view(4, 3, 2)[:, ::2]),
                 lambda: la.layer_norm_backward(x, x, mean[:3].contiguous(), rstd), lambda: la.layer_norm_backward(x, x.to(BF16), mean, rstd),
                 lambda: la.layer_norm_backward(x, x.clone(), mean, rstd, out=x),
                 lambda: la.layer_norm_backward(x, x, mean, rstd, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(la.LaError):
            call()


def test_rows_of_nothing(la):
    x = torch.empty(5, 0, device="cuda", dtype=torch.bfloat16)
    y, mean, rstd = la.layer_norm(x, want_stats=True)
    assert y.shape == x.shape and not mean.any() and not rstd.any()
    assert all(t.numel() == 0 for t in la.layer_norm_backward(x, y, mean, rstd))
