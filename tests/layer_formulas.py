"""The formulas of the sequence-layer operators in 64 bits, on the CPU, token by token and element by element: what the tests compare with."""
import torch


def delta_rule(q, k, v, g, beta, scale, S0):
    """One sequence: q, k [T, hk, dk], v [T, hv, dv], g, beta [T, hv], S0 [hv, dk, dv]; returns (o, final state)."""
    group = v.shape[1] // q.shape[1]
    q, k = (x.repeat_interleave(group, 1) for x in (q, k))
    S, o = S0, []
    for t in range(q.shape[0]):
        S = torch.exp(g[t])[:, None, None] * S
        u = beta[t][:, None] * (v[t] - (S * k[t][:, :, None]).sum(1))
        S = S + k[t][:, :, None] * u[:, None, :]
        o.append(scale * (S * q[t][:, :, None]).sum(1))
    return (torch.stack(o) if o else v + 0.0), S


def delta_rule_bars(q, k, v, g, beta, scale, S0, ob, Sb):
    """Gradients of one sequence by differentiating the recurrence above."""
    x = [t.clone().requires_grad_() for t in (q, k, v, g, beta, S0)]
    o, S = delta_rule(*x[:5], scale, x[5])
    out = torch.autograd.grad([o, S], x, [ob, Sb], allow_unused=True)
    return [torch.zeros_like(a) if b is None else b for a, b in zip(x, out)]


def layer_norm(x, w, c, eps):
    mean = x.mean(-1)
    rstd = 1.0 / torch.sqrt(((x - mean[..., None]) ** 2).mean(-1) + eps)
    return (x - mean[..., None]) * rstd[..., None] * w + c, mean, rstd


def layer_norm_bars(x, w, eps, yb):
    _, mean, rstd = layer_norm(x, w, 0.0, eps)
    h = (x - mean[..., None]) * rstd[..., None]
    t = yb * w
    xb = rstd[..., None] * (t - t.mean(-1, keepdim=True) - h * (t * h).mean(-1, keepdim=True))
    dims = tuple(range(x.dim() - 1))
    return xb, (yb * h).sum(dims), yb.sum(dims)


# How far results may be off, as the 2-norm of the difference over that of the result.  A result in 16 bits is rounded once: by at most
# 2^-8 (bf16, 8 significant bits) or 2^-11 (f16, 11 of them) of each element; the sums behind it are in 32 bits.  Results in 32 bits carry the rounding of sums and
# products of up to some hundred terms, 2^-24 each and growing with their root, and of the recurrence's dependent steps.
ROUNDING = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 0.0, torch.float64: 0.0}
SUMS = {torch.bfloat16: 2e-6, torch.float16: 2e-6, torch.float32: 2e-6, torch.float64: 2e-14}


def tolerance(dtype):
    return ROUNDING[dtype] + SUMS[dtype]


def rel(x, ref):
    x, ref = x.detach().double().cpu(), ref.detach().double().cpu()
    assert x.shape == ref.shape, (x.shape, ref.shape)
    if not ref.numel():
        return 0.0
    assert torch.isfinite(x).all()
    norm = float(ref.norm())
    return float((x - ref).norm()) / norm if norm else float(x.norm())
