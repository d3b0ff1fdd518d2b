"""The operators of a gated linear-recurrence layer and of its training step, as they are timed: what a
program that trains or serves such a layer asks of this library.

Kinds of pass (``case["kind"]``):

* ``step``    -- the gated delta rule for one new token of every running sequence: a row of the state cache
  per sequence is read, updated in place and answered from.
* ``forward`` -- the gated delta rule over whole prompts, of one length or packed one behind another, with the
  state at their ends.
* ``train``   -- the same over a training batch, and its gradient.
* ``norm``    -- layer norm of a block of rows as serving calls it.
* ``norm_train`` -- layer norm and its gradient, the weight's and the bias's among it.
* ``clip``    -- the norm over all gradients of a model, and the gradients scaled to a largest norm.

The gated delta rule, for one head with key size dk and value size dv, S_0 the initial state [dk, dv]:

    S_t = a_t S_{t-1} + k_t u_t^T,   a_t = exp(g_t),   u_t = beta_t (v_t - a_t S_{t-1}^T k_t),
    o_t = scale S_t^T q_t;

value head h reads key head h // (Hv / Hk).  ``listed`` gives fixed cases, ``draw`` one more case of the same
ranges; inputs are drawn on the GPU from the seed alone.  ``exact`` gives the same outputs in 64 bits.
"""
import math

import torch

own = False  # whether run() calls this library's operators or computes them in their plain form

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
MAX_NORM = 1.0


def listed():
    return [
        # one sequence being generated: a token through one layer, latency
        {"name": "step_one_bf16", "kind": "step", "dtype": "bf16", "batch": 1, "slots": 4, "hk": 16, "hv": 32, "dk": 128, "dv": 128},
        # a server's full batch of running sequences, their states scattered over a larger cache
        {"name": "step_many_bf16", "kind": "step", "dtype": "bf16", "batch": 128, "slots": 160, "hk": 16, "hv": 32, "dk": 128, "dv": 128},
        # one long prompt through a layer of few heads
        {"name": "forward_prompt_bf16", "kind": "forward", "dtype": "bf16", "batch": 1, "tokens": 8192, "packed": False, "hk": 8, "hv": 16,
         "dk": 128, "dv": 128},
        # prompts of very different lengths packed one behind another, odd head sizes
        {"name": "forward_packed_f16", "kind": "forward", "dtype": "f16", "batch": 13, "tokens": 6001, "packed": True, "hk": 12, "hv": 12,
         "dk": 72, "dv": 100},
        # a training batch
        {"name": "train_bf16", "kind": "train", "dtype": "bf16", "batch": 2, "tokens": 4096, "packed": False, "hk": 16, "hv": 32, "dk": 128, "dv": 128},
        # a small model in single precision, sizes that are multiples of nothing, shared key heads
        {"name": "train_ragged_f32", "kind": "train", "dtype": "f32", "batch": 3, "tokens": 333, "packed": False, "hk": 2, "hv": 6, "dk": 48, "dv": 65},
        # a few rows between two layers of a model that answers token by token
        {"name": "norm_few_bf16", "kind": "norm", "dtype": "bf16", "rows": 16, "n": 2048},
        # a training batch's activations
        {"name": "norm_train_bf16", "kind": "norm_train", "dtype": "bf16", "rows": 16384, "n": 4096},
        # an odd width in single precision
        {"name": "norm_train_ragged_f32", "kind": "norm_train", "dtype": "f32", "rows": 4099, "n": 1023},
        # the hyperparameters and inducing inputs of a small model: many tiny tensors
        {"name": "clip_small_f32", "kind": "clip", "dtype": "f32", "tensors": 24, "elements": 20000},
        # the gradients of a language model of a few hundred tensors, matrices in 16 bits, vectors in 32
        {"name": "clip_model_bf16", "kind": "clip", "dtype": "bf16", "tensors": 290, "elements": 200000000},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["step", "forward", "forward", "train", "train", "norm", "norm_train", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    c = {"kind": kind, "dtype": dtype}
    if kind in ("norm", "norm_train"):
        n = _log_int(rng, 64, 16384)
        c.update(rows=_log_int(rng, 1, max(2, min(16384, (1 << 26) // n))) if kind == "norm_train" else _log_int(rng, 1, 512), n=n)
        return c
    if kind == "clip":
        c.update(tensors=_log_int(rng, 1, 400), elements=_log_int(rng, 1 << 12, 1 << 27))
        return c
    c.update(hk=rng.choice([1, 2, 3, 4, 8, 16]), dk=rng.choice([64, 128, 128, rng.randint(8, 128)]), dv=rng.choice([64, 128, 128, rng.randint(8, 160)]))
    c["hv"] = c["hk"] * rng.choice([1, 1, 2, 3])
    if kind == "step":
        c["batch"] = _log_int(rng, 1, 128)
        c["slots"] = c["batch"] + rng.randint(0, 32)
        return c
    c["packed"] = kind == "forward" and rng.random() < 0.5
    limit = (1 << 18 if kind == "forward" else 1 << 16) // c["hv"]  # tokens in all
    c["batch"] = rng.choice([1, 2, _log_int(rng, 1, 16)])
    total = _log_int(rng, 16 * c["batch"], max(64 * c["batch"], min(limit, 16384)))
    c["tokens"] = total if c["packed"] else max(1, min(total // c["batch"], 8192))
    return c


# -----------------------------------------------------------------------------------------------
# inputs
# -----------------------------------------------------------------------------------------------
class _Draw:
    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(710087170 + seed)
        self.dt = DTYPES[dtype]

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def rand(self, *shape):
        return torch.rand(*shape, generator=self.g, device="cuda")

    def low(self, *shape):
        return self.normal(*shape).to(self.dt)


def _unit(x):
    return x / x.square().sum(-1, keepdim=True).sqrt().clamp_min(1e-6)


def _lengths(count, total):
    """`count` lengths of a packed batch, the first a single token, the others growing: they sum to `total`."""
    w = torch.arange(1, count + 1, dtype=torch.float64) ** 2
    ends = (w.cumsum(0) / w.sum() * (total - 1)).floor().long() + 1
    return torch.cat([torch.zeros(1, dtype=torch.long), torch.ones(1, dtype=torch.long), ends[1:]]) if count > 1 else torch.tensor([0, total])


def _sizes(count, total):
    """Sizes of a model's gradients: three of four are vectors' (small), the rest share what is left; odd ones among them."""
    i = torch.arange(count, dtype=torch.float64)
    w = torch.where(i % 4 == 0, 1.0 + (i % 7), 0.0005 * (1.0 + (i % 5)))
    n = (w / w.sum() * max(total - count, 0)).floor().long() + 1
    return [int(x) for x in n]


def prepare(case, seed):
    kind, d = case["kind"], _Draw(seed, case["dtype"])
    s = {"case": case}
    if kind in ("norm", "norm_train"):
        rows, n = case["rows"], case["n"]
        channel = torch.exp(0.5 * d.normal(n))  # channels of different spread, rows with a mean
        s["x"] = (d.normal(rows, n) * channel + 0.3 * d.normal(rows, 1)).to(d.dt)
        s["weight"], s["bias"] = (1.0 + 0.1 * d.normal(n)).to(d.dt), (0.1 * d.normal(n)).to(d.dt)
        s["y_bar"] = d.low(rows, n) if kind == "norm_train" else None
        return s
    if kind == "clip":
        sizes = _sizes(case["tensors"], case["elements"])
        # one flat buffer for the matrices, one for the vectors (which stay in 32 bits), a view of it for each tensor
        flat = {}
        for which, dt in (("matrices", d.dt), ("vectors", torch.float32)):
            mine = [n for i, n in enumerate(sizes) if (i % 4 == 0) == (which == "matrices")]
            x = (d.normal(sum(mine)) * (0.01 if which == "matrices" else 0.1)).to(dt)
            y = torch.empty_like(x)
            flat[which] = (y, list(zip(x.split(mine), y.split(mine))))
        s["out"] = {which: y for which, (y, _) in flat.items()}
        pairs = flat["matrices"][1] + flat["vectors"][1]
        s["grads"], s["clipped"] = [x for x, _ in pairs], [y for _, y in pairs]
        return s
    b, hk, hv, dk, dv = case["batch"], case["hk"], case["hv"], case["dk"], case["dv"]
    step, packed = kind == "step", case.get("packed", False)
    lead = (b,) if step else (1, case["tokens"]) if packed else (b, case["tokens"])
    s["q"], s["k"] = (_unit(d.normal(*lead, hk, dk)).to(d.dt) for _ in range(2))
    s["v"] = d.low(*lead, hv, dv)
    rate = torch.exp(math.log(0.002) + math.log(250.0) * d.rand(hv))  # heads that forget slowly and ones that forget at once
    s["g"] = -rate * torch.nn.functional.softplus(d.normal(*lead, hv) + 0.5)
    s["beta"] = torch.sigmoid(d.normal(*lead, hv))
    s["scale"] = dk ** -0.5
    if step:
        s["state"] = 0.2 * d.normal(case["slots"], hv, dk, dv)
        s["slots"] = torch.argsort(d.rand(case["slots"]))[:b].to(torch.int32)
        return s
    s["initial_state"] = 0.2 * d.normal(b, hv, dk, dv)
    s["offsets"] = _lengths(b, case["tokens"]).to(torch.int32).cuda() if packed else None
    if packed:
        s["longest"] = int(_lengths(b, case["tokens"]).diff().max())
    if kind == "train":
        s["o_bar"], s["state_bar"] = d.low(*lead, hv, dv), 0.2 * d.normal(b, hv, dk, dv)
    return s


# -----------------------------------------------------------------------------------------------
# one pass
# -----------------------------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    return (_run_own if own else _run_plain)(kind, s)


def _run_own(kind, s):
    import paper_1710_08717_amd as la

    if kind == "step":
        o = la.delta_rule_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["state"], slots=s["slots"], scale=s["scale"])
        return {"o": o, "state": s["state"]}
    if kind == "forward":
        o, state, _ = la.delta_rule(s["q"], s["k"], s["v"], s["g"], s["beta"], scale=s["scale"], initial_state=s["initial_state"],
                                    offsets=s["offsets"], want_state=True)
        return {"o": o, "state": state}
    if kind == "train":
        x = (s["q"], s["k"], s["v"], s["g"], s["beta"])
        o, state, saved = la.delta_rule(*x, scale=s["scale"], initial_state=s["initial_state"], want_state=True, keep=True)
        bars = la.delta_rule_backward(*x, s["o_bar"], scale=s["scale"], initial_state=s["initial_state"], state_bar=s["state_bar"], saved=saved)
        return {"o": o, "state": state, **dict(zip(("q_bar", "k_bar", "v_bar", "g_bar", "beta_bar", "initial_state_bar"), bars))}
    if kind == "norm":
        return {"y": la.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS)[0]}
    if kind == "norm_train":
        y, mean, rstd = la.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, want_stats=True)
        bars = la.layer_norm_backward(s["x"], s["y_bar"], mean, rstd, s["weight"])
        return {"y": y, **dict(zip(("x_bar", "weight_bar", "bias_bar"), bars))}
    norm = la.clip_gradients(s["grads"], MAX_NORM, out=s["clipped"])
    return {"norm": norm, **s["out"]}


CHUNK = 64


def _plain_rule(q, k, v, g, beta, scale, S):
    """The rule over [sequences, T, heads, ...] in 32 bits by chunks of 64 tokens: within a chunk the u_t solve a unit lower-triangular
    system, whose inverse is a product of six factors (its strict part is nilpotent)."""
    b, T, hk, dk = q.shape
    hv, pad = v.shape[2], -T % CHUNK
    heads = lambda x: torch.nn.functional.pad(x.float().transpose(1, 2), (0, 0, 0, pad)).unflatten(2, (-1, CHUNK))  # noqa: E731
    q, k = (heads(x).repeat_interleave(hv // hk, 1) for x in (q, k))
    v, g, beta = heads(v), heads(g[..., None])[..., 0].cumsum(-1), heads(beta[..., None])
    q = q * scale
    decay = torch.exp((g[..., :, None] - g[..., None, :]).tril()).tril()
    kt = k.transpose(-1, -2)
    N = -(beta * (k @ kt) * decay).tril(-1)
    eye = torch.eye(CHUNK, device=q.device)
    N2 = N @ N
    N4 = N2 @ N2
    N8 = N4 @ N4
    N16 = N8 @ N8
    inv = (eye + N) @ (eye + N2) @ (eye + N4) @ (eye + N8) @ (eye + N16) @ (eye + N16 @ N16)
    eg = torch.exp(g)[..., None]
    last = g[..., -1:]
    u, w = inv @ (beta * v), inv @ (beta * eg * k)
    p, qg = (q @ kt) * decay, q * eg
    kl = (k * torch.exp(last - g)[..., None]).transpose(-1, -2)
    keep = torch.exp(last)[..., None]
    o = []
    for c in range(q.shape[2]):
        uc = u[:, :, c] - w[:, :, c] @ S
        o.append(qg[:, :, c] @ S + p[:, :, c] @ uc)
        S = keep[:, :, c] * S + kl[:, :, c] @ uc
    return torch.cat(o, 2)[:, :, :T].transpose(1, 2), S


def _plain_norm(x, weight, bias):
    x, mean = x.float(), x.float().mean(-1, keepdim=True)
    c = x - mean
    rstd = torch.rsqrt(c.square().mean(-1, keepdim=True) + EPS)
    return c * rstd * weight.float() + bias.float(), c * rstd, rstd


def _run_plain(kind, s):
    dt = DTYPES[s["case"]["dtype"]]
    if kind == "step":
        group = s["v"].shape[1] // s["q"].shape[1]
        q, k = (s[x].float().repeat_interleave(group, 1) for x in ("q", "k"))
        at = s["slots"].long()
        S = s["state"][at] * torch.exp(s["g"])[..., None, None]
        u = s["beta"][..., None] * (s["v"].float() - (S * k[..., None]).sum(-2))
        S = S + k[..., None] * u[..., None, :]
        s["state"][at] = S
        return {"o": (s["scale"] * (S * q[..., None]).sum(-2)).to(dt), "state": s["state"]}
    if kind == "forward":
        x = [s[n] for n in ("q", "k", "v", "g", "beta")]
        if s["offsets"] is None:
            o, S = _plain_rule(*x, s["scale"], s["initial_state"])
            return {"o": o.to(dt), "state": S}
        # every sequence padded to the longest: k, beta and g of the padding are zero, so that the state passes it unchanged
        at = s["offsets"][:-1, None].long() + torch.arange(s["longest"], device="cuda")
        inside = at < s["offsets"][1:, None]
        at = at.clamp(max=x[0].shape[1] - 1)
        x = [y[0][at] * inside.view(*inside.shape, *[1] * (y.dim() - 2)) for y in x]
        o, S = _plain_rule(*x, s["scale"], s["initial_state"])
        return {"o": o[inside][None].to(dt), "state": S}
    if kind == "train":
        x = [s[n].float().requires_grad_() for n in ("q", "k", "v")] + [s[n].clone().requires_grad_() for n in ("g", "beta", "initial_state")]
        with torch.enable_grad():
            o, S = _plain_rule(*x[:5], s["scale"], x[5])
            bars = torch.autograd.grad((o, S), x, (s["o_bar"].float(), s["state_bar"]))
        names = ("q_bar", "k_bar", "v_bar", "g_bar", "beta_bar", "initial_state_bar")
        return {"o": o.detach().to(dt), "state": S.detach(), **{n: y.to(dt) if n in names[:3] else y for n, y in zip(names, bars)}}
    if kind in ("norm", "norm_train"):
        y, h, rstd = _plain_norm(s["x"], s["weight"], s["bias"])
        if kind == "norm":
            return {"y": y.to(dt)}
        yb = s["y_bar"].float()
        t = yb * s["weight"].float()
        xb = rstd * (t - t.mean(-1, keepdim=True) - h * (t * h).mean(-1, keepdim=True))
        return {"y": y.to(dt), "x_bar": xb.to(dt), "weight_bar": (yb * h).sum(0).to(dt), "bias_bar": yb.sum(0).to(dt)}
    squares = torch.stack([x.float().square().sum() for x in s["grads"]])
    norm = squares.sum().sqrt()
    factor = (MAX_NORM / norm).clamp(max=1.0)
    for x, y in zip(s["grads"], s["clipped"]):
        y.copy_(x.float() * factor)
    return {"norm": norm, **s["out"]}


# -----------------------------------------------------------------------------------------------
# the same outputs in 64 bits, from the definitions: token by token
# -----------------------------------------------------------------------------------------------
def _exact_rule(q, k, v, g, beta, scale, S0, keep):
    """Outputs, final state, and with `keep` every state before its token; all [sequences, T, heads, ...] in 64 bits."""
    T, S, o, states = q.shape[1], S0, [], []
    for t in range(T):
        if keep:
            states.append(S)
        S = S * g[:, t].exp()[..., None, None]
        u = beta[:, t, :, None] * (v[:, t] - (S * k[:, t, :, :, None]).sum(2))
        S = S + k[:, t, :, :, None] * u[:, :, None, :]
        o.append(scale * (S * q[:, t, :, :, None]).sum(2))
    return (torch.stack(o, 1) if o else v), S, states


def _exact_backward(q, k, v, g, beta, scale, states, ob, Sb):
    T = q.shape[1]
    qb, kb, vb, gb, bb = (torch.empty_like(x) for x in (q, k, v, g, beta))
    for t in reversed(range(T)):
        a, kt, qt, bt = g[:, t].exp()[..., None], k[:, t], scale * q[:, t], beta[:, t, :, None]
        old = states[t]
        p = a * (old * kt[..., None]).sum(2)   # what the decayed state answers for the key
        r = v[:, t] - p
        u = bt * r
        new = a[..., None] * old + kt[..., None] * u[:, :, None, :]
        Sb = Sb + qt[..., None] * ob[:, t, :, None, :]
        qb[:, t] = scale * (new * ob[:, t, :, None, :]).sum(3)
        ub = (Sb * kt[..., None]).sum(2)
        pb = -bt * ub
        kb[:, t] = (Sb * u[:, :, None, :]).sum(3) + a * (old * pb[:, :, None, :]).sum(3)
        vb[:, t], bb[:, t] = -pb, (ub * r).sum(-1)
        gb[:, t] = a[..., 0] * (Sb * old).sum((2, 3)) + (pb * p).sum(-1)
        Sb = a[..., None] * (Sb + kt[..., None] * pb[:, :, None, :])
        states[t] = None
    return qb, kb, vb, gb, bb, Sb


def exact(case, seed):
    kind, s = case["kind"], prepare(case, seed)
    D = lambda n: s[n].double()  # noqa: E731
    if kind in ("norm", "norm_train"):
        x, w = D("x"), D("weight")
        n = x.shape[1]
        mean = x.sum(1, keepdim=True) / n
        sd = (((x - mean) ** 2).sum(1, keepdim=True) / n + EPS).sqrt()
        h = (x - mean) / sd
        out = {"y": h * w + D("bias")}
        if kind == "norm_train":  # d y_i / d x_j = w_i ((i == j) - 1/n - h_i h_j / n) / sd
            yb = D("y_bar")
            out["x_bar"] = (yb * w - ((yb * w).sum(1, keepdim=True) + h * (yb * w * h).sum(1, keepdim=True)) / n) / sd
            out["weight_bar"], out["bias_bar"] = (yb * h).sum(0), yb.sum(0)
        return out
    if kind == "clip":
        norm = math.sqrt(sum(float(x.double().pow(2).sum()) for x in s["grads"]))
        factor = min(1.0, MAX_NORM / norm) if norm else 1.0
        whole = {}
        for which, want in (("matrices", 0), ("vectors", 1)):
            count = s["case"]["tensors"]
            first = (count + 3) // 4
            mine = s["grads"][:first] if want == 0 else s["grads"][first:]
            whole[which] = torch.cat([x.double() for x in mine]) * factor if mine else torch.empty(0, dtype=torch.float64, device="cuda")
        return {"norm": torch.tensor(norm, dtype=torch.float64, device="cuda"), **whole}
    group = case["hv"] // case["hk"]
    wide = lambda n: D(n).repeat_interleave(group, -2)  # noqa: E731
    x = [wide("q"), wide("k"), D("v"), D("g"), D("beta")]
    if kind == "step":
        at = s["slots"].long()
        o, S, _ = _exact_rule(*[y[:, None] for y in x], s["scale"], s["state"][at].double(), False)
        state = D("state")
        state[at] = S
        return {"o": o[:, 0], "state": state}
    if kind == "forward" and s["offsets"] is not None:
        ends = _lengths(case["batch"], case["tokens"]).tolist()
        parts = [_exact_rule(*[y[:, a:z] for y in x], s["scale"], s["initial_state"][i:i + 1].double(), False)
                 for i, (a, z) in enumerate(zip(ends[:-1], ends[1:]))]
        return {"o": torch.cat([p[0] for p in parts], 1), "state": torch.cat([p[1] for p in parts])}
    o, S, states = _exact_rule(*x, s["scale"], D("initial_state"), kind == "train")
    out = {"o": o, "state": S}
    if kind == "train":
        bars = list(_exact_backward(*x, s["scale"], states, D("o_bar"), D("state_bar")))
        for i in (0, 1):  # a key head's gradient: the sum over the value heads that read it
            bars[i] = bars[i].unflatten(2, (-1, group)).sum(3)
        out.update(zip(("q_bar", "k_bar", "v_bar", "g_bar", "beta_bar", "initial_state_bar"), bars))
    return out


# -----------------------------------------------------------------------------------------------
# what a pass cannot do without
# -----------------------------------------------------------------------------------------------
def work(case):
    """Inputs read once, outputs written once; operations of the recurrence as it is written (per token and value head 6 dk dv forward:
    the answer for the key, the update, the answer for the query; twice that for the gradient).  The norm of the gradients is known only
    when all of them were read, so the scaling reads them again."""
    kind, e = case["kind"], SIZE[case["dtype"]]
    if kind in ("norm", "norm_train"):
        rows, n = case["rows"], case["n"]
        if kind == "norm":
            return {"bytes": e * (2 * rows * n + 2 * n), "flops": 8 * rows * n}
        return {"bytes": e * (5 * rows * n + 5 * n) + 16 * rows, "flops": 22 * rows * n}
    if kind == "clip":
        sizes = _sizes(case["tensors"], case["elements"])
        m, v = sum(sizes[::4]), sum(sizes) - sum(sizes[::4])
        return {"bytes": 3 * (e * m + 4 * v) + 4, "flops": 3 * (m + v)}
    b, hk, hv, dk, dv = (case[x] for x in ("batch", "hk", "hv", "dk", "dv"))
    tokens = b if kind == "step" else case["tokens"] * (1 if case["packed"] else b)
    states = 2 * 4 * b * hv * dk * dv
    bytes_ = tokens * (e * (2 * hk * dk + 2 * hv * dv) + 8 * hv) + states
    flops = tokens * hv * 6 * dk * dv
    if kind == "train":
        bytes_ += tokens * (e * (4 * hk * dk + 3 * hv * dv) + 16 * hv) + states + 4 * b * hv * dk * dv
        flops *= 3
    return {"bytes": bytes_, "flops": flops}
