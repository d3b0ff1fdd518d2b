"""A recurrent sequence model that learns to recall: trained with the gated delta rule, layer norm and clipped gradients, then served token by token.

Every token of a sequence's first part gives a key and a value; every token of the rest gives one of those keys, and the value that came with it is to
be predicted.  A block is  x + W_o delta_rule(W layer_norm(x)):  one product gives q, k, v and the two gates of all heads, and v goes into the
operator as the view of it that it is.  Serving runs the prompt with delta_rule, keeps the states, and answers the queries with delta_rule_step.

    python examples/recall.py [--steps 300] [--batch 32] [--pairs 24] [--width 128] [--layers 2]
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1710_08717_amd as la  # noqa: E402


class LayerNorm(torch.autograd.Function):
    """la.layer_norm with its backward pass"""

    @staticmethod
    def forward(ctx, x, weight, bias):
        y, mean, rstd = la.layer_norm(x, weight, bias, want_stats=True)
        ctx.save_for_backward(x, mean, rstd, weight)
        return y

    @staticmethod
    def backward(ctx, y_bar):
        x, mean, rstd, weight = ctx.saved_tensors
        return la.layer_norm_backward(x, y_bar.contiguous(), mean, rstd, weight)


class DeltaRule(torch.autograd.Function):
    """la.delta_rule with its backward pass; what the forward pass keeps goes with it"""

    @staticmethod
    def forward(ctx, q, k, v, g, beta):
        o, _, kept = la.delta_rule(q, k, v, g, beta, keep=True)
        ctx.save_for_backward(q, k, v, g, beta, kept)
        return o

    @staticmethod
    def backward(ctx, o_bar):
        *inputs, kept = ctx.saved_tensors
        return la.delta_rule_backward(*inputs, o_bar.contiguous(), saved=kept)[:5]


def product(x, weight):
    """x weight^T as one matrix product over all tokens"""
    return (x.flatten(0, -2) @ weight.to(x.dtype).T).unflatten(0, x.shape[:-1])


class Block(torch.nn.Module):
    def __init__(self, width, key_heads, value_heads, head):
        super().__init__()
        self.sizes = (key_heads * head, key_heads * head, value_heads * head, value_heads, value_heads)
        self.key_heads, self.value_heads, self.head = key_heads, value_heads, head
        self.weight, self.bias = torch.nn.Parameter(torch.ones(width)), torch.nn.Parameter(torch.zeros(width))
        self.project = torch.nn.Parameter(torch.randn(sum(self.sizes), width) * width ** -0.5)
        self.out = torch.nn.Parameter(torch.randn(width, value_heads * head) * (value_heads * head) ** -0.5)
        self.decay = torch.nn.Parameter(torch.full((value_heads,), -4.0))  # of a state at the start: exp(-softplus(-4)), about 0.98 a token

    def inputs(self, y):
        """q, k, v, g, beta of the normalised tokens; the last axis of y is the width"""
        lead = y.shape[:-1]
        q, k, v, a, b = product(y, self.project).split(self.sizes, dim=-1)
        q, k = (F.normalize(x.reshape(*lead, self.key_heads, self.head).float(), dim=-1).to(y.dtype) for x in (q, k))
        v = v.unflatten(-1, (self.value_heads, self.head))  # a view: its tokens lie a row of the product apart
        return q, k, v, -F.softplus(a.float() + self.decay), torch.sigmoid(b.float())

    def forward(self, x):
        o = DeltaRule.apply(*self.inputs(LayerNorm.apply(x, self.weight, self.bias)))
        return x + product(o.flatten(-2), self.out)

    @torch.no_grad()
    def prompt(self, x):
        """the block of a whole prompt, and the state after it"""
        q, k, v, g, beta = self.inputs(la.layer_norm(x, self.weight, self.bias)[0])
        o, state, _ = la.delta_rule(q, k, v, g, beta, want_state=True)
        return x + product(o.flatten(-2), self.out), state

    @torch.no_grad()
    def step(self, x, state):
        """one token of every sequence; the state is updated in place"""
        q, k, v, g, beta = self.inputs(la.layer_norm(x, self.weight, self.bias)[0])
        o = la.delta_rule_step(q, k, v, g, beta, state)
        return x + product(o.flatten(-2), self.out)


class Recall(torch.nn.Module):
    def __init__(self, keys, values, width, layers, key_heads=1, value_heads=2, head=64, dtype=torch.bfloat16):
        super().__init__()
        self.dtype = dtype
        self.keys, self.values = torch.nn.Parameter(torch.randn(keys, width)), torch.nn.Parameter(torch.randn(values + 1, width))
        self.blocks = torch.nn.ModuleList(Block(width, key_heads, value_heads, head) for _ in range(layers))
        self.weight, self.bias = torch.nn.Parameter(torch.ones(width)), torch.nn.Parameter(torch.zeros(width))
        self.answer = torch.nn.Parameter(torch.randn(values, width) * width ** -0.5)

    def embed(self, key, value):
        return (self.keys[key] + self.values[value]).to(self.dtype)

    def logits(self, y):
        return product(y, self.answer).float()

    def forward(self, key, value):
        x = self.embed(key, value)
        for block in self.blocks:
            x = block(x)
        return self.logits(LayerNorm.apply(x, self.weight, self.bias))

    @torch.no_grad()
    def prompt(self, key, value):
        x, states = self.embed(key, value), []
        for block in self.blocks:
            x, state = block.prompt(x)
            states.append(state)
        return self.logits(la.layer_norm(x, self.weight, self.bias)[0]), states

    @torch.no_grad()
    def step(self, key, value, states):
        x = self.embed(key, value)
        for block, state in zip(self.blocks, states):
            x = block.step(x, state)
        return self.logits(la.layer_norm(x, self.weight, self.bias)[0])


def sequences(batch, pairs, queries, keys, values, generator):
    """(keys, values, targets) of `pairs` tokens that give a value and `queries` that ask for one; value `values` stands for none"""
    order = torch.rand(batch, keys, generator=generator, device="cuda").argsort(1)[:, :pairs]
    given = torch.randint(values, (batch, pairs), generator=generator, device="cuda")
    ask = torch.randint(pairs, (batch, queries), generator=generator, device="cuda")
    key = torch.cat([order, order.gather(1, ask)], 1)
    value = torch.cat([given, torch.full_like(ask, values)], 1)
    return key, value, given.gather(1, ask)


def train(model, steps, batch, pairs, queries, keys, values, rate=3e-3, max_norm=1.0, seed=0, report=None):
    """The losses of `steps` training steps"""
    generator = torch.Generator("cuda").manual_seed(seed)
    parameters = list(model.parameters())
    rule = torch.optim.Adam(parameters, lr=rate)
    losses = []
    for step in range(steps):
        key, value, target = sequences(batch, pairs, queries, keys, values, generator)
        logits = model(key, value)[:, pairs:]
        loss = F.cross_entropy(logits.reshape(-1, values), target.reshape(-1))
        rule.zero_grad()
        loss.backward()
        norm = la.clip_gradients([p.grad for p in parameters], max_norm)
        rule.step()
        losses.append(loss.detach())
        if report and (step + 1) % report == 0:
            right = (logits.argmax(-1) == target).float().mean()
            print(f"step {step + 1}: loss {loss.item():.4f}, {100 * right.item():.1f} % right, gradient norm {norm.item():.3f}", flush=True)
    return torch.stack(losses).tolist()


def serve(model, batch, pairs, queries, keys, values, seed=1):
    """Answers one query at a time after the prompt: the share of right ones, and the logits of steps and of whole sequences"""
    key, value, target = sequences(batch, pairs, queries, keys, values, torch.Generator("cuda").manual_seed(seed))
    _, states = model.prompt(key[:, :pairs], value[:, :pairs])
    steps = torch.stack([model.step(key[:, t], value[:, t], states) for t in range(pairs, pairs + queries)], 1)
    whole = model.prompt(key, value)[0][:, pairs:]
    return (steps.argmax(-1) == target).float().mean().item(), steps, whole


def main():
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=300)
    parser.add_argument("--batch", type=int, default=32)
    parser.add_argument("--pairs", type=int, default=24)
    parser.add_argument("--queries", type=int, default=40)
    parser.add_argument("--keys", type=int, default=64)
    parser.add_argument("--values", type=int, default=16)
    parser.add_argument("--width", type=int, default=128)
    parser.add_argument("--layers", type=int, default=2)
    a = parser.parse_args()
    torch.manual_seed(0)
    model = Recall(a.keys, a.values, a.width, a.layers).cuda()
    train(model, a.steps, a.batch, a.pairs, a.queries, a.keys, a.values, report=max(1, a.steps // 10))
    right, steps, whole = serve(model, a.batch, a.pairs, a.queries, a.keys, a.values)
    print(f"served token by token: {100 * right:.1f} % right; largest difference from whole sequences {(steps - whole).abs().max().item():.3g}")


if __name__ == "__main__":
    main()
