"""The operators together, as the example uses them: training lowers the loss far below chance's, the gradient of the whole model agrees with differences of
its loss, and serving by single tokens gives what whole sequences give."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
KEYS, VALUES = 32, 8


def _model(dtype, seed=0):
    import recall

    torch.manual_seed(seed)
    return recall, recall.Recall(KEYS, VALUES, 64, 2, dtype=dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_training_learns_to_recall(dtype):
    recall, model = _model(dtype)
    losses = recall.train(model, 120, 32, 12, 20, KEYS, VALUES)
    assert math.log(VALUES) * 0.5 < losses[0]
    assert sum(losses[-10:]) / 10 < 0.5 * math.log(VALUES)  # chance gives log(VALUES)
    right, _, _ = recall.serve(model, 32, 12, 20, KEYS, VALUES)
    assert right > 0.6  # chance: 1 / VALUES


def test_steps_after_a_prompt_equal_whole_sequences():
    """in float32 to its rounding: the logits are of order 1 to 10, some hundred sums of 64 to 128 terms lie between: 1e-3 is far above their rounding
    (1e-7 each, times the growth over two layers) and far below what a lost or doubled token would change"""
    recall, model = _model(torch.float32, seed=3)
    with torch.no_grad():
        _, steps, whole = recall.serve(model, 5, 13, 9, KEYS, VALUES)
    assert (steps - whole).abs().max().item() < 1e-3


def test_gradient_of_the_model_against_differences():
    """The derivative along the gradient's own direction is its norm; central differences of the float32 loss (about 2, rounding 2e-7, step 1e-2
    along a unit vector) are good to 2e-5 and, with third derivatives of order 10, to 2e-4; the norm is of order 1."""
    recall, model = _model(torch.float32, seed=4)
    parameters = list(model.parameters())
    key, value, target = recall.sequences(8, 12, 20, KEYS, VALUES, torch.Generator("cuda").manual_seed(5))

    def loss():
        return torch.nn.functional.cross_entropy(model(key, value)[:, 12:].double().reshape(-1, VALUES), target.reshape(-1))

    loss().backward()
    grads = [p.grad.clone() for p in parameters]
    norm = recall.la.clip_gradients([g.clone() for g in grads], 1e30)
    values = []
    for sign in (1, -1):
        with torch.no_grad():
            for p, g in zip(parameters, grads):
                p.add_(g, alpha=sign * 1e-2 / norm.item())
            values.append(loss().item())
            for p, g in zip(parameters, grads):
                p.sub_(g, alpha=sign * 1e-2 / norm.item())
    assert abs((values[0] - values[1]) / 2e-2 - norm.item()) < 0.01 * norm.item()
