"""The example that runs the training operators and the compressor together: its gradient against automatic
differentiation in binary64, and a short run that has to learn while it sends less than full gradients."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_worker_gradient_agrees_with_automatic_differentiation():
    import finetune as F

    model = F.Model(vocab=37, width=24, hidden=40, blocks=2, tokens=400, dtype=torch.float32, p=0.0)
    flat = model.initial(3)
    worker = F.Worker(model, pairs=5, steps=9, seed=1)
    worker.reference(model, model.initial(4))
    row = torch.empty_like(flat)
    worker.preference_gradient(model, flat, row, step=0)

    x = flat.double().requires_grad_(True)
    P = model.views(x)
    s = y = None
    for k in range(model.blocks + 1):
        branch = P["E"][worker.inputs] if k == 0 else (y @ P[f"W1_{k}"]).relu() @ P[f"W2_{k}"]
        s = branch if s is None else s + branch
        y = torch.nn.functional.layer_norm(s, (model.width,), P[f"w{k}"], P[f"b{k}"], 1e-5)
    logp = torch.log_softmax(y @ P["E"].t(), 1).gather(1, worker.labels[:, None])[:, 0]
    diff = ((logp - worker.ref.double()) * worker.mask).view(2, worker.pairs, -1).sum(2)
    loss = torch.nn.functional.softplus(-0.5 * (diff[0] - diff[1])).mean()
    (want,) = torch.autograd.grad(loss, x)
    assert abs(worker.loss.item() - loss.item()) < 1e-5
    # float32 products over up to 90 rows and 40 columns: a few hundred roundings of 6e-8 against the gradient's own size
    torch.backends.cuda.matmul.allow_tf32 = False
    assert (row.double() - want).norm() < 1e-4 * want.norm()


def test_short_run_learns_and_sends_less():
    import finetune as F

    h = F.train(steps=40, policy_steps=4, log=lambda *_: None)
    assert h["loss"][39] < 0.5 * h["loss"][0] and h["margin"][-1] > 1.0
    assert all(v == v for v in h["loss"]) and all(0.0 <= r <= 1.0 for r in h["reward"])
    assert h["bits"] < 0.8 * h["full"]
