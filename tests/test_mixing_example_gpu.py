"""The example with attention blocks: its gradient against automatic differentiation in binary64, and a run of it."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def reference_gradient(model, flat, worker):
    """Gradient and loss of the worker's preference loss, without the operators."""
    x = flat.double().requires_grad_(True)
    P = model.views(x)
    n, w, seqs = worker.inputs.numel(), model.width, 2 * worker.pairs
    steps, d = n // seqs, model.dim
    position = torch.arange(steps, device=flat.device).double()
    angle = position[:, None] * model.freq.double()
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    hidden = torch.triu(torch.full((steps, steps), float("-inf"), device=flat.device, dtype=torch.float64), 1)

    def heads(t, weight):
        t = t.view(seqs, steps, -1, d)
        t = t / (t.square().mean(-1, keepdim=True) + 1e-6).sqrt() * weight
        a, b = t[..., :d // 2], t[..., d // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    s = y = None
    for k in range(model.blocks + 1):
        if model.attends(k):
            qkv = y @ P[f"Wqkv_{k}"]
            q, kk = heads(qkv[:, :w], P[f"wq{k}"]), heads(qkv[:, w:w + model.keys], P[f"wk{k}"])
            v = qkv[:, w + model.keys:].view(seqs, steps, -1, d)
            share = model.heads // kk.shape[2]
            kk, v = kk.repeat_interleave(share, 2), v.repeat_interleave(share, 2)
            p = torch.softmax(torch.einsum("sihd,sjhd->shij", q, kk) * d ** -0.5 + hidden, -1)
            branch = torch.einsum("shij,sjhd->sihd", p, v).reshape(n, w) @ P[f"Wo_{k}"]
        else:
            branch = P["E"][worker.inputs] if k == 0 else (y @ P[f"W1_{k}"]).relu() @ P[f"W2_{k}"]
        s = branch if s is None else s + branch
        y = torch.nn.functional.layer_norm(s, (w,), P[f"w{k}"], P[f"b{k}"], 1e-5)
    logp = torch.log_softmax(y @ P["E"].t(), 1).gather(1, worker.labels[:, None])[:, 0]
    diff = ((logp - worker.ref.double()) * worker.mask).view(2, worker.pairs, -1).sum(2)
    loss = torch.nn.functional.softplus(-0.5 * (diff[0] - diff[1])).mean()
    return torch.autograd.grad(loss, x)[0], loss.item()


@pytest.mark.parametrize("dtype,heads,steps", [(torch.float32, 2, 9), (torch.float32, 4, 70), (torch.bfloat16, 4, 70), (torch.float16, 2, 140)])
def test_worker_gradient_agrees_with_automatic_differentiation(dtype, heads, steps):
    import finetune as F

    torch.backends.cuda.matmul.allow_tf32 = False
    model = F.Model(vocab=37, width=64, hidden=40, blocks=2, tokens=10 * steps, dtype=dtype, p=0.0, heads=heads)
    flat = model.initial(3)
    worker = F.Worker(model, pairs=5, steps=steps, seed=1)
    worker.reference(model, model.initial(4))
    row = torch.empty_like(flat)
    worker.preference_gradient(model, flat, row, step=0, scale=64.0)
    want, loss = reference_gradient(model, flat, worker)
    # float32: a few hundred roundings of 6e-8 against the gradient's own size.  The 16-bit types round the parameters and the results of some
    # thirty steps forwards and backwards, each by at most eps / 2 of its size and all by chance: eps / 2 sqrt(30) < 3 eps, and the loss's
    # sums over an answer's tokens pass the errors of its log-probabilities on: as much again for each of the two.
    limit = 1e-4 if dtype == torch.float32 else 12 * torch.finfo(dtype).eps
    assert (row.double() - want).norm() < limit * want.norm()
    again = torch.empty_like(row)
    worker.preference_gradient(model, flat, again, step=0, scale=64.0)
    if dtype == torch.float32:
        assert (row - again).norm() <= 1e-5 * row.norm()      # the products are a library's


def test_short_run_with_attention():
    import finetune as F

    h = F.train(steps=4, policy_steps=2, pairs=8, length=20, heads=2, log=lambda *_: None)
    assert len(h["loss"]) == 6 and all(v == v for v in h["loss"]) and all(0.0 <= r <= 1.0 for r in h["reward"])
