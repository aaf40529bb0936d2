"""Workers fine-tune a small language model with compressed gradients.

n workers hold pairs of answers (preferred, rejected).  Each computes the gradient of the preference loss of its own pairs
with the training operators between ordinary matrix products, the gradients go as rows X_i through the adaptive
compressor (AdaCGD.compress: EF21/3PC difference, level choice, estimator update, server mean), and the server's mean moves
the parameters.  A second phase lets the workers sample answers and goes on with the clipped policy loss.

    python examples/finetune.py [--steps 60] [--policy-steps 20] [--workers 4] [--heads 0]

The model is a residual network: s_0 = drop(E[token]), y_0 = norm(s_0), then per block
s = s + drop(relu(y W1) W2), y = norm(s), and logits y E^T.  Without heads it sees the current token only; with heads each block has
a causal attention in front, s = s + drop(attention(q, k, v) Wo) with q, k, v = y Wqkv, queries and keys normed and rotated by head.  Data is synthetic: preferred answers follow
next = (5 token + 3) mod vocab, rejected ones are random.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2211_00188_b200 as adacgd  # noqa: E402


class Model:
    """Parameters as views of one flat vector; `run` fills a flat gradient of the same layout."""

    def __init__(self, vocab, width, hidden, blocks, tokens, dtype=torch.bfloat16, p=0.1, device="cuda", heads=0, key_heads=1):
        self.vocab, self.width, self.hidden, self.p, self.dtype = vocab, width, hidden, p, dtype
        self.heads, self.blocks = heads, blocks * (2 if heads else 1)
        self.attends = lambda k: heads > 0 and k % 2 == 1          # blocks 1, 3, ... where there are heads
        shapes = [("E", (vocab, width)), ("w0", (width,)), ("b0", (width,))]
        if heads:
            self.dim, self.keys = width // heads, width // heads * key_heads
            self.freq = 10000.0 ** (-torch.arange(self.dim // 2, device=device, dtype=torch.float32) / (self.dim // 2))
        for k in range(1, self.blocks + 1):
            if self.attends(k):
                shapes += [(f"Wqkv_{k}", (width, width + 2 * self.keys)), (f"Wo_{k}", (width, width)), (f"wq{k}", (self.dim,)), (f"wk{k}", (self.dim,))]
            else:
                shapes += [(f"W1_{k}", (width, hidden)), (f"W2_{k}", (hidden, width))]
            shapes += [(f"w{k}", (width,)), (f"b{k}", (width,))]
        self.shapes, self.size = shapes, sum(torch.Size(s).numel() for _, s in shapes)
        self.device = device
        self.ops = adacgd.TrainingOps(tokens, width)

    def views(self, flat):
        out, at = {}, 0
        for name, shape in self.shapes:
            n = torch.Size(shape).numel()
            out[name] = flat[at:at + n].view(shape)
            at += n
        return out

    def initial(self, seed):
        g = torch.Generator(device=self.device).manual_seed(seed)
        flat = torch.empty(self.size, device=self.device)
        for name, v in self.views(flat).items():
            if v.dim() == 2:
                v.normal_(0, 0.5 * v.shape[0 if name != "E" else 1] ** -0.5, generator=g)
            else:
                v.fill_(1.0 if name[0] == "w" else 0.0)
        return flat

    def forward(self, flat, tokens, p, seed, sequences=1):
        """Logits and what the backward pass needs.  `seed` decides the dropout masks; the block's number is the offset.  Tokens are
        those of `sequences` sequences of one length."""
        P = {k: v.to(self.dtype) for k, v in self.views(flat).items()}
        n = tokens.numel()
        new = lambda cols=self.width: torch.empty(n, cols, dtype=self.dtype, device=self.device)  # noqa: E731
        kept = []
        branch, s = new(), None
        self.ops.embedding(tokens, P["E"], branch)
        position = torch.arange(n, device=self.device) % (n // sequences)
        for k in range(self.blocks + 1):
            c = {}
            if self.attends(k):
                w, h = self.width, self.keys
                c["qkv"] = kept[-1]["y"] @ P[f"Wqkv_{k}"]
                c["q"], c["k"], c["out"] = new(), new(h), new()
                c["lse"] = torch.empty(self.heads, n, device=self.device)
                self.ops.qk_norm(c["qkv"][:, :w], c["qkv"][:, w:w + h], c["q"], c["k"], position, self.freq, head_dim=self.dim, q_weight=P[f"wq{k}"],
                                 k_weight=P[f"wk{k}"])
                self.ops.attention(c["q"], c["k"], c["qkv"][:, w + h:], c["out"], heads=self.heads, lse=c["lse"], sequences=sequences)
                branch = c["out"] @ P[f"Wo_{k}"]
            elif k:
                c["a"] = kept[-1]["y"] @ P[f"W1_{k}"]
                c["g"] = c["a"].relu()
                branch = c["g"] @ P[f"W2_{k}"]
            y, total = new(), new()
            mean, rstd = torch.empty(n, device=self.device), torch.empty(n, device=self.device)
            self.ops.layer_norm(branch, y, weight=P[f"w{k}"], bias=P[f"b{k}"], residual=s, sum_out=total, mean=mean, rstd=rstd, p=p,
                                seed=seed, offset=k)
            kept.append(dict(c, y=y, s=total, mean=mean, rstd=rstd))
            s = total
        return kept[-1]["y"] @ P["E"].t(), (P, kept, tokens, p, seed, sequences, position)

    def backward(self, dlogits, state, flat_grad, scale):
        """Gradient of the loss into flat_grad, from scale * dloss/dlogits."""
        P, kept, tokens, p, seed, sequences, position = state
        G = self.views(flat_grad)
        dy, ds = dlogits @ P["E"], None
        G["E"].copy_(dlogits.t() @ kept[-1]["y"])
        for k in range(self.blocks, -1, -1):
            c = kept[k]
            branch, stream = torch.empty_like(dy), torch.empty_like(dy)
            dw, db = torch.empty_like(P[f"w{k}"]), torch.empty_like(P[f"w{k}"])
            self.ops.layer_norm_backward(dy, c["s"], c["mean"], c["rstd"], branch, weight=P[f"w{k}"], dweight=dw, dbias=db, dsum=ds,
                                         dresidual=stream, p=p, seed=seed, offset=k)
            G[f"w{k}"].copy_(dw)
            G[f"b{k}"].copy_(db)
            if self.attends(k):
                w, h = self.width, self.keys
                G[f"Wo_{k}"].copy_(c["out"].t() @ branch)
                dout, dqkv = branch @ P[f"Wo_{k}"].t(), torch.empty_like(c["qkv"])
                dq, dk, dot = torch.empty_like(c["q"]), torch.empty_like(c["k"]), torch.empty_like(c["lse"])
                self.ops.attention_backward(dout, c["q"], c["k"], c["qkv"][:, w + h:], c["out"], c["lse"], dot, dq, dk, dqkv[:, w + h:],
                                            heads=self.heads, sequences=sequences)
                dwq, dwk = torch.empty_like(P[f"wq{k}"]), torch.empty_like(P[f"wk{k}"])
                self.ops.qk_norm_backward(dq, dk, c["qkv"][:, :w], c["qkv"][:, w:w + h], dqkv[:, :w], dqkv[:, w:w + h], position, self.freq,
                                          head_dim=self.dim, q_weight=P[f"wq{k}"], k_weight=P[f"wk{k}"], dq_weight=dwq, dk_weight=dwk)
                G[f"wq{k}"].copy_(dwq)
                G[f"wk{k}"].copy_(dwk)
                G[f"Wqkv_{k}"].copy_(kept[k - 1]["y"].t() @ dqkv)
                dy = dqkv @ P[f"Wqkv_{k}"].t()
                ds = stream
            elif k:
                G[f"W2_{k}"].copy_(c["g"].t() @ branch)
                da = (branch @ P[f"W2_{k}"].t()) * (c["a"] > 0)
                G[f"W1_{k}"].copy_(kept[k - 1]["y"].t() @ da)
                dy = da @ P[f"W1_{k}"].t()
                ds = stream
            else:
                self.ops.embedding_backward(tokens, branch, G["E"], base=G["E"])
        flat_grad.div_(scale)


def answers(gen, pairs, steps, vocab, follow, device):
    """Token sequences [pairs, steps + 1]: following the rule, or random."""
    t = torch.randint(vocab, (pairs, steps + 1), generator=gen, device=device)
    if follow:
        for k in range(steps):
            t[:, k + 1] = (5 * t[:, k] + 3) % vocab
    return t


class Worker:
    def __init__(self, model, pairs, steps, seed):
        dev = model.device
        gen = torch.Generator(device=dev).manual_seed(seed)
        good, bad = answers(gen, pairs, steps, model.vocab, True, dev), answers(gen, pairs, steps, model.vocab, False, dev)
        bad[:, 0] = good[:, 0]                                       # the same prompt
        both = torch.cat([good, bad])
        self.inputs, self.labels = both[:, :-1].reshape(-1), both[:, 1:].reshape(-1)
        length = torch.randint(steps // 2, steps + 1, (2 * pairs, 1), generator=gen, device=dev)   # answers of uneven lengths
        self.mask = (torch.arange(steps, device=dev)[None] < length).reshape(-1)
        self.pairs, self.steps, self.seed, self.gen = pairs, steps, seed, gen
        self.ref = torch.empty(self.labels.numel(), device=dev)
        self.loss, self.margin = torch.empty(1, device=dev), torch.empty(pairs, device=dev)

    def reference(self, model, flat):
        logits, _ = model.forward(flat, self.inputs, 0.0, 0, 2 * self.pairs)
        model.ops.token_logp(logits, self.labels, self.ref, mask=self.mask)

    def preference_gradient(self, model, flat, row, step, scale=1024.0):
        logits, state = model.forward(flat, self.inputs, model.p, self.seed * 1000003 + step, 2 * self.pairs)
        model.ops.preference_loss(logits, self.labels, self.ref, self.loss, logits, mask=self.mask, sequences=2 * self.pairs, beta=0.5,
                                  grad_scale=scale, margin=self.margin)          # the gradient takes the logits' place
        model.backward(logits, state, row, scale)

    def policy_gradient(self, model, flat, row, step, scale=1024.0):
        """Samples an answer to every prompt, rewards rule-following tokens, one clipped step."""
        dev, n = model.device, 2 * self.pairs
        tokens = torch.empty(n, self.steps + 1, dtype=torch.long, device=dev)
        tokens[:, 0] = self.inputs.view(n, self.steps)[:, 0]
        for k in range(self.steps):
            seen = tokens[:, 0 if model.heads else k:k + 1]         # without heads the last token is all that counts
            logits, _ = model.forward(flat, seen.contiguous().view(-1), 0.0, 0, n)
            logits = logits.view(n, seen.shape[1], -1)[:, -1]
            tokens[:, k + 1] = torch.multinomial(logits.float().softmax(1), 1, generator=self.gen)[:, 0]
        inputs, labels = tokens[:, :-1].reshape(-1), tokens[:, 1:].reshape(-1)
        reward = (labels == (5 * inputs + 3) % model.vocab).float()
        advantage = (reward - reward.mean()) / (reward.std() + 1e-3)
        old, ref = torch.empty_like(advantage), torch.empty_like(advantage)
        logits, state = model.forward(flat, inputs, 0.0, 0, n)
        model.ops.token_logp(logits, labels, old)
        ref_logits, _ = model.forward(self.start, inputs, 0.0, 0, n)
        model.ops.token_logp(ref_logits, labels, ref)
        model.ops.policy_loss(logits, labels, old, advantage, self.loss, logits, sequences=n, ref_logp=ref, kl_beta=0.01,
                              per_sequence=True, grad_scale=scale)
        model.backward(logits, state, row, scale)
        return reward.mean()


def train(steps=60, policy_steps=20, workers=4, vocab=96, width=64, hidden=128, blocks=2, pairs=16, length=24, gamma=0.1, policy_gamma=0.4, zeta=1.0,
          seed=0, dtype=torch.bfloat16, log=print, heads=0):
    model = Model(vocab, width, hidden, blocks, 2 * pairs * length, dtype, heads=heads)
    crew = [Worker(model, pairs, length, 100 * seed + i) for i in range(workers)]
    flat = model.initial(seed)
    d = model.size
    ladder = adacgd.protocol.topk_ladder(d, (0.01, 0.1, 0.5))
    engine = adacgd.AdaCGD(workers, d, ladder, zeta)
    X, Y, G = (torch.zeros(workers, d, device=model.device) for _ in range(3))
    mean = torch.empty(d, device=model.device)
    level = torch.zeros(workers, dtype=torch.int32, device=model.device)
    bits = torch.zeros(workers, dtype=torch.int64, device=model.device)
    for w in crew:
        w.reference(model, flat)
    history = {"loss": [], "margin": [], "reward": [], "bits": 0, "levels": []}
    for step in range(steps + policy_steps):
        phase = "preference" if step < steps else "policy"
        if step == steps:
            for w in crew:
                w.start = flat.clone()
        rewards = []
        for i, w in enumerate(crew):
            if phase == "preference":
                w.preference_gradient(model, flat, X[i], step)
            else:
                rewards.append(w.policy_gradient(model, flat, X[i], step))
        if step == 0:
            G.copy_(X)                                    # g_i^0 = grad f_i(x^0), sent in full
            Y.copy_(X)
            mean.copy_(X.mean(0))
            sent = workers * adacgd.message_bits((adacgd.TOPK, d), d)
        else:
            engine.compress(X, G, Y, mean_out=mean, level=level, bits=bits)
            X, Y = Y, X                                   # this step's gradients are the next step's y
            sent = int(bits.sum().item())
        flat.sub_(mean, alpha=gamma if phase == "preference" else policy_gamma)
        history["bits"] += sent
        history["levels"].append(level.tolist())
        history["loss"].append(float(torch.stack([w.loss for w in crew]).mean()))
        if phase == "preference":
            history["margin"].append(float(torch.stack([w.margin for w in crew]).mean()))
            note = f"margin {history['margin'][-1]:8.3f}"
        else:
            history["reward"].append(float(torch.stack(rewards).mean()))
            note = f"reward {history['reward'][-1]:8.3f}"
        if step % 10 == 0 or step == steps + policy_steps - 1:
            log(f"{phase:10s} step {step:3d}  loss {history['loss'][-1]:8.4f}  {note}  levels {history['levels'][-1]}  sent {sent / 8e3:9.1f} kB")
    history["full"] = workers * 32 * d * (steps + policy_steps)
    log(f"sent {history['bits'] / 8e6:.2f} MB in all; full gradients would be {history['full'] / 8e6:.2f} MB")
    return history


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--policy-steps", type=int, default=20)
    p.add_argument("--workers", type=int, default=4)
    p.add_argument("--heads", type=int, default=0, help="attention heads of a block (0: the model sees the current token only)")
    a = p.parse_args()
    train(a.steps, a.policy_steps, a.workers, heads=a.heads)
