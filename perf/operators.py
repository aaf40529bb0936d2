"""Cases of the training operators: residual + dropout + layer norm with its backward pass, dropout alone, token
log-probabilities, and the two losses that start a fine-tuning worker's backward pass (preference loss over pairs of
answers, clipped policy loss with a KL term).

`run` computes an operator either in elementary torch operations in 32 bits (`own` false) or by the package's entry
points (`own` true).  Tokens are rows; a "vocab" is the length of a row of logits.
"""
import math

import torch

own = False

# One operator context serves a whole program: it is made for the largest shapes met here.
MAX_TOKENS = 1 << 17
MAX_COLS = 16384
_ops = None

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
LARGEST_NORM = 32768 * 8192      # elements of the largest listed norm and dropout cases
LARGEST_LOGITS = 4096 * 131072   # logits of the largest listed loss case


def listed():
    return [
        # one token of a model that answers: residual stream of 4096, no dropout; latency counts
        dict(name="norm_one_token", op="norm", rows=1, cols=4096, dtype="bf16", param="bf16", residual=True, p=0.0),
        # a training step's block, the largest: 32768 tokens of width 8192 with dropout on the branch
        dict(name="norm_wide", op="norm", rows=32768, cols=8192, dtype="bf16", param="bf16", residual=True, p=0.1),
        # plain layer norm of an odd width in 32 bits (a small encoder's head)
        dict(name="norm_backward_odd", op="norm_backward", rows=4099, cols=1001, dtype="f32", param="f32", residual=False, p=0.0),
        # the largest block's backward pass, weights kept in 32 bits
        dict(name="norm_backward_wide", op="norm_backward", rows=32768, cols=8192, dtype="bf16", param="f32", residual=True, p=0.1),
        # dropout on a small odd activation
        dict(name="dropout_small", op="dropout", rows=257, cols=1001, dtype="f32", residual=False, p=0.5),
        # dropout on the largest block
        dict(name="dropout_wide", op="dropout", rows=32768, cols=8192, dtype="bf16", residual=False, p=0.1),
        # scoring one short answer of eight tokens
        dict(name="logp_one_answer", op="logp", seqs=1, steps=8, vocab=32000, dtype="bf16"),
        # reference log-probabilities of a batch, odd vocabulary
        dict(name="logp_batch_odd", op="logp", seqs=16, steps=512, vocab=50001, dtype="bf16"),
        # four short pairs in 32 bits
        dict(name="preference_small", op="preference", seqs=8, steps=24, vocab=8000, dtype="f32", packed=False, smoothing=0.0),
        # four pairs of 512 tokens
        dict(name="preference_batch", op="preference", seqs=8, steps=512, vocab=32000, dtype="bf16", packed=False, smoothing=0.1),
        # sixteen short packed answers of uneven lengths, odd small vocabulary
        dict(name="policy_small_packed", op="policy", seqs=16, steps=33, vocab=1001, dtype="f16", packed=True, per_sequence=True),
        # the largest batch of logits
        dict(name="policy_wide", op="policy", seqs=8, steps=512, vocab=131072, dtype="bf16", packed=False, per_sequence=False),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _size(rng, low, high):
    """A size of [low, high], even over its logarithm: an odd number, eight times an odd number, or a power of two."""
    n = _log_uniform(rng, low, high)
    kind = rng.randrange(3)
    if kind == 0:
        n |= 1
    elif kind == 1:
        n = 8 * (max(1, n // 8) | 1)
    else:
        n = 1 << max(0, n.bit_length() - 1)
    return max(low, n if n <= high else 1 << (high.bit_length() - 1))


def draw(rng):
    op = rng.choice(("norm", "norm_backward", "dropout", "logp", "preference", "policy"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op in ("norm", "norm_backward", "dropout"):
        cols = _size(rng, 64, 16384)
        rows = _size(rng, 1, 65536)
        most = LARGEST_NORM * 2 // SIZE[dtype]
        while rows * cols > most:
            rows = max(1, rows // 2)
        case = dict(op=op, rows=rows, cols=cols, dtype=dtype, residual=rng.random() < 0.6,
                    p=rng.choice((0.0, 0.05, 0.1, 0.5)) if op != "dropout" else rng.choice((0.05, 0.1, 0.5)))
        if op != "dropout":
            case["param"] = rng.choice((dtype, "f32"))
        return case
    vocab = _size(rng, 500, 140000)
    steps = _size(rng, 1, 2048)
    seqs = 2 * _size(rng, 1, 32)
    most = LARGEST_LOGITS // SIZE[dtype]  # half the bytes of the largest listed batch
    while seqs * steps * vocab > most:
        if steps > 64:
            steps //= 2
        else:
            seqs = max(2, seqs // 4 * 2)
            steps = max(1, steps - steps // 4)
    case = dict(op=op, seqs=seqs, steps=steps, vocab=vocab, dtype=dtype)
    if op == "preference":
        case.update(packed=rng.random() < 0.5, smoothing=rng.choice((0.0, 0.1)))
    elif op == "policy":
        case.update(packed=rng.random() < 0.5, per_sequence=rng.random() < 0.5)
    return case


# ----------------------------------------------------------------------------- inputs

def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    state = {"case": case}
    dt = TYPES[case["dtype"]]

    def normal(*shape, scale=1.0, mean=0.0, dtype=torch.float32):
        t = torch.randn(*shape, generator=gen, device=dev, dtype=dtype)
        if scale != 1.0:
            t *= scale
        if mean != 0.0:
            t += mean
        return t

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device=dev)

    if case["op"] in ("norm", "norm_backward", "dropout"):
        rows, cols, p = case["rows"], case["cols"], case["p"]
        state["p"], state["seed"], state["offset"] = p, int(seed) * 7919 + 12345, int(seed) % 97
        if case["op"] == "dropout":
            state["x"] = normal(rows, cols, dtype=dt)
            state["residual"] = normal(rows, cols, dtype=dt) if case["residual"] else None
            state["y"] = torch.empty_like(state["x"])
            return state
        pt = TYPES[case["param"]]
        state["weight"] = normal(cols, scale=0.2, mean=1.0).to(pt)
        if case["op"] == "norm":
            state["bias"] = normal(cols, scale=0.2).to(pt)
            state["x"] = normal(rows, cols, dtype=dt)
            # a residual stream grows along the blocks and has a few large channels
            state["residual"] = (normal(rows, cols, scale=2.0, dtype=dt) + normal(cols, scale=0.5, dtype=dt)) if case["residual"] else None
            state["y"] = torch.empty_like(state["x"])
            state["sum"] = torch.empty_like(state["x"]) if case["residual"] or p > 0 else None
            state["mean"] = torch.empty(rows, device=dev)
            state["rstd"] = torch.empty(rows, device=dev)
            return state
        s = normal(rows, cols, scale=2.0, dtype=dt) + normal(cols, scale=0.5, dtype=dt)
        state["s"] = s
        mean, rstd = torch.empty(rows, device=dev), torch.empty(rows, device=dev)
        for a in range(0, rows, 4096):  # what the forward pass keeps, a few rows at a time
            b = s[a:a + 4096].float()
            mean[a:a + 4096] = b.mean(1)
            rstd[a:a + 4096] = ((b - b.mean(1, keepdim=True)).square().mean(1) + 1e-5).rsqrt()
        state["mean"], state["rstd"] = mean, rstd
        state["dy"] = normal(rows, cols, scale=0.1, dtype=dt)
        state["dsum"] = normal(rows, cols, scale=0.1, dtype=dt) if case["residual"] else None
        state["dx"] = torch.empty_like(s)
        state["dresidual"] = torch.empty_like(s) if case["residual"] and p > 0 else None
        state["dweight"] = torch.empty_like(state["weight"])
        state["dbias"] = torch.empty_like(state["weight"])
        return state

    seqs, steps, vocab = case["seqs"], case["steps"], case["vocab"]
    n = seqs * steps
    packed = case.get("packed", False)
    logits = normal(n, vocab, scale=2.0, dtype=dt)
    labels = torch.randint(vocab, (n,), generator=gen, device=dev)
    # the labelled entry stands out, as it does in a model that has learnt something
    logits.scatter_add_(1, labels[:, None], normal(n, 1, scale=3.0, mean=6.0).to(dt))
    # prompts are not counted, nor is the padding behind an answer: two thirds of the tokens are, on average
    pos = torch.arange(steps, device=dev)[None]
    first = (uniform(seqs, 1) * (steps / 3)).floor()
    last = steps - (uniform(seqs, 1) * (steps / 3)).floor()
    state["mask"] = ((pos >= first) & (pos < last)).reshape(n)
    state["start"] = None
    if packed:  # answers of uneven lengths, one behind the other
        cuts = torch.randint(n + 1, (seqs - 1,), generator=gen, device=dev).sort().values
        edge = torch.zeros(1, dtype=cuts.dtype, device=dev)
        state["start"] = torch.cat([edge, cuts, edge + n]).to(torch.int32)
    logp = torch.empty(n, device=dev)
    for a in range(0, n, 1024):
        b = logits[a:a + 1024].float()
        top = b.amax(1, keepdim=True)
        logp[a:a + 1024] = b.gather(1, labels[a:a + 1024, None])[:, 0] - top[:, 0] - (b - top).exp().sum(1).log()
    state["logits"], state["labels"] = logits, labels
    if case["op"] == "logp":
        state["logp"] = torch.empty(n, device=dev)
        return state
    state["dlogits"] = torch.empty_like(logits)
    state["loss"] = torch.empty(1, device=dev)
    if case["op"] == "preference":
        # the model has moved from its reference token by token, and a little further on some answers than on others
        drift = normal(seqs, scale=0.05)
        state["ref_logp"] = logp + normal(n, scale=0.25) + drift.repeat_interleave(steps)
        state["margin"] = torch.empty(seqs // 2, device=dev)
        state["seq_logp"] = torch.empty(seqs, device=dev)
        state["beta"], state["smoothing"] = 0.1, case["smoothing"]
        return state
    state["old_logp"] = logp + normal(n, scale=0.15)
    state["ref_logp"] = logp + normal(n, scale=0.25)
    state["advantages"] = normal(n)
    state["logp"] = torch.empty(n, device=dev)
    state["stats"] = torch.empty(3, device=dev)
    state["clip"], state["kl_beta"] = 0.2, 0.04
    return state


def _member(state):
    """[tokens, sequences]: 1 where the token belongs to the sequence."""
    n, seqs = state["labels"].numel(), state["case"]["seqs"]
    at = torch.arange(n, device=state["labels"].device)[:, None]
    if state["start"] is None:
        return (at // state["case"]["steps"] == torch.arange(seqs, device=at.device)[None]).float()
    start = state["start"].long()
    return ((at >= start[None, :-1]) & (at < start[None, 1:])).float()


def _sums(state, per_token):
    """The sum over each sequence's tokens."""
    if state["start"] is None:
        return per_token.view(state["case"]["seqs"], -1).sum(1)
    return (_member(state) * per_token[:, None]).sum(0)


# ----------------------------------------------------------------------------- the package's entry points

def _context():
    global _ops
    if _ops is None:
        import paper_2211_00188_b200 as adacgd
        _ops = adacgd.TrainingOps(MAX_TOKENS, MAX_COLS)
    return _ops


def _run_own(state):
    ops, case = _context(), state["case"]
    op = case["op"]
    if op == "norm":
        ops.layer_norm(state["x"], state["y"], weight=state["weight"], bias=state["bias"], residual=state["residual"],
                       sum_out=state["sum"], mean=state["mean"], rstd=state["rstd"], p=state["p"], seed=state["seed"],
                       offset=state["offset"])
        return _named(state, "y", "sum", "mean", "rstd")
    if op == "norm_backward":
        ops.layer_norm_backward(state["dy"], state["s"], state["mean"], state["rstd"], state["dx"], weight=state["weight"],
                                dweight=state["dweight"], dbias=state["dbias"], dsum=state["dsum"],
                                dresidual=state["dresidual"], p=state["p"], seed=state["seed"], offset=state["offset"])
        return _named(state, "dx", "dresidual", "dweight", "dbias")
    if op == "dropout":
        ops.dropout(state["x"], state["y"], p=state["p"], seed=state["seed"], offset=state["offset"], residual=state["residual"])
        return _named(state, "y")
    if op == "logp":
        ops.token_logp(state["logits"], state["labels"], state["logp"], mask=state["mask"])
        return _named(state, "logp")
    shape = {"seq_start": state["start"]} if state["start"] is not None else {"sequences": case["seqs"]}
    if op == "preference":
        ops.preference_loss(state["logits"], state["labels"], state["ref_logp"], state["loss"], state["dlogits"],
                            mask=state["mask"], beta=state["beta"], label_smoothing=state["smoothing"],
                            seq_logp=state["seq_logp"], margin=state["margin"], **shape)
        return _named(state, "loss", "margin", "seq_logp", "dlogits")
    ops.policy_loss(state["logits"], state["labels"], state["old_logp"], state["advantages"], state["loss"], state["dlogits"],
                    mask=state["mask"], ref_logp=state["ref_logp"], clip_low=state["clip"], clip_high=state["clip"],
                    kl_beta=state["kl_beta"], per_sequence=case["per_sequence"], logp=state["logp"], stats=state["stats"], **shape)
    return _named(state, "loss", "stats", "logp", "dlogits")


def _named(state, *names):
    return {k: state[k] for k in names if state[k] is not None}


# ----------------------------------------------------------------------------- plain forms, in 32 bits

def _kept(state, count, device):
    """Which of `count` elements dropout keeps: halves of Philox4x32-10 words (Salmon et al., SC 2011), the counter being
    the element's number divided by eight and the call's offset, the key the seed."""
    block = torch.arange((count + 7) // 8, device=device)
    low = 0xFFFFFFFF
    c0, c1 = block & low, block >> 32
    c2 = torch.full_like(block, state["offset"] & low)
    c3 = torch.full_like(block, (state["offset"] >> 32) & low)
    k0, k1 = state["seed"] & low, (state["seed"] >> 32) & low
    for _ in range(10):  # the generator's rounds
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], 1)
    return words.reshape(-1)[:count] >= _threshold(state["p"])


def _threshold(p):
    return int(p * 65536 + 0.5)


def _drop(state, x):
    """x in 32 bits -> dropout of it."""
    thr = _threshold(state["p"])
    if thr == 0:
        return x
    return torch.where(_kept(state, x.numel(), x.device).view(x.shape), x * (65536 / (65536 - thr)), torch.zeros((), device=x.device))


def _plain_norm(state):
    s = _drop(state, state["x"].float())
    if state["residual"] is not None:
        s = s + state["residual"].float()
    mean = s.mean(1)
    centred = s - mean[:, None]
    rstd = (centred.square().mean(1) + 1e-5).rsqrt()
    y = centred * rstd[:, None] * state["weight"].float() + state["bias"].float()
    out = {"y": y.to(state["x"].dtype), "mean": mean, "rstd": rstd}
    if state["sum"] is not None:
        out["sum"] = s.to(state["x"].dtype)
    return out


def _plain_norm_backward(state):
    dy = state["dy"].float()
    hat = (state["s"].float() - state["mean"][:, None]) * state["rstd"][:, None]
    g = dy * state["weight"].float()
    ds = state["rstd"][:, None] * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))
    if state["dsum"] is not None:
        ds = ds + state["dsum"].float()
    dt, pt = state["s"].dtype, state["weight"].dtype
    out = {"dx": _drop(state, ds).to(dt), "dweight": (dy * hat).sum(0).to(pt), "dbias": dy.sum(0).to(pt)}
    if state["dresidual"] is not None:
        out["dresidual"] = ds.to(dt)
    return out


def _plain_dropout(state):
    y = _drop(state, state["x"].float())
    if state["residual"] is not None:
        y = y + state["residual"].float()
    return {"y": y.to(state["x"].dtype)}


def _plain_logp(state):
    """Log-probabilities of the labels, and the softmax that the gradients need."""
    z = state["logits"].float()
    z = z - z.amax(1, keepdim=True)
    e = z.exp()
    total = e.sum(1)
    return z.gather(1, state["labels"][:, None])[:, 0] - total.log(), e / total[:, None]


def _dlogits(state, per_token, softmax):
    """dL/dlogits from dL/dlogp."""
    d = softmax * -per_token[:, None]
    d.scatter_add_(1, state["labels"][:, None], per_token[:, None])
    return d.to(state["logits"].dtype)


def _log_sigmoid(h):
    return h.clamp(max=0.0) - (1 + (-h.abs()).exp()).log()


def _plain_preference(state):
    pairs, beta, e = state["case"]["seqs"] // 2, state["beta"], state["smoothing"]
    counted = state["mask"].float()
    logp, softmax = _plain_logp(state)
    ratio = _sums(state, (logp - state["ref_logp"]) * counted)
    h = beta * (ratio[:pairs] - ratio[pairs:])
    loss = (-(1 - e) * _log_sigmoid(h) - e * _log_sigmoid(-h)).mean()
    dh = (e / (1 + (-h).exp()) - (1 - e) / (1 + h.exp())) * (beta / pairs)
    per_seq = torch.cat([dh, -dh])
    per_token = (per_seq[:, None].expand(-1, state["case"]["steps"]).reshape(-1) if state["start"] is None
                 else (_member(state) * per_seq[None]).sum(1)) * counted
    return {"loss": loss.view(1), "margin": h, "seq_logp": _sums(state, logp * counted), "dlogits": _dlogits(state, per_token, softmax)}


def _plain_policy(state):
    counted = state["mask"].float()
    logp, softmax = _plain_logp(state)
    total = counted.sum()
    if state["case"]["per_sequence"]:
        lengths = _sums(state, counted)
        each = torch.where(lengths > 0, 1 / lengths, torch.zeros_like(lengths)) / (lengths > 0).sum()
        w = (each[:, None].expand(-1, state["case"]["steps"]).reshape(-1) if state["start"] is None
             else (_member(state) * each[None]).sum(1)) * counted
    else:
        w = counted / total
    a = state["advantages"]
    ratio = (logp - state["old_logp"]).exp()
    free, held = ratio * a, ratio.clamp(1 - state["clip"], 1 + state["clip"]) * a
    back = state["ref_logp"] - logp
    kl = back.exp() - back - 1
    loss = (w * (state["kl_beta"] * kl - torch.minimum(free, held))).sum()
    per_token = w * (torch.where(free <= held, -free, torch.zeros_like(free)) + state["kl_beta"] * (1 - back.exp()))
    stats = torch.stack([(counted * kl).sum() / total, (counted * (free > held)).sum() / total, total])
    return {"loss": loss.view(1), "stats": stats, "logp": logp * counted, "dlogits": _dlogits(state, per_token, softmax)}


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "logp":
        return {"logp": _plain_logp_only(state)}
    return {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "dropout": _plain_dropout,
            "preference": _plain_preference, "policy": _plain_policy}[op](state)


def _plain_logp_only(state):
    z = state["logits"].float()
    z = z - z.amax(1, keepdim=True)
    return (z.gather(1, state["labels"][:, None])[:, 0] - z.exp().sum(1).log()) * state["mask"].float()


# ----------------------------------------------------------------------------- work of one pass

def work(case):
    size = SIZE[case["dtype"]]
    if case["op"] in ("norm", "norm_backward", "dropout"):
        rows, cols = case["rows"], case["cols"]
        n, drop = rows * cols, case["p"] > 0
        if case["op"] == "dropout":
            return {"bytes": n * size * (3 if case["residual"] else 2), "flops": n * 2}
        par = cols * SIZE[case["param"]]
        if case["op"] == "norm":  # x [and the residual] in, y [and the sum] out, two statistics a row
            arrays = 2 + (1 if case["residual"] else 0) + (1 if case["residual"] or drop else 0)
            return {"bytes": n * size * arrays + 2 * par + 8 * rows, "flops": n * 8}
        arrays = 3 + (1 if case["residual"] else 0) + (1 if case["residual"] and drop else 0)
        return {"bytes": n * size * arrays + 3 * par + 8 * rows, "flops": n * 14}
    n, vocab = case["seqs"] * case["steps"], case["vocab"]
    counted = n * 2 / 3  # on average
    if case["op"] == "logp":
        return {"bytes": counted * vocab * size + 13 * n, "flops": counted * vocab * 4}
    # counted rows of logits in, every row of their gradient out
    return {"bytes": (counted + n) * vocab * size + 25 * n, "flops": counted * vocab * 6}


# ----------------------------------------------------------------------------- the definitions, in 64 bits

def _exact_kept(state, count, device):
    """As the definition has it, by 16-bit pieces: no product here passes 64 bits."""
    block = torch.arange((count + 7) // 8, device=device)
    word = [block % 2 ** 32, block // 2 ** 32, torch.zeros_like(block) + state["offset"] % 2 ** 32,
            torch.zeros_like(block) + state["offset"] // 2 ** 32 % 2 ** 32]
    key = [state["seed"] % 2 ** 32, state["seed"] // 2 ** 32 % 2 ** 32]

    def product(a, m):
        small, large = a * (m % 65536), a * (m // 65536)
        large = large + small // 65536
        return large // 65536, large % 65536 * 65536 + small % 65536

    for r in range(10):
        ah, al = product(word[0], 0xD2511F53)
        bh, bl = product(word[2], 0xCD9E8D57)
        word = [torch.bitwise_xor(torch.bitwise_xor(bh, word[1]), (key[0] + r * 0x9E3779B9) % 2 ** 32), bl,
                torch.bitwise_xor(torch.bitwise_xor(ah, word[3]), (key[1] + r * 0xBB67AE85) % 2 ** 32), al]
    halves = torch.empty(block.numel(), 4, 2, dtype=torch.int32, device=device)
    for k in range(4):
        halves[:, k, 0], halves[:, k, 1] = word[k] % 65536, word[k] // 65536
    return halves.view(-1)[:count] >= math.floor(state["p"] * 65536 + 0.5)


def _exact_drop(state, x):
    keep = 1 - math.floor(state["p"] * 65536 + 0.5) / 65536
    return x if keep == 1 else x / keep * _exact_kept(state, x.numel(), x.device).view(x.shape)


def exact(case, seed):
    state = prepare(case, seed)
    f = torch.float64
    if case["op"] == "dropout":
        y = _exact_drop(state, state["x"].to(f))
        return {"y": y if state["residual"] is None else y + state["residual"].to(f)}
    if case["op"] == "norm":
        s = _exact_drop(state, state["x"].to(f))
        s = s if state["residual"] is None else s + state["residual"].to(f)
        var, mean = torch.var_mean(s, 1, unbiased=False)
        rstd = 1 / torch.sqrt(var + 1e-5)
        out = {"y": (s - mean[:, None]) * rstd[:, None] * state["weight"].to(f) + state["bias"].to(f), "mean": mean, "rstd": rstd}
        return out if state["sum"] is None else dict(out, sum=s)
    if case["op"] == "norm_backward":
        # the row's statistics are inputs, so their derivatives are written out: d mean / d s = 1/n, d rstd / d s = -rstd^2 hat / n
        n = case["cols"]
        dy, rstd = state["dy"].to(f), state["rstd"].to(f)[:, None]
        centred = state["s"].to(f) - state["mean"].to(f)[:, None]
        up = dy * state["weight"].to(f)
        ds = up * rstd - (up * rstd).sum(1, keepdim=True) / n - centred * rstd ** 3 * (up * centred).sum(1, keepdim=True) / n
        ds = ds if state["dsum"] is None else ds + state["dsum"].to(f)
        out = {"dx": _exact_drop(state, ds), "dweight": torch.einsum("ij,ij->j", dy, centred * rstd), "dbias": dy.sum(0)}
        return out if state["dresidual"] is None else dict(out, dresidual=ds)
    z = state["logits"].to(f).requires_grad_(case["op"] != "logp")
    mask = state["mask"]
    logp = z.gather(1, state["labels"][:, None])[:, 0] - torch.logsumexp(z, 1)
    logp = torch.where(mask, logp, torch.zeros((), dtype=f, device=z.device))
    if case["op"] == "logp":
        return {"logp": logp}
    seqs, n = case["seqs"], case["seqs"] * case["steps"]
    start = torch.arange(0, n + 1, case["steps"], device=z.device) if state["start"] is None else state["start"].long()
    which = torch.searchsorted(start, torch.arange(n, device=z.device), right=True) - 1
    if case["op"] == "preference":
        sums = torch.zeros(seqs, dtype=f, device=z.device).index_add(0, which, logp)
        ref = torch.where(mask, state["ref_logp"].to(f), torch.zeros_like(logp))
        ratio = (sums - torch.zeros_like(sums).index_add(0, which, ref)).view(2, -1)
        h = state["beta"] * (ratio[0] - ratio[1])
        e = state["smoothing"]
        loss = (1 - e) * torch.nn.functional.softplus(-h).mean() + e * torch.nn.functional.softplus(h).mean()
        (dz,) = torch.autograd.grad(loss, z)
        return {"loss": loss.detach().view(1), "margin": h.detach(), "seq_logp": sums.detach(), "dlogits": dz}
    count = torch.zeros(seqs, dtype=f, device=z.device).index_add(0, which, mask.to(f))
    w = mask / (count[which] * (count > 0).sum()) if case["per_sequence"] else mask / count.sum()
    w = torch.where(mask, w, torch.zeros_like(w))
    a, c = state["advantages"].to(f), state["clip"]
    ratio = torch.exp(logp - state["old_logp"].to(f))
    back = torch.where(mask, state["ref_logp"].to(f) - logp, torch.zeros_like(logp))
    bound = torch.where(a >= 0, a * (1 + c), a * (1 - c))  # the clipped term caps the gain from either side
    gain = torch.minimum(ratio * a, bound)
    kl = torch.expm1(back) - back
    loss = (w * (state["kl_beta"] * kl - gain)).sum()
    (dz,) = torch.autograd.grad(loss, z)
    total = mask.sum()
    stats = torch.stack([kl.sum() / total, ((ratio * a > bound) & mask).sum() / total, total.to(f)])
    return {"loss": loss.detach().view(1), "stats": stats.detach(), "logp": logp.detach(), "dlogits": dz}
