"""Cases of the operators that mix tokens in a worker's training step: embedding lookup and its gradient, the norm and
rotation of queries and keys with its backward pass, attention and its backward pass.

`run` computes an operator either in elementary torch operations in 32 bits (`own` false) or by the package's entry
points (`own` true).  Tokens are rows; heads lie side by side in a row.
"""
import math

import numpy as np
import torch

own = False

# One operator context serves a whole program: it is made for the largest shapes met here.
MAX_TOKENS = 1 << 17
MAX_COLS = 16384
_ops = None

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
LARGEST_ROWS = 32768 * 4096            # elements of the largest listed embedding output
LARGEST_TABLE = 131072 * 4096          # and of its table
LARGEST_HEADS = 32768 * 40 * 128       # elements of the largest listed queries and keys
LARGEST_PAIRS = 32 * 8192 * 8192 * 128  # heads x queries x keys x head size of the largest listed attention


def listed():
    return [
        # the prompt of one short answer
        dict(name="embedding_prompt", op="embedding", tokens=24, vocab=32000, cols=4096, dtype="bf16", masked=False),
        # a training step's tokens, large vocabulary
        dict(name="embedding_batch", op="embedding", tokens=32768, vocab=131072, cols=4096, dtype="bf16", masked=False),
        # a small vocabulary of odd size and width in 32 bits, padding left out
        dict(name="embedding_grad_odd", op="embedding_backward", tokens=1023, vocab=1001, cols=333, dtype="f32", out="f32", masked=True, base=False),
        # a training step's tokens, their gradient for a large table
        dict(name="embedding_grad_batch", op="embedding_backward", tokens=32768, vocab=131072, cols=4096, dtype="bf16", out="bf16", masked=False, base=False),
        # one token of a model that answers
        dict(name="qk_norm_one_token", op="qk_norm", tokens=1, heads=32, kv=8, dim=128, dtype="bf16", param="bf16", rotate=1.0, neighbours=False, far=100000),
        # a training step's queries and keys
        dict(name="qk_norm_batch", op="qk_norm", tokens=32768, heads=32, kv=8, dim=128, dtype="bf16", param="bf16", rotate=1.0, neighbours=False, far=0),
        # heads of odd length in 32 bits, rotated in neighbouring pairs, only a part of each
        dict(name="qk_norm_grad_odd", op="qk_norm_backward", tokens=777, heads=6, kv=2, dim=50, dtype="f32", param="f32", rotate=0.5, neighbours=True, far=0),
        # a training step's queries and keys, backwards
        dict(name="qk_norm_grad_batch", op="qk_norm_backward", tokens=32768, heads=32, kv=8, dim=128, dtype="bf16", param="f32", rotate=1.0, neighbours=False, far=0),
        # eight padded answers seen in both directions (a reward model's batch)
        dict(name="attention_padded", op="attention", seqs=8, steps=100, heads=4, kv=4, dim=64, dtype="f16", causal=False, layout="padded"),
        # one long document
        dict(name="attention_long", op="attention", seqs=1, steps=8192, heads=32, kv=8, dim=128, dtype="bf16", causal=True, layout="equal"),
        # sixteen answers of uneven lengths, packed one behind the other
        dict(name="attention_grad_packed", op="attention_backward", seqs=16, steps=256, heads=16, kv=4, dim=64, dtype="f16", causal=True, layout="packed"),
        # one long document, backwards
        dict(name="attention_grad_long", op="attention_backward", seqs=1, steps=8192, heads=32, kv=8, dim=128, dtype="bf16", causal=True, layout="equal"),
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
    op = rng.choice(("embedding", "embedding_backward", "qk_norm", "qk_norm_backward", "attention", "attention_backward"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op in ("embedding", "embedding_backward"):
        out = rng.choice((dtype, "f32"))
        size = max(SIZE[dtype], SIZE[out])
        tokens, vocab, cols = _size(rng, 1, 65536), _size(rng, 500, 140000), _size(rng, 64, 8192)
        while tokens * cols > LARGEST_ROWS * 2 // size:
            tokens = max(1, tokens // 2)
        base = op == "embedding_backward" and rng.random() < 0.4
        while vocab * cols > LARGEST_TABLE * 2 // size // (2 if base else 1):
            cols = cols // 2
        case = dict(op=op, tokens=tokens, vocab=vocab, cols=cols, dtype=dtype, masked=rng.random() < 0.4)
        return case if op == "embedding" else dict(case, out=out, base=base)
    kv = rng.choice((1, 2, 3, 4, 8))
    heads = kv * rng.choice((1, 1, 2, 4))
    if op in ("qk_norm", "qk_norm_backward"):
        dim = rng.choice((32, 50, 64, 72, 96, 128, 128, 256))
        tokens = _size(rng, 1, 65536)
        while tokens * (heads + kv) * dim > LARGEST_HEADS * 2 // SIZE[dtype]:
            tokens = max(1, tokens // 2)
        return dict(op=op, tokens=tokens, heads=heads, kv=kv, dim=dim, dtype=dtype, param=rng.choice((dtype, "f32")),
                    rotate=rng.choice((1.0, 1.0, 0.5, 0.0)), neighbours=rng.random() < 0.4, far=rng.choice((0, 0, 5000, 1000000)))
    dtype = rng.choice(("bf16", "bf16", "f16"))
    dim = rng.choice((32, 64, 64, 80, 96, 128, 128))
    layout = rng.choice(("equal", "packed", "padded"))
    seqs, steps = _size(rng, 1, 64), _size(rng, 1, 8192)
    pairs = lambda: heads * dim * seqs * steps * (steps if layout != "packed" else seqs * steps)  # noqa: E731  (as the plain form takes them)
    while pairs() > LARGEST_PAIRS * (1 if op == "attention" else 0.5) or seqs * steps > 65536:
        if seqs > 4 and rng.random() < 0.5:
            seqs //= 2
        else:
            steps = max(1, steps * 2 // 3)
    return dict(op=op, seqs=seqs, steps=steps, heads=heads, kv=kv, dim=dim, dtype=dtype, causal=rng.random() < 0.6, layout=layout)


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

    def uniform(*shape, dtype=torch.float32):
        return torch.rand(*shape, generator=gen, device=dev, dtype=dtype)

    op = case["op"]
    if op in ("embedding", "embedding_backward"):
        n, vocab, cols = case["tokens"], case["vocab"], case["cols"]
        # the r-th most frequent word comes about once in r words, and its number says nothing of its rank
        rank = (vocab ** uniform(n, dtype=torch.float64)).floor().long().clamp(1, vocab) - 1
        state["tokens"] = torch.randperm(vocab, generator=gen, device=dev)[rank]
        state["mask"] = uniform(n) < 0.8 if case["masked"] else None
        state["scale"] = math.sqrt(cols)
        if op == "embedding":
            state["table"] = normal(vocab, cols, scale=cols ** -0.5, dtype=dt)
            state["out"] = torch.empty(n, cols, dtype=dt, device=dev)
            return state
        state["dout"] = normal(n, cols, scale=0.1, dtype=dt)
        ot = TYPES[case["out"]]
        state["base"] = normal(vocab, cols, scale=0.1, dtype=ot) if case["base"] else None  # of tied output weights
        state["dtable"] = torch.empty(vocab, cols, dtype=ot, device=dev)
        return state

    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    if op in ("qk_norm", "qk_norm_backward"):
        n, pt = case["tokens"], TYPES[case["param"]]
        pairs = int(dim * case["rotate"]) // 2
        # q, k and v come out of one product side by side: rows are strided
        qkv = normal(n, (heads + 2 * kv) * dim, dtype=dt)
        state["q"], state["k"] = qkv[:, :heads * dim], qkv[:, heads * dim:(heads + kv) * dim]
        state["q_weight"], state["k_weight"] = (normal(dim, scale=0.2, mean=1.0).to(pt) for _ in range(2))
        state["freq"] = 10000.0 ** (-torch.arange(pairs, device=dev, dtype=torch.float32) / pairs) if pairs else None
        state["positions"] = (torch.arange(n, device=dev) % 4096 + case["far"]) if pairs else None
        if op == "qk_norm":
            state["q_out"], state["k_out"] = torch.empty(n, heads * dim, dtype=dt, device=dev), torch.empty(n, kv * dim, dtype=dt, device=dev)
            return state
        state["dq_out"], state["dk_out"] = normal(n, heads * dim, scale=0.1, dtype=dt), normal(n, kv * dim, scale=0.1, dtype=dt)
        dqkv = torch.zeros_like(qkv)
        state["dq"], state["dk"] = dqkv[:, :heads * dim], dqkv[:, heads * dim:(heads + kv) * dim]
        state["dq_weight"], state["dk_weight"] = torch.empty(dim, dtype=pt, device=dev), torch.empty(dim, dtype=pt, device=dev)
        return state

    seqs, steps, layout = case["seqs"], case["steps"], case["layout"]
    n = seqs * steps
    # normed and rotated queries and keys; values straight from the product
    state["q"], state["k"] = normal(n, heads * dim, scale=1.2, dtype=dt), normal(n, kv * dim, scale=1.2, dtype=dt)
    state["v"] = normal(n, (heads + 2 * kv) * dim, dtype=dt)[:, (heads + kv) * dim:]
    state["start"] = state["mask"] = None
    if layout == "packed":  # uneven lengths, one behind the other
        cuts = torch.randint(n + 1, (seqs - 1,), generator=gen, device=dev).sort().values
        edge = torch.zeros(1, dtype=cuts.dtype, device=dev)
        state["start"] = torch.cat([edge, cuts, edge + n]).to(torch.int32)
    if layout == "padded":
        last = steps - (uniform(seqs, 1) * (steps / 2)).floor()
        state["mask"] = (torch.arange(steps, device=dev)[None] < last).reshape(n)
    state["scale"] = dim ** -0.5
    state["out"], state["lse"] = torch.empty(n, heads * dim, dtype=dt, device=dev), torch.empty(heads, n, device=dev)
    if op == "attention":
        return state
    first = _plain_attention(state)  # what the forward pass keeps
    state["out"], state["lse"] = first["out"], first["lse"]
    state["dout"] = normal(n, heads * dim, scale=0.1, dtype=dt)
    state["row_dot"] = torch.empty(heads, n, device=dev)
    state["dq"], state["dk"], state["dv"] = torch.empty_like(state["q"]), torch.empty_like(state["k"]), torch.empty(n, kv * dim, dtype=dt, device=dev)
    return state


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
    if op == "embedding":
        ops.embedding(state["tokens"], state["table"], state["out"], scale=state["scale"], mask=state["mask"])
        return _named(state, "out")
    if op == "embedding_backward":
        ops.embedding_backward(state["tokens"], state["dout"], state["dtable"], scale=state["scale"], mask=state["mask"], base=state["base"])
        return _named(state, "dtable")
    if op == "qk_norm":
        ops.qk_norm(state["q"], state["k"], state["q_out"], state["k_out"], state["positions"], state["freq"], head_dim=case["dim"],
                    q_weight=state["q_weight"], k_weight=state["k_weight"], eps=1e-6, interleaved=case["neighbours"])
        return _named(state, "q_out", "k_out")
    if op == "qk_norm_backward":
        ops.qk_norm_backward(state["dq_out"], state["dk_out"], state["q"], state["k"], state["dq"], state["dk"], state["positions"],
                             state["freq"], head_dim=case["dim"], q_weight=state["q_weight"], k_weight=state["k_weight"],
                             dq_weight=state["dq_weight"], dk_weight=state["dk_weight"], eps=1e-6, interleaved=case["neighbours"])
        return _named(state, "dq", "dk", "dq_weight", "dk_weight")
    shape = {"seq_start": state["start"]} if state["start"] is not None else {"sequences": case["seqs"]}
    shape.update(heads=case["heads"], causal=case["causal"], scale=state["scale"], mask=state["mask"])
    if op == "attention":
        ops.attention(state["q"], state["k"], state["v"], state["out"], lse=state["lse"], **shape)
        return _named(state, "out", "lse")
    ops.attention_backward(state["dout"], state["q"], state["k"], state["v"], state["out"], state["lse"], state["row_dot"],
                           state["dq"], state["dk"], state["dv"], **shape)
    return _named(state, "dq", "dk", "dv")


def _named(state, *names):
    return {k: state[k] for k in names}


# ----------------------------------------------------------------------------- plain forms, in 32 bits

def _plain_embedding(state):
    rows = state["table"][state["tokens"]].float() * state["scale"]
    if state["mask"] is not None:
        rows = rows * state["mask"][:, None]
    return {"out": rows.to(state["table"].dtype)}


def _plain_embedding_backward(state):
    rows, dtable = state["dout"].float() * state["scale"], state["dtable"]
    if state["mask"] is not None:
        rows = rows * state["mask"][:, None]
    total = torch.zeros(dtable.shape, device=dtable.device) if state["base"] is None else state["base"].float()
    return {"dtable": total.index_add(0, state["tokens"], rows).to(dtable.dtype)}


def _turned(x, state, back=False):
    """Heads x [tokens, heads, dim] rotated by their position's angles, or back; angles in 64 bits."""
    if state["freq"] is None:
        return x
    pairs = state["freq"].numel()
    angle = state["positions"].double()[:, None] * state["freq"].double()
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if back:
        s = -s
    if state["case"]["neighbours"]:
        a, b = x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]
        front = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = x[..., :pairs], x[..., pairs:2 * pairs]
        front = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([front, x[..., 2 * pairs:]], -1)


def _plain_qk_norm(state):
    out = {}
    for name in ("q", "k"):
        x = state[name].float().unflatten(1, (-1, state["case"]["dim"]))
        h = x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * state[name + "_weight"].float()
        out[name + "_out"] = _turned(h, state).flatten(1).to(state[name].dtype)
    return out


def _plain_qk_norm_backward(state):
    out = {}
    for name in ("q", "k"):
        dim, w = state["case"]["dim"], state[name + "_weight"]
        x = state[name].float().unflatten(1, (-1, dim))
        dn = _turned(state[f"d{name}_out"].float().unflatten(1, (-1, dim)), state, back=True)
        r = (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
        g = dn * w.float()
        out["d" + name] = (r * (g - x * r.square() * (g * x).mean(-1, keepdim=True))).flatten(1).to(state[name].dtype)
        out[f"d{name}_weight"] = (dn * x * r).sum((0, 1)).to(w.dtype)
    return out


def _allowed(state):
    """[batch, 1, 1, queries, keys] truth values, a batch being a sequence, or all of the packed ones."""
    case, dev = state["case"], state["q"].device
    n = case["seqs"] * case["steps"]
    if state["start"] is None:
        at = torch.arange(case["steps"], device=dev)
        ok = torch.ones(case["seqs"], case["steps"], case["steps"], dtype=torch.bool, device=dev)
    else:
        at = torch.arange(n, device=dev)
        seq = torch.bucketize(at, state["start"][1:].long(), right=True)
        ok = (seq[:, None] == seq[None])[None]
    if case["causal"]:
        ok = ok & (at[:, None] >= at[None])
    if state["mask"] is not None:
        m = state["mask"].view(ok.shape[0], -1)
        ok = ok & m[:, None] & m[:, :, None]
    return ok[:, None, None]


def _heads(x, state, count):
    """[tokens, count * dim] -> [batch, key heads, heads that share one, tokens, dim] in 32 bits"""
    case = state["case"]
    batch = 1 if state["start"] is not None else case["seqs"]
    return x.float().view(batch, -1, case["kv"], count // case["kv"], case["dim"]).permute(0, 2, 3, 1, 4)


def _rows(x, dtype):
    """Back to rows of tokens."""
    return x.permute(0, 3, 1, 2, 4).flatten(2).flatten(0, 1).to(dtype)


def _plain_attention(state):
    case, dt = state["case"], state["q"].dtype
    q, k, v = _heads(state["q"], state, case["heads"]), _heads(state["k"], state, case["kv"]), _heads(state["v"], state, case["kv"])
    s = (q * state["scale"]) @ k.transpose(-1, -2)
    s = s.masked_fill_(~_allowed(state), -math.inf)
    top = s.amax(-1, keepdim=True).clamp(min=-3e38)  # rows without a key
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / total.clamp(min=1e-38)
    lse = (top + total.log())[..., 0]
    lse = torch.where(total[..., 0] > 0, lse, torch.full_like(lse, -math.inf))
    return {"out": _rows(out, dt), "lse": lse.permute(1, 2, 0, 3).reshape(case["heads"], -1)}


def _plain_attention_backward(state):
    case, dt = state["case"], state["q"].dtype
    q, k, v = _heads(state["q"], state, case["heads"]), _heads(state["k"], state, case["kv"]), _heads(state["v"], state, case["kv"])
    dout, out = _heads(state["dout"], state, case["heads"]), _heads(state["out"], state, case["heads"])
    lse = state["lse"].view(case["kv"], case["heads"] // case["kv"], q.shape[0], -1).permute(2, 0, 1, 3)[..., None]
    p = ((q * state["scale"]) @ k.transpose(-1, -2)).sub_(lse).masked_fill_(~_allowed(state), -math.inf).exp_()
    dv = (p.transpose(-1, -2) @ dout).sum(2, keepdim=True)
    delta = (dout * out).sum(-1, keepdim=True)
    ds = (dout @ v.transpose(-1, -2)).sub_(delta).mul_(p).mul_(state["scale"])
    dk = (ds.transpose(-1, -2) @ q).sum(2, keepdim=True)
    return {"dq": _rows(ds @ k, dt), "dk": _rows(dk, dt), "dv": _rows(dv, dt)}


def run(state):
    if own:
        return _run_own(state)
    return {"embedding": _plain_embedding, "embedding_backward": _plain_embedding_backward, "qk_norm": _plain_qk_norm,
            "qk_norm_backward": _plain_qk_norm_backward, "attention": _plain_attention,
            "attention_backward": _plain_attention_backward}[state["case"]["op"]](state)


# ----------------------------------------------------------------------------- work of one pass

def _distinct(case):
    """Expected number of different tokens that count."""
    r = np.arange(1, case["vocab"] + 1, dtype=np.float64)
    n = case["tokens"] * (0.8 if case["masked"] else 1.0)
    return float(-np.expm1(n * np.log1p(-np.log((r + 1) / r) / math.log(case["vocab"] + 1))).sum())


def _pairs(case):
    """Expected pairs of a query and a key that it sees."""
    seqs, steps = case["seqs"], case["steps"]
    if case["layout"] == "packed":  # pieces of a line cut at random: the mean square of a length is 2 L^2 / (q (q + 1))
        squares = 2.0 * (seqs * steps) ** 2 / (seqs + 1)
    elif case["layout"] == "padded":  # lengths even between a half and the whole
        squares = seqs * steps ** 2 * 7 / 12
    else:
        squares = float(seqs) * steps ** 2
    return squares / 2 if case["causal"] else squares


def work(case):
    size, op = SIZE[case["dtype"]], case["op"]
    if op in ("embedding", "embedding_backward"):
        n, cols = case["tokens"], case["cols"]
        if op == "embedding":
            return {"bytes": _distinct(case) * cols * size + n * cols * size + 8 * n, "flops": n * cols}
        counted = n * (0.8 if case["masked"] else 1.0)
        return {"bytes": counted * cols * size + case["vocab"] * cols * SIZE[case["out"]] * (2 if case["base"] else 1) + 8 * n, "flops": 2 * counted * cols}
    if op in ("qk_norm", "qk_norm_backward"):
        elements = case["tokens"] * (case["heads"] + case["kv"]) * case["dim"]
        par = case["dim"] * SIZE[case["param"]]
        if op == "qk_norm":
            return {"bytes": 2 * elements * size + 2 * par + 8 * case["tokens"], "flops": elements * 8}
        return {"bytes": 3 * elements * size + 4 * par + 8 * case["tokens"], "flops": elements * 16}
    n, q, k = case["seqs"] * case["steps"], case["heads"] * case["dim"], case["kv"] * case["dim"]
    per = case["heads"] * case["dim"] * _pairs(case)
    if op == "attention":
        return {"bytes": n * size * 2 * (q + k) + 4 * n * case["heads"], "flops": 4 * per}
    return {"bytes": n * size * 4 * (q + k) + 4 * n * case["heads"], "flops": 10 * per}


# ----------------------------------------------------------------------------- the definitions, in 64 bits

def _exact_turn(x, state):
    """Pairs as complex numbers, multiplied by exp(i angle)."""
    if state["freq"] is None:
        return x
    p = state["freq"].numel()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), state["positions"].double()[:, None] * state["freq"].double())[:, None]
    first = slice(0, 2 * p, 2) if state["case"]["neighbours"] else slice(0, p)
    second = slice(1, 2 * p, 2) if state["case"]["neighbours"] else slice(p, 2 * p)
    z = torch.complex(x[..., first], x[..., second]) * turn
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_qk(state, backward):
    out, f = {}, torch.float64
    for name in ("q", "k"):
        dim = state["case"]["dim"]
        x = state[name].to(f).unflatten(1, (-1, dim)).requires_grad_(backward)
        w = state[name + "_weight"].to(f).requires_grad_(backward)
        y = _exact_turn(x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / dim + 1e-6) * w, state)
        if not backward:
            out[name + "_out"] = y.flatten(1)
            continue
        dx, dw = torch.autograd.grad(y, (x, w), state[f"d{name}_out"].to(f).view_as(y))
        out["d" + name], out[f"d{name}_weight"] = dx.flatten(1), dw
    return out


def _exact_attention(state, backward):
    """Head by head and sequence by sequence."""
    case, f = state["case"], torch.float64
    dim, group, n = case["dim"], case["heads"] // case["kv"], case["seqs"] * case["steps"]
    edges = state["start"].tolist() if state["start"] is not None else list(range(0, n + 1, case["steps"]))
    counted = torch.ones(n, dtype=torch.bool, device=state["q"].device) if state["mask"] is None else state["mask"]
    out = {k: torch.zeros(n, state[k].shape[1], dtype=f, device=counted.device) for k in (("dq", "dk", "dv") if backward else ("out",))}
    lse = torch.full((case["heads"], n), -math.inf, dtype=f, device=counted.device)
    for a, b in zip(edges[:-1], edges[1:]):
        at = torch.arange(a, b, device=counted.device)[counted[a:b]]
        if not at.numel():
            continue
        hidden = torch.triu(torch.full((at.numel(), at.numel()), -math.inf, dtype=f, device=at.device), 1) if case["causal"] else 0.0
        for h in range(case["heads"]):
            mine, shared = slice(h * dim, (h + 1) * dim), slice(h // group * dim, (h // group + 1) * dim)
            q, k, v = state["q"][at, mine].to(f), state["k"][at, shared].to(f), state["v"][at, shared].to(f)
            s = torch.einsum("id,jd->ij", q, k) * state["scale"] + hidden
            if not backward:
                out["out"][at, mine], lse[h, at] = torch.softmax(s, 1) @ v, torch.logsumexp(s, 1)
                continue
            p, do = torch.exp(s - state["lse"][h, at].to(f)[:, None]), state["dout"][at, mine].to(f)
            ds = p * (do @ v.T - torch.einsum("id,id->i", do, state["out"][at, mine].to(f))[:, None])
            out["dq"][at, mine] = state["scale"] * ds @ k
            out["dk"][at, shared] += state["scale"] * ds.T @ q
            out["dv"][at, shared] += p.T @ do
    return out if backward else dict(out, lse=lse)


def exact(case, seed):
    op, f = case["op"], torch.float64
    if op in ("attention", "attention_backward"):
        if case["heads"] * case["seqs"] > 4096:  # many short products, one after the other
            return None
        return _exact_attention(prepare(case, seed), op == "attention_backward")
    state = prepare(case, seed)
    if op in ("qk_norm", "qk_norm_backward"):
        return _exact_qk(state, op == "qk_norm_backward")
    scale = state["scale"]
    counted = torch.ones_like(state["tokens"], dtype=torch.bool) if state["mask"] is None else state["mask"]
    if op == "embedding":
        out = torch.zeros(state["out"].shape, dtype=f, device=counted.device)
        out[counted] = torch.index_select(state["table"], 0, state["tokens"][counted]).to(f) * scale
        return {"out": out}
    # one column of ones for each token: a sparse product adds up what belongs to a word
    at = torch.nonzero(counted)[:, 0]
    who = torch.stack([state["tokens"][at], at])
    pick = torch.sparse_coo_tensor(who, torch.full((at.numel(),), scale, dtype=f, device=at.device), (case["vocab"], case["tokens"]))
    total = torch.sparse.mm(pick, state["dout"].to(f))
    return {"dtable": total if state["base"] is None else total + state["base"].to(f)}
