"""Lookup, norm and rotation of queries and keys, attention, and their backward passes on the device, against the binary64 restatement.

Tolerances (u(T): rounding of a stored result, E = 2^-24, as in test_training_gpu.py).
  lookup    one product; a gradient adds c terms: u |out| + (c + 4) E sum|terms|.
  qk_norm   r is off by at most (dim / 8 + 8) E, an angle by 4 E, a pair mixes two elements: u |out| + 2 K E max|n| over the head,
            K = dim / 8 + 24.  Backward the same with r (|g| + |x r| mean|g x r|) in n's place; a weight's gradient adds N terms.
  attention a score is a sum of dim products, added in any order with a rounding or truncation of 2 E each: it is off by d = 2 (dim + 16) E
            scale |q|.|k| (sums of absolute values), an exponential by 2 d + 8 E more than that, relatively.  p is rounded to T where T has 16 bits
            (UP), so out is off by u |out| + (UP + 2 d + (keys + 32) E) sum p|v|; in float16 a p below 2^-14 of its row's largest is off by 2^-25
            of that.  Backward: p as before, with lse's own rounding; ds by (UP + 2 d + 2 (dim + 16) E) p (|dout||v| + |dout||out|), and every
            sum by E a term.  An exponential below 2^-126 is 0: a term of a sum is then off by up to 2^-126 of its other factors.
"""
import numpy as np
import pytest
import torch

import paper_2211_00188_b200 as pkg
from oracle import training_oracle as O
from test_training_gpu import E, TINY, TYPES, U, close, dev, host, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    return pkg.TrainingOps(70000, 32768)


def ints(a, dtype=torch.int64):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(dtype)


def truths(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


# ----------------------------------------------------------------------------- lookup

WIDTHS = [(1, 0, 0), (8, 0, 0), (7, 0, 0), (64, 8, 0), (65, 3, 1), (1001, 0, 0), (1032, 0, 0), (4104, 8, 0)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cols,extra,shift", WIDTHS)
@pytest.mark.parametrize("masked", [False, True])
def test_embedding(ops, dtype, cols, extra, shift, masked):
    dt, rng = TYPES[dtype], np.random.default_rng(cols)
    n, vocab = 37, 19
    table = strided(dev(rng.normal(size=(vocab, cols)), dt), extra, shift)
    out = strided(torch.full((n, cols), 5.0, dtype=dt, device="cuda"), extra, shift)
    tok = rng.integers(0, vocab, n)
    tok[3], tok[8], tok[9] = -1, vocab, vocab - 1
    mask = rng.random(n) < 0.7 if masked else None
    if masked:
        mask[8] = False                                       # a token out of range that does not count
    ops.embedding(ints(tok, torch.int32 if masked else torch.int64), table, out, scale=0.37, mask=truths(mask))
    want = O.embedding(tok, host(table), float(np.float32(0.37)), mask)
    close(out, want, (U[dt] + 2 * E) * np.abs(want) + TINY[dt], "out")
    if extra:
        assert torch.isnan(out._base[shift:shift + n * (cols + extra)].view(n, cols + extra)[:, cols:]).all()


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("n,vocab,cols,extra,shift", [(0, 5, 9, 0, 0), (1, 1, 8, 0, 0), (33, 40, 7, 0, 0), (200, 3, 24, 0, 0), (1023, 700, 65, 3, 1),
                                                      (2500, 33, 136, 8, 0), (700, 600, 2056, 0, 0)])
@pytest.mark.parametrize("kind", ["plain", "masked", "base", "place"])
def test_embedding_backward(ops, dtype, out, n, vocab, cols, extra, shift, kind):
    dt, ot, rng = TYPES[dtype], TYPES[out], np.random.default_rng(n + cols)
    tok = rng.zipf(1.4, n) % (vocab + 2) - 1                   # some out of range, some very frequent
    mask = rng.random(n) < 0.6 if kind == "masked" else None
    d = strided(dev(rng.normal(size=(n, cols)), dt), extra, shift)
    if mask is not None:
        d[torch.from_numpy(~mask).cuda()] = float("nan")       # not read
    base = strided(dev(rng.normal(size=(vocab, cols)), ot), extra, shift) if kind in ("base", "place") else None
    before = None if base is None else host(base)
    g = base if kind == "place" else strided(torch.full((vocab, cols), 7.0, dtype=ot, device="cuda"), extra, shift)
    ops.embedding_backward(ints(tok), d, g, scale=1.7, mask=truths(mask), base=base)
    s = float(np.float32(1.7))
    dh = np.nan_to_num(host(d))
    want = O.embedding_backward(tok, dh, vocab, s, mask, before)
    size = O.embedding_backward(tok, np.abs(dh), vocab, s, mask)
    count = O.embedding_backward(tok, np.ones((n, 1)), vocab, 1.0, mask)
    close(g, want, (U[ot] + 2 * E) * np.abs(want) + (count + 4) * E * size + TINY[ot], "dtable")
    if extra:
        assert torch.isnan(g._base[shift:shift + vocab * (cols + extra)].view(vocab, cols + extra)[:, cols:]).all()
    if kind == "place":                                       # rows without tokens keep their bits
        idle = torch.from_numpy(count[:, 0] == 0).cuda()
        assert torch.equal(g[idle], dev(before, ot)[idle])


@pytest.mark.parametrize("n,vocab", [(2048, 511), (2049, 512), (4097, 513), (20000, 131071), (65537, 262143), (70000, 2)])
def test_embedding_backward_of_many_tokens(ops, n, vocab):
    """Token counts around what one CTA sorts, vocabularies around one, two and three passes.  Small whole numbers: the sums are exact."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    tok = (vocab ** torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)).long().clamp(max=vocab) - 1
    tok = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.2, vocab - 1 - tok, tok)
    d = torch.randint(-3, 4, (n, 16), generator=gen, device="cuda").float()
    g = torch.full((vocab, 16), 9.0, device="cuda")
    ops.embedding_backward(tok, d, g)
    want = torch.zeros(vocab, 16, dtype=torch.float64, device="cuda").index_add_(0, tok, d.double())
    assert torch.equal(g.double(), want)
    again = torch.empty_like(g)
    f = torch.randn(n, 16, generator=gen, device="cuda")
    ops.embedding_backward(tok, f, g)
    ops.embedding_backward(tok, f, again)
    assert torch.equal(g, again)                              # the same bits


def test_embedding_gradient_agrees_with_differences():
    rng = np.random.default_rng(5)
    tok, table, up = rng.integers(0, 4, 9), rng.normal(size=(4, 3)), rng.normal(size=(9, 3))
    got = O.embedding_backward(tok, up, 4, 1.3)
    for v in range(4):
        for c in range(3):
            a, b = table.copy(), table.copy()
            a[v, c] += 1e-4
            b[v, c] -= 1e-4
            d = ((O.embedding(tok, a, 1.3) - O.embedding(tok, b, 1.3)) * up).sum() / 2e-4
            assert abs(d - got[v, c]) < 1e-9


# ----------------------------------------------------------------------------- norm and rotation

HEADS = [(1, 1, 1, 8, 4), (3, 2, 1, 16, 5), (5, 4, 2, 64, 32), (5, 3, 3, 50, 12), (4, 2, 1, 72, 36), (9, 4, 1, 96, 24), (6, 5, 1, 128, 64),
         (2, 3, 1, 256, 128), (2, 2, 2, 256, 30), (3, 2, 1, 272, 60), (2, 1, 1, 512, 256), (4, 2, 0, 33, 16), (4, 2, 1, 128, 0), (300, 2, 1, 40, 16)]


def rotary_case(n, heads, kv, dim, pairs, dt, extra, shift):
    rng = np.random.default_rng(n * dim + pairs)
    make = lambda c, s=1.0: strided(dev(rng.normal(size=(n, c)) * s, dt), extra, shift)  # noqa: E731
    q, k = make(heads * dim), make(kv * dim) if kv else None
    freq = torch.tensor(10000.0 ** (-np.arange(pairs) / max(pairs, 1)), dtype=torch.float32, device="cuda") if pairs else None
    pos = rng.integers(0, 3_000_000, n) if pairs else None
    if pairs:
        pos[0] = 0
    return rng, make, q, k, freq, pos


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,heads,kv,dim,pairs", HEADS)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("extra,shift,param", [(0, 0, "f32"), (8, 0, None), (3, 1, "f32")])
def test_qk_norm_and_backward(ops, dtype, n, heads, kv, dim, pairs, interleaved, extra, shift, param):
    dt = TYPES[dtype]
    pt = TYPES[param] if param else dt
    rng, make, q, k, freq, pos = rotary_case(n, heads, kv, dim, pairs, dt, extra, shift)
    qw, kw = (dev(rng.normal(size=dim) * 0.3 + 1, pt) for _ in range(2))
    if param is None:
        qw = None                                              # weights of one
    kw = kw if kv else None
    p = None if pos is None else ints(pos, torch.int32 if extra else torch.int64)
    common = dict(head_dim=dim, q_weight=qw, k_weight=kw, eps=1e-5, interleaved=interleaved)
    qo, ko = make(heads * dim), make(kv * dim) if kv else None
    ops.qk_norm(q, k, qo, ko, p, freq, **common)
    dqo, dko = make(heads * dim, 0.1), make(kv * dim, 0.1) if kv else None
    dq, dk = make(heads * dim), make(kv * dim) if kv else None
    dqw, dkw = torch.empty(dim, dtype=pt, device="cuda"), torch.empty(dim, dtype=pt, device="cuda") if kv else None
    ops.qk_norm_backward(dqo, dko, q, k, dq, dk, p, freq, dq_weight=dqw, dk_weight=dkw, **common)
    f = [] if freq is None else host(freq)
    K = dim / 8 + 24
    eps = float(np.float32(1e-5))
    for x, w, out, dout, dx, dw in ((q, qw, qo, dqo, dq, dqw), (k, kw, ko, dko, dk, dkw)):
        if x is None:
            continue
        wh = None if w is None else host(w)
        want = O.qk_norm(host(x), dim, wh, eps, pos, f, interleaved)
        h = host(x).reshape(n, -1, dim)
        r = 1 / np.sqrt((h * h).mean(2, keepdims=True) + eps)
        one = np.ones(dim) if wh is None else np.abs(wh)
        top = (np.abs(h) * r * one).max(2, keepdims=True) + 0 * h
        close(out, want, U[dt] * np.abs(want) + 2 * K * E * top.reshape(want.shape) + TINY[dt], "out")
        wdx, wdw = O.qk_norm_backward(host(dout), host(x), dim, wh, eps, pos, f, interleaved)
        dn = O._turned(host(dout).reshape(h.shape), pos, f, interleaved, back=True)
        amp = np.abs(host(dout).reshape(h.shape)).max(2, keepdims=True)
        g = 2 * amp * one.max()
        lim = r * (g + np.abs(h * r).max(2, keepdims=True) * (g * np.abs(h * r)).mean(2, keepdims=True)) + 0 * h
        close(dx, wdx, U[dt] * np.abs(wdx) + 2 * K * E * lim.reshape(wdx.shape) + TINY[dt], "dx")
        N = n * h.shape[1]
        close(dw, wdw, U[pt] * np.abs(wdw) + ((N + 8) * E * (np.abs(dn * h * r)).sum((0, 1)) + 2 * K * E * (2 * amp * np.abs(h * r)).sum((0, 1))) + TINY[pt],
              "dweight")
        if extra:
            c = x.shape[1]
            for t in (out, dx):
                assert torch.isnan(t._base[shift:shift + n * (c + extra)].view(n, c + extra)[:, c:]).all()


def test_qk_norm_in_place_and_in_slices(ops):
    gen = torch.Generator(device="cuda").manual_seed(1)
    n, h, kv, d = 200, 6, 2, 64
    qkv = torch.randn(n, (h + 2 * kv) * d, generator=gen, device="cuda", dtype=torch.bfloat16)
    q, k = qkv[:, :h * d], qkv[:, h * d:(h + kv) * d]
    freq = torch.rand(32, generator=gen, device="cuda")
    pos = torch.arange(n, device="cuda")
    qo, ko = torch.empty(n, h * d, dtype=q.dtype, device="cuda"), torch.empty(n, kv * d, dtype=q.dtype, device="cuda")
    ops.qk_norm(q, k, qo, ko, pos, freq, head_dim=d)
    values = qkv[:, (h + kv) * d:].clone()
    dqo, dko = torch.randn_like(qo), torch.randn_like(ko)
    dq, dk = torch.empty_like(qo), torch.empty_like(ko)
    ops.qk_norm_backward(dqo, dko, q, k, dq, dk, pos, freq, head_dim=d)
    ops.qk_norm_backward(dqo, dko, q, k, dqo, dko, pos, freq, head_dim=d)
    assert torch.equal(dq, dqo) and torch.equal(dk, dko)
    ops.qk_norm(q, k, q, k, pos, freq, head_dim=d)
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(qkv[:, (h + kv) * d:], values)


def test_rotation_of_far_positions(ops):
    """Angles of positions beyond 32 bits: the product with the frequency is reduced before it is rounded."""
    pos = np.array([0, 2 ** 24 + 1, 2 ** 31 + 5, 2 ** 40 + 3])
    freq = torch.tensor([1.0, 0.1, 1e-3, 1e-7], device="cuda")
    x = dev(np.tile([1.0, 0.0], (4, 4)))
    out = torch.empty_like(x)
    ops.qk_norm(x, None, out, None, ints(pos), freq, head_dim=8, eps=0.0, interleaved=True)
    turns = pos[:, None] * host(freq)[None]
    want = np.stack([np.cos(turns), np.sin(turns)], 2).reshape(4, 8) * np.sqrt(2)
    # an angle is off by two roundings of 53 bits
    close(out, want, 8 * E * np.sqrt(2) + 0 * want + (np.repeat(turns, 2, 1) * 2.0 ** -51), "out")


def test_qk_norm_gradients_agree_with_differences():
    rng = np.random.default_rng(2)
    x, up, w = rng.normal(size=(3, 12)), rng.normal(size=(3, 12)), rng.normal(size=6)
    kw = dict(eps=1e-3, positions=[0, 5, 9], freq=[0.7, 0.2])
    for inter in (False, True):
        dx, dw = O.qk_norm_backward(up, x, 6, w, interleaved=inter, **kw)
        f = lambda x_, w_: (O.qk_norm(x_, 6, w_, interleaved=inter, **kw) * up).sum()  # noqa: E731
        for i in np.ndindex(x.shape):
            e = np.zeros_like(x)
            e[i] = 1e-5
            assert abs((f(x + e, w) - f(x - e, w)) / 2e-5 - dx[i]) < 1e-7
        for i in range(6):
            e = np.zeros(6)
            e[i] = 1e-5
            assert abs((f(x, w + e) - f(x, w - e)) / 2e-5 - dw[i]) < 1e-7


# ----------------------------------------------------------------------------- attention

def attention_case(n, heads, kv, dim, dt, seed=0, extra=0, shift=0, size=1.0):
    rng = np.random.default_rng(seed + n * dim)
    make = lambda c, s=1.0: strided(dev(rng.normal(size=(n, c)) * s, dt), extra, shift)  # noqa: E731
    return rng, make, make(heads * dim, size), make(kv * dim, size), make(kv * dim)


def score_tol(q, k, heads, scale):
    """d of the docstring: an upper bound over all pairs."""
    n, dim = len(q), q.shape[1] // heads
    a = np.abs(np.nan_to_num(q, posinf=0, neginf=0)).reshape(n, -1, dim)
    b = np.abs(np.nan_to_num(k, posinf=0, neginf=0)).reshape(n, -1, dim)
    group = a.shape[1] // b.shape[1]
    worst = 0.0
    for h in range(heads):
        worst = max(worst, (a[:, h] @ b[:, h // group].T).max())
    return 2 * (dim + 16) * E * scale * worst


def check_attention(ops, q, k, v, heads, dt, make, causal, mask, kw, scale=None, left=0):
    n, dim = q.shape[0], q.shape[1] // heads
    out = make(heads * dim)
    out.fill_(3.0)
    lse = torch.full((heads, n), 3.0, device="cuda")
    ops.attention(q, k, v, out, heads=heads, lse=lse, causal=causal, mask=truths(mask), scale=scale, **kw)
    okw = {a: (host(b).astype(int) if isinstance(b, torch.Tensor) else b) for a, b in kw.items()}
    s = float(np.float32(dim ** -0.5 if scale is None else scale))
    want, wlse = O.attention(host(q), host(k), host(v), heads, causal=causal, mask=mask, scale=s, **okw)
    none = np.isnan(wlse)
    used = n - left
    assert torch.equal(out[used:], torch.full_like(out[used:], 3.0)) and (lse[:, used:] == 3.0).all()
    d = score_tol(host(q), host(k), heads, s)
    size, _ = O.attention(host(q), host(k), np.abs(np.nan_to_num(host(v))), heads, causal=causal, mask=mask, scale=s, **okw)
    up = U[dt] if dt != torch.float32 else 0.0
    tiny = 2.0 ** -24 * np.abs(np.nan_to_num(host(v))).max() * n if dt == torch.float16 else 0.0
    tol = U[dt] * np.abs(want) + (up + 2 * d + (n + 32) * E) * size + tiny + TINY[dt]
    close(out[:used], want[:used], tol[:used], "out")
    assert not none[:, :used].any()
    close(lse[:, :used], wlse[:, :used], d + 8 * E * (1 + np.abs(np.where(np.isinf(wlse), 0, wlse)))[:, :used] + n * E, "lse")
    return out, lse, d


def check_attention_backward(ops, q, k, v, out, lse, heads, dt, make, causal, mask, kw, d, scale=None, left=0, dout=None):
    n, dim, kc = q.shape[0], q.shape[1] // heads, k.shape[1]
    dout = make(heads * dim, 0.5) if dout is None else dout
    dq, dk, dv = make(heads * dim), make(kc), make(kc)
    for t in (dq, dk, dv):
        t.fill_(3.0)
    dot = torch.full((heads, n), 3.0, device="cuda")
    ops.attention_backward(dout, q, k, v, out, lse, dot, dq, dk, dv, heads=heads, causal=causal, mask=truths(mask), scale=scale, **kw)
    okw = {a: (host(b).astype(int) if isinstance(b, torch.Tensor) else b) for a, b in kw.items()}
    s = float(np.float32(dim ** -0.5 if scale is None else scale))
    r = O.attention_backward(host(dout), host(q), host(k), host(v), host(out), host(lse), heads, causal=causal, mask=mask, scale=s, **okw)
    up = U[dt] if dt != torch.float32 else 0.0
    finite = lambda t: np.abs(np.nan_to_num(host(t), posinf=0, neginf=0))  # noqa: E731
    wl = np.abs(np.where(np.isfinite(host(lse)), host(lse), 0)).max()
    group = heads * dim // kc
    flushed = 2.0 ** -126 * (1 + 2 * dim * finite(dout).max() * max(finite(v).max(), finite(out).max()))
    step = (2.0 ** -25 if dt == torch.float16 else 0.0) + flushed
    common = up + 2 * d + 8 * E * (1 + wl) + 2 * (dim + 16) * E + (n * group + 32) * E
    used = n - left
    for name, got, size, low in (("dq", dq, r["aq"], finite(k).max() * n * s), ("dk", dk, r["ak"], finite(q).max() * n * group * s),
                                 ("dv", dv, r["av"], finite(dout).max() * n * group)):
        assert torch.equal(got[used:], torch.full_like(got[used:], 3.0)), name
        tol = U[dt] * np.abs(r[name]) + common * size + step * low + TINY[dt]
        close(got[:used], r[name][:used], tol[:used], name)
    do, oo = (np.nan_to_num(host(t)).reshape(n, heads, dim) for t in (dout, out))
    close(dot[:, :used], r["row_dot"][:, :used], (dim + 8) * E * (np.abs(do) * np.abs(oo)).sum(2).T[:, :used] + 2.0 ** -126, "row_dot")
    return dq, dk, dv


SHAPES = [  # lengths of the sequences, heads, key heads, head length
    ([1], 1, 1, 8), ([1, 1, 1], 2, 1, 64), ([2, 7], 2, 2, 16), ([63, 64, 65], 2, 1, 64), ([127], 2, 1, 128), ([128, 128], 2, 2, 64),
    ([129, 3], 4, 2, 128), ([255, 0, 257], 2, 1, 64), ([256], 4, 1, 128), ([300, 17, 0, 0, 200], 2, 2, 80), ([513], 1, 1, 128), ([640, 130], 2, 1, 32),
    ([70, 90], 2, 1, 50), ([45], 2, 1, 192), ([100, 33], 2, 2, 256), ([40, 60], 3, 3, 7)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("extra,shift", [(0, 0), (8, 8), (5, 1)])
def test_attention_and_backward(ops, dtype, shape, causal, masked, extra, shift):
    lengths, heads, kv, dim = SHAPES[shape]
    dt, n = TYPES[dtype], sum(lengths)
    rng, make, q, k, v = attention_case(n, heads, kv, dim, dt, shape, extra, shift, 1.2)
    mask = rng.random(n) < 0.7 if masked else None
    kw = dict(seq_start=ints(np.cumsum([0] + lengths), torch.int32))
    out, lse, d = check_attention(ops, q, k, v, heads, dt, make, causal, mask, kw)
    check_attention_backward(ops, q, k, v, out, lse, heads, dt, make, causal, mask, kw, d)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("steps,seqs,dim", [(1, 5, 64), (40, 6, 64), (130, 2, 128), (260, 1, 64)])
def test_attention_of_a_padded_batch(ops, dtype, causal, steps, seqs, dim):
    """Equal runs, padding behind (and in one sequence before) the counted tokens, one sequence wholly masked; the padding holds NaN and infinities."""
    dt, n, heads, kv = TYPES[dtype], steps * seqs, 2, 1
    rng, make, q, k, v = attention_case(n, heads, kv, dim, dt, 7)
    last = rng.integers(1, steps + 1, seqs)
    mask = np.arange(steps)[None] < last[:, None]
    if seqs > 2:
        mask[1] = False
        mask[2] = np.arange(steps) >= steps // 2
    mask = mask.reshape(n)
    off = torch.from_numpy(~mask).cuda()
    for j, t in enumerate((q, k, v)):
        t[off] = (float("nan"), float("inf"), float("-inf"))[j]
    kw = dict(sequences=seqs)
    out, lse, d = check_attention(ops, q, k, v, heads, dt, make, causal, mask, kw, scale=0.3)
    assert not out[off].any() and torch.isinf(lse[:, off]).all()
    dout = make(heads * dim, 0.5)
    dout[off] = float("nan")
    out[off] = float("inf")
    lse[:, off] = float("nan")
    dq, dk, dv = check_attention_backward(ops, q, k, v, out, lse, heads, dt, make, causal, mask, kw, d, scale=0.3, dout=dout)
    assert not dq[off].any() and not dk[off].any() and not dv[off].any()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim", [64, 128, 24])
def test_attention_keeps_sequences_apart(ops, dtype, dim):
    """A sequence of NaN reaches none of its neighbours, rows of no sequence stay as they are, edges outside the batch are cut off."""
    dt, heads, kv = TYPES[dtype], 2, 1
    lengths = [70, 33, 150]
    n, left = sum(lengths) + 9, 9
    rng, make, q, k, v = attention_case(n, heads, kv, dim, dt, 3)
    start = ints(np.cumsum([0] + lengths), torch.int32)
    kw = dict(seq_start=start)
    out, lse, d = check_attention(ops, q, k, v, heads, dt, make, False, None, kw, left=left)
    dout = make(heads * dim, 0.5)
    grads = check_attention_backward(ops, q, k, v, out, lse, heads, dt, make, False, None, kw, d, left=left, dout=dout)
    bad = [t.clone() for t in (q, k, v, dout)]
    for t in bad:
        t[70:103] = float("nan")
        t[253:] = float("inf")
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    ops.attention(*bad[:3], out2, heads=heads, lse=lse2, causal=False, **kw)
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[70:103] = False
    keep[253:] = False
    assert torch.equal(out2[keep], out[keep]) and torch.equal(lse2[:, keep], lse[:, keep])
    assert torch.isnan(out2[70:103]).all()
    g2 = [torch.empty_like(t) for t in grads]
    dot = torch.empty_like(lse)
    ops.attention_backward(bad[3], *bad[:3], out2, lse2, dot, *g2, heads=heads, causal=False, **kw)
    for a, b in zip(grads, g2):
        assert torch.equal(a[keep], b[keep]) and torch.isnan(b[70:103]).all()
    wide = torch.tensor([-5, 70, 103, 10 ** 6], dtype=torch.int32, device="cuda")    # cut off at 0 and n
    inside = torch.tensor([0, 70, 103, n], dtype=torch.int32, device="cuda")
    a, b = torch.empty_like(out), torch.empty_like(out)
    ops.attention(q, k, v, a, heads=heads, seq_start=wide)
    ops.attention(q, k, v, b, heads=heads, seq_start=inside)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_of_large_scores(ops, dtype, dim):
    """Scores far from zero, rising along the row: the running maximum moves on every tile.  And infinities that count."""
    dt, heads, n = TYPES[dtype], 1, 400
    rng, make, q, k, v = attention_case(n, heads, 1, dim, dt, 5)
    q.fill_(0.0)
    q[:, 0] = 8.0
    k[:, 0] = torch.arange(n, device="cuda").to(dt) * 0.25
    kw = dict(sequences=1)
    out, lse, d = check_attention(ops, q, k, v, heads, dt, make, True, None, kw, scale=1.0)
    check_attention_backward(ops, q, k, v, out, lse, heads, dt, make, True, None, kw, d, scale=1.0)
    k[:, 0] = -k[:, 0] - 50.0
    out, lse, d = check_attention(ops, q, k, v, heads, dt, make, False, None, kw, scale=1.0)
    check_attention_backward(ops, q, k, v, out, lse, heads, dt, make, False, None, kw, d, scale=1.0)
    q[:, 0] = 1.0
    k[7, 0] = float("-inf")                                   # a key that no row gives weight: as if it were not there
    out2 = torch.empty_like(out)
    ops.attention(q, k, v, out2, heads=1, sequences=1, causal=False, scale=1.0)
    assert torch.isfinite(out2).all()


def test_attention_repeats_itself(ops):
    for dt, dim in ((torch.bfloat16, 128), (torch.float16, 64), (torch.float32, 64)):
        n, heads, kv = 1500, 4, 2
        _, make, q, k, v = attention_case(n, heads, kv, dim, dt, 9)
        first = None
        for _ in range(3):
            out, lse = make(heads * dim), torch.empty(heads, n, device="cuda")
            dq, dk, dv, dot = make(heads * dim), make(kv * dim), make(kv * dim), torch.empty(heads, n, device="cuda")
            ops.attention(q, k, v, out, heads=heads, lse=lse, sequences=3)
            ops.attention_backward(q, q, k, v, out, lse, dot, dq, dk, dv, heads=heads, sequences=3)
            got = (out, lse, dq, dk, dv, dot)
            if first is not None:
                assert all(torch.equal(a, b) for a, b in zip(first, got))
            first = got


def test_attention_gradients_agree_with_differences():
    rng = np.random.default_rng(4)
    q, k, v, up = rng.normal(size=(7, 8)), rng.normal(size=(7, 4)), rng.normal(size=(7, 4)), rng.normal(size=(7, 8))
    mask = np.array([1, 1, 0, 1, 1, 1, 1], bool)
    for causal in (False, True):
        kw = dict(seq_start=[0, 4, 7], causal=causal, mask=mask, scale=0.7)
        out, lse = O.attention(q, k, v, 2, **kw)
        r = O.attention_backward(up, q, k, v, out, lse, 2, **kw)
        for name, x in (("dq", q), ("dk", k), ("dv", v)):
            for i in np.ndindex(x.shape):
                old = x[i]
                x[i] = old + 1e-5
                a = (O.attention(q, k, v, 2, **kw)[0] * up).sum()
                x[i] = old - 1e-5
                b = (O.attention(q, k, v, 2, **kw)[0] * up).sum()
                x[i] = old
                assert abs((a - b) / 2e-5 - r[name][i]) < 1e-7, (name, i)


# ----------------------------------------------------------------------------- streams, graphs, refusals

def layer(ops, t, seqs):
    """All of them as a layer runs them, forwards and backwards; every tensor is t's."""
    ops.embedding(t["tok"], t["table"], t["x"], scale=2.0)
    torch.mm(t["x"], t["wqkv"], out=t["qkv"])
    hd, kd = t["q"].shape[1], t["k"].shape[1]
    q, k, v = t["qkv"][:, :hd], t["qkv"][:, hd:hd + kd], t["qkv"][:, hd + kd:]
    ops.qk_norm(q, k, t["q"], t["k"], t["pos"], t["freq"], head_dim=64, q_weight=t["w"], k_weight=t["w"])
    ops.attention(t["q"], t["k"], v, t["out"], heads=4, lse=t["lse"], sequences=seqs)
    ops.attention_backward(t["dout"], t["q"], t["k"], v, t["out"], t["lse"], t["dot"], t["dq"], t["dk"], t["dqkv"][:, hd + kd:], heads=4, sequences=seqs)
    ops.qk_norm_backward(t["dq"], t["dk"], q, k, t["dqkv"][:, :hd], t["dqkv"][:, hd:hd + kd], t["pos"], t["freq"], head_dim=64, q_weight=t["w"],
                         k_weight=t["w"], dq_weight=t["dqw"], dk_weight=t["dkw"])
    torch.mm(t["dqkv"], t["wqkv"].t(), out=t["dx"])
    ops.embedding_backward(t["tok"], t["dx"], t["dtable"], scale=2.0)


def layer_tensors(n, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    t = dict(tok=torch.randint(500, (n,), generator=gen, device="cuda"), table=r(500, 96), x=r(n, 96), wqkv=r(96, 512) * 0.1, qkv=r(n, 512), q=r(n, 256),
             k=r(n, 128), pos=torch.arange(n, device="cuda") % 100, freq=torch.rand(32, generator=gen, device="cuda"), w=r(64) * 0.1 + 1, out=r(n, 256),
             lse=torch.zeros(4, n, device="cuda"), dout=r(n, 256), dot=torch.zeros(4, n, device="cuda"), dq=r(n, 256), dk=r(n, 128), dqkv=r(n, 512),
             dqw=r(64), dkw=r(64), dx=r(n, 96), dtable=r(500, 96))
    return t


RESULTS = ("out", "lse", "dqkv", "dqw", "dkw", "dtable")


def test_a_layer_on_streams_and_in_graphs():
    n = 600
    ops = pkg.TrainingOps(n, 512)
    want = layer_tensors(n, 1)
    layer(ops, want, 2)
    torch.cuda.synchronize()
    other, t = torch.cuda.Stream(), layer_tensors(n, 1)
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):                            # calls made on a stream that is not the context's
        layer(ops, t, 2)
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda.synchronize()
    for name in RESULTS:
        assert torch.equal(t[name], want[name]), name
    side = torch.cuda.Stream()
    mine = pkg.TrainingOps(n, 512, stream=side)
    graphs, sets = [], [layer_tensors(n, 1), layer_tensors(n, 2)]
    side.wait_stream(torch.cuda.current_stream())
    for s in sets:                                            # two graphs that share the context's workspace
        with torch.cuda.stream(side):
            layer(mine, s, 2)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            layer(mine, s, 2)
        graphs.append(g)
    second = {name: sets[1][name].clone() for name in RESULTS}
    for s in sets:
        for name in RESULTS:
            s[name].zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(3):
            for g in graphs:
                g.replay()
    side.synchronize()
    for name in RESULTS:
        assert torch.equal(sets[0][name], want[name]) and torch.equal(sets[1][name], second[name]), name
    mine.close()
    ops.close()


def test_refusals(ops):
    x = torch.randn(6, 32, device="cuda")
    o, tok, tab = torch.empty_like(x), torch.zeros(6, dtype=torch.int64, device="cuda"), torch.randn(9, 32, device="cuda")
    dt = torch.empty_like(tab)
    k, v = torch.randn(6, 16, device="cuda"), torch.randn(6, 16, device="cuda")
    ko, lse, f = torch.empty_like(k), torch.empty(4, 6, device="cuda"), torch.ones(4, device="cuda")
    pos = torch.arange(6, device="cuda")
    w = torch.ones(8, device="cuda")
    big = torch.randn(6, 80, device="cuda")
    dq, dk, dv = torch.empty_like(x), torch.empty_like(k), torch.empty_like(k)
    grad = torch.empty(6, 32, device="cuda", requires_grad=True)
    att = dict(heads=4, sequences=2)
    wrong = [
        lambda: ops.embedding(tok.float(), tab, o), lambda: ops.embedding(tok[:5], tab, o), lambda: ops.embedding(tok, tab, o[:, :31]),
        lambda: ops.embedding(tok, tab.bfloat16(), o), lambda: ops.embedding(tok, tab, o, mask=torch.ones(6, device="cuda")),
        lambda: ops.embedding(tok.cpu(), tab, o), lambda: ops.embedding(tok, tab.t(), o), lambda: ops.embedding(tok, tab, grad),
        lambda: ops.embedding_backward(tok, x, dt[:, :31]), lambda: ops.embedding_backward(tok, x, dt.bfloat16()),
        lambda: ops.embedding_backward(tok, x.bfloat16(), dt.half()), lambda: ops.embedding_backward(tok, x, dt, base=tab[:8]),
        lambda: ops.embedding_backward(tok, x, None),
        lambda: ops.qk_norm(x, k, o, ko, head_dim=0), lambda: ops.qk_norm(x, k, o, ko, head_dim=5), lambda: ops.qk_norm(x, k, o, None, head_dim=8),
        lambda: ops.qk_norm(x, None, o, ko, head_dim=8), lambda: ops.qk_norm(x, k, o, ko, None, f, head_dim=8),
        lambda: ops.qk_norm(x, k, o, ko, pos, torch.ones(5, device="cuda"), head_dim=8), lambda: ops.qk_norm(x, k, o, ko, pos, f.double(), head_dim=8),
        lambda: ops.qk_norm(x, k, o, ko, pos[:5], f, head_dim=8), lambda: ops.qk_norm(x, k, o, ko, head_dim=8, q_weight=w[:7]),
        lambda: ops.qk_norm(x, k, o, ko, head_dim=8, q_weight=w.half()), lambda: ops.qk_norm(x, k[:5], o, ko, head_dim=8),
        lambda: ops.qk_norm_backward(x, None, x, k, o, ko, head_dim=8), lambda: ops.qk_norm_backward(x, k, x, k, o, None, head_dim=8),
        lambda: ops.attention(x, k, v, o, heads=4), lambda: ops.attention(x, k, v, o, heads=0, sequences=1), lambda: ops.attention(x, k, v, o, heads=5, sequences=1),
        lambda: ops.attention(x, k[:, :12], v, o, **att), lambda: ops.attention(x, big[:, :24], big[:, 24:48], o, **att), lambda: ops.attention(x, k, v[:, :8], o, **att),
        lambda: ops.attention(x, k, v, o, lse=lse[:3], **att), lambda: ops.attention(x, k, v, o, lse=lse.half(), **att),
        lambda: ops.attention(x, k, v, grad, **att), lambda: ops.attention(x.expand(6, 32)[:1].expand(6, 32), k, v, o, **att),
        lambda: ops.attention(x, k, v, o, heads=4, seq_start=torch.zeros(3, dtype=torch.int64, device="cuda")),
        lambda: ops.attention(x, k, v, o, heads=4, sequences=1, seq_start=torch.zeros(3, dtype=torch.int32, device="cuda")),
        lambda: ops.attention_backward(x, x, k, v, x, lse, None, dq, dk, dv, **att), lambda: ops.attention_backward(x, x, k, v, x, None, lse, dq, dk, dv, **att),
        lambda: ops.attention_backward(x, x, k, v, x, lse, torch.empty_like(lse), dq, dk[:, :8], dv, **att),
    ]
    for i, call in enumerate(wrong):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"refusal {i} went through")
    dot = torch.empty_like(lse)
    library = [
        lambda: ops.embedding(tok, tab, o, scale=float("inf")), lambda: ops.embedding(tok, tab, tab[:6]), lambda: ops.embedding(tok, x, x),
        lambda: ops.embedding_backward(tok, x, dt, scale=float("nan")), lambda: ops.embedding_backward(tok, x, x, base=x),
        lambda: ops.embedding_backward(tok, x, dt[:6], base=dt[1:7]), lambda: ops.embedding_backward(tok, x, x),
        lambda: ops.qk_norm(x, k, o, ko, head_dim=8, eps=-1.0), lambda: ops.qk_norm(x, x, o, o, head_dim=8), lambda: ops.qk_norm(x, o, o, x, head_dim=8),
        lambda: ops.qk_norm(x, x, x, o, head_dim=8), lambda: ops.qk_norm(big[:, :32], big[:, 32:48], big[:, 8:40], ko, head_dim=8),
        lambda: ops.qk_norm_backward(x, k, x, k, dq, dk, head_dim=8, q_weight=w, dq_weight=w),
        lambda: ops.attention(x, k, v, x, **att), lambda: ops.attention(x, k, v, o, heads=4, sequences=4), lambda: ops.attention(x, k, v, o, heads=4, sequences=0),
        lambda: ops.attention(x, k, v, o, heads=4, sequences=1, scale=0.0), lambda: ops.attention(x, k, v, o, heads=4, sequences=1, scale=float("inf")),
        lambda: ops.attention(x, k, v, o, heads=4, seq_start=torch.zeros(1, dtype=torch.int32, device="cuda")),
        lambda: ops.attention_backward(x, x, k, v, x, lse, lse, dq, dk, dv, **att), lambda: ops.attention_backward(x, x, k, v, x, lse, dot, x, dk, dv, **att),
        lambda: ops.attention_backward(x, x, k, v, x, lse, dot, dq, dk, dk, **att),
    ]
    before = ops.launch_count()
    for i, call in enumerate(library):
        with pytest.raises(pkg.AdacgdError) as e:
            call()
            pytest.fail(f"library refusal {i} went through")
        assert e.value.status == 1 and "adacgd_" in str(e.value), i
    assert ops.launch_count() == before
    small = pkg.TrainingOps(4, 8)
    for call in (lambda: small.embedding_backward(tok, x, dt), lambda: small.qk_norm_backward(x, k, x, k, dq, dk, head_dim=8)):
        with pytest.raises(pkg.AdacgdError):
            call()
    small.close()


def test_no_tokens(ops):
    e = lambda c: torch.empty(0, c, device="cuda")  # noqa: E731
    t = torch.zeros(0, dtype=torch.int64, device="cuda")
    ops.embedding(t, torch.randn(3, 8, device="cuda"), e(8))
    g = torch.full((3, 8), 4.0, device="cuda")
    ops.embedding_backward(t, e(8), g)
    assert not g.any()
    ops.qk_norm(e(16), e(8), e(16), e(8), t, torch.ones(2, device="cuda"), head_dim=8)
    dw = torch.full((8,), 4.0, device="cuda")
    ops.qk_norm_backward(e(16), e(8), e(16), e(8), e(16), e(8), head_dim=8, q_weight=torch.ones(8, device="cuda"), dq_weight=dw)
    assert not dw.any()
    lse = torch.empty(2, 0, device="cuda")
    ops.attention(e(16), e(8), e(8), e(16), heads=2, lse=lse, sequences=1)
    ops.attention_backward(e(16), e(16), e(8), e(8), e(16), lse, torch.empty(2, 0, device="cuda"), e(16), e(8), e(8), heads=2, sequences=1)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("count", [31, 32, 40, 1000])
def test_attention_of_many_sequences(ops, dtype, count):
    """More sequences than a warp looks at in one round, empty ones among them."""
    rng = np.random.default_rng(count)
    lengths = rng.integers(0, 4, count)
    lengths[rng.integers(0, count)] = 150
    dt, n = TYPES[dtype], int(lengths.sum())
    _, make, q, k, v = attention_case(n, 2, 1, 64, dt, count)
    kw = dict(seq_start=ints(np.concatenate([[0], np.cumsum(lengths)]), torch.int32))
    out, lse, d = check_attention(ops, q, k, v, 2, dt, make, True, None, kw)
    check_attention_backward(ops, q, k, v, out, lse, 2, dt, make, True, None, kw, d)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("counted", [(300, 420), (0, 130), (560, 700), (128, 256), (699, 700)])
def test_attention_of_tiles_without_a_counted_token(ops, dtype, causal, counted):
    """Whole tiles of padding in front of and behind the tokens, and a hole among them; the padding holds NaN."""
    dt, n, heads, kv, dim = TYPES[dtype], 700, 2, 1, 64
    rng, make, q, k, v = attention_case(n, heads, kv, dim, dt, counted[0])
    mask = np.zeros(n, bool)
    mask[counted[0]:counted[1]] = True
    if counted[1] - counted[0] > 50:
        mask[counted[0] + 20:counted[0] + 30] = False
    off = torch.from_numpy(~mask).cuda()
    for t in (q, k, v):
        t[off] = float("nan")
    kw = dict(sequences=1)
    out, lse, d = check_attention(ops, q, k, v, heads, dt, make, causal, mask, kw)
    dout = make(heads * dim, 0.5)
    dout[off] = float("nan")
    check_attention_backward(ops, q, k, v, out, lse, heads, dt, make, causal, mask, kw, d, dout=dout)


@pytest.mark.parametrize("size", [1e-4, 1.0, 200.0])
def test_small_and_large_gradients_in_float16(ops, size):
    """ds is brought into the type's range before it is rounded: gradients of 1e-4 keep its eleven bits, gradients of 200 do not overflow."""
    dt, n, heads, kv, dim = torch.float16, 1000, 2, 1, 64
    _, make, q, k, v = attention_case(n, heads, kv, dim, dt, 12)
    out, lse = make(heads * dim), torch.empty(heads, n, device="cuda")
    ops.attention(q, k, v, out, heads=heads, lse=lse, sequences=1, causal=False)
    dout = make(heads * dim, size)
    dq, dk, dv, dot = make(heads * dim), make(kv * dim), make(kv * dim), torch.empty(heads, n, device="cuda")
    ops.attention_backward(dout, q, k, v, out, lse, dot, dq, dk, dv, heads=heads, sequences=1, causal=False)
    r = O.attention_backward(host(dout), host(q), host(k), host(v), host(out), host(lse), heads, sequences=1, causal=False)
    for name, got in (("dq", dq), ("dk", dk), ("dv", dv)):
        # p or ds and the result are each off by at most 2^-11 of themselves, by chance in a sum: less than 2^-10 of the whole; the results' own
        # smallest step, 2^-24, adds half of itself an element
        lim = 2.0 ** -10 * np.linalg.norm(r[name]) + 2.0 ** -25 * np.sqrt(r[name].size)
        assert np.linalg.norm(host(got) - r[name]) < lim, name
