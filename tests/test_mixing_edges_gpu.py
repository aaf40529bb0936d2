"""Calls of the operators that mix tokens which the formulas allow and an ordinary batch does not make.  Tolerances: see test_mixing_gpu.py."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2211_00188_b200 as pkg
from oracle import training_oracle as O
from test_mixing_gpu import attention_case, ints, score_tol
from test_training_gpu import TYPES, U, close, dev, host, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    return pkg.TrainingOps(70000, 32768)


# ----------------------------------------------------------------------------- attention

class Both:
    """Attention and its backward pass on tensors of its own."""

    def __init__(self, ops, n, heads, kv, dim, dt, seed=0, **kw):
        self.ops, self.heads, self.kw = ops, heads, kw
        _, make, self.q, self.k, self.v = attention_case(n, heads, kv, dim, dt, seed)
        self.dout, self.out = make(heads * dim, 0.5), make(heads * dim)
        self.dq, self.dk, self.dv = make(heads * dim), make(kv * dim), make(kv * dim)
        self.lse, self.dot = torch.empty(heads, n, device="cuda"), torch.empty(heads, n, device="cuda")

    def forward(self):
        self.ops.attention(self.q, self.k, self.v, self.out, heads=self.heads, lse=self.lse, **self.kw)

    def backward(self):
        self.ops.attention_backward(self.dout, self.q, self.k, self.v, self.out, self.lse, self.dot, self.dq, self.dk, self.dv, heads=self.heads, **self.kw)

    def __call__(self):
        self.forward()
        self.backward()

    def results(self):
        return self.out, self.lse, self.dot, self.dq, self.dk, self.dv

    def fill(self, value):
        for t in self.results():
            t.fill_(value)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim", [64, 128])
def test_only_empty_sequences(ops, dtype, dim):
    """Tokens, but every sequence empty: nothing is written, and a call right behind it, in a stream's order or in a graph, has the bits it has alone."""
    dt = TYPES[dtype]
    ordinary = Both(ops, 700, 4, 2, dim, dt, 1, sequences=2)
    ordinary()
    want = [t.clone() for t in ordinary.results()]
    starts = [ints([at] * 4, torch.int32) for at in (0, 300)]
    empty = [Both(ops, 300, 4, 2, dim, dt, 2, seq_start=s) for s in starts]
    for e in empty:
        e.fill(3.0)
    ordinary.fill(0.0)
    for e in empty:
        e()
    ordinary()
    for e in empty:
        assert all((t == 3.0).all() for t in e.results())
    for a, b in zip(ordinary.results(), want):
        assert torch.equal(a, b)
    side = torch.cuda.Stream()
    mine = pkg.TrainingOps(1000, 512, stream=side)
    for b in [ordinary] + empty:
        b.ops = mine
    ordinary.fill(0.0)
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for e in empty:
            e()
        ordinary()
    with torch.cuda.stream(side):
        for _ in range(3):
            graph.replay()
    side.synchronize()
    for e in empty:
        assert all((t == 3.0).all() for t in e.results())
    for a, b in zip(ordinary.results(), want):
        assert torch.equal(a, b)
    del graph
    mine.close()


def float16_case(ops, lengths, heads, kv, dim, seed, causal):
    start = ints(np.cumsum([0] + list(lengths)), torch.int32)
    b = Both(ops, sum(lengths), heads, kv, dim, torch.float16, seed, seq_start=start, causal=causal)
    b.q *= 1.2
    b.dout *= 0.01
    return b


def part(b, rows):
    """The same tensors cut to the rows of one sequence, which then stands alone."""
    n = rows.stop - rows.start
    alone = Both(b.ops, n, b.heads, b.k.shape[1] * b.heads // b.q.shape[1], b.q.shape[1] // b.heads, b.q.dtype, 0, sequences=1, causal=b.kw["causal"])
    for name in ("q", "k", "v", "dout"):
        getattr(alone, name).copy_(getattr(b, name)[rows])
    return alone


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim,heads,kv", [(64, 2, 2), (128, 4, 2), (8, 9, 1), (80, 3, 1)])
@pytest.mark.parametrize("other", ["large", "infinite dout", "infinite v", "nothing"])
def test_float16_gradients_of_a_sequence_do_not_depend_on_another(ops, causal, dim, heads, kv, other):
    """ds is brought into the type's range by a power of two; what decides it is the row's or the sequence's own.  A neighbour 10^5 times larger, or
    infinite, changes no bit."""
    lengths = [200, 333, 140]
    b = float16_case(ops, lengths, heads, kv, dim, dim + heads, causal)
    if other == "nothing":
        b.dout[200:533] = 0.0
    elif other == "large":
        b.dout[200:533] *= 1e5
        b.v[200:533] *= 10
    elif other == "infinite v":
        b.v[300, 0] = float("inf")
    else:
        b.dout[300, 1] = float("-inf")
    b()
    for rows in (slice(0, 200), slice(533, 673)):
        alone = part(b, rows)
        alone()
        for name in ("out", "dq", "dk", "dv"):
            assert torch.equal(getattr(b, name)[rows], getattr(alone, name)), name
        assert torch.equal(b.lse[:, rows], alone.lse) and torch.equal(b.dot[:, rows], alone.dot)


def test_float16_gradients_of_a_key_head_do_not_depend_on_another(ops):
    b = float16_case(ops, [300, 90], 4, 2, 64, 3, True)
    b()
    want = [t.clone() for t in (b.dq, b.dk, b.dv)]
    b.dout[:, 128:] *= 1e5
    b.v[:, 64:] = float("inf")
    b()
    for got, w, cols in zip((b.dq, b.dk, b.dv), want, (128, 64, 64)):
        assert torch.equal(got[:, :cols], w[:, :cols])


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("value", [5e4, float("inf"), float("nan")])
def test_float16_gradients_of_a_query_do_not_depend_on_another(ops, causal, value):
    """One row of dout far above the others: their dq keeps its bits, which are those of the formula.  dq_i adds n terms scale ds_ij k_j; ds is rounded in
    binary16 (2^-11 of itself, or 2^-25 of its smallest step), multiplied so that 2 |dout_i| max|v| is at least 2^13."""
    n, heads, dim = 500, 2, 64
    b = float16_case(ops, [n], heads, 1, dim, 5, causal)
    b()
    want = b.dq.clone()
    b.dout[123] = value
    b()
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[123] = False
    assert torch.equal(b.dq[keep], want[keep])
    b.dout[123] = 0.0
    r = O.attention_backward(host(b.dout), host(b.q), host(b.k), host(b.v), host(b.out), host(b.lse), heads, sequences=1, causal=causal)
    s, E = dim ** -0.5, 2.0 ** -24
    d = score_tol(host(b.q), host(b.k), heads, s)
    wl = np.abs(host(b.lse)).max()
    size = np.linalg.norm(host(b.dout).reshape(n, heads, dim), axis=2).repeat(dim, 1)
    top = np.linalg.norm(host(b.v), axis=1).max()
    tol = 2.0 ** -11 * np.abs(r["dq"]) + (2.0 ** -11 + 2 * d + 8 * E * (1 + wl) + 2 * (dim + 16) * E + (n + 32) * E) * r["aq"]
    tol = tol + s * n * np.abs(host(b.k)).max() * 2.0 ** -25 * 2.002 * size * top / 2.0 ** 13 + 2.0 ** -25
    k = host(keep).astype(bool)
    close(want[keep], r["dq"][k], tol[k], "dq")


@pytest.mark.parametrize("causal", [False, True])
def test_float16_gradients_with_rows_far_apart(ops, causal):
    """Rows of dout over nine powers of ten, the largest in the middle: every row of dq has the accuracy of its own size."""
    n, heads, dim = 400, 2, 128
    b = float16_case(ops, [n], heads, 2, dim, 6, causal)
    b.forward()
    b.dout[:] = torch.randn_like(b.dout.float()).mul_(10.0 ** torch.linspace(-4, 2.5, n, device="cuda")[:, None]).half()
    b.backward()
    r = O.attention_backward(host(b.dout), host(b.q), host(b.k), host(b.v), host(b.out), host(b.lse), heads, sequences=1, causal=causal)
    got = host(b.dq).reshape(n, heads, dim)
    err = np.linalg.norm(got - r["dq"].reshape(n, heads, dim), axis=2)
    # as in test_small_and_large_gradients_in_float16, for each row; the terms of a row may cancel, so against the norm of their sizes
    lim = 2.0 ** -10 * np.linalg.norm(r["aq"].reshape(n, heads, dim), axis=2) + 2.0 ** -25 * np.sqrt(dim)
    assert (err < lim).all(), (err / lim).max()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,dim", [(128, 64), (384, 128)])
def test_keys_of_no_weight_have_none(ops, dtype, n, dim):
    """exp(-2000) is 0 in 64 bits too: values near the type's largest behind such scores reach nothing."""
    dt = TYPES[dtype]
    q, k, v = (torch.zeros(n, dim, device="cuda", dtype=dt) for _ in range(3))
    q[:, 0] = 1.0
    idle = torch.rand(n, generator=torch.Generator().manual_seed(n)).cuda() < 0.8
    idle[0] = False
    k[idle, 0] = -2000.0
    v[idle] = 6e4 if dtype == "f16" else 1e38
    v[~idle, 1] = 1.0
    out, lse = torch.empty_like(q), torch.empty(1, n, device="cuda")
    ops.attention(q, k, v, out, heads=1, lse=lse, sequences=1, causal=False, scale=1.0)
    want = torch.zeros_like(out)
    want[:, 1] = 1.0
    assert torch.equal(out[:, :1], want[:, :1]) and torch.equal(out[:, 2:], want[:, 2:])
    # the exponentials of the others are all 1, some by a polynomial that is off by 2.7e-6; the sum and the result add their roundings
    close(out, host(want), 2.7e-6 + (n + 32) * 2.0 ** -24 + U[dt] + np.zeros((n, dim)), "out")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("masked", [False, True])
def test_large_scores_of_other_rows_change_no_bit(ops, dtype, dim, causal, masked):
    """Rows of the next sequence, or that do not count, lie in the same tile of queries.  Their scores rise far from one tile of keys to the next, while
    those of the rows that count hardly do: the results are the bits of the sequence that stands alone, or of a batch whose masked rows hold zeros."""
    dt, n, heads = TYPES[dtype], 400, 2
    b = Both(ops, n, heads, 1, dim, dt, dim, causal=causal)
    start = ints([0, 200, 400], torch.int32)
    mask = torch.ones(n, dtype=torch.bool, device="cuda")
    if masked:
        mask[170:200:3] = False
        mask[360::2] = False
    b.kw.update(seq_start=start, mask=mask if masked else None)
    b.q.mul_(0.5)
    b.k[:, 5], b.k[0:128, 5], b.k[200:328, 5] = 0.0, 1.0, 1.0
    b.q[:, 5] = 0.0
    b.q[:, dim + 5] = 0.0
    plain = b.q.clone()
    b()
    want = [t.clone() for t in b.results()]
    for name, rows in (("next", slice(200, 400)), ("masked", ~mask)):
        b.q.copy_(plain)
        b.q[rows, 5] = 300.0
        b.q[rows, dim + 5] = 200.0
        b()
        keep = torch.zeros(n, dtype=torch.bool, device="cuda")
        keep[:200] = True
        if name == "masked":
            keep[:] = True
        for got, w, by_row in zip(b.results(), want, (True, False, False, True, True, True)):
            assert torch.equal(got[keep], w[keep]) if by_row else torch.equal(got[:, keep], w[:, keep]), name


# ----------------------------------------------------------------------------- norm and rotation

# head length, pairs, neighbours, extra columns, first element: each of the kernels' ways to a pair; heads longer than their rotated front
FRONTS = [(64, 16, True, 0, 0), (64, 0, False, 0, 0), (128, 16, False, 0, 0), (256, 24, False, 0, 0), (72, 8, False, 0, 0), (72, 12, False, 0, 0),
          (72, 10, False, 0, 0), (40, 8, True, 0, 0), (40, 0, True, 0, 0), (50, 12, True, 0, 0), (50, 12, False, 0, 0), (64, 16, True, 3, 1),
          (130, 0, False, 0, 0), (272, 60, True, 0, 0)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("dim,pairs,interleaved,extra,shift", FRONTS)
@pytest.mark.parametrize("where", ["x", "weight", "dout"])
def test_infinities_outside_the_rotated_front(ops, dtype, dim, pairs, interleaved, extra, shift, where):
    """An element that is not turned takes nothing from another one: an infinity there reaches what the formulas say, and no neighbour, in its own place or
    in a weight's gradient."""
    dt, rng, n, heads, kv, E = TYPES[dtype], np.random.default_rng(dim + pairs), 9, 3, 2, 2.0 ** -24
    make = lambda c, s=1.0: strided(dev(rng.normal(size=(n, c)) * s, dt), extra, shift)  # noqa: E731
    x, dout, w = [make(heads * dim), make(kv * dim)], [make(heads * dim, 0.1), make(kv * dim, 0.1)], [dev(rng.normal(size=dim) * 0.3 + 1) for _ in range(2)]
    places = {2 * pairs + 1, (2 * pairs + dim) // 2, dim - 1}
    for j, e in enumerate(places):
        for c in (0, 1):
            if where == "weight":
                w[c][e] = float("inf")
            else:
                (x if where == "x" else dout)[c][2 + 2 * j, (j % 2) * dim + e] = float("inf")
    pos, freq = rng.integers(1, 5000, n), torch.rand(pairs, device="cuda")
    rot = dict(positions=ints(pos), freq=freq) if pairs else {}
    out, dx, dw = [make(heads * dim), make(kv * dim)], [make(heads * dim), make(kv * dim)], [torch.empty(dim, device="cuda") for _ in range(2)]
    common = dict(head_dim=dim, q_weight=w[0], k_weight=w[1], eps=1e-5, interleaved=interleaved, **rot)
    ops.qk_norm(*x, *out, **common)
    ops.qk_norm_backward(*dout, *x, *dx, dq_weight=dw[0], dk_weight=dw[1], **common)
    K, eps, f = dim / 8 + 24, float(np.float32(1e-5)), host(freq)
    size = lambda t: np.abs(np.nan_to_num(t, nan=0.0, posinf=0.0, neginf=0.0))  # noqa: E731
    with np.errstate(all="ignore"):
        for c in (0, 1):
            wh, h, up = host(w[c]), host(x[c]).reshape(n, -1, dim), host(dout[c])
            want = O.qk_norm(host(x[c]), dim, wh, eps, pos, f, interleaved)
            r = 1 / np.sqrt((size(h) ** 2).mean(2, keepdims=True) + eps)
            hr, one, amp = size(h) * r, size(wh), size(up).reshape(h.shape).max(2, keepdims=True)
            top = (hr * one).max(2, keepdims=True) + 0 * hr
            close(out[c], want, U[dt] * np.abs(want) + 2 * K * E * top.reshape(want.shape) + 2.0 ** -25, "out")
            wdx, wdw = O.qk_norm_backward(up, host(x[c]), dim, wh, eps, pos, f, interleaved)
            g = 2 * amp * one.max()
            lim = r * (g + hr.max(2, keepdims=True) * (g * hr).mean(2, keepdims=True)) + 0 * hr
            close(dx[c], wdx, U[dt] * np.abs(wdx) + 2 * K * E * lim.reshape(wdx.shape) + 2.0 ** -25, "dx")
            close(dw[c], wdw, 2.0 ** -24 * np.abs(wdw) + ((n * h.shape[1] + 8) + 4 * K) * E * (2 * amp * hr).sum((0, 1)), "dweight")


# ----------------------------------------------------------------------------- the most tokens

class Inputs(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("sequences", C.c_int64), ("seq_start", C.c_void_p), ("mask", C.c_void_p)] + \
        [f for n in "qkv" for f in ((n, C.c_void_p), (n + "_stride", C.c_int64))] + \
        [("heads", C.c_int32), ("key_heads", C.c_int32), ("head_dim", C.c_int32), ("causal", C.c_int32), ("scale", C.c_float), ("dtype", C.c_int32)]


class Forward(C.Structure):
    _fields_ = [("in_", Inputs), ("out", C.c_void_p), ("out_stride", C.c_int64), ("lse", C.c_void_p)]


class Gradient(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("vocab", C.c_int64), ("cols", C.c_int64), ("ids", C.c_void_p), ("mask", C.c_void_p)] + \
        [f for n in ("dout", "base", "dtable") for f in ((n, C.c_void_p), (n + "_stride", C.c_int64))] + \
        [("scale", C.c_float), ("dtype", C.c_int32), ("table_dtype", C.c_int32), ("id_bytes", C.c_int32)]


def test_more_tokens_than_32_bit_places_are_refused():
    """The checks alone: a context for 2^31 - 1 tokens, whose workspace would take 51 GB and is never touched, and matrices that are not there."""
    lib = pkg.load_training_library()
    need, ctx, small = C.c_size_t(), C.c_void_p(), torch.zeros(4096, dtype=torch.uint8, device="cuda")
    most = 2 ** 31 - 2 ** 24
    assert lib.adacgd_train_workspace_bytes(2 ** 31 - 1, 8, C.byref(need)) == 0
    assert small.data_ptr() % 256 == 0
    assert lib.adacgd_train_init(C.byref(ctx), 2 ** 31 - 1, 8, small.data_ptr(), need.value, torch.cuda.current_stream().cuda_stream) == 0
    at = small.data_ptr()
    for tokens in (2 ** 31 - 1, most + 1):
        g = Gradient(tokens=tokens, vocab=5, cols=8, ids=at, dout=at, dout_stride=8, dtable=at, dtable_stride=8, scale=1.0, id_bytes=4)
        a = Forward(in_=Inputs(tokens=tokens, sequences=1, q=at, q_stride=8, k=at, k_stride=8, v=at, v_stride=8, heads=1, key_heads=1, head_dim=8, scale=1.0),
                    out=at, out_stride=8)
        for call, args in ((lib.adacgd_embedding_backward, g), (lib.adacgd_attention, a)):
            assert call(ctx, C.byref(args)) == 1
            assert b"MAX_RUN" in lib.adacgd_train_last_error(ctx)
    assert lib.adacgd_train_launch_count(ctx) == 0
    torch.cuda.synchronize()
    lib.adacgd_train_destroy(ctx)


# ----------------------------------------------------------------------------- lookup

@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n", [0, 40])
@pytest.mark.parametrize("cols", [24, 1001, 2056])
def test_a_gradient_of_no_token_that_counts(ops, dtype, n, cols):
    """Every row is written all the same: 0, or the base's; in place nothing is."""
    dt, vocab = TYPES[dtype], 77
    tok = torch.arange(n, device="cuda") % vocab
    dout = torch.full((n, cols), float("nan"), device="cuda", dtype=dt)
    mask = torch.zeros(n, dtype=torch.bool, device="cuda")
    base = torch.randn(vocab, cols, device="cuda").to(dt)
    g = torch.full_like(base, 5.0)
    ops.embedding_backward(tok, dout, g, mask=mask)
    assert not g.any()
    ops.embedding_backward(tok, dout, g, mask=mask, base=base)
    assert torch.equal(g, base)
    ops.embedding_backward(tok, dout, g, mask=mask, base=g)
    assert torch.equal(g, base)
