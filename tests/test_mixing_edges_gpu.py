"""Calls of the operators that mix tokens which the formulas allow and an ordinary batch does not make.  Tolerances: see test_mixing_gpu.py."""
import numpy as np
import pytest
import torch

import paper_2211_00188_b200 as pkg
from oracle import training_oracle as O
from test_mixing_gpu import attention_case, ints
from test_training_gpu import TYPES, close, dev, host, strided

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
