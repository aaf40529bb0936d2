"""The training operators on the device against their binary64 restatement (oracle/training_oracle.py).

Tolerances.  u(T) is the rounding of a stored result: 2^-24 (float32), 2^-11 (float16), 2^-8 (bfloat16), plus half the
smallest subnormal of float16.  E = 2^-24 is the rounding of the arithmetic in between.
  norm      out = h w + b, |h| <= (|s| + |mean|) rstd.  A sum of `cols` terms is a chain of at most cols / 128 + 16 additions
            (a thread's share, then trees), so mean and rstd are off by at most K E, K = cols / 128 + 32, relative to the
            row's largest |s| and to rstd: |error| <= u |out| + K E (max|s| rstd |w| + |out| + |b|).
  logits    an exponential is within 2^-21 of its value for the terms that count (2^-22 from the hardware, the rounding of the
            argument weighted by the term) and a sum adds a chain of vocab / 128 + 32 roundings: log-probabilities are off by
            at most L = (vocab / 128 + 64) E + 4 E max|z|.  A gradient c (1{y} - softmax) is off by
            u |d| + |c| (softmax L + 4 E) + |error of c|.
"""
import numpy as np
import pytest
import torch

import paper_2211_00188_b200 as pkg
from oracle import training_oracle as O

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}   # flushed exponentials: 2^-126


@pytest.fixture(scope="module")
def ops():
    return pkg.TrainingOps(70000, 32768)


def dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(dtype)


def host(t):
    return t.double().cpu().numpy()


def strided(t, extra=0, shift=0):
    """The same matrix inside a larger allocation: row stride cols + extra, first element `shift` elements in."""
    rows, cols = t.shape
    buf = torch.full((rows * (cols + extra) + shift + 8,), float("nan"), dtype=t.dtype, device=t.device)
    v = buf[shift:shift + rows * (cols + extra)].view(rows, cols + extra)[:, :cols]
    v.copy_(t)
    return v


def close(got, want, tol, what=""):
    got = host(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, (what, got.shape, want.shape)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), what
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), what
    ok = ~(nan | inf)
    err = np.abs(got - want)[ok]
    lim = np.broadcast_to(tol, want.shape)[ok]
    bad = err > lim
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {(err / np.maximum(lim, 1e-300)).max():.3g} x the tolerance"


# ----------------------------------------------------------------------------- dropout

@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols,extra,shift", [(1, 1, 0, 0), (1, 7, 0, 0), (3, 8, 0, 0), (5, 17, 0, 0), (5, 17, 3, 1),
                                                   (33, 64, 0, 0), (33, 64, 8, 0), (33, 64, 0, 3), (7, 1001, 0, 0), (2, 4099, 5, 2)])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(ops, dtype, rows, cols, extra, shift, residual):
    dt = TYPES[dtype]
    rng = np.random.default_rng(rows * cols + extra)
    x, res = dev(rng.normal(size=(rows, cols)), dt), dev(rng.normal(size=(rows, cols)), dt)
    xs, rs = strided(x, extra, shift), strided(res, extra, shift)
    out = strided(torch.zeros_like(x), extra, shift)
    ops.dropout(xs, out, p=0.25, seed=2 ** 40 + 3, offset=2 ** 33 + 5, residual=rs if residual else None)
    want = O.drop(host(x), 0.25, 2 ** 40 + 3, 2 ** 33 + 5)
    if residual:
        want = want + host(res)
    # one product, one sum, one rounding to the type
    close(out, want, (U[dt] + 2 * E) * (np.abs(want) + (np.abs(host(res)) * 2 * E if residual else 0)) + TINY[dt], "dropout")
    keep = O.kept(0, rows * cols, 0.25, 2 ** 40 + 3, 2 ** 33 + 5).reshape(rows, cols)
    if not residual:
        assert np.array_equal(host(out) != 0, keep & (host(x) != 0))
    buf = out._base if out._base is not None else out
    if extra:   # nothing outside the columns is written
        full = buf[shift:shift + rows * (cols + extra)].view(rows, cols + extra)
        assert torch.isnan(full[:, cols:]).all()


def test_dropout_extremes(ops):
    x = dev(np.array([[np.inf, np.nan, -np.inf, 1.0, 2.0, 3.0, -0.0, 5.0, 6.0]]))
    out = torch.empty_like(x)
    ops.dropout(x, out, p=1.0, seed=1)
    assert not out.any()                                         # dropped infinities and NaN are zero
    ops.dropout(x, out, p=0.0, seed=1)
    assert torch.equal(out.view(torch.int32), x.view(torch.int32))
    ops.dropout(x, out, p=0.5, seed=3)
    assert np.array_equal(np.isfinite(host(out)) | O.kept(0, 9, 0.5, 3, 0), np.ones((1, 9), bool))
    y = x.clone()
    ops.dropout(y, y, p=0.5, seed=3)                             # in place
    assert torch.equal(y.view(torch.int32), out.view(torch.int32))
    e = torch.empty(0, 5, device="cuda")
    ops.dropout(e, torch.empty_like(e), p=0.5, seed=1)           # no rows


def test_dropout_backward_is_the_same_mask_and_calls_are_independent(ops):
    x, g = torch.randn(64, 129, device="cuda") + 10, torch.randn(64, 129, device="cuda") + 10
    y, dx, other = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    ops.dropout(x, y, p=0.5, seed=11, offset=4)
    ops.dropout(g, dx, p=0.5, seed=11, offset=4)
    ops.dropout(x, other, p=0.5, seed=11, offset=5)
    assert torch.equal(y != 0, dx != 0)
    n = x.numel()
    same = ((y != 0) == (other != 0)).sum().item()
    assert abs(same - n / 2) < 5 * (n / 4) ** 0.5                # agreement by chance, five standard deviations


def test_dropout_numbers_elements_past_32_bits(ops):
    n = 2 ** 32 + 4096 + 24
    x = torch.ones(1, n, dtype=torch.float16, device="cuda")
    ops.dropout(x, x, p=0.5, seed=9, offset=1)
    for first in (0, 2 ** 31 - 64, 2 ** 32 - 64, n - 128):
        got = x[0, first:first + 128].cpu().numpy() != 0
        assert np.array_equal(got, O.kept(first, 128, 0.5, 9, 1)), first


# ----------------------------------------------------------------------------- layer norm

NORM_SHAPES = [(1, 1), (3, 1), (1, 2), (2, 7), (5, 8), (1, 33), (300, 64), (17, 255), (9, 256), (4, 1000), (33, 1001), (3, 1024),
               (150, 2048), (2, 4097), (3, 8192), (1, 8200), (2, 12345), (3, 16384), (2, 16385), (2, 20000), (1, 32768)]


def norm_tol(want, s, mean, rstd, w, b, dt, cols):
    big = np.abs(s).max(1, keepdims=True)
    w = np.ones(cols) if w is None else np.abs(w)
    b = np.zeros(cols) if b is None else np.abs(b)
    K = cols / 128 + 32
    return U[dt] * np.abs(want) + K * E * (big * rstd[:, None] * w + np.abs(want) + b) + TINY[dt]


def run_norm(ops, rows, cols, dt, pt, p, residual, affine, extra=0, shift=0, spread=1.0, offset=0.0, seed=0):
    rng = np.random.default_rng(rows * 31 + cols + seed)
    x = dev(rng.normal(size=(rows, cols)) * spread + offset, dt)
    res = dev(rng.normal(size=(rows, cols)) * 2 + offset, dt) if residual else None
    w = dev(rng.normal(size=cols) * 0.3 + 1, pt) if affine else None
    b = dev(rng.normal(size=cols) * 0.3, pt) if affine else None
    out, total = strided(torch.zeros_like(x), extra, shift), strided(torch.zeros_like(x), extra, shift)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    ops.layer_norm(strided(x, extra, shift), out, weight=w, bias=b, eps=1e-5, residual=strided(res, extra, shift) if residual else None,
                   sum_out=total, mean=mean, rstd=rstd, p=p, seed=77, offset=3)
    hw, hb = (host(w), host(b)) if affine else (None, None)
    want, s, m, r = O.layer_norm(host(x), hw, hb, float(np.float32(1e-5)), None if res is None else host(res), p, 77, 3)
    K = cols / 128 + 32
    big = np.abs(s).max(1)
    close(total, s, U[dt] * np.abs(s) + 4 * E * (np.abs(s) + (np.abs(host(res)) if residual else 0)) + TINY[dt], "sum")
    close(mean, m, K * E * big, "mean")
    # the variance is a mean of squares about a mean that is off by K E max|s|
    close(rstd, r, r * (K * E + K * E * big * r), "rstd")
    close(out, want, norm_tol(want, s, m, r, hw, hb, dt, cols), "out")
    if extra:
        assert torch.isnan(out._base[shift:shift + rows * (cols + extra)].view(rows, cols + extra)[:, cols:]).all()
    return total, mean, rstd, w


@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
@pytest.mark.parametrize("dtype,param", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32")])
def test_norm_forward(ops, rows, cols, dtype, param):
    run_norm(ops, rows, cols, TYPES[dtype], TYPES[param], 0.0, False, True)
    run_norm(ops, rows, cols, TYPES[dtype], TYPES[param], 0.1, True, True)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols,extra,shift", [(5, 64, 8, 0), (5, 64, 0, 1), (5, 64, 3, 0), (4, 1001, 2, 5), (3, 8193, 7, 1)])
def test_norm_forward_strides(ops, dtype, rows, cols, extra, shift):
    run_norm(ops, rows, cols, TYPES[dtype], TYPES[dtype], 0.2, True, True, extra, shift)


def test_norm_forward_without_parameters_and_with_a_large_mean(ops):
    run_norm(ops, 6, 1000, torch.float32, torch.float32, 0.0, False, False)
    run_norm(ops, 6, 1000, torch.float32, torch.float32, 0.3, False, False)
    run_norm(ops, 6, 1000, torch.float32, torch.float32, 0.0, True, True, spread=0.1, offset=300.0)
    run_norm(ops, 6, 5000, torch.bfloat16, torch.float32, 0.0, True, True, offset=50.0)


def test_norm_optional_outputs_and_in_place(ops):
    x, res = torch.randn(12, 520, device="cuda", dtype=torch.bfloat16), torch.randn(12, 520, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(520, device="cuda", dtype=torch.bfloat16)
    out, total = torch.empty_like(x), torch.empty_like(x)
    ops.layer_norm(x, out, weight=w, residual=res, sum_out=total, p=0.1, seed=4)
    alone = torch.empty_like(x)
    ops.layer_norm(x, alone, weight=w, residual=res, p=0.1, seed=4)
    assert torch.equal(alone, out)
    a, r = x.clone(), res.clone()
    ops.layer_norm(a, a, weight=w, residual=r, sum_out=r, p=0.1, seed=4)     # both outputs in place of the inputs
    assert torch.equal(a, out) and torch.equal(r, total)


def test_norm_row_with_nan_stays_alone(ops):
    x = torch.randn(4, 300, device="cuda")
    x[1, 5], x[2, 7] = float("nan"), float("inf")
    out = torch.empty_like(x)
    ops.layer_norm(x, out)
    assert torch.isnan(out[1]).all() and torch.isnan(out[2]).any()
    assert torch.isfinite(out[0]).all() and torch.isfinite(out[3]).all()
    z = torch.zeros(2, 40, device="cuda")                                    # no variance: only eps holds the quotient
    o = torch.ones_like(z)
    ops.layer_norm(z, o)
    assert not o.any()


def run_norm_backward(ops, rows, cols, dt, pt, p, extra_grad, extra=0, shift=0, weight=True):
    rng = np.random.default_rng(rows * 17 + cols)
    s = dev(rng.normal(size=(rows, cols)) * 2 + 0.3, dt)
    dy, dsum = dev(rng.normal(size=(rows, cols)), dt), dev(rng.normal(size=(rows, cols)), dt)
    w = dev(rng.normal(size=cols) * 0.3 + 1, pt) if weight else None
    hs = host(s)
    mean, rstd = dev(hs.mean(1)), dev(1 / np.sqrt(hs.var(1) + 1e-5))
    dx, dres = strided(torch.zeros_like(s), extra, shift), strided(torch.zeros_like(s), extra, shift)
    dw, db = torch.empty(cols, dtype=pt, device="cuda"), torch.empty(cols, dtype=pt, device="cuda")
    ops.layer_norm_backward(strided(dy, extra, shift), strided(s, extra, shift), mean, rstd, dx, weight=w, dweight=dw, dbias=db,
                            dsum=strided(dsum, extra, shift) if extra_grad else None, dresidual=dres, p=p, seed=5, offset=9)
    hw, hd = host(w) if weight else np.ones(cols), host(dy)
    wx, wr, ww, wb = O.layer_norm_backward(hd, hs, host(mean), host(rstd), hw, host(dsum) if extra_grad else None, p, 5, 9)
    r = host(rstd)[:, None]
    h = np.abs(hs - host(mean)[:, None]) * r + E * np.abs(hs) * r
    g = np.abs(hd * hw)
    K = cols / 128 + 32
    mag = r * (g + g.mean(1, keepdims=True) + h * (g * h).mean(1, keepdims=True)) + (np.abs(host(dsum)) if extra_grad else 0)
    close(dres, wr, U[dt] * np.abs(wr) + K * E * mag + TINY[dt], "dresidual")
    scale = 1.0 if p == 0 else 65536 / (65536 - O.threshold(p))
    close(dx, wx, U[dt] * np.abs(wx) + K * E * mag * scale + TINY[dt], "dx")
    # a chain of at most rows + 32 products and sums
    chain = (rows + 32) * E
    close(dw, ww, U[pt] * np.abs(ww) + chain * (np.abs(hd) * h).sum(0) + TINY[pt], "dweight")
    close(db, wb, U[pt] * np.abs(wb) + chain * np.abs(hd).sum(0) + TINY[pt], "dbias")
    if extra:
        assert torch.isnan(dx._base[shift:shift + rows * (cols + extra)].view(rows, cols + extra)[:, cols:]).all()


@pytest.mark.parametrize("rows,cols", NORM_SHAPES + [(1000, 24), (777, 520), (4000, 40)])
@pytest.mark.parametrize("dtype,param", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32")])
def test_norm_backward(ops, rows, cols, dtype, param):
    run_norm_backward(ops, rows, cols, TYPES[dtype], TYPES[param], 0.0, False)
    run_norm_backward(ops, rows, cols, TYPES[dtype], TYPES[param], 0.2, True)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols,extra,shift", [(5, 64, 8, 0), (5, 64, 0, 1), (40, 64, 3, 0), (9, 1001, 2, 5), (3, 8193, 7, 1)])
def test_norm_backward_strides(ops, dtype, rows, cols, extra, shift):
    run_norm_backward(ops, rows, cols, TYPES[dtype], TYPES[dtype], 0.2, True, extra, shift)
    run_norm_backward(ops, rows, cols, TYPES[dtype], TYPES[dtype], 0.0, False, extra, shift, weight=False)


def test_norm_backward_optional_outputs_in_place_and_no_rows(ops):
    dy, s = torch.randn(50, 300, device="cuda"), torch.randn(50, 300, device="cuda")
    mean, rstd = s.mean(1), (s.var(1, unbiased=False) + 1e-5).rsqrt()
    w = torch.randn(300, device="cuda")
    dx, dw, db = torch.empty_like(s), torch.empty_like(w), torch.empty_like(w)
    ops.layer_norm_backward(dy, s, mean, rstd, dx, weight=w, dweight=dw, dbias=db)
    only, db2 = torch.empty_like(s), torch.empty_like(w)
    ops.layer_norm_backward(dy, s, mean, rstd, only, weight=w)
    assert torch.equal(only, dx)
    ops.layer_norm_backward(dy, s, mean, rstd, only, weight=w, dbias=db2)
    assert torch.equal(db2, db)
    g, dw2 = dy.clone(), torch.empty_like(w)
    ops.layer_norm_backward(g, s, mean, rstd, g, weight=w, dweight=dw2)      # dx in place of dout
    assert torch.equal(g, dx) and torch.equal(dw2, dw)
    e = torch.empty(0, 300, device="cuda")
    ops.layer_norm_backward(e, e, mean[:0], rstd[:0], e.clone(), weight=w, dweight=dw, dbias=db)
    assert not dw.any() and not db.any()


def test_norm_gradient_agrees_with_differences_of_the_forward_pass(ops):
    torch.manual_seed(0)
    x, up = torch.randn(6, 40, device="cuda"), torch.randn(6, 40, device="cuda")
    w, b = torch.randn(40, device="cuda"), torch.randn(40, device="cuda")
    mean, rstd, total = torch.empty(6, device="cuda"), torch.empty(6, device="cuda"), torch.empty_like(x)
    out, dx = torch.empty_like(x), torch.empty_like(x)
    kw = dict(p=0.25, seed=8, offset=1)
    ops.layer_norm(x, out, weight=w, bias=b, sum_out=total, mean=mean, rstd=rstd, **kw)
    ops.layer_norm_backward(up, total, mean, rstd, dx, weight=w, **kw)
    step = 2.0 ** -6
    dirs = torch.randn(20, 6, 40, device="cuda")
    for v in dirs:
        hi, lo = torch.empty_like(x), torch.empty_like(x)
        ops.layer_norm(x + step * v, hi, weight=w, bias=b, **kw)
        ops.layer_norm(x - step * v, lo, weight=w, bias=b, **kw)
        want = ((hi.double() - lo.double()) * up.double()).sum().item() / (2 * step)
        got = (dx.double() * v.double()).sum().item()
        # step^2 = 2.4e-4 times a third derivative of order 10 (|v|^3 over 240 entries), against sums of order 15
        assert abs(got - want) < 0.05 + 0.01 * abs(want)


# ----------------------------------------------------------------------------- logits

def make_rows(n, vocab, dt, seed=0, scale=2.0):
    rng = np.random.default_rng(seed + n + vocab)
    z = rng.normal(size=(n, vocab)) * scale
    y = rng.integers(0, vocab, n)
    z[np.arange(n), y] += 4
    return dev(z, dt), torch.from_numpy(y).cuda(), rng


def logp_tol(z, vocab):
    z = np.where(np.isfinite(z), np.abs(z), 0)
    return (vocab / 128 + 64) * E + 4 * E * z.max(1)


def grad_tol(want, per_token, soft, tol, dt, scale=1.0, c_err=0.0):
    c = np.abs(per_token)[:, None] * abs(scale)
    return U[dt] * np.abs(want) + c * (soft * tol[:, None] + 4 * E) + np.broadcast_to(c_err, per_token.shape)[:, None] * abs(scale) + TINY[dt]


ROW_SHAPES = [(1, 1), (2, 2), (3, 7), (5, 8), (4, 33), (40, 100), (6, 1000), (7, 1001), (2, 1024), (3, 4097), (9, 8192), (2, 16385),
              (3, 32000), (2, 32768), (2, 32769), (5, 50001), (2, 65536), (1, 131072), (2, 150001), (1, 262144), (1, 262145), (2, 300007)]


@pytest.mark.parametrize("n,vocab", ROW_SHAPES)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_token_logp(ops, n, vocab, dtype):
    z, y, _ = make_rows(n, vocab, TYPES[dtype])
    logp, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ops.token_logp(z, y, logp, lse=lse)
    wl, ws, _ = O.token_logp(host(z), y.cpu().numpy())
    tol = logp_tol(host(z), vocab)
    close(logp, wl, tol, "logp")
    close(lse, ws, tol, "lse")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab,extra,shift", [(64, 8, 0), (64, 0, 1), (61, 3, 0), (5000, 1, 3), (33000, 8, 0), (33000, 0, 5), (70001, 1, 1)])
def test_token_logp_strides_masks_and_label_types(ops, dtype, vocab, extra, shift):
    z, y, rng = make_rows(6, vocab, TYPES[dtype])
    mask = torch.tensor([True, False, True, True, False, True], device="cuda")
    zs = strided(z, extra, shift)
    zs[1] = float("nan")
    zs[4] = float("inf")                                    # rows that do not count are not looked at
    y2 = y.clone()
    y2[1], y2[4] = -100, vocab + 7
    logp = torch.full((6,), 9.0, device="cuda")
    ops.token_logp(zs, y2.to(torch.int32), logp, mask=mask.to(torch.uint8))
    want = O.token_logp(host(z), y.cpu().numpy(), mask.cpu().numpy())[0]
    close(logp, want, logp_tol(host(z), vocab), "logp")


@pytest.mark.parametrize("vocab", [40, 3000, 40000, 290001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_of_minus_infinity_and_lowest_values(ops, vocab, dtype):
    dt = TYPES[dtype]
    z, y, _ = make_rows(8, vocab, dt)
    lowest = torch.finfo(dt).min
    z[0, : vocab // 2] = -float("inf")
    z[1, :] = -float("inf")
    z[1, 3] = 1.5
    z[2, :] = -float("inf")                                  # nothing left: NaN
    z[3, 5:] = lowest                                        # the type's lowest value, as masks have it
    z[4, :] = lowest
    z[5, 2] = float("nan")
    z[6, :] = -float("inf")
    z[6, 7] = 2.0                                            # everything but one entry
    y[0], y[1], y[3], y[6] = vocab - 1, 3, 2, 0              # row 6: the label itself has probability zero
    logp = torch.empty(8, device="cuda")
    ops.token_logp(z, y, logp)
    wl = O.token_logp(host(z), y.cpu().numpy())[0]
    tol = logp_tol(host(z), vocab) + np.where(np.abs(wl) > 1e30, np.abs(wl) * 4 * E, 0)
    tol[4] = (vocab / 128 + 64) * E + 4 * E * np.log(vocab)  # equal entries: log(1 / vocab)
    assert np.isnan(wl[2]) and np.isnan(wl[5]) and wl[6] == -np.inf
    close(logp, wl, tol, "logp")
    # a gradient row of the finite cases: probability zero gives gradient zero
    n = 8
    loss, d = torch.empty(1, device="cuda"), torch.empty_like(z)
    keep = torch.tensor([1, 1, 0, 1, 1, 0, 0, 0], device="cuda", dtype=torch.bool)
    old = torch.nan_to_num(logp)
    ops.policy_loss(z, y, old, torch.ones(n, device="cuda"), loss, d, mask=keep)
    want = O.policy(host(z), y.cpu().numpy(), host(old), np.ones(n), keep.cpu().numpy())
    soft = O.token_logp(host(z), y.cpu().numpy(), keep.cpu().numpy())[2]
    close(d, want["dlogits"], grad_tol(want["dlogits"], want["per_token"], soft, tol, dt, c_err=0.2 * (tol + 4 * E)), "dlogits")
    assert not d[2].any() and not d[5].any()


def test_label_out_of_range_is_nan_and_stays_in_its_row(ops):
    z, y, _ = make_rows(4, 500, torch.float32)
    y[1], y[2] = -1, 500
    logp = torch.empty(4, device="cuda")
    ops.token_logp(z, y, logp)
    assert torch.isnan(logp[1:3]).all() and torch.isfinite(logp[[0, 3]]).all()
    d, loss = torch.empty_like(z), torch.empty(1, device="cuda")
    ops.policy_loss(z, y, torch.zeros(4, device="cuda"), torch.ones(4, device="cuda"), loss, d)
    assert torch.isnan(loss).all() and torch.isfinite(d[[0, 3]]).all()


def test_rows_past_32_bit_offsets(ops):
    vocab, stride, n = 1000, 2 ** 28 + 1, 12                 # the last row starts past 2^31 elements
    buf = torch.empty(stride * (n - 1) + vocab, dtype=torch.bfloat16, device="cuda")
    z = buf.as_strided((n, vocab), (stride, 1))
    src, y, _ = make_rows(n, vocab, torch.bfloat16)
    z.copy_(src)
    near = strided(src, 1)                                   # the same rows, misaligned alike, close together
    logp, loss, a = torch.empty(n, device="cuda"), torch.empty(1, device="cuda"), torch.ones(n, device="cuda")
    ops.token_logp(z, y, logp)
    want = O.policy(host(src), y.cpu().numpy(), host(logp), np.ones(n))
    close(logp, want["logp"], logp_tol(host(src), vocab), "logp")
    ops.policy_loss(near, y, logp, a, loss, near)
    ops.policy_loss(z, y, logp, a, loss, z)                  # in place, across the large stride
    assert torch.equal(z, near)
    out = torch.empty_like(src)
    z.copy_(src), near.copy_(src)
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ops.layer_norm(z, out, mean=mean, rstd=rstd)
    ref = torch.empty_like(src)
    ops.layer_norm(near, ref)
    assert torch.equal(out, ref)
    dx, dz = torch.empty_like(src), torch.empty_like(src)
    dw, dw2 = torch.empty(vocab, device="cuda", dtype=torch.bfloat16), torch.empty(vocab, device="cuda", dtype=torch.bfloat16)
    ops.layer_norm_backward(out, near, mean, rstd, dx, dweight=dw)
    ops.layer_norm_backward(out, z, mean, rstd, dz, dweight=dw2)
    assert torch.equal(dx, dz) and torch.equal(dw, dw2)


# ----------------------------------------------------------------------------- preference loss

def starts(n, seqs, rng):
    cuts = np.sort(rng.integers(0, n + 1, seqs - 1))
    return np.concatenate([[0], cuts, [n]]).astype(np.int32)


PREF_SHAPES = [(2, 1, 5), (2, 3, 8), (4, 5, 1001), (6, 4, 33), (8, 24, 2000), (2, 40, 8193), (4, 3, 32001), (2, 2, 131072), (2, 2, 270001)]


@pytest.mark.parametrize("seqs,steps,vocab", PREF_SHAPES)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kind,packed", [("sigmoid", False), ("sigmoid", True), ("hinge", False), ("square", True)])
def test_preference_loss(ops, seqs, steps, vocab, dtype, kind, packed):
    dt, n = TYPES[dtype], seqs * steps
    z, y, rng = make_rows(n, vocab, dt, seed=3)
    mask = rng.random(n) < 0.7
    start = starts(n, seqs, rng) if packed else None
    logp0 = O.token_logp(host(z), y.cpu().numpy())[0]
    ref = dev(logp0 + rng.normal(size=n) * 0.3)
    e = 0.1 if kind == "sigmoid" and packed else 0.0
    norm = kind == "square"
    beta, scale = 0.25, 64.0
    loss, margin = torch.empty(1, device="cuda"), torch.empty(seqs // 2, device="cuda")
    sums, d = torch.empty(seqs, device="cuda"), torch.full_like(z, 7.0)
    where = dict(seq_start=torch.from_numpy(start).cuda()) if packed else dict(sequences=seqs)
    ops.preference_loss(z, y, ref, loss, d, mask=torch.from_numpy(mask).cuda(), beta=beta, kind=kind, label_smoothing=e,
                        length_normalized=norm, grad_scale=scale, margin=margin, seq_logp=sums, **where)
    b32, e32 = float(np.float32(beta)), float(np.float32(e))
    want = O.preference(host(z), y.cpu().numpy(), host(ref), mask, None if packed else seqs, start, b32, kind, e32, norm, scale)
    tol = logp_tol(host(z), vocab)
    rows = [(a, b) for a, b in O.runs(n, seqs, start)]
    counts = np.array([max(1, mask[a:b].sum()) for a, b in rows])
    per = np.array([tol[a:b][mask[a:b]].sum() for a, b in rows]) / (counts if norm else 1)   # a sequence's sum of errors
    close(sums, want["seq_logp"], per + 4 * E * np.abs(want["seq_logp"]), "seq_logp")
    herr = b32 * (per[:seqs // 2] + per[seqs // 2:]) + 4 * E * np.abs(want["margin"])
    close(margin, want["margin"], herr, "margin")
    slope = np.abs(2 * (want["margin"] / b32 - 0.5 / b32) / b32) if kind == "square" else np.ones(seqs // 2)
    curve = 2 / b32 ** 2 if kind == "square" else 0.25
    if kind == "hinge":
        assert np.all(np.abs(want["margin"] - 1) > herr)
    close(loss, np.array([want["loss"]]), ((slope * herr).mean() + curve * (herr ** 2).mean() + 4 * E * abs(want["loss"])), "loss")
    soft = O.token_logp(host(z), y.cpu().numpy(), mask)[2]
    cerr = np.zeros(n)
    for q, (a, b) in enumerate(rows):
        k = 1.0 / counts[q] if norm else 1.0
        cerr[a:b] = (0.0 if kind == "hinge" else curve) * herr[q % (seqs // 2)] * b32 * k / (seqs // 2)
    cerr = (cerr + 4 * E * np.abs(want["per_token"])) * mask
    close(d, want["dlogits"], grad_tol(want["dlogits"], want["per_token"], soft, tol, dt, scale, cerr), "dlogits")
    assert not host(d)[~mask].any()
    again, margin2 = torch.empty(1, device="cuda"), torch.empty(seqs // 2, device="cuda")
    ops.preference_loss(z, y, ref, again, mask=torch.from_numpy(mask).cuda(), beta=beta, kind=kind, label_smoothing=e,
                        length_normalized=norm, margin=margin2, **where)                    # loss only
    assert torch.equal(again, loss) and torch.equal(margin2, margin)
    ops.preference_loss(z, y, ref, again, z, mask=torch.from_numpy(mask).cuda(), beta=beta, kind=kind, label_smoothing=e,
                        length_normalized=norm, grad_scale=scale, **where)                  # in place, the same bits
    assert torch.equal(z, d) and torch.equal(again, loss)


def test_preference_with_empty_sequences_and_no_tokens(ops):
    z, y, _ = make_rows(3, 50, torch.float32)
    ref = torch.zeros(3, device="cuda")
    loss, margin, sums, d = (torch.empty(k, device="cuda") for k in (1, 2, 4, 1))
    d = torch.full_like(z, 3.0)
    start = torch.tensor([0, 2, 2, 3, 3], dtype=torch.int32, device="cuda")     # two sequences without tokens
    ops.preference_loss(z, y, ref, loss, d, seq_start=start, margin=margin, seq_logp=sums)
    want = O.preference(host(z), y.cpu().numpy(), host(ref), None, None, start.cpu().numpy(), float(np.float32(0.1)))
    close(margin, want["margin"], 1e-5, "margin")
    close(loss, np.array([want["loss"]]), 1e-5, "loss")
    none = torch.zeros(3, dtype=torch.bool, device="cuda")
    ops.preference_loss(z, y, ref, loss, d, seq_start=start, mask=none, margin=margin, seq_logp=sums)
    assert not d.any() and not margin.any() and not sums.any()
    assert abs(loss.item() - np.log(2)) < 4 * E
    e = torch.empty(0, 50, device="cuda")
    ops.preference_loss(e, y[:0], ref[:0], loss, e.clone(), sequences=2)
    assert abs(loss.item() - np.log(2)) < 4 * E


def test_large_margins_do_not_overflow(ops):
    z, y, _ = make_rows(4, 64, torch.float32)
    loss, margin, d = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(z)
    for shift in (-2000.0, 2000.0):
        ref = torch.zeros(4, device="cuda")
        ref[:2] = shift
        ops.preference_loss(z, y, ref, loss, d, sequences=2, beta=1.0, margin=margin)
        want = O.preference(host(z), y.cpu().numpy(), host(ref), sequences=2, beta=1.0)
        close(loss, np.array([want["loss"]]), 1e-6 * max(1.0, abs(want["loss"])), "loss")
        close(d, want["dlogits"], 1e-5 * np.ones_like(want["dlogits"]), "dlogits")


# ----------------------------------------------------------------------------- policy loss

@pytest.mark.parametrize("seqs,steps,vocab", PREF_SHAPES + [(1, 1, 1), (3, 7, 500), (16, 33, 1001), (1, 600, 40)])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("per_sequence,packed,with_ref", [(False, False, True), (True, True, True), (True, False, False)])
def test_policy_loss(ops, seqs, steps, vocab, dtype, per_sequence, packed, with_ref):
    dt, n = TYPES[dtype], seqs * steps
    z, y, rng = make_rows(n, vocab, dt, seed=5)
    mask = rng.random(n) < 0.7
    start = starts(n, seqs, rng) if packed else None
    logp0 = O.token_logp(host(z), y.cpu().numpy())[0]
    old, ref = dev(logp0 + rng.normal(size=n) * 0.2), dev(logp0 + rng.normal(size=n) * 0.3)
    adv = dev(rng.normal(size=n))
    lo, hi, kb, scale = 0.2, 0.25, 0.05 if with_ref else 0.0, 128.0
    loss, stats, logp, d = torch.empty(1, device="cuda"), torch.empty(3, device="cuda"), torch.empty(n, device="cuda"), torch.full_like(z, 7.0)
    kw = dict(mask=torch.from_numpy(mask).cuda(), ref_logp=ref if with_ref else None, clip_low=lo, clip_high=hi, kl_beta=kb,
              per_sequence=per_sequence, grad_scale=scale)
    kw.update(dict(seq_start=torch.from_numpy(start).cuda()) if packed else dict(sequences=seqs))
    ops.policy_loss(z, y, old, adv, loss, d, logp=logp, stats=stats, **kw)
    f = lambda v: float(np.float32(v))  # noqa: E731
    want = O.policy(host(z), y.cpu().numpy(), host(old), host(adv), mask, None if packed else seqs, start, host(ref) if with_ref else None,
                    f(lo), f(hi), f(kb), per_sequence, scale)
    tol = logp_tol(host(z), vocab)
    r = np.exp(want["logp"] - host(old))
    edge = np.minimum(np.abs(r - (1 - f(lo))), np.abs(r - (1 + f(hi))))
    assert np.all((edge > 4 * r * (tol + 4 * E)) | ~mask), "an input sits on the corner of the clip"
    close(logp, want["logp"], tol, "logp")
    u = host(ref) - want["logp"]
    w = np.where(mask, 1.0 / max(1, mask.sum()), 0.0)
    if per_sequence:
        w = np.zeros(n)
        used = sum(mask[a:b].any() for a, b in O.runs(n, seqs, start))
        for a, b in O.runs(n, seqs, start):
            if mask[a:b].any():
                w[a:b] = mask[a:b] / (used * mask[a:b].sum())
    # the ratio's relative error is the log-probability's and a few roundings; so is exp(u)'s
    terr = (tol + 8 * E) * (r * np.abs(host(adv)) + kb * (np.exp(u) + 1 + np.abs(u)))
    close(loss, np.array([want["loss"]]), 2 * (w * terr).sum() + 8 * E * (w * r * np.abs(host(adv))).sum() + 1e-30, "loss")
    k = max(1, mask.sum())
    close(stats, want["stats"], np.array([((tol + 8 * E) * (np.exp(u) + 1 + np.abs(u)) * mask).sum() / k + 4 * E, 4 * E, 0.5]), "stats")
    soft = O.token_logp(host(z), y.cpu().numpy(), mask)[2]
    cerr = w * terr * 2 + 4 * E * np.abs(want["per_token"])
    close(d, want["dlogits"], grad_tol(want["dlogits"], want["per_token"], soft, tol, dt, scale, cerr), "dlogits")
    again = torch.empty(1, device="cuda")
    ops.policy_loss(z, y, old, adv, again, **kw)                                  # loss only
    assert torch.equal(again, loss)
    ops.policy_loss(z, y, old, adv, again, z, **kw)                               # in place, the same bits
    assert torch.equal(z, d) and torch.equal(again, loss)


def test_policy_nothing_counts_and_no_tokens(ops):
    z, y, _ = make_rows(6, 70, torch.bfloat16)
    v = torch.ones(6, device="cuda")
    loss, stats, d = torch.full((1,), 5.0, device="cuda"), torch.full((3,), 5.0, device="cuda"), torch.full_like(z, 2.0)
    none = torch.zeros(6, dtype=torch.bool, device="cuda")
    for per in (False, True):
        ops.policy_loss(z, y, v, v, loss, d, mask=none, sequences=2, per_sequence=per, stats=stats)
        assert loss.item() == 0 and not d.any() and not stats.any()
    e = torch.empty(0, 70, device="cuda")
    ops.policy_loss(e, y[:0], v[:0], v[:0], loss, e.clone(), sequences=3, stats=stats)
    assert loss.item() == 0 and not stats.any()


def test_policy_nan_inputs_reach_the_loss(ops):
    z, y, _ = make_rows(3, 64, torch.float32)
    one = torch.ones(3, device="cuda")
    for old, adv in ((torch.tensor([0.0, float("nan"), 0.0], device="cuda"), one), (one, torch.tensor([1.0, float("nan"), 1.0], device="cuda"))):
        loss = torch.empty(1, device="cuda")
        ops.policy_loss(z, y, old, adv, loss)
        assert torch.isnan(loss).all()


def test_loss_gradients_agree_with_differences(ops):
    z, y, rng = make_rows(8, 30, torch.float32, seed=9, scale=1.0)
    logp = O.token_logp(host(z), y.cpu().numpy())[0]
    old, ref, adv = dev(logp + 0.05 * rng.normal(size=8)), dev(logp + 0.3 * rng.normal(size=8)), dev(rng.normal(size=8))
    loss, d = torch.empty(1, device="cuda"), torch.empty_like(z)
    calls = [lambda a, g: ops.policy_loss(a, y, old, adv, loss, g, ref_logp=ref, kl_beta=0.5),
             lambda a, g: ops.preference_loss(a, y, ref, loss, g, sequences=4, beta=0.7)]
    step = 2.0 ** -5
    for call in calls:
        call(z, d)
        for _ in range(10):
            v = torch.randn_like(z)
            v /= v.norm()
            call(z + step * v, None)
            up = loss.item()
            call(z - step * v, None)
            want = (up - loss.item()) / (2 * step)
            got = (d.double() * v.double()).sum().item()
            # step^2 / 6 times a third derivative of order 1, and 2^-24 / step of rounding
            assert abs(got - want) < 2e-3


# ----------------------------------------------------------------------------- whole calls

def test_calls_repeat_bit_for_bit(ops):
    z, y, rng = make_rows(64, 5003, torch.bfloat16)
    v = torch.randn(64, device="cuda")
    loss, d, stats = torch.empty(1, device="cuda"), torch.empty_like(z), torch.empty(3, device="cuda")
    x, s = torch.randn(700, 1500, device="cuda"), torch.randn(700, 1500, device="cuda")
    mean, rstd = s.mean(1), s.var(1).rsqrt()
    dx, dw, db = torch.empty_like(x), torch.empty(1500, device="cuda"), torch.empty(1500, device="cuda")
    seen = []
    for _ in range(5):
        ops.policy_loss(z, y, v, v, loss, d, sequences=8, per_sequence=True, stats=stats)
        one = [loss.clone(), d.clone(), stats.clone()]
        ops.preference_loss(z, y, v, loss, d, sequences=8)
        one += [loss.clone(), d.clone()]
        ops.layer_norm_backward(x, s, mean, rstd, dx, dweight=dw, dbias=db)
        seen.append(one + [dx.clone(), dw.clone(), db.clone()])
    for other in seen[1:]:
        assert all(torch.equal(a, b) for a, b in zip(seen[0], other))


def test_calls_from_another_stream_are_ordered(ops):
    side = torch.cuda.Stream()
    x = torch.zeros(4096, 4096, device="cuda")
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for k in range(20):
            x.fill_(float(k))              # the context's stream has to wait for this
            ops.dropout(x, out, p=0.0, seed=0)
            x.fill_(-1.0)                  # and this for the context's stream
            got = out[::1024, ::1024].clone()
            assert (got == k).all()
    torch.cuda.current_stream().wait_stream(side)


def test_a_call_can_be_captured_in_a_graph():
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ops = pkg.TrainingOps(256, 2048, stream=side)
        z, y, _ = make_rows(64, 3001, torch.bfloat16)
        v = torch.zeros(64, device="cuda")
        loss, d = torch.empty(1, device="cuda"), torch.empty_like(z)
        ops.policy_loss(z, y, v, v + 1, loss, d, sequences=4, per_sequence=True)
        want = (loss.clone(), d.clone())
        g = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(g, stream=side):
            ops.policy_loss(z, y, v, v + 1, loss, d, sequences=4, per_sequence=True)
        for _ in range(3):
            loss.zero_(), d.zero_()
            g.replay()
            side.synchronize()
            assert torch.equal(loss, want[0]) and torch.equal(d, want[1])


def test_refusals(ops):
    x, w = torch.randn(4, 16, device="cuda"), torch.randn(16, device="cuda")
    out, st = torch.empty_like(x), torch.empty(4, device="cuda")
    z, y, v = torch.randn(6, 10, device="cuda"), torch.zeros(6, dtype=torch.int64, device="cuda"), torch.zeros(6, device="cuda")
    loss, d = torch.empty(1, device="cuda"), torch.empty_like(z)
    big = torch.randn(8, 32, device="cuda")
    wide = torch.empty(1, pkg.training.MAX_COLS + 1, device="cuda")
    i32 = torch.tensor([0, 6], dtype=torch.int32, device="cuda")
    python = [  # refused by the binding
        lambda: ops.dropout(x.double(), out, p=0.1, seed=0),
        lambda: ops.dropout(x, out.half(), p=0.1, seed=0),
        lambda: ops.dropout(x, out[:3], p=0.1, seed=0),
        lambda: ops.dropout(x.t(), out.t(), p=0.1, seed=0),
        lambda: ops.dropout(x.cpu(), out, p=0.1, seed=0),
        lambda: ops.dropout(x[0], out[0], p=0.1, seed=0),
        lambda: ops.dropout(x, out[:1].expand(4, 16), p=0.1, seed=0),
        lambda: ops.layer_norm(x, out, weight=w.half()),
        lambda: ops.layer_norm(x, out, weight=w[:8]),
        lambda: ops.layer_norm(x.half(), out.half(), weight=w.half(), bias=w),
        lambda: ops.layer_norm(x, out, mean=st.half()),
        lambda: ops.layer_norm_backward(x, x, st[:2], st, out),
        lambda: ops.token_logp(z, y.float(), v),
        lambda: ops.token_logp(z, y[:3], v),
        lambda: ops.token_logp(z, y, v, mask=v),
        lambda: ops.preference_loss(z, y, v, loss, d),
        lambda: ops.preference_loss(z, y, v, loss, d, sequences=2, kind="other"),
        lambda: ops.preference_loss(z, y, v, loss, d, sequences=2, seq_start=i32),
        lambda: ops.preference_loss(z, y, v, loss, d, seq_start=i32.long()),
        lambda: ops.policy_loss(z, y, v, v, loss, d, per_sequence=True),
        lambda: ops.policy_loss(z, y, v, v[:2], loss, d),
        lambda: ops.policy_loss(z, y, v, v, loss, d.half()),
    ]
    for k, call in enumerate(python):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"python refusal {k} went through")
    library = [  # refused by the C entry points
        lambda: ops.dropout(x, out, p=1.5, seed=0),
        lambda: ops.dropout(x, out, p=float("nan"), seed=0),
        lambda: ops.dropout(big[:4, :16], big[1:5, :16], p=0.1, seed=0),        # overlapping, not the same matrix
        lambda: ops.dropout(big[:4, :16], big[:4, 8:24], p=0.1, seed=0),
        lambda: ops.layer_norm(x, out, eps=-1.0),
        lambda: ops.layer_norm(x, out, sum_out=out),
        lambda: ops.layer_norm(wide, torch.empty_like(wide)),
        lambda: ops.layer_norm(x, out, mean=st, rstd=st),
        lambda: ops.layer_norm(x[:1], w.view(1, 16), weight=w),
        lambda: ops.layer_norm_backward(x, x, st, st, out, dresidual=out),
        lambda: ops.layer_norm_backward(x, x, st, st, out, weight=w, dweight=w),
        lambda: ops.layer_norm_backward(*(torch.empty(70001, 4, device="cuda"),) * 2, *(torch.empty(70001, device="cuda"),) * 2,
                                        torch.empty(70001, 4, device="cuda")),  # more rows than the context has room for
        lambda: ops.token_logp(z, y, v, lse=v),
        lambda: ops.preference_loss(z, y, v, loss, d, sequences=3),             # odd
        lambda: ops.preference_loss(z, y, v, loss, d, sequences=4),             # does not divide
        lambda: ops.preference_loss(z, y, v, loss, d, sequences=2, beta=0.0),
        lambda: ops.preference_loss(z, y, v, loss, d, sequences=2, label_smoothing=0.6),
        lambda: ops.preference_loss(z, y, v, loss, d, sequences=2, label_smoothing=0.1, kind="hinge"),
        lambda: ops.preference_loss(z, y, v, loss, d, sequences=2, grad_scale=float("inf")),
        lambda: ops.preference_loss(z, y, v, v[:1], d, sequences=2),            # loss inside ref_logp
        lambda: ops.policy_loss(z, y, v, v, loss, d, kl_beta=0.1),              # no reference
        lambda: ops.policy_loss(z, y, v, v, loss, d, clip_low=1.5),
        lambda: ops.policy_loss(z, y, v, v, loss, d, clip_high=-0.1),
        lambda: ops.policy_loss(z, y, v, v, loss, d, logp=v),
    ]
    before = ops.launch_count()
    for k, call in enumerate(library):
        with pytest.raises(pkg.AdacgdError) as e:
            call()
            pytest.fail(f"library refusal {k} went through")
        assert e.value.status == 1 and "adacgd_" in str(e.value), k
    assert ops.launch_count() == before
    left, right = big[:, :16], big[:, 16:]
    ops.dropout(left, right, p=0.0, seed=0)                                     # columns of one matrix do not overlap
    assert torch.equal(left, right)
    small = pkg.TrainingOps(4, 8)
    with pytest.raises(pkg.AdacgdError):
        small.token_logp(z, y, v)
    with pytest.raises(pkg.AdacgdError):
        small.layer_norm_backward(x, x, st, st, out)
    small.close()
    with pytest.raises(RuntimeError):
        small.dropout(x, out, p=0.1, seed=0)


@pytest.mark.parametrize("steps,vocab,dtype", [(1024, 40, "bf16"), (1025, 40, "bf16"), (2500, 1001, "f32"), (2500, 520, "f16")])
@pytest.mark.parametrize("per_sequence", [False, True])
@pytest.mark.parametrize("masked", [False, True])
def test_policy_loss_of_many_tokens(ops, steps, vocab, dtype, per_sequence, masked):
    """Token counts on both sides of the sizes at which the sums move to kernels of their own."""
    seqs, dt = 2, TYPES[dtype]
    n = seqs * steps
    z, y, rng = make_rows(n, vocab, dt, seed=8)
    mask = rng.random(n) < 0.6 if masked else np.ones(n, bool)
    logp0 = O.token_logp(host(z), y.cpu().numpy())[0]
    old, adv = dev(logp0 + 0.05), dev(rng.normal(size=n))
    loss, stats, d = torch.empty(1, device="cuda"), torch.empty(3, device="cuda"), torch.empty_like(z)
    ops.policy_loss(z, y, old, adv, loss, d, mask=torch.from_numpy(mask).cuda() if masked else None, sequences=seqs,
                    per_sequence=per_sequence, stats=stats)
    f = lambda v: float(np.float32(v))  # noqa: E731
    want = O.policy(host(z), y.cpu().numpy(), host(old), host(adv), mask, seqs, None, None, f(0.2), f(0.2), 0.0, per_sequence, 1.0)
    tol = logp_tol(host(z), vocab)
    r = np.exp(want["logp"] - host(old))
    w = mask / max(1, mask.sum())
    if per_sequence:
        w = np.concatenate([m / (2 * m.sum()) for m in np.split(mask, 2)])
    terr = (tol + 8 * E) * r * np.abs(host(adv))
    close(loss, np.array([want["loss"]]), 2 * (w * terr).sum() + 8 * E * (w * r * np.abs(host(adv))).sum(), "loss")
    assert stats[2].item() == mask.sum() and stats[1].item() == pytest.approx(want["stats"][1], abs=4 * E)
    soft = O.token_logp(host(z), y.cpu().numpy(), mask)[2]
    close(d, want["dlogits"], grad_tol(want["dlogits"], want["per_token"], soft, tol, dt, 1.0, w * terr * 2 + 4 * E * np.abs(want["per_token"])),
          "dlogits")


@pytest.mark.parametrize("packed", [False, True])
def test_preference_loss_of_long_sequences(ops, packed):
    """Pairs long enough to be summed by several CTAs."""
    seqs, steps, vocab = 4, 3000, 24
    n = seqs * steps
    z, y, rng = make_rows(n, vocab, torch.float32, seed=4, scale=1.0)
    mask = rng.random(n) < 0.8
    ref = dev(O.token_logp(host(z), y.cpu().numpy())[0] + rng.normal(size=n) * 0.01)
    start = np.array([0, 1, 700, 7000, n], np.int32) if packed else None
    loss, margin, sums, d = torch.empty(1, device="cuda"), torch.empty(2, device="cuda"), torch.empty(4, device="cuda"), torch.empty_like(z)
    kw = dict(seq_start=torch.from_numpy(start).cuda()) if packed else dict(sequences=seqs)
    ops.preference_loss(z, y, ref, loss, d, beta=0.5, mask=torch.from_numpy(mask).cuda(), margin=margin, seq_logp=sums, **kw)
    want = O.preference(host(z), y.cpu().numpy(), host(ref), mask, None if packed else seqs, start, beta=0.5)
    # every token's log-probability is off by at most `tol`, all of them the same way at worst
    tol = logp_tol(host(z), vocab)
    assert abs(loss.item() - want["loss"]) <= 0.5 * (tol * mask).sum() + 4 * E * abs(want["loss"])
    close(margin, want["margin"], 0.5 * (tol * mask).sum() + 4 * E * np.abs(want["margin"]), "margin")
    close(sums, want["seq_logp"], (tol * mask).sum() + 4 * E * np.abs(want["seq_logp"]), "seq_logp")
    top = np.abs(want["dlogits"]).max()
    close(d, want["dlogits"], top * (0.5 * (tol * mask).sum() + 32 * E) + 1e-30 + 0 * want["dlogits"], "dlogits")
