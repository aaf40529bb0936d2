"""Inputs at the edge of what the training operators take, against the binary64 restatement (oracle/training_oracle.py).  Tolerances and
their derivation are those of test_training_gpu.py unless a test says otherwise."""
import numpy as np
import pytest
import torch

import paper_2211_00188_b200 as pkg
from oracle import training_oracle as O
from test_training_gpu import E, TINY, TYPES, U, close, dev, grad_tol, host, logp_tol, make_rows, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    return pkg.TrainingOps(70000, 32768)


# ----------------------------------------------------------------------------- counting tokens

def masks(n, which, rng):
    m = np.zeros(n, bool)
    if which == "all":
        m[:] = True
    elif which == "last":
        m[-1] = True
    elif which == "rest":
        m[n // 16 * 16 + 8:] = True                          # what lies behind the eighth token after the last whole sixteen
    else:
        m[:] = rng.random(n) < 0.6
        m[0] = True
    return m


@pytest.mark.parametrize("n", [9, 10, 12, 13, 15, 31, 41, 1005, 2047])
@pytest.mark.parametrize("vocab", [5, 40, 64, 65, 200])
@pytest.mark.parametrize("which", ["all", "last", "rest", "some"])
@pytest.mark.parametrize("shift", [0, 1])
def test_policy_loss_counts_every_token(ops, n, vocab, which, shift):
    z, y, rng = make_rows(n, vocab, torch.float32, seed=11)
    mask = masks(n, which, rng)
    buf = torch.zeros(n + 16, dtype=torch.bool, device="cuda")
    dm = buf[shift:shift + n]                                # a mask on 16 bytes, and one off them
    dm.copy_(torch.from_numpy(mask))
    buf[shift + n:] = True                                   # behind the mask: not part of it
    logp0 = O.token_logp(host(z), y.cpu().numpy())[0]
    old, adv = dev(logp0 + 0.05), dev(rng.normal(size=n))
    loss, stats, d = torch.empty(1, device="cuda"), torch.empty(3, device="cuda"), torch.empty_like(z)
    ops.policy_loss(z, y, old, adv, loss, d, mask=dm, stats=stats)
    f = lambda v: float(np.float32(v))  # noqa: E731
    want = O.policy(host(z), y.cpu().numpy(), host(old), host(adv), mask, 1, None, None, f(0.2), f(0.2))
    assert stats[2].item() == mask.sum()
    tol = logp_tol(host(z), vocab)
    r = np.exp(want["logp"] - host(old))
    w = mask / mask.sum()
    terr = (tol + 8 * E) * r * np.abs(host(adv))
    close(loss, np.array([want["loss"]]), 2 * (w * terr).sum() + 8 * E * (w * r * np.abs(host(adv))).sum(), "loss")
    soft = O.token_logp(host(z), y.cpu().numpy(), mask)[2]
    close(d, want["dlogits"], grad_tol(want["dlogits"], want["per_token"], soft, tol, torch.float32, 1.0,
                                       w * terr * 2 + 4 * E * np.abs(want["per_token"])), "dlogits")


# ----------------------------------------------------------------------------- NaN

@pytest.mark.parametrize("per_sequence", [False, True])      # one kernel, three kernels
@pytest.mark.parametrize("with_ref", [False, True])
@pytest.mark.parametrize("what", ["label", "old", "advantage"])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", [40, 500])
def test_policy_gradient_of_a_nan_ratio_is_nan(ops, per_sequence, with_ref, what, dtype, vocab):
    z, y, _ = make_rows(6, vocab, TYPES[dtype])
    logp = O.token_logp(host(z), y.cpu().numpy())[0]
    old, ref, adv = dev(logp), dev(logp + 0.1), torch.ones(6, device="cuda")
    bad = [1, 4]
    if what == "label":
        y[1], y[4] = -1, vocab
    else:
        (old if what == "old" else adv)[bad] = float("nan")
    loss, d = torch.empty(1, device="cuda"), torch.zeros_like(z)
    ops.policy_loss(z, y, old, adv, loss, d, sequences=2, per_sequence=per_sequence, ref_logp=ref if with_ref else None,
                    kl_beta=0.1 if with_ref else 0.0)
    assert torch.isnan(loss).all()
    assert torch.isnan(d[bad]).all()
    assert torch.isfinite(d[[0, 2, 3, 5]]).all()
    want = O.policy(host(z), y.cpu().numpy(), host(old), host(adv), None, 2, ref_logp=host(ref) if with_ref else None,
                    kl_beta=0.1 if with_ref else 0.0, per_sequence=per_sequence)
    assert np.array_equal(np.isnan(want["dlogits"]), np.isnan(host(d)))


@pytest.mark.parametrize("per_sequence", [False, True])
def test_policy_without_advantage_has_no_gradient_whatever_the_ratio(ops, per_sequence):
    """exp(logp - old) = e^100 is no number of binary32; times an advantage of zero it is zero all the same."""
    z, y, _ = make_rows(4, 60, torch.float32)
    logp = O.token_logp(host(z), y.cpu().numpy())[0]
    old, adv = dev(logp - 100), torch.tensor([0.0, 0.0, 2.0, 0.0], device="cuda")
    loss, stats, d = torch.empty(1, device="cuda"), torch.empty(3, device="cuda"), torch.full_like(z, 3.0)
    ops.policy_loss(z, y, old, adv, loss, d, sequences=2, per_sequence=per_sequence, stats=stats)
    want = O.policy(host(z), y.cpu().numpy(), host(old), host(adv), None, 2, per_sequence=per_sequence)
    assert not d.any() and not want["dlogits"].any()             # the third token is clipped
    close(loss, np.array([want["loss"]]), 4 * E, "loss")
    assert stats[1].item() == 0.25


# ----------------------------------------------------------------------------- logits far from zero

def far_rows(dt, vocab):
    """Rows whose logits lie near a distant value, equal or a few units of the type apart, and their labels."""
    rng = np.random.default_rng(vocab)
    rows = []
    for at in (-1e10, 1e10, -1e30, 1e30, -2.2e38, 3e9, -4194304.0, 4194304.0, 2.0 ** 23):
        rows.append(np.full(vocab, at))
    if dt == torch.float32:
        for at in (-4194304.0, 4194304.0):                       # half a unit apart there, on both sides of a power of two
            rows.append(at + rng.integers(-8, 9, vocab) * 0.5)
            rows.append(at + np.sort(rng.integers(-8, 9, vocab)) * 0.5)
    else:
        rows.append(np.where(rng.random(vocab) < 0.5, 2048.0, 2048.0 + (16.0 if dt == torch.bfloat16 else 2.0)))
    z = dev(np.stack(rows), dt)
    y = torch.from_numpy(rng.integers(0, vocab, len(rows))).cuda()
    return z, y


@pytest.mark.parametrize("vocab", [7, 40, 3000, 40000, 290001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_far_from_zero(ops, vocab, dtype):
    """A row that is masked as a whole by -1e10 or -1e30 is a uniform one.  Differences of such logits are exact, so the tolerance goes
    by the largest difference and not by the logits."""
    dt = TYPES[dtype]
    z, y = far_rows(dt, vocab)
    n = len(y)
    logp = torch.empty(n, device="cuda")
    ops.token_logp(z, y, logp)
    hz = host(z)
    wl, _, soft = O.token_logp(hz, y.cpu().numpy())
    tol = (vocab / 128 + 64) * E + 4 * E * (hz.max(1) - hz.min(1) + np.log(vocab))
    close(logp, wl, tol, "logp")
    loss, d = torch.empty(1, device="cuda"), torch.empty_like(z)
    adv = torch.ones(n, device="cuda")
    ops.policy_loss(z, y, dev(wl), adv, loss, d)
    per = -np.exp(wl - host(dev(wl))) / n
    want = np.zeros_like(hz)
    want -= per[:, None] * soft
    want[np.arange(n), y.cpu().numpy()] += per
    close(d, want, grad_tol(want, per, soft, tol, dt, c_err=(2 * tol + 8 * E) / n), "dlogits")
    seqs = n // 2 * 2
    margin, sums = torch.empty(seqs // 2, device="cuda"), torch.empty(seqs, device="cuda")
    ops.preference_loss(z[:seqs], y[:seqs], torch.zeros(seqs, device="cuda"), loss, d[:seqs], sequences=seqs, seq_logp=sums, margin=margin)
    close(sums, wl[:seqs], tol[:seqs] + 4 * E * np.abs(wl[:seqs]), "seq_logp")


def test_label_at_the_types_lowest_value_has_a_finite_logp(ops):
    """A label that a mask has set to the type's lowest value: its log-probability is that value, not -inf, and two of them differ
    by nothing."""
    for dtype in ("f32", "bf16"):
        dt = TYPES[dtype]
        for vocab in (40, 3000, 40000, 290001):
            z, y, _ = make_rows(4, vocab, dt)
            lowest = torch.finfo(dt).min
            z[torch.arange(4, device="cuda"), y] = lowest
            logp = torch.empty(4, device="cuda")
            ops.token_logp(z, y, logp)
            # beside a number of 2^127 log s is nothing: one rounding of the product and one of the result
            close(logp, np.full(4, float(lowest)), 4 * E * abs(float(lowest)), "logp")
            loss, margin, d = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(z)
            ops.preference_loss(z, y, logp, loss, d, sequences=2, margin=margin)
            # the reference is the value itself: no NaN from the difference of two such
            assert torch.isfinite(margin).all() and torch.isfinite(loss).all() and not torch.isnan(d).any()


# ----------------------------------------------------------------------------- accuracy of log-probabilities

@pytest.mark.parametrize("dtype,n,vocab", [("bf16", 4096, 4000), ("bf16", 2048, 50001), ("bf16", 1024, 131072), ("f32", 2048, 8000), ("f16", 4096, 300)])
def test_log_probabilities_are_at_least_as_exact_as_the_plain_form(ops, dtype, n, vocab):
    """Root mean square error over many tokens against binary64, beside that of the formula in elementary binary32 operations
    (which has the maximum subtracted first).  Errors of a few roundings each, independent from row to row: with a thousand rows the two
    figures are known to a few per cent."""
    dt = TYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    z = (torch.randn(n, vocab, generator=gen, device="cuda") * 2).to(dt)
    y = torch.randint(vocab, (n,), generator=gen, device="cuda")
    z.scatter_add_(1, y[:, None], (torch.randn(n, 1, generator=gen, device="cuda") * 3 + 6).to(dt))
    logp, lse, plogp = (torch.empty(n, device="cuda") for _ in range(3))
    ops.token_logp(z, y, logp, lse=lse)
    ops.policy_loss(z, y, torch.zeros(n, device="cuda"), torch.ones(n, device="cuda"), torch.empty(1, device="cuda"), logp=plogp)
    f = z.float()
    top = f.amax(1, keepdim=True)
    total = (f - top).exp().sum(1)
    plain = f.gather(1, y[:, None])[:, 0] - top[:, 0] - total.log()
    plain_lse = top[:, 0] + total.log()
    wide = z.double()
    want_lse = torch.logsumexp(wide, 1)
    want = wide.gather(1, y[:, None])[:, 0] - want_lse
    rms = lambda a, b: (a.double() - b).square().mean().sqrt().item()  # noqa: E731
    assert rms(logp, want) <= rms(plain, want)
    assert rms(plogp, want) <= rms(plain, want)
    assert rms(lse, want_lse) <= 1.25 * rms(plain_lse, want_lse)      # both end in one rounding of the same size


@pytest.mark.parametrize("vocab", [7, 1001, 40000, 290001])
def test_rows_on_both_sides_of_the_largest_offset(ops, vocab):
    """Logits around +-2^21, where the kernels' form of the exponent changes, a quarter or half a unit apart: one thread's share of a row
    may lie below it, another's beyond.  Differences are exact, as above."""
    rng = np.random.default_rng(vocab)
    steps = rng.integers(-40, 41, vocab) * 0.25
    rows = [at + s for at in (-2.0 ** 21, 2.0 ** 21) for s in (steps, np.sort(steps), np.sort(steps)[::-1])]
    z = dev(np.stack(rows))
    y = torch.from_numpy(rng.integers(0, vocab, len(rows))).cuda()
    logp = torch.empty(len(rows), device="cuda")
    ops.token_logp(z, y, logp)
    hz = host(z)
    wl, _, soft = O.token_logp(hz, y.cpu().numpy())
    tol = (vocab / 128 + 64) * E + 4 * E * (hz.max(1) - hz.min(1) + np.log(vocab))
    close(logp, wl, tol, "logp")
    loss, d = torch.empty(1, device="cuda"), torch.empty_like(z)
    ops.policy_loss(z, y, dev(wl), torch.ones(len(rows), device="cuda"), loss, d)
    per = -np.exp(wl - host(dev(wl))) / len(rows)
    want = -per[:, None] * soft
    want[np.arange(len(rows)), y.cpu().numpy()] += per
    close(d, want, grad_tol(want, per, soft, tol, torch.float32, c_err=(2 * tol + 8 * E) / len(rows)), "dlogits")


# ----------------------------------------------------------------------------- layer norm, backward

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(9, 64), (9, 65), (40, 1001), (300, 1024), (5, 8192), (3, 16384), (3, 20001)])
@pytest.mark.parametrize("scale", [1e22, 1e25, 1e-22])
@pytest.mark.parametrize("with_dsum", [False, True])
@pytest.mark.parametrize("shift", [0, 1])
def test_norm_backward_of_rows_with_a_large_or_small_spread(ops, dtype, rows, cols, scale, with_dsum, shift):
    """rstd is far from one, its square no number of binary32; every factor of the formula is.  `shift`: off the runs."""
    dt = TYPES[dtype]
    rng = np.random.default_rng(rows + cols)
    s = dev(rng.normal(size=(rows, cols)) * scale, dt)
    hs = host(s)
    mean, rstd = dev(hs.mean(1)), dev(1 / hs.std(1))
    dy, w = dev(rng.normal(size=(rows, cols)), dt), dev(rng.normal(size=cols) * 0.3 + 1)
    dsum = dev(rng.normal(size=(rows, cols)) / scale, dt) if with_dsum else None
    dx, dw = strided(torch.zeros_like(s), 0, shift), torch.empty(cols, device="cuda")
    ops.layer_norm_backward(strided(dy, 0, shift), strided(s, 0, shift), mean, rstd, dx, weight=w, dweight=dw,
                            dsum=strided(dsum, 0, shift) if with_dsum else None)
    hd, hw = host(dy), host(w)
    want, _, ww, _ = O.layer_norm_backward(hd, hs, host(mean), host(rstd), hw, host(dsum) if with_dsum else None)
    r = host(rstd)[:, None]
    h = np.abs(hs - host(mean)[:, None]) * r + E * np.abs(hs) * r
    g = np.abs(hd * hw)
    K = cols / 128 + 32
    mag = r * (g + g.mean(1, keepdims=True) + h * (g * h).mean(1, keepdims=True)) + (np.abs(host(dsum)) if with_dsum else 0)
    close(dx, want, U[dt] * np.abs(want) + K * E * mag + TINY[dt], "dx")
    close(dw, ww, (rows + 33) * E * (np.abs(hd) * h).sum(0), "dweight")


@pytest.mark.parametrize("cols", [41, 47, 49, 82, 94, 98, 976, 1001, 8200, 20000])
@pytest.mark.parametrize("p", [0.0, 0.25])
def test_norm_backward_takes_out_a_constant_exactly(ops, cols, p):
    """dout constant, h = +-1 in pairs: every sum is exact in binary32 (multiples of 2^20 below 2^44), mean(g) is g and mean(g h)
    is 0, so ds is 0.  1 / cols is no binary number, and a product with its rounding misses g by a unit in the last place for some cols."""
    rows = 5
    s = torch.zeros(rows, cols, device="cuda")
    s[:, 0:cols // 2 * 2:2], s[:, 1:cols // 2 * 2:2] = 1.0, -1.0
    dy = torch.full_like(s, 2.0 ** 20)
    dx = torch.empty_like(s)
    ops.layer_norm_backward(dy, s, torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda"), dx, p=p, seed=1)
    assert not dx.any()


# ----------------------------------------------------------------------------- terms of weight zero

def test_preference_without_smoothing_survives_an_impossible_answer(ops):
    """A rejected answer of probability zero: h = +inf, -log sigma(h) = 0.  The smoothing term has weight zero and is left out."""
    z, y, _ = make_rows(4, 70, torch.float32)
    z[3, y[3]] = -float("inf")
    ref = torch.zeros(4, device="cuda")
    loss, margin, d = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(z)
    ops.preference_loss(z, y, ref, loss, d, sequences=2, margin=margin)
    assert margin.item() == float("inf") and loss.item() == 0.0 and not d.any()
    z2 = torch.cat([z[2:], z[:2]]).contiguous()                  # now the preferred one
    y2 = torch.cat([y[2:], y[:2]])
    ops.preference_loss(z2, y2, ref, loss, d, sequences=2, margin=margin)
    assert margin.item() == -float("inf") and loss.item() == float("inf")


@pytest.mark.parametrize("per_sequence", [False, True])
def test_policy_statistics_without_the_kl_term_leave_the_loss_alone(ops, per_sequence):
    """kl_beta = 0 with ref_logp: the KL statistic may overflow, loss and gradient are those without it."""
    z, y, rng = make_rows(6, 300, torch.float32)
    logp = O.token_logp(host(z), y.cpu().numpy())[0]
    old, adv, ref = dev(logp + 0.05), dev(rng.normal(size=6)), dev(logp + 0.1)
    ref[2] = 200.0                                               # exp(u) overflows binary32
    loss, stats, d = torch.empty(1, device="cuda"), torch.empty(3, device="cuda"), torch.empty_like(z)
    other, e = torch.empty(1, device="cuda"), torch.empty_like(z)
    ops.policy_loss(z, y, old, adv, loss, d, sequences=2, per_sequence=per_sequence, ref_logp=ref, stats=stats)
    ops.policy_loss(z, y, old, adv, other, e, sequences=2, per_sequence=per_sequence)
    assert torch.isfinite(other).all() and torch.equal(loss, other) and torch.equal(d, e)
    assert stats[0].item() == float("inf")


# ----------------------------------------------------------------------------- automatic differentiation

def test_calls_are_outside_automatic_differentiation(ops):
    """An output that is part of a recorded graph is refused, and what a call writes counts as modified in place."""
    x = torch.randn(4, 16, device="cuda")
    w = torch.randn(16, device="cuda", requires_grad=True)
    out = torch.empty_like(x)
    ops.layer_norm(x, out, weight=w)                             # inputs may require gradients; the call is not recorded
    assert not out.requires_grad
    grad = torch.empty(4, 16, device="cuda", requires_grad=True)
    vec = torch.empty(4, device="cuda", requires_grad=True)
    z, y, v = torch.randn(6, 10, device="cuda"), torch.zeros(6, dtype=torch.int64, device="cuda"), torch.zeros(6, device="cuda")
    loss, one = torch.empty(1, device="cuda"), torch.empty(1, device="cuda", requires_grad=True)
    refused = [lambda: ops.dropout(x, grad, p=0.1, seed=0), lambda: ops.layer_norm(x, grad), lambda: ops.layer_norm(x, out, mean=vec),
               lambda: ops.layer_norm(x, out, sum_out=grad),
               lambda: ops.layer_norm_backward(x, x, v[:4], v[:4], out, weight=w, dweight=w),
               lambda: ops.token_logp(z, y, v.clone().requires_grad_()), lambda: ops.preference_loss(z, y, v, one, sequences=2),
               lambda: ops.policy_loss(z, y, v, v, loss, z.clone().requires_grad_())]
    before = ops.launch_count()
    for k, call in enumerate(refused):
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
            pytest.fail(f"refusal {k} went through")
    assert ops.launch_count() == before
    with torch.no_grad():
        ops.layer_norm(x, grad)                                  # nothing is being recorded
    ops.layer_norm(x, out)
    assert torch.equal(grad.detach(), out)
    a = torch.randn(4, 16, device="cuda", requires_grad=True)
    s = a * 1.0
    t = s.square().sum()                                         # keeps s
    with torch.no_grad():
        ops.dropout(x, s, p=0.0, seed=0)                         # overwrites it
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        t.backward()
    with torch.inference_mode():
        i = torch.empty(4, 16, device="cuda")
    ops.dropout(x, i, p=0.0, seed=0)                             # inference tensors have no version to count
    assert torch.equal(i, x)
    versions = (out._version, loss._version)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ops.layer_norm(x, out)                                   # by way of another stream too
    torch.cuda.current_stream().wait_stream(side)
    ops.policy_loss(z, y, v, v, loss)
    assert out._version == versions[0] + 1 and loss._version == versions[1] + 1


def test_one_token_norm_repeats_bit_for_bit(ops):
    x, res = (torch.randn(1, 4096, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    w, b = (torch.randn(4096, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    seen = []
    for _ in range(200):
        out, total, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
        ops.layer_norm(x, out, weight=w, bias=b, residual=res, sum_out=total, mean=mean, rstd=rstd)
        seen.append((out, total, mean, rstd))
    for other in seen[1:]:
        assert all(torch.equal(a, c) for a, c in zip(seen[0], other))


@pytest.mark.parametrize("n,vocab", [(1024, 8000), (512, 100003)])
def test_policy_loss_is_at_least_as_exact_as_the_plain_form(ops, n, vocab):
    """Errors of loss and gradient against binary64 over eight batches (root mean square), beside those of the formula in elementary
    binary32 operations.  Ratios are near one, so what counts is the difference of log-probabilities.  The gradient's error is relative;
    the loss is a sum of terms of both signs that may come out anywhere near zero, so its error is taken as it is."""
    lo = hi = float(np.float32(0.2))
    kb = float(np.float32(0.04))
    found = np.zeros((8, 4))
    for k in range(8):
        gen = torch.Generator(device="cuda").manual_seed(1000 + k)
        normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
        z, y = normal(n, vocab) * 2, torch.randint(vocab, (n,), generator=gen, device="cuda")
        z.scatter_add_(1, y[:, None], normal(n, 1) * 3 + 6)
        true = torch.log_softmax(z.double(), 1)
        at = true.gather(1, y[:, None])[:, 0]
        old, ref, A = (at + 0.15 * normal(n)).float(), (at + 0.25 * normal(n)).float(), normal(n)

        def rest(logp, soft, old, ref, A):
            r, u = (logp - old).exp(), ref - logp
            gain, held = r * A, r.clamp(1 - lo, 1 + hi) * A
            loss = (kb * (u.exp() - u - 1) - torch.minimum(gain, held)).sum() / n
            slope = (torch.where(gain <= held, -gain, torch.zeros_like(gain)) + kb * (1 - u.exp())) / n
            d = soft * -slope[:, None]
            return loss, d.scatter_add_(1, y[:, None], slope[:, None])

        exact_loss, exact_d = rest(at, true.exp(), old.double(), ref.double(), A.double())
        e = (z - z.amax(1, keepdim=True)).exp()
        total = e.sum(1)
        plain = (z - z.amax(1, keepdim=True)).gather(1, y[:, None])[:, 0] - total.log()
        plain_loss, plain_d = rest(plain, e / total[:, None], old, ref, A)
        loss, d = torch.empty(1, device="cuda"), torch.empty_like(z)
        ops.policy_loss(z, y, old, A, loss, d, ref_logp=ref, clip_low=0.2, clip_high=0.2, kl_beta=0.04)
        off = lambda v, w: ((v.double() - w).norm() / w.norm()).item()  # noqa: E731
        miss = lambda v: abs(v.item() - exact_loss.item())  # noqa: E731
        found[k] = miss(loss), miss(plain_loss), off(d, exact_d), off(plain_d, exact_d)
    own_loss, plain_loss, own_d, plain_d = np.sqrt((found ** 2).mean(0))
    assert own_loss <= plain_loss and own_d <= plain_d, found


@pytest.mark.parametrize("value", [-3e4, -1e9, -1e30, None])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [40, 3000, 290001])
def test_a_masked_label_is_the_same_under_the_same_model(ops, value, dtype, vocab):
    """Labels that a mask has set to a low value (None: the type's lowest), with the log-probabilities of the same logits as the old policy's
    and the reference's: ratios are one and margins zero, although a log-probability of -1e9 is only given to the nearest 64."""
    dt = TYPES[dtype]
    z, y, rng = make_rows(8, vocab, dt)
    z[torch.arange(8, device="cuda"), y] = torch.finfo(dt).min if value is None else value
    logp, loss, margin, d = torch.empty(8, device="cuda"), torch.empty(1, device="cuda"), torch.empty(2, device="cuda"), torch.empty_like(z)
    stats = torch.empty(3, device="cuda")
    ops.token_logp(z, y, logp)
    ops.preference_loss(z, y, logp, loss, d, sequences=4, margin=margin)
    assert not margin.any() and abs(loss.item() - np.log(2)) < 4 * E
    A = dev(rng.normal(size=8))
    ops.policy_loss(z, y, logp, A, loss, d, ref_logp=logp, kl_beta=0.1, stats=stats)
    assert abs(loss.item() + A.double().mean().item()) <= 4 * E * A.abs().mean().item()
    assert stats[0].item() == 0 and stats[1].item() == 0
    got = d.double()[torch.arange(8, device="cuda"), y]                  # -A / n (1 - 0): the label's own probability is zero
    close(got, -host(A) / 8, (U[dt] + 4 * E) * np.abs(host(A)) / 8, "dlogits")
