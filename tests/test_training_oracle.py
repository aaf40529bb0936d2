"""Pins of the binary64 restatement that the training operators are tested against, and the host side of their C ABI
(symbols, checks of arguments).  No GPU."""
import ctypes as C
import os
import re

import numpy as np
import pytest

import paper_2211_00188_b200 as pkg
from oracle import training_oracle as O
from paper_2211_00188_b200 import build as builder
from paper_2211_00188_b200 import training as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    builder.build()
    return pkg.load_training_library()


def test_generator_gives_the_published_vectors():
    # known answers of the generator's authors for Philox4x32 with ten rounds
    assert O.philox_words([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert O.philox_words([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert O.philox_words([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == \
        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_dropout_keeps_the_share_and_the_expectation():
    x = np.ones(40000)
    y = O.drop(x, 0.3, 7, 1)
    thr = O.threshold(0.3)
    assert set(np.unique(y)) == {0.0, 65536.0 / (65536 - thr)}
    share = (y > 0).mean()
    assert abs(share - (1 - thr / 65536)) < 5 * np.sqrt(0.3 * 0.7 / 40000)   # five standard deviations
    assert not np.array_equal(y, O.drop(x, 0.3, 7, 2)) and not np.array_equal(y, O.drop(x, 0.3, 8, 1))
    assert np.array_equal(O.drop(x, 0.0, 7, 1), x) and not O.drop(x, 1.0, 7, 1).any()


def difference(f, x, step):
    g = np.zeros_like(x)
    for i in range(x.size):
        a, b = x.copy(), x.copy()
        a.flat[i] += step
        b.flat[i] -= step
        g.flat[i] = (f(a) - f(b)) / (2 * step)
    return g


def test_norm_gradients_agree_with_differences():
    rng = np.random.default_rng(0)
    x, res, up, down = (rng.normal(size=(3, 7)) for _ in range(4))
    w, b = rng.normal(size=7), rng.normal(size=7)
    kw = dict(p=0.3, seed=5, offset=2)

    def value(x_=x, r_=res, w_=w, b_=b):
        out, s, _, _ = O.layer_norm(x_, w_, b_, 1e-5, r_, **kw)
        return (up * out).sum() + (down * s).sum()

    _, s, mean, rstd = O.layer_norm(x, w, b, 1e-5, res, **kw)
    dx, dres, dw, db = O.layer_norm_backward(up, s, mean, rstd, w, down, **kw)
    # central differences: step^2 times the third derivative (of order 1) and rounding / step: 1e-8 either way
    for got, want in ((dx, difference(lambda v: value(x_=v), x, 1e-4)), (dres, difference(lambda v: value(r_=v), res, 1e-4)),
                      (dw, difference(lambda v: value(w_=v), w, 1e-4)), (db, difference(lambda v: value(b_=v), b, 1e-4))):
        assert np.abs(got - want).max() < 1e-6


@pytest.mark.parametrize("kind,normalized,smoothing", [("sigmoid", False, 0.0), ("sigmoid", True, 0.2), ("hinge", False, 0.0),
                                                       ("square", True, 0.0)])
def test_preference_gradient_agrees_with_differences(kind, normalized, smoothing):
    rng = np.random.default_rng(1)
    z = rng.normal(size=(10, 5))
    labels, ref = rng.integers(0, 5, 10), rng.normal(size=10) - 2
    mask = np.array([1, 1, 0, 1, 1, 0, 0, 1, 1, 1])
    start = [0, 3, 5, 7, 10]        # sequence 2 has one counted token at most
    kw = dict(mask=mask, seq_start=start, beta=0.3, kind=kind, label_smoothing=smoothing, length_normalized=normalized)
    got = O.preference(z, labels, ref, **kw)
    assert np.all(np.abs(got["margin"] - 1) > 1e-2)     # away from the hinge's corner
    want = difference(lambda v: O.preference(v, labels, ref, **kw)["loss"], z, 1e-4)
    assert np.abs(got["dlogits"] - want).max() < 1e-6


@pytest.mark.parametrize("per_sequence", [False, True])
def test_policy_gradient_agrees_with_differences(per_sequence):
    rng = np.random.default_rng(2)
    z = rng.normal(size=(9, 6))
    labels = rng.integers(0, 6, 9)
    mask = np.array([1, 0, 1, 1, 0, 0, 1, 1, 1])
    logp = O.token_logp(z, labels)[0]
    old, ref, adv = logp + rng.normal(size=9) * 0.4, logp + rng.normal(size=9) * 0.4, rng.normal(size=9)
    r = np.exp(logp - old)
    assert np.all(np.abs(r - 0.8) > 1e-2) and np.all(np.abs(r - 1.25) > 1e-2)   # away from the corners of the clip
    kw = dict(mask=mask, seq_start=[0, 4, 6, 9], ref_logp=ref, clip_low=0.2, clip_high=0.25, kl_beta=0.3, per_sequence=per_sequence)
    got = O.policy(z, labels, old, adv, **kw)
    assert got["stats"][1] > 0                        # some token is clipped
    want = difference(lambda v: O.policy(v, labels, old, adv, **kw)["loss"], z, 1e-4)
    assert np.abs(got["dlogits"] - want).max() < 1e-6


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "adacgd_train.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(adacgd_[a-z_]+)\s*\(", text)))
    assert sorted(pkg.TRAIN_SYMBOLS) == names
    for name in names:
        assert hasattr(lib, name), name


def test_workspace_bytes_and_null_arguments(lib):
    n = C.c_size_t(0)
    assert lib.adacgd_train_workspace_bytes(1000, 1024, C.byref(n)) == 0 and n.value > 0
    small = n.value
    assert lib.adacgd_train_workspace_bytes(1000, 2048, C.byref(n)) == 0 and n.value > small
    for args in ((0, 8), (2 ** 31, 8), (8, 0), (8, T.MAX_COLS + 1)):
        assert lib.adacgd_train_workspace_bytes(*args, C.byref(n)) == 1
        assert b"adacgd_train_workspace_bytes" in lib.adacgd_train_last_error(None)
    assert lib.adacgd_train_workspace_bytes(8, 8, None) == 1
    ctx = C.c_void_p()
    assert lib.adacgd_train_init(None, 8, 8, None, 0, None) == 1
    assert lib.adacgd_train_init(C.byref(ctx), 8, 8, None, 0, None) == 1 and not ctx.value
    assert lib.adacgd_train_init(C.byref(ctx), 8, 8, C.c_void_p(8), 1 << 30, None) == 1
    assert lib.adacgd_train_init(C.byref(ctx), 8, 8, C.c_void_p(256), 16, None) == 4
    for name in ("adacgd_dropout", "adacgd_layer_norm", "adacgd_layer_norm_backward", "adacgd_preference_loss", "adacgd_policy_loss"):
        assert getattr(lib, name)(None, None) == 1
    assert lib.adacgd_token_logp(None, None, None, None) == 1
    assert lib.adacgd_train_launch_count(None) == 0
    lib.adacgd_train_destroy(None)


def test_no_device_is_an_error_not_a_fallback(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("device present")
    ctx, n = C.c_void_p(), C.c_size_t(0)
    assert lib.adacgd_train_workspace_bytes(8, 8, C.byref(n)) == 0
    assert lib.adacgd_train_init(C.byref(ctx), 8, 8, C.c_void_p(4096), n.value, None) == 5 and not ctx.value
    with pytest.raises(RuntimeError):
        pkg.TrainingOps(8, 8)
