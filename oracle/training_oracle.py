"""Plain numpy restatement, in binary64, of the training operators of include/adacgd_train.h.  Test infrastructure:
shares no code with the kernels, written from the formulas of the header, slow.

Arrays are numpy; inputs are converted to binary64 first, so the results are exact but for binary64 rounding.
"""
from __future__ import annotations

import numpy as np

M32 = 0xFFFFFFFF


def philox_words(counter, key):
    """Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC 2011) of one counter (four words) under a key (two words)."""
    c, k = [int(v) for v in counter], [int(v) for v in key]
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & M32, (a >> 32) ^ c[3] ^ k[1], a & M32]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return c


def threshold(p):
    return int(np.floor(65536 * p + 0.5))


def kept(first, count, p, seed, offset):
    """Truth values of elements first .. first + count - 1."""
    out = np.empty(count, dtype=bool)
    key = (seed & M32, (seed >> 32) & M32)
    words, block = None, None
    for i in range(count):
        b, j = divmod(first + i, 8)
        if b != block:
            words, block = philox_words((b & M32, (b >> 32) & M32, offset & M32, (offset >> 32) & M32), key), b
        out[i] = ((words[j >> 1] >> (16 * (j & 1))) & 0xFFFF) >= threshold(p)
    return out


def drop(x, p, seed, offset):
    x = np.asarray(x, dtype=np.float64)
    thr = threshold(p)
    if thr == 0:
        return x.copy()
    if thr == 65536:
        return np.zeros_like(x)
    k = kept(0, x.size, p, seed, offset).reshape(x.shape)
    return np.where(k, x * (65536.0 / (65536.0 - thr)), 0.0)


def layer_norm(x, weight=None, bias=None, eps=1e-5, residual=None, p=0.0, seed=0, offset=0):
    """(out, s, mean, rstd)"""
    s = drop(x, p, seed, offset)
    if residual is not None:
        s = np.asarray(residual, dtype=np.float64) + s
    mean = s.mean(1)
    rstd = 1.0 / np.sqrt(((s - mean[:, None]) ** 2).mean(1) + eps)
    h = (s - mean[:, None]) * rstd[:, None]
    out = h * (1.0 if weight is None else np.asarray(weight, np.float64)) + (0.0 if bias is None else np.asarray(bias, np.float64))
    return out, s, mean, rstd


def layer_norm_backward(dout, s, mean, rstd, weight=None, dsum=None, p=0.0, seed=0, offset=0):
    """(dx, dresidual, dweight, dbias)"""
    dout, s = np.asarray(dout, np.float64), np.asarray(s, np.float64)
    mean, rstd = np.asarray(mean, np.float64)[:, None], np.asarray(rstd, np.float64)[:, None]
    h = (s - mean) * rstd
    g = dout * (1.0 if weight is None else np.asarray(weight, np.float64))
    ds = rstd * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    if dsum is not None:
        ds = ds + np.asarray(dsum, np.float64)
    return drop(ds, p, seed, offset), ds, (dout * h).sum(0), dout.sum(0)


def token_logp(logits, labels, mask=None):
    """(logp, lse, softmax); rows that do not count: 0, 0 and 0.  All -inf, or a label out of range: NaN."""
    z = np.asarray(logits, np.float64)
    n, v = z.shape
    logp, lse, soft = np.zeros(n), np.zeros(n), np.zeros((n, v))
    for t in range(n):
        if mask is not None and not mask[t]:
            continue
        m = z[t].max()
        if m == -np.inf:
            lse[t], logp[t], soft[t] = -np.inf, np.nan, np.nan
            continue
        e = np.exp(z[t] - m)
        lse[t] = m + np.log(e.sum())
        soft[t] = e / e.sum()
        y = int(labels[t])
        logp[t] = (z[t, y] - m) - np.log(e.sum()) if 0 <= y < v else np.nan   # not z - lse: m may be huge
    return logp, lse, soft


def runs(tokens, sequences=None, seq_start=None):
    if seq_start is None:
        each = tokens // sequences
        return [(q * each, (q + 1) * each) for q in range(sequences)]
    return [(int(a), int(b)) for a, b in zip(seq_start[:-1], seq_start[1:])]


def _dlogits(per_token, labels, soft, counted):
    d = np.zeros_like(soft)
    for t in np.flatnonzero(counted):
        d[t] = -per_token[t] * soft[t]
        if 0 <= int(labels[t]) < soft.shape[1]:
            d[t, int(labels[t])] += per_token[t]
    return d


def preference(logits, labels, ref_logp, mask=None, sequences=None, seq_start=None, beta=0.1, kind="sigmoid",
               label_smoothing=0.0, length_normalized=False, grad_scale=1.0):
    """dict(loss, margin, seq_logp, dlogits, per_token)"""
    n = len(labels)
    counted = np.ones(n, bool) if mask is None else np.asarray(mask).astype(bool)
    logp, _, soft = token_logp(logits, labels, counted)
    ref = np.asarray(ref_logp, np.float64)
    rr = runs(n, sequences, seq_start)
    diff, total, inv = [], [], []
    for a, b in rr:
        c = counted[a:b]
        k = 1.0 / c.sum() if length_normalized and c.sum() else 1.0
        diff.append(k * (logp[a:b][c] - ref[a:b][c]).sum())
        total.append(k * logp[a:b][c].sum())
        inv.append(k)
    half = len(rr) // 2
    h = beta * (np.array(diff[:half]) - np.array(diff[half:]))
    if kind == "sigmoid":
        e = label_smoothing
        loss = (1 - e) * np.logaddexp(0, -h) + (e * np.logaddexp(0, h) if e else 0.0)      # weight zero: left out
        g = e / (1 + np.exp(-h)) - (1 - e) / (1 + np.exp(h))
    elif kind == "hinge":
        loss, g = np.maximum(0, 1 - h), np.where(h < 1, -1.0, 0.0)
    else:
        u = h / beta - 1 / (2 * beta)
        loss, g = u * u, 2 * u / beta
    per_token = np.zeros(n)
    for q, (a, b) in enumerate(rr):
        sign = 1.0 if q < half else -1.0
        per_token[a:b] = sign * g[q % half] * beta * inv[q] / half * counted[a:b]
    return dict(loss=loss.mean(), margin=h, seq_logp=np.array(total), per_token=per_token,
                dlogits=grad_scale * _dlogits(per_token, labels, soft, counted))


def policy(logits, labels, old_logp, advantages, mask=None, sequences=None, seq_start=None, ref_logp=None, clip_low=0.2,
           clip_high=0.2, kl_beta=0.0, per_sequence=False, grad_scale=1.0):
    """dict(loss, logp, stats, dlogits, per_token)"""
    n = len(labels)
    counted = np.ones(n, bool) if mask is None else np.asarray(mask).astype(bool)
    logp, _, soft = token_logp(logits, labels, counted)
    w = np.zeros(n)
    if per_sequence:
        rr = runs(n, sequences, seq_start)
        used = sum(1 for a, b in rr if counted[a:b].any())
        for a, b in rr:
            if counted[a:b].any():
                w[a:b] = counted[a:b] / (used * counted[a:b].sum())
    elif counted.any():
        w = counted / counted.sum()
    loss, kl_sum, clipped = 0.0, 0.0, 0
    per_token = np.zeros(n)
    for t in np.flatnonzero(counted):
        A, r = float(advantages[t]), np.exp(logp[t] - float(old_logp[t]))
        gain, held = r * A, min(max(r, 1 - clip_low), 1 + clip_high) * A
        l, c = (-held, 0.0) if gain > held else (-gain, -gain)        # NaN goes through
        if ref_logp is not None:
            u = float(ref_logp[t]) - logp[t]
            if kl_beta:                                                # weight zero: left out
                l += kl_beta * (np.expm1(u) - u)
                c += kl_beta * -np.expm1(u)
            kl_sum += np.expm1(u) - u
        clipped += gain > held
        loss += w[t] * l
        per_token[t] = w[t] * c
    k = counted.sum()
    return dict(loss=loss, logp=logp, stats=np.array([kl_sum / k if k else 0.0, clipped / k if k else 0.0, k]),
                per_token=per_token, dlogits=grad_scale * _dlogits(per_token, labels, soft, counted))


def embedding(tokens, table, scale=1.0, mask=None):
    table = np.asarray(table, np.float64)
    out = np.zeros((len(tokens), table.shape[1]))
    for t, v in enumerate(tokens):
        if mask is None or mask[t]:
            out[t] = scale * table[int(v)] if 0 <= int(v) < len(table) else np.nan
    return out


def embedding_backward(tokens, dout, vocab, scale=1.0, mask=None, base=None):
    dout = np.asarray(dout, np.float64)
    total = np.zeros((vocab, dout.shape[1]))
    for t, v in enumerate(tokens):
        if (mask is None or mask[t]) and 0 <= int(v) < vocab:
            total[int(v)] += dout[t]
    return scale * total + (0.0 if base is None else np.asarray(base, np.float64))


def _turned(x, positions, freq, interleaved, back=False):
    """x [tokens, heads, dim] with its pairs turned."""
    y = x.copy()
    for i, f in enumerate(freq):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, len(freq) + i)
        angle = np.asarray(positions, np.float64) * float(f) * (-1.0 if back else 1.0)
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        y[..., p], y[..., q] = x[..., p] * c - x[..., q] * s, x[..., q] * c + x[..., p] * s
    return y


def qk_norm(x, head_dim, weight=None, eps=1e-6, positions=None, freq=(), interleaved=False):
    """q or k alone; [tokens, heads * head_dim]"""
    x = np.asarray(x, np.float64)
    h = x.reshape(len(x), -1, head_dim)
    n = h / np.sqrt((h * h).mean(2, keepdims=True) + eps) * (1.0 if weight is None else np.asarray(weight, np.float64))
    return _turned(n, positions, freq, interleaved).reshape(x.shape)


def qk_norm_backward(dout, x, head_dim, weight=None, eps=1e-6, positions=None, freq=(), interleaved=False):
    """(dx, dweight)"""
    x = np.asarray(x, np.float64)
    h = x.reshape(len(x), -1, head_dim)
    dn = _turned(np.asarray(dout, np.float64).reshape(h.shape), positions, freq, interleaved, back=True)
    r = 1.0 / np.sqrt((h * h).mean(2, keepdims=True) + eps)
    g = dn * (1.0 if weight is None else np.asarray(weight, np.float64))
    dx = r * (g - h * r * (g * h * r).mean(2, keepdims=True))
    return dx.reshape(x.shape), (dn * h * r).sum((0, 1))


def _seen(a, b, causal, counted):
    """[queries, keys] of rows a .. b"""
    ok = counted[a:b, None] & counted[None, a:b]
    return np.tril(ok) if causal else ok


def attention(q, k, v, heads, sequences=None, seq_start=None, causal=True, scale=None, mask=None):
    """(out, lse); rows of no sequence: NaN"""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n, dim = len(q), q.shape[1] // heads
    group = heads * dim // k.shape[1]
    scale = dim ** -0.5 if scale is None else scale
    counted = np.ones(n, bool) if mask is None else np.asarray(mask).astype(bool)
    out, lse = np.full(q.shape, np.nan), np.full((heads, n), np.nan)
    for a, b in runs(n, sequences, seq_start):
        ok = _seen(a, b, causal, counted)
        for h in range(heads):
            mine, shared = slice(h * dim, (h + 1) * dim), slice(h // group * dim, (h // group + 1) * dim)
            for i in range(a, b):
                sees = a + np.flatnonzero(ok[i - a])
                if not len(sees):
                    out[i, mine], lse[h, i] = 0.0, -np.inf
                    continue
                s = scale * (k[sees, shared] @ q[i, mine])
                m = s.max()
                e = np.exp(s - m)
                lse[h, i] = m + np.log(e.sum())
                out[i, mine] = (e / e.sum()) @ v[sees, shared]
    return out, lse


def attention_backward(dout, q, k, v, out, lse, heads, sequences=None, seq_start=None, causal=True, scale=None, mask=None):
    """dict(dq, dk, dv, row_dot), and what a tolerance is made of: sums of the absolute values of the terms (aq, ak, av).
    Rows of no sequence: NaN."""
    dout, q, k, v, out, lse = (np.asarray(x, np.float64) for x in (dout, q, k, v, out, lse))
    n, dim = len(q), q.shape[1] // heads
    group = heads * dim // k.shape[1]
    scale = dim ** -0.5 if scale is None else scale
    counted = np.ones(n, bool) if mask is None else np.asarray(mask).astype(bool)
    r = {"dq": np.full(q.shape, np.nan), "dk": np.full(k.shape, np.nan), "dv": np.full(k.shape, np.nan), "row_dot": np.full((heads, n), np.nan),
         "aq": np.zeros(q.shape), "ak": np.zeros(k.shape), "av": np.zeros(k.shape)}
    for a, b in runs(n, sequences, seq_start):
        ok = _seen(a, b, causal, counted)
        for name in ("dq", "dk", "dv"):
            r[name][a:b] = 0.0
        c = counted[a:b, None]
        for h in range(heads):
            mine, shared = slice(h * dim, (h + 1) * dim), slice(h // group * dim, (h // group + 1) * dim)
            qs, do, os = (np.where(c, x[a:b, mine], 0.0) for x in (q, dout, out))
            ks, vs = (np.where(c, x[a:b, shared], 0.0) for x in (k, v))
            with np.errstate(over="ignore", invalid="ignore"):
                p = np.where(ok, np.exp(scale * (qs @ ks.T) - np.where(counted[a:b], lse[h, a:b], 0.0)[:, None]), 0.0)
            dot = (do * os).sum(1)
            r["row_dot"][h, a:b] = dot
            dp = do @ vs.T
            ds = p * (dp - dot[:, None])
            r["dq"][a:b, mine] += scale * ds @ ks
            r["dk"][a:b, shared] += scale * ds.T @ qs
            r["dv"][a:b, shared] += p.T @ do
            # a rounded ds is off by its own rounding and by those of p (relative to ds) and of the sums in dp and dot
            ad = p * (np.abs(do) @ np.abs(vs).T + (np.abs(do) * np.abs(os)).sum(1)[:, None])
            r["aq"][a:b, mine] += scale * ad @ np.abs(ks)
            r["ak"][a:b, shared] += scale * ad.T @ np.abs(qs)
            r["av"][a:b, shared] += p.T @ np.abs(do)
    return r
