"""Plain double-precision definitions of the operators of a gated recurrent and of a selective state-space language model -- TEST
INFRASTRUCTURE ONLY.

Every function takes and returns float64 arrays; 8- and 32-bit whole numbers are held as the numbers they are."""
from __future__ import annotations

import numpy as np

from . import _d, round_to


def rms_norm_q8(x, r, g, eps, dtype):
    """(q, s, y): y = x (+ r), rounded to `dtype` as it is stored, is what the norm is of."""
    y = _d(x) if r is None else round_to(_d(x) + _d(r), dtype)
    with np.errstate(invalid="ignore"):
        n = y * _d(g) / np.sqrt((y * y).mean(axis=1, keepdims=True) + eps)
        s = np.abs(n).max(axis=1) / 127.0
    whole = np.isfinite(y).all(axis=1)
    some = whole & (s > 0)
    q = np.zeros_like(n)
    q[some] = np.rint(n[some] / s[some][:, None])
    return q, np.where(whole, s, np.nan), y


def dense_q8(x, sx, w, sw, b=None):
    y = (_d(x) @ _d(w).T) * _d(sx)[:, None] * _d(sw)[None, :]        # whole numbers below 2^53: the sum is exact
    return y if b is None else y + _d(b)


def _gates(z):
    z = z.reshape(z.shape[0], 2, -1)
    f = z[:, 0]
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-f)), 1.0 / (1.0 + np.exp(f)), z[:, 1]


def linear_scan(z, h0, keep=None, states=False):
    """(h, hT), and with states=True the state before every row as well."""
    z, state = _d(z), _d(h0).copy()
    B, D = state.shape
    T = z.shape[0] // B
    a, rest, v = (t.reshape(B, T, D) for t in _gates(z))
    keep = np.ones((B, T)) if keep is None else np.asarray(keep).reshape(B, T)
    h, before = np.zeros((B, T, D)), np.zeros((B, T, D))
    for b in range(B):
        for t in range(T):
            before[b, t] = state[b]
            if keep[b, t] == 0:
                continue
            if keep[b, t] == 2:
                before[b, t] = 0.0
                state[b] = rest[b, t] * v[b, t]
            else:
                state[b] = a[b, t] * state[b] + rest[b, t] * v[b, t]
            h[b, t] = state[b]
    out = (h.reshape(B * T, D), state)
    return out + (before,) if states else out


def linear_scan_grad(z, h0, dh, dhT, keep=None):
    """(dz, dh0)"""
    z, h0 = _d(z), _d(h0)
    B, D = h0.shape
    T = z.shape[0] // B
    before = linear_scan(z, h0, keep, states=True)[2]
    a, rest, v = (t.reshape(B, T, D) for t in _gates(z))
    keep = np.ones((B, T)) if keep is None else np.asarray(keep).reshape(B, T)
    dh, G = _d(dh).reshape(B, T, D), _d(dhT).copy()
    dz = np.zeros((B, T, 2, D))
    for b in range(B):
        for t in range(T - 1, -1, -1):
            if keep[b, t] == 0:
                continue
            G[b] = G[b] + dh[b, t]
            dz[b, t, 0] = G[b] * (before[b, t] - v[b, t]) * a[b, t] * rest[b, t]
            dz[b, t, 1] = G[b] * rest[b, t]
            G[b] = 0.0 if keep[b, t] == 2 else a[b, t] * G[b]
    return dz.reshape(B * T, 2 * D), G


def _softmax(x):
    """(ln p, p, entropy) of the rows; a row of -inf alone has ln p = -inf, p = 0, entropy 0."""
    x = _d(x)
    m = x.max(axis=1, keepdims=True)
    with np.errstate(all="ignore"):
        rel = np.where(np.isneginf(m), -np.inf, x - m)
        e = np.exp(rel)
        total = e.sum(axis=1, keepdims=True)
        logs = np.where(np.isneginf(m), -np.inf, rel - np.log(total))
        p = np.where(np.isneginf(m), 0.0, e / total)
        ent = -np.where(p == 0, 0.0, p * logs).sum(axis=1)
    return logs, p, ent


def token_logprobs(x, tok, top=0):
    """(lp, ent) and, with top > 0, (top_lp, top_id)."""
    x, tok = _d(x), np.asarray(tok).astype(np.int64)
    logs, _, ent = _softmax(x)
    given = (tok >= 0) & (tok < x.shape[1])
    lp = np.where(given, logs[np.arange(len(tok)), np.where(given, tok, 0)], 0.0)
    broken = np.isnan(x).any(axis=1) | np.isposinf(x).any(axis=1)
    lp[broken] = np.nan
    ent = np.where(broken, np.nan, ent)
    if not top:
        return lp, ent
    ids = np.empty((len(tok), top))
    for i, row in enumerate(x):
        # largest first, the earlier one of equals; NaN above everything
        order = sorted(range(len(row)), key=lambda j: (0, 0.0, j) if np.isnan(row[j]) else (1, -row[j], j))
        ids[i] = order[:top]
    top_lp = logs[np.arange(len(tok))[:, None], ids.astype(np.int64)]
    top_lp[broken] = np.nan
    return lp, ent, top_lp, ids


def token_logprobs_grad(x, tok, dlp, dent):
    x, tok = _d(x), np.asarray(tok).astype(np.int64)
    logs, p, ent = _softmax(x)
    given = (tok >= 0) & (tok < x.shape[1])
    dlp = np.where(given, _d(dlp), 0.0)
    dead = np.isneginf(x).all(axis=1)
    with np.errstate(invalid="ignore"):
        dx = -dlp[:, None] * p - _d(dent)[:, None] * np.where(p == 0, 0.0, p * (logs + ent[:, None]))
    dx[np.arange(len(tok)), np.where(given, tok, 0)] += dlp
    dx[dead] = 0.0
    return dx


# ---- a selective state-space language model -------------------------------------------------------------------------------
def _sigmoid(v):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-v))


def _documents(keep, b, T):
    """The rows of sequence b that are tokens, each with whether a document begins there."""
    return [(t, keep[b, t] == 2) for t in range(T) if keep[b, t] != 0]


def _sequences(x, s0, keep):
    B = s0.shape[0]
    T = x.shape[0] // B
    return B, T, np.ones((B, T)) if keep is None else np.asarray(keep).reshape(B, T)


def causal_conv(x, w, b, s0, keep=None, silu=False, grads=None):
    """(y, sT); grads = (dy, dsT): (dx, dw, db, ds0).  A token is what an integer names: t >= 0 a row, -1 - j the state's token j, None zeros."""
    x, w, bias, s0 = _d(x), _d(w), _d(b), _d(s0)
    B, T, keep = _sequences(x, s0, keep)
    D, K = w.shape
    x = x.reshape(B, T, D)
    y, sT = np.zeros((B, T, D)), np.zeros_like(s0)
    if grads:
        dy, dsT = _d(grads[0]).reshape(B, T, D), _d(grads[1])
        dx, dw, db, ds0 = np.zeros((B, T, D)), np.zeros_like(w), np.zeros(D), np.zeros_like(s0)

    def add(i, seq, v):
        if seq is not None:
            (dx[i] if seq >= 0 else ds0[i])[seq if seq >= 0 else -1 - seq] += v

    for i in range(B):
        seen = [-1 - j for j in range(K - 1)]
        value = lambda q: np.zeros(D) if q is None else x[i, q] if q >= 0 else s0[i, -1 - q]
        for t, begins in _documents(keep, i, T):
            if begins:
                seen = [None] * (K - 1)
            taps = seen + [t]
            u = bias + sum(w[:, k] * value(q) for k, q in enumerate(taps))
            s = _sigmoid(u)
            y[i, t] = u * s if silu else u
            if grads:
                g = dy[i, t] * (s + u * s * (1 - s) if silu else 1.0)
                db += g
                for k, q in enumerate(taps):
                    dw[:, k] += g * value(q)
                    add(i, q, w[:, k] * g)
            seen = taps[1:]
        for j, q in enumerate(seen):
            sT[i, j] = value(q)
            if grads:
                add(i, q, dsT[i, j])
    if grads:
        return dx.reshape(B * T, D), dw, db, ds0
    return y.reshape(B * T, D), sT


def causal_conv_grad(x, w, b, s0, dy, dsT, keep=None, silu=False):
    return causal_conv(x, w, b, s0, keep, silu, (dy, dsT))


def softplus(v):
    return np.maximum(v, 0.0) + np.log1p(np.exp(-np.abs(v)))


def selective_scan(x, dt, bc, a, skip, h0, z=None, keep=None, grads=None):
    """(y, hT); grads = (dy, dhT): (dx, ddt, dbc, da, dskip, dh0[, dz])."""
    x, dt, bc, a, skip, h0 = (_d(v) for v in (x, dt, bc, a, skip, h0))
    B, T, keep = _sequences(x, h0, keep)
    D, N = a.shape
    x, dt, bc = x.reshape(B, T, D), dt.reshape(B, T, D), bc.reshape(B, T, 2, N)
    gate = None if z is None else _d(z).reshape(B, T, D)
    y, hT = np.zeros((B, T, D)), h0.copy()
    if grads:
        dy, dhT = _d(grads[0]).reshape(B, T, D), _d(grads[1])
        dx, ddt, dz, dbc = (np.zeros_like(v) for v in (x, dt, x, bc))
        da, dskip, dh0 = np.zeros_like(a), np.zeros_like(skip), dhT.copy()
    for i in range(B):
        tokens, before = _documents(keep, i, T), {}
        for t, begins in tokens:
            if begins:
                hT[i] = 0.0
            before[t] = hT[i].copy()
            s = softplus(dt[i, t])
            hT[i] = np.exp(s[:, None] * a) * hT[i] + (s * x[i, t])[:, None] * bc[i, t, 0]
            y[i, t] = hT[i] @ bc[i, t, 1] + skip * x[i, t]
            if gate is not None:
                y[i, t] *= gate[i, t] * _sigmoid(gate[i, t])
        for t, begins in reversed(tokens) if grads else ():
            Bt, Ct = bc[i, t]
            s, xt = softplus(dt[i, t]), x[i, t]
            e = np.exp(s[:, None] * a)
            h = e * before[t] + (s * xt)[:, None] * Bt
            du = dy[i, t]
            if gate is not None:
                zt = gate[i, t]
                sg = _sigmoid(zt)
                dz[i, t] = du * (h @ Ct + skip * xt) * (sg + zt * sg * (1 - sg))
                du = du * zt * sg
            G = dh0[i] + du[:, None] * Ct
            decayed = G * e * before[t]
            dx[i, t] = du * skip + s * (G @ Bt)
            ddt[i, t] = ((decayed * a).sum(1) + xt * (G @ Bt)) * _sigmoid(dt[i, t])
            dbc[i, t, 0], dbc[i, t, 1] = (s * xt) @ G, du @ h
            da += decayed * s[:, None]
            dskip += du * xt
            dh0[i] = 0.0 if begins else G * e
    if grads:
        return (dx.reshape(B * T, D), ddt.reshape(B * T, D), dbc.reshape(B * T, 2 * N), da, dskip, dh0) + (() if gate is None else (dz.reshape(B * T, D),))
    return y.reshape(B * T, D), hT


def selective_scan_grad(x, dt, bc, a, skip, h0, dy, dhT, z=None, keep=None):
    return selective_scan(x, dt, bc, a, skip, h0, z, keep, (dy, dhT))


def dense_logprobs(x, w, tok):
    """(lp, lse)"""
    with np.errstate(all="ignore"):
        logits = _d(x) @ _d(w).T
        m = logits.max(axis=1)
        lse = np.where(np.isneginf(m), -np.inf, m + np.log(np.exp(logits - np.where(np.isneginf(m), 0.0, m)[:, None]).sum(axis=1)))
        tok = np.asarray(tok).astype(np.int64)
        given = (tok >= 0) & (tok < logits.shape[1])
        lp = logits[np.arange(len(tok)), np.where(given, tok, 0)] - lse
    return np.where(given, np.where(np.isneginf(lse), -np.inf, lp), 0.0), lse


def dense_logprobs_grad(x, w, tok, lse, dlp, dlse, parts=False):
    """(dx, dw); parts: dl as well."""
    x, w, lse, dlse = (_d(v) for v in (x, w, lse, dlse))
    tok = np.asarray(tok).astype(np.int64)
    given = (tok >= 0) & (tok < w.shape[0])
    dlp = np.where(given, _d(dlp), 0.0)
    takes_part = (dlp != 0) | (dlse != 0)
    x = np.where(takes_part[:, None], x, 0.0)
    with np.errstate(all="ignore"):
        p = np.where(np.isneginf(lse)[:, None], 0.0, np.exp(x @ w.T - lse[:, None]))
        dl = (dlse - dlp)[:, None] * p
    dl[np.arange(len(tok)), np.where(given, tok, 0)] += dlp
    dl[~takes_part] = 0.0
    return (dl @ w, dl.T @ x) + ((dl,) if parts else ())
