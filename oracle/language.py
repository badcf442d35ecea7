"""Plain double-precision definitions of the operators of a gated recurrent language model -- TEST INFRASTRUCTURE ONLY.

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
