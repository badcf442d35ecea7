"""Cases of the operators of a selective state-space language model, and bounds on how far 32-bit arithmetic may be off.

Half a step of f32 is F.  An exponential of v is off by its argument's rounding, twice |v| F with that of the constant it is taken by, and its
own last bit, 2 F; so is a sigmoid, with 4 F more of its sum and reciprocal."""
import numpy as np

from oracle import language as L
from language_helpers import U, tensor

F = U["f32"]


def sigmoid(v):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-v))


def flags(rng, b, t, how):
    """keep of b sequences of t rows: None, "some" (documents of some eight tokens, padding anywhere), "ends" (padding behind, a sequence without a token)."""
    if how is None:
        return None
    keep = np.where(rng.uniform(size=(b, t)) < 0.12, 2, 1)
    if how == "some":
        keep = np.where(rng.uniform(size=(b, t)) < 0.25, 0, keep)
        keep[rng.integers(0, b)] = np.where(rng.uniform(size=t) < 0.9, 0, 1)
        keep = np.where(keep == 1, rng.choice([1, 1, 3, -1], size=keep.shape), keep)
    else:
        for i in range(b):
            keep[i, t - rng.integers(0, t // 2 + 1):] = 0
        keep[b - 1] = 0
    return keep.reshape(-1).astype(np.float64)


def poison(rng, a, keep):
    """NaN and infinities in the rows that are padding."""
    if keep is not None:
        rows = np.flatnonzero(keep == 0)
        a[rows] = rng.choice([np.nan, np.inf, -np.inf], size=(len(rows), 1))
    return a


# ---- the convolution -------------------------------------------------------------------------------------------------------
def conv_case(b, t, d, k, dtype, w_dtype, how, seed=0):
    """Operands as device tensors and as the numbers these hold: x, w, b, s0, dy, dsT, keep."""
    rng = np.random.default_rng(seed)
    keep = flags(rng, b, t, how)
    made = [(poison(rng, rng.normal(size=(b * t, d)), keep), dtype), (rng.uniform(-1, 1, size=(d, k)), w_dtype), (rng.normal(size=d), "f32"),
            (rng.normal(size=(b, k - 1, d)), dtype), (poison(rng, rng.normal(size=(b * t, d)), keep), dtype), (rng.normal(size=(b, k - 1, d)), dtype)]
    if keep is not None:
        made.append((keep, "i8"))
    both = [tensor(a, dt) + (dt,) for a, dt in made]
    return [(tt, dt) for tt, _, dt in both], [a for _, a, _ in both] + ([None] if keep is None else [])


def conv_bounds(x, w, b, s0, dy, dsT, keep, silu, dtype):
    """[y, dx, dw, db, ds0] bounds.  u: a product and a sum a tap.  The bounds of sums are sums of the terms' bounds and sizes: the linear operator
    on absolute values."""
    def clean(a):
        return np.abs(a) if keep is None else np.where((keep == 0)[:, None], 0.0, np.abs(a))

    K, rows = w.shape[1], x.shape[0]
    x, w_, s0_ = np.where(np.isfinite(x), x, 0.0), np.abs(w), np.abs(s0)
    u, _ = L.causal_conv(x, w, b, s0, keep)
    size, _ = L.causal_conv(clean(x), w_, np.abs(b), s0_, keep)
    eu = (K + 2) * F * size
    s = sigmoid(u)
    if silu:
        # slope of u s: at most 1.1; of s + u s (1 - s): at most 0.5
        y, g = u * s, s + u * s * (1 - s)
        ey = 1.1 * eu + np.abs(y) * (2 * np.abs(u) + 8) * F
        eg = 0.5 * eu + (s + np.abs(u) * s * (1 - s)) * (4 * np.abs(u) + 16) * F
    else:
        y, g, ey, eg = u, np.ones_like(u), eu, 0 * u
    last = U[dtype] if dtype == "bf16" else F
    dy = clean(np.where(np.isfinite(dy), dy, 0.0))
    eg = dy * (eg + F * np.abs(g))                             # of a row's derivative by u
    ag = dy * np.abs(g)
    zero, wide = np.zeros_like(s0), np.zeros_like(b)
    ex, ew, eb, es = L.causal_conv_grad(clean(x), w_, wide, s0_, eg, zero, keep)
    ax, aw, ab, as_ = L.causal_conv_grad(clean(x), w_, wide, s0_, ag, np.abs(dsT), keep)
    depth = rows / 16 + 100                                    # of the sum of a channel's rows
    return [ey + last * np.abs(y) + 1e-40, ex + ((K + 2) * F + last) * ax + 1e-40, ew + depth * F * aw + 1e-40, eb + depth * F * ab + 1e-40,
            es + ((K + 2) * F + last) * as_ + 1e-40]


# ---- the scan ---------------------------------------------------------------------------------------------------------------
def scan_case(b, t, d, n, dtype, gated, how, seed=0):
    """Operands: x, dt, bc, a, skip, h0, dy, dhT, z, keep."""
    rng = np.random.default_rng(seed)
    keep = flags(rng, b, t, how)
    a = -rng.uniform(0.05, 4.0, size=(d, n))
    a[0, 0] = 0.0
    a[-1, -1] = 0.01                                           # a state that grows
    made = [(poison(rng, rng.normal(size=(b * t, d)), keep), dtype), (poison(rng, rng.normal(size=(b * t, d)) - 1.5, keep), dtype),
            (poison(rng, rng.normal(size=(b * t, 2 * n)), keep), dtype), (a, "f32"), (rng.normal(size=d), "f32"), (rng.normal(size=(b, d, n)), "f32"),
            (poison(rng, rng.normal(size=(b * t, d)), keep), dtype), (rng.normal(size=(b, d, n)), "f32"),
            (poison(rng, rng.normal(size=(b * t, d)), keep), dtype) if gated else None, (keep, "i8") if keep is not None else None]
    both = [None if m is None else tensor(*m) + (m[1],) for m in made]
    return [None if m is None else (m[0], m[2]) for m in both], [None if m is None else m[1] for m in both]


def scan_bounds(x, dt, bc, a, skip, h0, dy, dhT, z, keep, dtype):
    """Bounds of (y, hT) and of (dx, ddt, dbc, da, dskip, dh0, dz).

    softplus: an exponential, a sum, a logarithm, a quotient: (2 |dt| + 20) F of itself.  A gate e = exp(s a): its argument by 4 F and that, the
    sum of many where rows are joined to chunks: T F more, and 2 F.  A state is off by what the one before is, decayed, by the gate's share and by
    three roundings; a derivative likewise.  Sums of n terms: n F of the terms' sizes."""
    B, D, N = h0.shape
    T = x.shape[0] // B
    fine = lambda v: np.where(np.isfinite(v), v, 0.0)
    x, dt, dy = (fine(v).reshape(B, T, D) for v in (x, dt, dy))
    bc = fine(bc).reshape(B, T, 2, N)
    zz = None if z is None else fine(z).reshape(B, T, D)
    keep = np.ones((B, T)) if keep is None else keep.reshape(B, T)
    last = U[dtype] if dtype == "bf16" else F
    y, dx, ddt, dz = (np.zeros((B, T, D)) for _ in range(4))
    dbc, da, dskip = np.zeros((B, T, 2, N)), np.zeros((D, N)), np.zeros(D)
    ehT, edh0 = np.zeros((B, D, N)), np.zeros((B, D, N))
    s = L.softplus(dt)
    es = (2 * np.abs(dt) + 20) * F
    sig = sigmoid(dt)
    for i in range(B):
        h, eh, kept = h0[i].copy(), np.zeros((D, N)), {}
        rows = [t for t in range(T) if keep[i, t] != 0]
        for t in rows:
            if keep[i, t] == 2:
                h, eh = np.zeros((D, N)), np.zeros((D, N))
            st, ss = s[i, t][:, None], es[i, t][:, None]
            e = np.exp(st * a)
            re = np.abs(st * a) * ((4 + T) * F + ss) + 3 * F
            u = (s[i, t] * x[i, t])[:, None] * bc[i, t, 0]
            kept[t] = h, eh, e, re
            ah = e * np.abs(h) + np.abs(u)
            eh = e * eh + e * np.abs(h) * re + np.abs(u) * (ss + 3 * F) + 2 * F * ah
            h = e * h + u
            C = np.abs(bc[i, t, 1])
            ar, er = np.abs(h) @ C + np.abs(skip * x[i, t]), eh @ C
            er = er + (N + 4) * F * ar
            r = h @ bc[i, t, 1] + skip * x[i, t]
            kept[t] += (r, er)
            if zz is None:
                y[i, t] = er + last * np.abs(r)
            else:
                zt = zz[i, t]
                gate = np.abs(zt) * sigmoid(zt)
                y[i, t] = gate * (er + np.abs(r) * ((2 * np.abs(zt) + 10) * F + last))
        ehT[i] = eh
        G, eG = np.abs(dhT[i]), np.zeros((D, N))
        for t in reversed(rows):
            h, eh, e, re, r, er = kept[t]
            Bt, Ct = np.abs(bc[i, t])
            st, ss, xt = s[i, t], es[i, t], np.abs(x[i, t])
            du, rdu = np.abs(dy[i, t]), np.zeros(D)
            if zz is not None:
                zt = zz[i, t]
                sg = sigmoid(zt)
                slope = sg + np.abs(zt) * sg * (1 - sg)
                dz[i, t] = du * slope * (er + np.abs(r) * ((4 * np.abs(zt) + 20) * F + last))
                du, rdu = du * np.abs(zt) * sg, (2 * np.abs(zt) + 10) * F
            eG = eG + (du * (rdu + 2 * F))[:, None] * Ct
            G = G + du[:, None] * Ct
            eG = eG + F * G
            dec = G * e * np.abs(h)
            edec = (eG * np.abs(h) + G * eh + G * np.abs(h) * (re + 3 * F)) * e
            gb, egb = G @ Bt, eG @ Bt + (N + 3) * F * (G @ Bt)
            ga, ega = (dec * np.abs(a)).sum(1), (edec * np.abs(a)).sum(1) + (N + 3) * F * (dec * np.abs(a)).sum(1)
            dx[i, t] = du * np.abs(skip) * (rdu + 3 * F + last) + st * (egb + gb * (ss + 3 * F + last))
            ddt[i, t] = sig[i, t] * (ega + xt * egb + (ga + xt * gb) * ((2 * np.abs(dt[i, t]) + 12) * F + last))
            sx = st * xt
            dbc[i, t, 0] = sx @ eG + (sx * (ss + (D + 4) * F + last)) @ G
            hn = e * np.abs(h) + sx[:, None] * Bt
            ehn = e * eh + e * np.abs(h) * (re + F) + (sx * (ss + 4 * F))[:, None] * Bt
            dbc[i, t, 1] = du @ ehn + (du * (rdu + (D + 4) * F + last)) @ hn
            depth = B * T * F
            da += edec * st[:, None] + dec * (st * (ss + depth))[:, None] + 4 * F * dec * st[:, None]
            dskip += du * xt * (rdu + 3 * F + depth)
            eG = np.where(keep[i, t] == 2, 0.0, eG * e + G * e * (re + 2 * F))
            G = np.where(keep[i, t] == 2, 0.0, G * e)
        edh0[i] = eG
    tiny = 1e-40
    # states of a few of the joined rows' products below f32
    return [y.reshape(B * T, D) + tiny, ehT + F * 1e-30 + tiny], [dx.reshape(B * T, D) + tiny, ddt.reshape(B * T, D) + tiny, dbc.reshape(B * T, 2 * N) + tiny, da + tiny, dskip + tiny,
                                                                  edh0 + tiny] + ([] if zz is None else [dz.reshape(B * T, D) + tiny])


# ---- the loss ---------------------------------------------------------------------------------------------------------------
def loss_case(m, v, k, dtype, seed=0, std=2.0):
    """Operands: x, w, tok, dlp, dlse.  A tenth of the rows without a target (on either side of the vocabulary), a tenth that take no part."""
    rng = np.random.default_rng(seed)
    tok = rng.integers(0, v, size=m)
    tok = np.where(rng.uniform(size=m) < 0.1, rng.choice([-1, v, -2 ** 31, 2 ** 31 - 1], size=m), tok)
    dlp, dlse = -rng.uniform(0, 2, size=m), rng.normal(size=m)
    out = rng.uniform(size=m) < 0.1
    dlp, dlse = np.where(out, 0.0, dlp), np.where(out, 0.0, dlse)
    made = [(rng.normal(size=(m, k)), dtype), (rng.normal(size=(v, k)) * std / np.sqrt(k), dtype), (tok, "i32"), (dlp, "f32"), (dlse, "f32")]
    both = [tensor(a, dt) + (dt,) for a, dt in made]
    return [(t, dt) for t, _, dt in both], [a for _, a, _ in both]


def loss_bounds(x, w, tok, lse, dlp, dlse, dtype):
    """Bounds of (lp, lse) and (dx, dw).  A logit: 2 F of its terms' sizes for each of the K sums, which the matrix pipes may cut off.  A sum of exponentials:
    each by its argument and 2 F, their sums by V F / 16 + 60 F.  dl: the exponential, two roundings, one to x's type; sums of V and M terms as a logit's."""
    K, V, M = x.shape[1], w.shape[0], x.shape[0]
    size = np.abs(x) @ np.abs(w).T
    el = 2 * (K + 2) * F * size
    logits = x @ w.T
    p = np.exp(logits - lse[:, None])
    far = np.abs(logits - lse[:, None])
    elog = (p * (el + far * 3 * F)).sum(1) + (V / 16 + 60) * F + 4 * F * (np.abs(lse) + np.log(V) + 1)
    hit = np.take_along_axis(el, np.where((tok >= 0) & (tok < V), tok, 0).astype(np.int64)[:, None], 1)[:, 0]
    dx, dw, dl = L.dense_logprobs_grad(x, w, tok, lse, dlp, dlse, parts=True)
    one = np.where((tok >= 0) & (tok < V), dlp, 0.0)
    c = np.abs(dlse) + np.abs(one)
    # lse itself is the forward operator's, off by elog and a rounding
    edl = c[:, None] * p * (el + elog[:, None] + far * 3 * F + 6 * F) + (F + (U["bf16"] if dtype == "bf16" else 0)) * (c[:, None] * p + np.abs(dl))
    last = U[dtype] if dtype == "bf16" else F
    ex = edl @ np.abs(w) + 2 * (V + 80) * F * ((np.abs(dl) + edl) @ np.abs(w)) + last * np.abs(dx)
    takes = (one != 0) | (dlse != 0)
    ax = np.where(takes[:, None], np.abs(x), 0.0)
    ew = edl.T @ ax + 2 * (M + 80) * F * ((np.abs(dl) + edl).T @ ax) + last * np.abs(dw)
    return [hit + elog + 2 * F * (np.abs(lse) + 50), elog], [ex + 1e-40, ew + 1e-40]
