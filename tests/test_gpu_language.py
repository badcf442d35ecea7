"""The operators of a recurrent language model on the GPU against their definitions in 64 bits."""
import numpy as np
import pytest

from oracle import language as L
from language_helpers import Call, GATE, U, scan_bounds, scan_grad_bounds, soft_bounds, tensor, within

pytestmark = pytest.mark.gpu

BF16, F32 = U["bf16"], U["f32"]


# ---- rms_norm_q8 ---------------------------------------------------------------------------------------------------------
def norm_case(m, d, dtype, residual, g_dtype, seed=0, x=None):
    rng = np.random.default_rng(seed)
    tx, x = tensor(rng.normal(size=(m, d)) * 2 if x is None else x, dtype)
    tg, g = tensor(rng.uniform(0.5, 1.5, size=d), g_dtype)
    operands, results = [(tx, dtype), (tg, g_dtype)], [("i8", (m, d)), ("f32", (m,))]
    r = None
    if residual:
        tr, r = tensor(rng.normal(size=(m, d)), dtype)
        operands.insert(1, (tr, dtype))
        results.append((dtype, (m, d)))
    call = Call("rms_norm_q8", operands, results, params=(len(operands) - 1,), eps=1e-5)
    return call, x, r, g


def check_norm(out, x, r, g, dtype, what):
    y = x
    if r is not None:
        y = out[2]
        # x + r is rounded to f32 and then to its type
        within(y, x + r, (F32 + (BF16 if dtype == "bf16" else 0)) * np.abs(x + r), what + " y")
    D = x.shape[1]
    q, s, _ = L.rms_norm_q8(y, None, g, float(np.float32(1e-5)), dtype)
    # half of the sum's D roundings, the mean's, eps', the root's, the scale's four
    within(out[1], s, np.where(np.isfinite(s), np.abs(s), 0) * (D / 2 + 10) * F32 + 1e-44, what + " s")
    # four roundings of a number of at most 127 before it is rounded to a whole one
    ok = s > 0
    n = (y[ok] * g) * (127 / np.abs(y[ok] * g).max(axis=1, keepdims=True))
    within(out[0][ok], n, 0.5 + 127 * 5 * F32, what + " q")
    assert not out[0][~ok].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,d", [(1, 1), (3, 2), (2, 63), (5, 64), (7, 65), (1, 515), (65, 1024), (3, 2047), (300, 520), (9, 4096), (2, 4099), (4, 8192), (3, 16384), (2, 20001), (1, 40000)])
def test_norm(m, d, dtype):
    for residual in (False, True):
        for g_dtype in {"f32", dtype}:
            what = f"norm {m}x{d} {dtype} r={residual} g={g_dtype}"
            print(what, flush=True)
            call, x, r, g = norm_case(m, d, dtype, residual, g_dtype, seed=m + d)
            check_norm(call.run().numbers(), x, r, g, dtype, what)


@pytest.mark.parametrize("d", [40, 515, 2048])
def test_norm_of_odd_rows(d):
    rng = np.random.default_rng(d)
    x = rng.normal(size=(9, d))
    x[0] = 0.0                                    # nothing
    x[1, d // 2] = np.inf
    x[2, d - 1] = np.nan
    x[3] *= 1e-30                                 # its squares are below f32
    x[4] *= 1e-37
    x[5] *= 1e25                                  # its squares are past f32: no scale
    x[6] *= 1e15
    x[7] = 0.0
    x[7, 0] = -3.0                                # one value
    x[8, 1] = -np.inf
    call, x, _, g = norm_case(9, d, "f32", False, "f32", x=x)
    out = call.run().numbers()
    assert np.isnan(out[1][[1, 2, 5, 8]]).all() and not out[0][[1, 2, 5, 8]].any()
    assert out[1][0] == 0 and not out[0][0].any()
    keep = [3, 6, 7]
    check_norm([t[keep] for t in out], x[keep], None, g, "f32", "norm of odd rows")
    assert abs(out[0][4]).max() == 127 and out[0][7, 0] == -127


@pytest.mark.parametrize("d", [1, 40, 515, 4096, 40000])
def test_norm_with_a_gain_that_is_no_number(d):
    """No row has a scale then, a row of zeros neither: 0 times NaN or infinity is NaN."""
    for gain in (np.nan, -np.nan, np.inf):
        for residual in (False, True):
            call, x, r, g = norm_case(4, d, "f32", residual, "f32", seed=d, x=np.concatenate([np.zeros((1, d)), np.random.default_rng(d).normal(size=(3, d))]))
            call.operands[-1][d // 2] = gain       # the gain
            if residual:
                call.operands[1][0] = 0.0
            out = call.run().numbers()
            assert np.isnan(out[1]).all() and not out[0].any(), (d, gain, residual)


@pytest.mark.parametrize("d,past", [(515, False), (4096, False), (4096, True), (40000, False), (40000, True)])
def test_norm_of_gains_near_the_end_of_f32(d, past):
    """A row's scale is within f32 where 127 steps of it are not; a scale past f32 is none."""
    x = np.zeros((2, d))
    x[0, d // 3] = -1.0
    x[1] = np.random.default_rng(d).normal(size=d)
    x[1, d // 3] = 0.5
    call, x, _, g = norm_case(2, d, "f32", False, "f32", x=x)
    call.operands[-1][d // 3] = 3.4e38 if past else 2e37
    g[d // 3] = float(call.operands[-1][d // 3])
    out = call.run().numbers()
    ref = L.rms_norm_q8(x, None, g, float(np.float32(1e-5)), "f32")[1]
    assert ref[0] * 127 > np.finfo(np.float32).max
    if past and ref[0] > np.finfo(np.float32).max:
        assert np.isnan(out[1][0]) and not out[0][0].any()
        out, x = [t[1:] for t in out], x[1:]
    check_norm(out, x, None, g, "f32", f"gains of {g.max():.1e}")


# ---- dense_q8 ------------------------------------------------------------------------------------------------------------
def q8_case(m, n, k, out, bias, w_param=True, seed=0, edge=False):
    rng = np.random.default_rng(seed)
    tx, x = tensor(np.full((m, k), -128) if edge else rng.integers(-128, 128, size=(m, k)), "i8")
    tw, w = tensor(np.full((n, k), -128) if edge else rng.integers(-128, 128, size=(n, k)), "i8")
    tsx, sx = tensor(rng.uniform(0.005, 0.05, size=m), "f32")
    tsw, sw = tensor(rng.uniform(1e-4, 1e-3, size=n), "f32")
    operands, b = [(tx, "i8"), (tsx, "f32"), (tw, "i8"), (tsw, "f32")], None
    if bias:
        tb, b = tensor(rng.normal(size=n), "f32")
        operands.append((tb, "f32"))
    return Call("dense_q8", operands, [(out, (m, n))], params=(2, 3, 4) if w_param else (), out_dtype=out), (x, sx, w, sw, b)


def check_q8(got, data, out, what):
    ref, bare = L.dense_q8(*data), np.abs(L.dense_q8(*data[:4]))
    # the sum's conversion, two factors, the bias' addition; the result's rounding
    within(got, ref, 3.01 * F32 * bare + (1.01 * F32 + (1.01 * BF16 if out == "bf16" else 0)) * (np.abs(ref) + 3 * F32 * bare), what)


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 65, 16), (3, 64, 17), (2, 1000, 127), (16, 33, 128), (17, 100, 129), (33, 96, 784), (8, 512, 1024), (64, 200, 1000),
                                   (100, 100, 100), (130, 257, 64), (257, 130, 256), (1, 4096, 4096), (5, 1000, 2500), (300, 520, 384), (1000, 1000, 784),
                                   (256, 256, 128), (512, 768, 640), (700, 900, 1100)])
def test_dense_q8(m, n, k):
    for out, bias, param in (("f32", True, True), ("bf16", False, True), ("f32", False, False), ("bf16", True, False)):
        what = f"dense_q8 {m}x{n}x{k} {out} bias={bias} param={param}"
        print(what, flush=True)
        call, data = q8_case(m, n, k, out, bias, param, seed=m + n + k)
        check_q8(call.run().numbers()[0], data, out, what)


def test_dense_q8_largest_sum():
    for m, n in ((3, 70), (300, 300)):
        call, data = q8_case(m, n, 131071, "f32", False, edge=True)
        check_q8(call.run().numbers()[0], data, "f32", "largest sum")


def test_dense_q8_scale_that_is_no_number():
    import torch
    call, data = q8_case(20, 70, 200, "f32", True)
    call.operands[1][7] = float("nan")
    got = call.run().numbers()[0]
    assert np.isnan(got[7]).all() and np.isfinite(np.delete(got, 7, 0)).all()


# ---- linear_scan ---------------------------------------------------------------------------------------------------------
def scan_keep(rng, b, t, how):
    if how is None:
        return None
    if how == "none":                             # nothing but padding
        return np.zeros(b * t)
    keep = np.ones((b, t))
    keep[rng.uniform(size=(b, t)) < 0.05] = 2
    keep[rng.uniform(size=(b, t)) < 0.1] = 0
    for i in range(b):
        keep[i, t - int(rng.integers(0, t + 1)):] = 0
    if how == "other":                            # any other value is a token
        keep[keep == 1] = np.where(rng.uniform(size=int((keep == 1).sum())) < 0.5, -1, 7)
    return keep.reshape(-1)


def scan_inputs(b, t, d, dtype, how, seed=0):
    rng = np.random.default_rng(seed)
    z = np.clip(rng.normal(size=(b * t, 2 * d)), -5, 5)
    z[:, :d] += 2.0
    keep = scan_keep(rng, b, t, how)
    tz, z = tensor(z, dtype)
    th, h0 = tensor(rng.normal(size=(b, d)), "f32")
    if keep is not None and (keep == 0).any():    # what stands in padding is not looked at
        import torch
        rows = torch.from_numpy(keep == 0).to(tz.device)
        tz[rows] = float("nan")
        z = np.where(keep[:, None] == 0, 0.0, z)
    operands = [(tz, dtype), (th, "f32")]
    tk = None if keep is None else tensor(keep, "i8")[0]
    return rng, z, h0, keep, operands, tk


def scan_case(b, t, d, dtype, how, seed=0, in_place=None):
    _, z, h0, keep, operands, tk = scan_inputs(b, t, d, dtype, how, seed)
    if tk is not None:
        operands = operands + [(tk, "i8")]
    return Call("linear_scan", operands, [(dtype, (b * t, d)), ("f32", (b, d))], in_place=in_place), z, h0, keep


def check_scan(out, z, h0, keep, dtype, what):
    after, _, last = scan_bounds(z, h0, keep)
    h, hT = L.linear_scan(z, h0, keep)
    after = after.reshape(h.shape)
    within(out[0], h, after + (BF16 * (np.abs(h) + after) if dtype == "bf16" else 0), what + " h")
    within(out[1], hT, last, what + " hT")


def grad_case(b, t, d, dtype, how, seed=0):
    rng, z, h0, keep, operands, tk = scan_inputs(b, t, d, dtype, how, seed)
    tdh, dh = tensor(rng.normal(size=(b * t, d)), dtype)
    tdT, dhT = tensor(rng.normal(size=(b, d)), "f32")
    if keep is not None and (keep == 0).any():
        import torch
        tdh[torch.from_numpy(keep == 0).to(tdh.device)] = float("inf")
        dh = np.where(keep[:, None] == 0, 0.0, dh)
    operands = operands + [(tdh, dtype), (tdT, "f32")] + ([(tk, "i8")] if tk is not None else [])
    return Call("linear_scan_grad", operands, [(dtype, (b * t, 2 * d)), ("f32", (b, d))]), z, h0, dh, dhT, keep


def check_grad(out, z, h0, dh, dhT, keep, dtype, what):
    states = L.linear_scan(z, h0, keep, states=True)[2]
    _, before, _ = scan_bounds(z, h0, keep)
    tf, tv, t0 = scan_grad_bounds(z, h0, dh, dhT, keep, states, before)
    dz, dh0 = L.linear_scan_grad(z, h0, dh, dhT, keep)
    tol = np.stack([tf, tv], 2).reshape(dz.shape)
    within(out[0], dz, tol + (BF16 * (np.abs(dz) + tol) if dtype == "bf16" else 0), what + " dz")
    within(out[1], dh0, t0, what + " dh0")


SCANS = [(1, 1, 1), (64, 1, 128), (3, 1, 65), (2, 2, 3), (1, 31, 64), (2, 33, 130), (3, 64, 515), (1, 100, 1024), (5, 129, 66), (2, 513, 63), (1, 1025, 256), (1, 3001, 40),
         (4, 2048, 129), (70, 5, 300), (33, 40, 2048)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,t,d", SCANS)
def test_scan(b, t, d, dtype):
    for how in (None, "some", "other", "none"):
        what = f"scan {b}x{t}x{d} {dtype} keep={how}"
        print(what, flush=True)
        call, z, h0, keep = scan_case(b, t, d, dtype, how, seed=b + t + d)
        check_scan(call.run().numbers(), z, h0, keep, dtype, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,t,d", SCANS)
def test_scan_grad(b, t, d, dtype):
    for how in (None, "some", "none"):
        what = f"scan grad {b}x{t}x{d} {dtype} keep={how}"
        print(what, flush=True)
        case = grad_case(b, t, d, dtype, how, seed=b + t + d)
        check_grad(case[0].run().numbers(), *case[1:], dtype, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,t,d", [(2, 9, 3), (3, 64, 66), (1, 3001, 40), (1, 6000, 130), (8, 300, 1024), (130, 260, 64)])
def test_documents_are_apart(b, t, d, dtype):
    """NaN and infinities of a document, of the state before a first token and behind the last one stay where the definition has them."""
    import torch
    rng, z, h0, keep, operands, tk = scan_inputs(b, t, d, dtype, "some", seed=t)
    keep = keep.reshape(b, t)
    keep[:, 0] = 2
    tk.view(b, t)[:, 0] = 2
    tz, th = operands[0][0], operands[1][0]
    tdh, dh = tensor(rng.normal(size=(b * t, d)), dtype)
    tdT, dhT = tensor(rng.normal(size=(b, d)), "f32")
    dh = np.where(keep.reshape(-1, 1) == 0, 0.0, dh)
    z, dh, tz, tdh = z.reshape(b, t, 2 * d), dh.reshape(b, t, d), tz.view(b, t, 2 * d), tdh.view(b, t, d)
    z[:, 0] = tz[:, 0].double().cpu().numpy()      # was padding or a token, and is a first one now
    dh[:, 0] = tdh[:, 0].double().cpu().numpy()
    if not np.isfinite(z[:, 0]).all():
        z[:, 0] = 0.5
        tz[:, 0] = 0.5
    for i in range(b):
        tokens, firsts = np.flatnonzero(keep[i] == 1), np.flatnonzero(keep[i] == 2)
        for n, t0 in enumerate(rng.choice(tokens, size=min(4, len(tokens)), replace=False)):
            c = int(rng.integers(0, d))
            if n % 2 == 0:
                z[i, t0, [c, d + c][n // 2]] = np.nan
                tz[i, t0, [c, d + c][n // 2]] = float("nan")
            else:
                dh[i, t0, c] = np.nan
                tdh[i, t0, c] = float("nan")
        c = int(rng.integers(0, d))
        dh[i, firsts[-1], c] = np.inf
        tdh[i, firsts[-1], c] = float("inf")
    h0[:, 0], th[:, 0] = np.nan, float("nan")
    dhT[:, d - 1], tdT[:, d - 1] = np.nan, float("nan")
    z, dh, tz, tdh, keep = z.reshape(b * t, 2 * d), dh.reshape(b * t, d), tz.view(b * t, 2 * d), tdh.view(b * t, d), keep.reshape(-1)
    types = [(dtype, (b * t, d)), ("f32", (b, d)), (dtype, (b * t, 2 * d)), ("f32", (b, d))]
    with np.errstate(invalid="ignore"):
        after, before, last = scan_bounds(z, h0, keep)
        states, (h, hT) = L.linear_scan(z, h0, keep, states=True)[2], L.linear_scan(z, h0, keep)
        tf, tv, t0 = scan_grad_bounds(z, h0, dh, dhT, keep, states, before)
        dz, dh0 = L.linear_scan_grad(z, h0, dh, dhT, keep)
    # padding, whose result is zero: the bounds stand for a state it does not show
    after, tol = (np.where(keep[:, None] == 0, 0.0, a.reshape(b * t, -1)) for a in (after, np.stack([tf, tv], 2)))
    out = Call("linear_scan", [(tz, dtype), (th, "f32"), (tk, "i8")], types[:2]).run().numbers()
    within(out[0], h, after + (BF16 * (np.abs(h) + after) if dtype == "bf16" else 0), "h")
    within(out[1], hT, last, "hT")
    out = Call("linear_scan_grad", [(tz, dtype), (th, "f32"), (tdh, dtype), (tdT, "f32"), (tk, "i8")], types[2:]).run().numbers()
    within(out[0], dz, tol + (BF16 * (np.abs(dz) + tol) if dtype == "bf16" else 0), "dz")
    within(out[1], dh0, t0, "dh0")
    assert not out[1].any()                        # nothing goes back past a first token


def test_scan_step_in_place():
    """A decoding step's new state over its old one."""
    for b, d, dtype in ((64, 1024, "f32"), (3, 77, "bf16")):
        call, z, h0, keep = scan_case(b, 1, d, dtype, "some", in_place={1: 1})
        check_scan(call.run().numbers(), z, h0, keep, dtype, "step in place")


def test_the_last_reader_of_a_state_may_write_over_it():
    """Two scans of one token from the same state: the second one's new state over it, the first one's beside it."""
    import torch
    from paper_1810_00952_amd import binding as B
    b, d = 5, 70
    rng = np.random.default_rng(1)
    z = [tensor(rng.normal(size=(b, 2 * d)), "f32") for _ in range(2)]
    th, h0 = tensor(rng.normal(size=(b, d)), "f32")
    g = B.Graph(B.Context())
    zi, hi = [g.input("f32", (b, 2 * d)) for _ in z], g.input("f32", (b, d))
    outs = [g.op("linear_scan", [v, hi], [("f32", (b, d)), ("f32", (b, d))])[1] for v in zi]
    for v in (*outs[0], *outs[1]):
        g.output(v)
    plan = g.plan()
    got = {v: torch.empty((b, d), device="cuda:0") for v in (*outs[0], outs[1][0])}
    bound = {**{v: t.data_ptr() for v, (t, _) in zip(zi, z)}, hi: th.data_ptr(), **{v: t.data_ptr() for v, t in got.items()}, outs[1][1]: th.data_ptr()}
    plan.run(bound, 0, 0, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    results = [[got[outs[0][0]], got[outs[0][1]]], [got[outs[1][0]], th]]
    for (_, zn), res in zip(z, results):
        check_scan([t.double().cpu().numpy() for t in res], zn, h0, None, "f32", "shared state")


def test_scan_steps_continue_a_sequence():
    """T single steps, each on the state of the one before, are the sequence: within the bound of either."""
    b, t, d = 2, 9, 70
    whole, z, h0, _ = scan_case(b, t, d, "f32", None)
    ref = L.linear_scan(z, h0)
    after, _, _ = scan_bounds(z, h0, None)
    state = h0
    for i in range(t):
        tz, _ = tensor(z.reshape(b, t, 2 * d)[:, i], "f32")
        th, _ = tensor(state, "f32")
        h, state = Call("linear_scan", [(tz, "f32"), (th, "f32")], [("f32", (b, d)), ("f32", (b, d))]).run().numbers()
        within(h, ref[0].reshape(b, t, d)[:, i], after[:, i], f"step {i}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,t,d", [(3, 1, 66), (2, 20, 66), (3, 90, 515), (1, 3001, 40), (1, 6000, 130), (8, 300, 1024), (130, 260, 64)])
def test_infinite_states_and_derivatives_stay_infinite(b, t, d, dtype):
    """Gates are above zero, so that an infinite state, and an infinite derivative on its way back, outlasts any number of them; the product of
    the gates of a run, of a tile, of many tiles, is far below f32."""
    for packed in (False, True):
        print(f"{b}x{t}x{d} {dtype} packed={packed}", flush=True)
        rng = np.random.default_rng(t + d)
        z = np.clip(rng.normal(size=(b, t, 2 * d)), -5, 5)
        z[:, :, :d:3] = -60.0                          # a third of the channels: two gates of e^-60 are below f32
        h0, dh, dhT = rng.normal(size=(b, d)), rng.normal(size=(b, t, d)), rng.normal(size=(b, d))
        h0[:, 0], h0[:, d // 2] = np.inf, -np.inf
        dhT[:, 1], dhT[:, d - 1] = np.inf, -np.inf
        keep = np.ones((b, t))
        for i in range(b):                             # and of a token's own candidate or derivative
            z[i, rng.integers(0, t), d + 2] = np.inf
            z[i, rng.integers(0, t), d + 3] = -np.inf
            dh[i, rng.integers(0, t), 4], dh[i, rng.integers(0, t), 6] = np.inf, -np.inf
        if packed:
            keep[:, 40::200] = 2
            keep[:, 7::50] = 0
            z[:, 7::50], dh[:, 7::50] = 0.0, 0.0
        tz, z = tensor(z.reshape(b * t, 2 * d), dtype)
        th, h0 = tensor(h0, "f32")
        tdh, dh = tensor(dh.reshape(b * t, d), dtype)
        tdT, dhT = tensor(dhT, "f32")
        tk, keep = tensor(keep.reshape(-1), "i8")
        last = [(tk, "i8")] if packed else []
        k = keep if packed else None
        got = Call("linear_scan", [(tz, dtype), (th, "f32")] + last, [(dtype, (b * t, d)), ("f32", (b, d))]).run().numbers()
        grad = Call("linear_scan_grad", [(tz, dtype), (th, "f32"), (tdh, dtype), (tdT, "f32")] + last, [(dtype, (b * t, 2 * d)), ("f32", (b, d))]).run().numbers()
        with np.errstate(invalid="ignore"):
            want = L.linear_scan(z, h0, k)
            wgrad = L.linear_scan_grad(z, h0, dh, dhT, k)
        for a, w, name in zip(got + grad, list(want) + list(wgrad), ("h", "hT", "dz", "dh0")):
            assert packed or np.isinf(w).any(), name
            np.testing.assert_array_equal(np.where(np.isfinite(w), 0.0, w), np.where(np.isfinite(a), 0.0, a), err_msg=name)


def test_scan_gates_at_their_ends():
    """Gates of +-infinity and far out: the state is kept or replaced, and nothing is NaN."""
    f = np.array([np.inf, -np.inf, 100.0, -100.0, 88.0, -88.0])
    z = np.stack([f, np.full(6, 3.0)], 1)
    tz, _ = tensor(z, "f32")
    th, _ = tensor([[2.0]], "f32")
    td, _ = tensor(np.ones((6, 1)), "f32")
    h, _ = Call("linear_scan", [(tz, "f32"), (th, "f32")], [("f32", (6, 1)), ("f32", (1, 1))]).run().numbers()
    np.testing.assert_allclose(h[:, 0], [2, 3, 3, 3, 3, 3], rtol=1e-6)
    dz, dh0 = Call("linear_scan_grad", [(tz, "f32"), (th, "f32"), (td, "f32"), (th, "f32")], [("f32", (6, 2)), ("f32", (1, 1))]).run().numbers()
    assert np.isfinite(dz).all() and dh0[0, 0] == 1.0


# ---- token_logprobs --------------------------------------------------------------------------------------------------------
def logits_case(m, v, dtype, masked, seed=0, spread=2.5):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(m, v)) * spread
    if masked:
        x[rng.uniform(size=(m, v)) < 0.3] = -np.inf
        x[0] = -np.inf                             # a row without any token
        if v > 1 and m > 1:
            x[1] = -np.inf
            x[1, v - 1] = 3.0                      # one with a single one
    tx, x = tensor(x, dtype)
    tok = rng.integers(0, v, size=m)
    tok[rng.uniform(size=m) < 0.2] = -1
    if m > 2:
        tok[2] = v                                 # not a column
    tt, _ = tensor(tok, "i32")
    return rng, tx, x, tt, tok


def check_logprobs(out, x, tok, top, what):
    ref = L.token_logprobs(x, tok, top)
    ln_s, ent = soft_bounds(x)

    def tol(lp):                                   # the logit less the maximum is one rounding, less ln S another
        return (ln_s[:, None] + 3 * F32 * np.abs(np.where(np.isfinite(lp), lp, 0)).reshape(len(tok), -1)).reshape(lp.shape)

    within(out[0], ref[0], tol(ref[0]), what + " lp")
    within(out[1], ref[1], ent, what + " ent")
    if top:
        np.testing.assert_array_equal(out[3], ref[3], err_msg=what + " ids")
        within(out[2], ref[2], tol(ref[2]), what + " top_lp")


LOGITS = [(1, 1), (3, 2), (2, 63), (5, 65), (1, 1000), (9, 1023), (4, 4096), (3, 10007), (2, 50001), (1, 65536), (5, 131072), (300, 700), (1100, 40), (2, 262147)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,v", LOGITS)
def test_logprobs(m, v, dtype):
    for masked in (False, True):
        _, tx, x, tt, tok = logits_case(m, v, dtype, masked, seed=m + v)
        for top in sorted({0, 1, min(8, v), min(32, v)}) if m * v < 1 << 17 else (0, min(20, v)):
            what = f"logprobs {m}x{v} {dtype} masked={masked} top={top}"
            print(what, flush=True)
            results = [("f32", (m,)), ("f32", (m,))] + ([("f32", (m, top)), ("i32", (m, top))] if top else [])
            check_logprobs(Call("token_logprobs", [(tx, dtype), (tt, "i32")], results, top=top).run().numbers(), x, tok, top, what)


@pytest.mark.parametrize("m,v", [(2, 700), (3, 9000), (2, 70000), (600, 300)])
def test_alternatives_among_equals(m, v):
    """Few different logits, all of them equal, the largest at the end, signed zeros: ties go to the lowest index."""
    rng = np.random.default_rng(v)
    for name, x in (("two values", rng.integers(0, 2, size=(m, v))), ("all equal", np.zeros((m, v))), ("rising", np.tile(np.arange(v) / 7.0, (m, 1))),
                    ("falling", np.tile(-np.arange(v) / 7.0, (m, 1))), ("zeros", np.where(rng.uniform(size=(m, v)) < 0.5, 0.0, -0.0)), ("few", np.where(np.arange(v) % 97 == 5, 1.0, -np.inf) + np.zeros((m, 1)))):
        print(name, flush=True)
        for dtype in ("f32", "bf16"):
            tx, stored = tensor(np.asarray(x, dtype=np.float64), dtype)
            tt, _ = tensor(np.zeros(m), "i32")
            call = Call("token_logprobs", [(tx, dtype), (tt, "i32")], [("f32", (m,)), ("f32", (m,)), ("f32", (m, 32)), ("i32", (m, 32))], top=32)
            check_logprobs(call.run().numbers(), stored, np.zeros(m, dtype=int), 32, f"{name} {dtype}")


@pytest.mark.parametrize("v", [5, 900, 70001])
def test_logits_that_are_no_numbers(v):
    rng = np.random.default_rng(v)
    x = rng.normal(size=(6, v))
    x[0, v - 1] = np.nan
    x[1, 1] = np.inf
    x[2, 0] = np.nan
    x[2, v - 2] = np.inf
    x[3, :] = np.nan
    x[4, :] = np.inf
    tok = np.array([0, 1, 2, 3, 4, 0])
    tt, _ = tensor(tok, "i32")
    for dtype in ("f32", "bf16"):
        tx, stored = tensor(x, dtype)
        lp, ent, top_lp, ids = Call("token_logprobs", [(tx, dtype), (tt, "i32")], [("f32", (6,)), ("f32", (6,)), ("f32", (6, 3)), ("i32", (6, 3))], top=3).run().numbers()
        assert np.isnan(lp[:5]).all() and np.isnan(ent[:5]).all() and np.isnan(top_lp[:5]).all()
        np.testing.assert_array_equal(ids, L.token_logprobs(stored, tok, 3)[3])
        assert np.isfinite(lp[5]) and np.isfinite(ent[5])
        ts, _ = tensor(np.ones(6), "f32")
        dx, = Call("token_logprobs_grad", [(tx, dtype), (tt, "i32"), (ts, "f32"), (ts, "f32")], [(dtype, (6, v))]).run().numbers()
        assert np.isnan(dx[:5]).all() and np.isfinite(dx[5]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [3, 700, 9000, 70001])
def test_logits_at_the_ends_of_their_type(v, dtype):
    """Masks of the type's lowest number: among other logits their p is 0, a row of nothing else is a uniform distribution; logits further apart
    than f32 reaches."""
    import torch
    low = float(torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min)
    rng = np.random.default_rng(v)
    x = rng.normal(size=(6, v))
    x[0] = low                                     # nothing but masks
    x[1] = np.where(np.arange(v) % 3 == 0, low, -np.inf)
    x[2, ::2] = low                                # some of them
    x[3] = np.where(np.arange(v) % 5 == 1, -low, 0.0)
    x[4] = np.where(np.arange(v) % 5 == 1, -low, low)
    x[5] = -np.inf
    x[5, v - 1] = low                              # one
    tx, x = tensor(x, dtype)
    tok = np.array([v - 1, 0, 1, 1, 1, v - 1])
    tt, _ = tensor(tok, "i32")
    ts, one = tensor(np.ones(6), "f32")
    out = Call("token_logprobs", [(tx, dtype), (tt, "i32")], [("f32", (6,)), ("f32", (6,)), ("f32", (6, 3)), ("i32", (6, 3))], top=3).run().numbers()
    dx, = Call("token_logprobs_grad", [(tx, dtype), (tt, "i32"), (ts, "f32"), (ts, "f32")], [(dtype, (6, v))]).run().numbers()
    lp, ent, top_lp, ids = L.token_logprobs(x, tok, 3)
    ln_s, tol_ent = soft_bounds(x)
    within(out[0], lp, ln_s + 3 * F32 * np.abs(lp), "lp")
    within(out[1], ent, tol_ent, "ent")
    np.testing.assert_array_equal(out[3], ids)
    shown = np.where(top_lp < low, -np.inf, top_lp)       # ln p past f32 is -inf in it
    within(out[2], shown, ln_s[:, None] + 3 * F32 * np.abs(np.where(np.isfinite(shown), shown, 0)), "top_lp")
    ref = L.token_logprobs_grad(x, tok, one, one)
    logs, p, _ = L._softmax(x)
    # |ln p| is at most ln V + 12 where p is not 0 in f32: the bound of a factor of that size on every term
    tol = p * (ln_s + tol_ent + 16 * F32)[:, None] * (2 + 2 * np.log(v) + 12) + 4 * F32 * np.abs(ref)
    within(dx, ref, tol + (BF16 * (np.abs(ref) + tol) if dtype == "bf16" else 0), "dx")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,v", LOGITS)
def test_logprobs_grad(m, v, dtype):
    for masked in (False, True):
        what = f"logprobs grad {m}x{v} {dtype} masked={masked}"
        print(what, flush=True)
        rng, tx, x, tt, tok = logits_case(m, v, dtype, masked, seed=m + v)
        tp, dlp = tensor(rng.normal(size=m), "f32")
        te, dent = tensor(rng.normal(size=m), "f32")
        if m > 2:
            tp[2] = float("nan")                   # without a target it is not looked at
        dx, = Call("token_logprobs_grad", [(tx, dtype), (tt, "i32"), (tp, "f32"), (te, "f32")], [(dtype, (m, v))]).run().numbers()
        ref = L.token_logprobs_grad(x, tok, dlp, dent)
        logs, p, ent = L._softmax(x)
        ln_s, tol_ent = soft_bounds(x)
        far = np.where(p > 0, np.abs(np.where(np.isfinite(logs), logs, 0)), 0.0)
        part = np.abs(dlp)[:, None] + np.abs(dent)[:, None] * (far + ent[:, None])
        tol = p * part * (ln_s[:, None] + (4 * far + 12) * F32) + np.abs(dent)[:, None] * p * (tol_ent + ln_s)[:, None] + 4 * F32 * (np.abs(ref) + p * part) + 1e-37 * (1 + part)
        within(dx, ref, tol + (BF16 * (np.abs(ref) + tol) if dtype == "bf16" else 0), what)


# ---- streams, graphs ---------------------------------------------------------------------------------------------------------
def some_calls():
    rng, tx, x, tt, tok = logits_case(7, 5003, "bf16", True)
    tp, _ = tensor(rng.normal(size=7), "f32")
    yield norm_case(33, 515, "bf16", True, "f32")[0]
    yield q8_case(40, 130, 515, "bf16", True, False)[0]
    yield q8_case(3, 130, 512, "f32", False, True)[0]
    yield scan_case(2, 300, 130, "bf16", "some")[0]
    yield scan_case(1, 4000, 64, "f32", None)[0]
    yield grad_case(2, 300, 130, "bf16", "some")[0]
    yield grad_case(1, 4000, 64, "f32", None)[0]
    yield Call("token_logprobs", [(tx, "bf16"), (tt, "i32")], [("f32", (7,)), ("f32", (7,)), ("f32", (7, 5)), ("i32", (7, 5))], top=5)
    yield Call("token_logprobs_grad", [(tx, "bf16"), (tt, "i32"), (tp, "f32"), (tp, "f32")], [("bf16", (7, 5003))])


def test_other_streams_graphs_and_the_same_bits_twice():
    import torch
    for call in some_calls():
        want = call.run().numbers()
        side = torch.cuda.Stream()
        for t in call.results:
            t.view(torch.uint8).fill_(0x5a)
        torch.cuda.synchronize()
        got = call.run(side).numbers()
        for a, b in zip(got, want):
            np.testing.assert_array_equal(a, b)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call.run()
        for _ in range(3):                        # replays between eager work on the same memory
            for t in call.results:
                t.view(torch.uint8).fill_(0x5a)
            call.workspace[:call.workspace_bytes].fill_(0xa5)
            graph.replay()
            for a, b in zip(call.numbers(), want):
                np.testing.assert_array_equal(a, b)
            for a, b in zip(call.run().numbers(), want):
                np.testing.assert_array_equal(a, b)


# ---- every form, operators together -------------------------------------------------------------------------------------------
@pytest.mark.parametrize("m,n,k", [(600, 2000, 200), (1500, 1500, 100), (2100, 2050, 144), (2048, 2304, 256), (9, 17, 5000), (40, 5000, 300), (70, 40, 3000)])
def test_dense_q8_forms(m, n, k):
    """Grids past the CUs, for each of the tiles, with ragged edges."""
    for out, bias in (("bf16", True), ("f32", False)):
        call, data = q8_case(m, n, k, out, bias, seed=m)
        check_q8(call.run().numbers()[0], data, out, f"dense_q8 {m}x{n}x{k} {out}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,t,d", [(8, 300, 1024), (6, 700, 1111), (40, 150, 515), (130, 260, 64)])
def test_scan_of_many_tiles(b, t, d, dtype):
    """Workgroups that walk over the tiles of their channels."""
    for how in (None, "some"):
        what = f"scan {b}x{t}x{d} {dtype} keep={how}"
        print(what, flush=True)
        call, z, h0, keep = scan_case(b, t, d, dtype, how, seed=t)
        check_scan(call.run().numbers(), z, h0, keep, dtype, what)
        case = grad_case(b, t, d, dtype, how, seed=t)
        check_grad(case[0].run().numbers(), *case[1:], dtype, what)


@pytest.mark.parametrize("b,t,d,dtype", [(8, 700, 1024, "bf16"), (40, 600, 515, "f32"), (9, 1300, 515, "bf16"), (5, 777, 515, "f32"), (1, 3001, 130, "bf16")])
def test_scan_of_long_documents(b, t, d, dtype):
    """Documents of some hundred tokens: waves of tokens alone beside ones with first tokens, with padding and with rows past the end, in the
    workgroups that walk (the first three) and in tiles of their own; one sequence of nothing but tokens; a document that holds NaN."""
    rng, z, h0, _, operands, _ = scan_inputs(b, t, d, dtype, None, seed=t)
    keep = np.ones((b, t))
    for i in range(1 if b > 1 else 0, b):
        keep[i, rng.choice(np.arange(1, t), size=max(1, t // 350), replace=False)] = 2
        keep[i, t - int(rng.integers(0, t // 3)):] = 0
    tdh, dh = tensor(rng.normal(size=(b * t, d)), dtype)
    tdT, dhT = tensor(rng.normal(size=(b, d)), "f32")
    z, dh, tz = z.reshape(b, t, 2 * d), dh.reshape(b, t, d), operands[0][0].view(b, t, 2 * d)
    at = int(np.flatnonzero(keep[b - 1] == 2)[0]) - 1      # the last token of a first document
    z[b - 1, at, d + 1], tz[b - 1, at, d + 1] = np.nan, float("nan")
    dh[keep == 0] = 0.0                                    # padding is not looked at
    z[keep == 0] = 0.0
    import torch
    tz[torch.from_numpy(keep == 0).to(tz.device)] = float("nan")
    z, dh, keep = z.reshape(b * t, 2 * d), dh.reshape(b * t, d), keep.reshape(-1)
    last = [(tensor(keep, "i8")[0], "i8")]
    with np.errstate(invalid="ignore"):
        after, before, end = scan_bounds(z, h0, keep)
        (h, hT), states = L.linear_scan(z, h0, keep), L.linear_scan(z, h0, keep, states=True)[2]
        tf, tv, t0 = scan_grad_bounds(z, h0, dh, dhT, keep, states, before)
        dz, dh0 = L.linear_scan_grad(z, h0, dh, dhT, keep)
    after, tol = (np.where(keep[:, None] == 0, 0.0, a.reshape(b * t, -1)) for a in (after, np.stack([tf, tv], 2)))
    out = Call("linear_scan", operands + last, [(dtype, (b * t, d)), ("f32", (b, d))]).run().numbers()
    within(out[0], h, after + (BF16 * (np.abs(h) + after) if dtype == "bf16" else 0), "h")
    within(out[1], hT, end, "hT")
    out = Call("linear_scan_grad", operands + [(tdh, dtype), (tdT, "f32")] + last, [(dtype, (b * t, 2 * d)), ("f32", (b, d))]).run().numbers()
    within(out[0], dz, tol + (BF16 * (np.abs(dz) + tol) if dtype == "bf16" else 0), "dz")
    within(out[1], dh0, t0, "dh0")


def session_of(build):
    """A graph's plan on torch tensors: build(graph) -> ({id: tensor}, {id: (dtype, shape)} of results)."""
    import torch
    from language_helpers import torch_type
    from paper_1810_00952_amd import binding as B
    g = B.Graph(B.Context())
    ins, outs = build(g)
    for v in outs:
        g.output(v)
    plan = g.plan()
    got = {v: torch.full(sh, 7, dtype=torch_type(dt), device="cuda:0") for v, (dt, sh) in outs.items()}
    ws = torch.full((max(256, plan.workspace_bytes()),), 0xa5, dtype=torch.uint8, device="cuda:0")
    plan.bind({v: t.data_ptr() for v, t in {**ins, **got}.items()}, ws.data_ptr(), ws.numel()).run(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return plan, [t.cpu() for t in got.values()]


@pytest.mark.parametrize("b,t,d,how", [(8, 300, 1024, None), (8, 300, 1024, "some"), (1, 2000, 130, "some"), (3, 20, 70, None), (40, 200, 515, None)])
def test_scan_gradient_takes_states_from_the_forward_pass(b, t, d, how):
    """In one plan with its forward pass the gradient is the same to the bit, and launches no pass for the states."""
    import torch
    dtype = "bf16"
    rng, z, h0, keep, operands, tk = scan_inputs(b, t, d, dtype, how, seed=5)
    tdh, _ = tensor(rng.normal(size=(b * t, d)), dtype)
    tdT, _ = tensor(rng.normal(size=(b, d)), "f32")
    last = [(tk, "i8")] if tk is not None else []
    dz, dh0 = Call("linear_scan_grad", operands + [(tdh, dtype), (tdT, "f32")] + last, [(dtype, (b * t, 2 * d)), ("f32", (b, d))]).run().results
    h, hT = Call("linear_scan", operands + last, [(dtype, (b * t, d)), ("f32", (b, d))]).run().results

    def build(g):
        ids = {k: g.input(dt, x.shape) for k, (x, dt) in dict(z=operands[0], h0=operands[1], dh=(tdh, dtype), dT=(tdT, "f32"), **({"keep": last[0]} if last else {})).items()}
        tail = [ids["keep"]] if last else []
        types = [(dtype, (b * t, d)), ("f32", (b, d)), (dtype, (b * t, 2 * d)), ("f32", (b, d))]
        _, a = g.op("linear_scan", [ids["z"], ids["h0"]] + tail, types[:2])
        _, c = g.op("linear_scan_grad", [ids["z"], ids["h0"], ids["dh"], ids["dT"]] + tail, types[2:])
        tensors = dict(z=operands[0][0], h0=operands[1][0], dh=tdh, dT=tdT, keep=tk)
        return {v: tensors[k] for k, v in ids.items()}, dict(zip(list(a) + list(c), types))

    plan, got = session_of(build)
    assert [s["kernel"] for s in plan.describe()["steps"]] == ["linear_scan", "linear_scan_grad"]
    for x, y in zip(got, (h, hT, dz, dh0)):
        assert torch.equal(x, y.cpu())


@pytest.mark.parametrize("m,v", [(5, 700), (3, 70000), (300, 5003)])
def test_logprobs_and_gradient_share_a_launch(m, v):
    """The pair gives the bits of the two calls alone; a gradient that reads the forward result comes behind it."""
    import torch
    dtype = "bf16"
    rng, tx, x, tt, tok = logits_case(m, v, dtype, True, seed=v)
    tp, _ = tensor(rng.normal(size=m), "f32")
    top = 6
    types = [("f32", (m,)), ("f32", (m,)), ("f32", (m, top)), ("i32", (m, top)), (dtype, (m, v))]
    alone = Call("token_logprobs", [(tx, dtype), (tt, "i32")], types[:4], top=top).run().results + Call(
        "token_logprobs_grad", [(tx, dtype), (tt, "i32"), (tp, "f32"), (tp, "f32")], types[4:]).run().results

    def build(g, own=False):
        ix, it, ip = g.input(dtype, (m, v)), g.input("i32", (m,)), g.input("f32", (m,))
        _, a = g.op("token_logprobs", [ix, it], types[:4], top=top)
        _, c = g.op("token_logprobs_grad", [ix, it, a[1] if own else ip, ip], types[4:])
        return {ix: tx, it: tt, ip: tp}, dict(zip(list(a) + list(c), types))

    plan, got = session_of(build)
    assert "token_logprobs_grad" in plan.describe()["steps"][0]["kernel"]
    for a, b in zip(got, alone):
        np.testing.assert_array_equal(a.double().numpy(), b.double().cpu().numpy())
    plan, got = session_of(lambda g: build(g, True))         # dlp is the entropy
    assert [s["kernel"] for s in plan.describe()["steps"]] == ["token_logprobs", "token_logprobs_grad"]
    want = Call("token_logprobs_grad", [(tx, dtype), (tt, "i32"), (alone[1], "f32"), (tp, "f32")], types[4:]).run().results[0]
    np.testing.assert_array_equal(got[4].double().numpy(), want.double().cpu().numpy())


@pytest.mark.parametrize("m,v,k", [(5, 700, 64), (3, 70000, 40), (300, 5003, 128)])
def test_values_between_a_loss_and_its_reader_share_the_workspace(m, v, k):
    """Logits, loss and gradient that nobody else sees live in one workspace: the results are those of a plan whose every value leaves it."""
    import torch
    rng = np.random.default_rng(v)
    tensors = dict(q=(rng.integers(-127, 128, size=(m, k)), "i8"), s=(rng.uniform(0.01, 0.03, size=m), "f32"), w=(rng.integers(-127, 128, size=(v, k)), "i8"),
                   sw=(rng.uniform(0.01, 0.02, size=v), "f32"), tok=(rng.integers(-1, v, size=m), "i32"), dlp=(rng.normal(size=m), "f32"), dent=(rng.normal(size=m), "f32"))
    tensors = {n: (tensor(a, dt)[0], dt) for n, (a, dt) in tensors.items()}
    row, wide, tops = ("f32", (m,)), ("bf16", (m, v)), [("f32", (m, 3)), ("i32", (m, 3))]

    def build(everything):
        def f(g):
            ids = {n: g.input(dt, t.shape) for n, (t, dt) in tensors.items()}
            x, = g.op("dense_q8", [ids[n] for n in ("q", "s", "w", "sw")], [wide], out_dtype="bf16")[1]
            made = g.op("token_logprobs", [x, ids["tok"]], [row, row] + tops, top=3)[1]
            dx, = g.op("token_logprobs_grad", [x, ids["tok"], ids["dlp"], ids["dent"]], [wide])[1]
            far, = g.op("neg", [dx], [wide])[1]
            loss, = g.op("neg", [made[0]], [row])[1]
            outs = {far: wide, loss: row}
            return {ids[n]: t for n, (t, _) in tensors.items()}, outs | (dict(zip([x, *made, dx], [wide, row, row, *tops, wide])) if everything else {})
        return f

    plan, got = session_of(build(False))
    assert any("token_logprobs | token_logprobs_grad" in s["kernel"] for s in plan.describe()["steps"])
    full, want = session_of(build(True))
    assert [s["kernel"] for s in full.describe()["steps"]] == [s["kernel"] for s in plan.describe()["steps"]] and plan.workspace_bytes() > full.workspace_bytes()
    for a, b in zip(got, want):
        assert torch.equal(a, b) and bool(torch.isfinite(a.float()).all())


@pytest.mark.parametrize("b,t,d,how", [(8, 300, 1024, "some"), (8, 300, 1024, None), (1, 2000, 130, "some"), (3, 20, 70, None)])
def test_values_between_a_scan_and_its_gradient_share_the_workspace(b, t, d, how):
    """The same of a recurrence whose operands and results are all values of the plan."""
    import torch
    _, z, h0, keep, operands, tk = scan_inputs(b, t, d, "f32", how, seed=9)
    tz = tensor(z, "f32")[0]
    wide, state, rows = ("f32", (b * t, 2 * d)), ("f32", (b, d)), ("f32", (b * t, d))

    def build(everything):
        def f(g):
            iz, ih = g.input(*wide), g.input(*state)
            tail = [g.input("i8", (b * t,))] if tk is not None else []
            z, = g.op("neg", [iz], [wide])[1]
            h0, = g.op("neg", [ih], [state])[1]
            h, hT = g.op("linear_scan", [z, h0] + tail, [rows, state])[1]
            dh, = g.op("neg", [h], [rows])[1]
            dT, = g.op("neg", [hT], [state])[1]
            dz, d0 = g.op("linear_scan_grad", [z, h0, dh, dT] + tail, [wide, state])[1]
            y, = g.op("neg", [dz], [wide])[1]
            y0, = g.op("neg", [d0], [state])[1]
            return {iz: tz, ih: operands[1][0], **{v: tk for v in tail}}, {y: wide, y0: state} | (dict(zip([z, h0, h, hT, dh, dT, dz, d0], [wide, state, rows, state, rows, state, wide, state])) if everything else {})
        return f

    plan, got = session_of(build(False))
    full, want = session_of(build(True))
    assert [s["kernel"] for s in full.describe()["steps"]] == [s["kernel"] for s in plan.describe()["steps"]] and plan.workspace_bytes() > full.workspace_bytes()
    for a, b_ in zip(got, want):
        assert torch.equal(a, b_) and bool(torch.isfinite(a).all())


def check_graph(spec, data, dtype):
    """Every call of a graph against its definition on what the library computed for its operands."""
    import torch
    import oracle as O
    from helpers import assert_close
    from paper_1810_00952_amd import harness
    for op in spec.ops:                             # everything leaves the plan
        for v in op.outputs:
            if v not in spec.outputs:
                spec.output(v)
    s = harness.Session(spec)
    s.load(data)
    s.run()
    torch.cuda.synchronize()
    val = {v: O.widen(harness.to_host(s.raw.get(v, t)), spec.values[v].type.dtype) for v, t in s.tensors.items()}    # raw: before it was packed
    for i, op in enumerate(spec.ops):
        a, out, what = [val[v] for v in op.inputs], [val[v] for v in op.outputs], f"call {i}: {op.kind}"
        if op.kind == "rms_norm_q8":
            check_norm(out, a[0], a[1] if len(a) == 3 else None, a[-1], dtype, what)
        elif op.kind == "dense_q8":
            check_q8(out[0], a + ([None] if len(a) == 4 else []), spec.values[op.outputs[0]].type.dtype, what)
        elif op.kind == "linear_scan":
            check_scan(out, a[0], a[1], a[2] if len(a) > 2 else None, dtype, what)
        elif op.kind == "linear_scan_grad":
            check_grad(out, a[0], a[1], a[2], a[3], a[4] if len(a) > 4 else None, dtype, what)
        elif op.kind == "token_logprobs":
            check_logprobs(out, a[0], a[1].astype(int), op.attrs.get("top", 0), what)
        elif op.kind == "token_logprobs_grad":
            assert_close(out[0], L.token_logprobs_grad(*a), dtype, what)
        else:                                       # the contractions that were there: their own gate
            f = {"dense": O.dense, "dense_grad_x": O.dense_grad_x, "dense_grad_w": O.dense_grad_w}[op.kind]
            assert_close(out[0], f(a[0], a[1]), dtype, what)
    return s


@pytest.mark.parametrize("args", [dict(), dict(batch=3, steps=37, dim=72, vocab=1001, top=0, packed=True), dict(batch=9, steps=1, dim=128), dict(batch=2, steps=70, dim=50, dtype="f32")])
def test_recurrent_lm(args):
    import workloads as W
    check_graph(*W.recurrent_lm(**args), args.get("dtype", "bf16"))


@pytest.mark.parametrize("args", [dict(), dict(batch=2, steps=150, dim=96, vocab=333, packed=True)])
def test_recurrent_lm_train(args):
    import workloads as W
    s = check_graph(*W.recurrent_lm_train(**args), "bf16")
    names = [k["kernel"] for k in s.plan.describe()["steps"]]
    assert sum("linear_scan" in n for n in names) == 2 and "token_logprobs | token_logprobs_grad" in names


def test_generation_continues_a_prompt():
    """A prompt, then its next tokens one at a time on the states it left: the states of the whole, each within the recurrence's bound of
    the steps before (the plan's other operators give the same bits for the same rows)."""
    import torch
    import workloads as W
    from paper_1810_00952_amd import harness
    b, t, d, layers = 3, 12, 64, 2
    spec, data = W.recurrent_lm(b, t, d, layers, 300, 4, "f32")
    whole = harness.Session(spec)
    whole.load(data)
    whole.run()
    step_spec, _ = W.recurrent_lm(b, 1, d, layers, 300, 4, "f32")
    step = harness.Session(step_spec)
    state = {f"h{l}": data[f"h{l}"] for l in range(layers)}
    lps = []
    for i in range(t):
        step.tensors = {}
        step.load({**data, "x": data["x"].reshape(b, t, d)[:, i], "tok": data["tok"].reshape(b, t)[:, i], **state})
        step.alloc()
        step.run()
        torch.cuda.synchronize()
        lps.append(step.output(0).cpu().numpy())
        state = {f"h{l}": step.tensors[step_spec.outputs[4 + l]].cpu().numpy() for l in range(layers)}
    # an 8-bit value next to a border may fall the other way where the state differs in its last bits: a step of 1/127 of a row's largest
    # in one of d summands a layer
    torch.cuda.synchronize()
    want = whole.output(0).cpu().numpy().reshape(b, t)
    assert np.abs(np.stack(lps, 1) - want).max() < layers * 6 * 3.0 / 127
    for l in range(layers):
        ref = whole.tensors[spec.outputs[4 + l]].cpu().numpy()
        assert np.abs(state[f"h{l}"] - ref).max() < layers * 6 * 3.0 / 127


def test_past_32_bits():
    """Rows behind the first 4 GB (2 G elements where a row index is multiplied) of each operator's largest operand."""
    import torch
    dev, f = "cuda:0", torch.float32

    def run(kind, operands, results, params=(), **attrs):
        from language_helpers import plan_of, torch_type
        plan, ids, outs = plan_of(kind, [(dt, t.shape) for t, dt in operands], results, params, **attrs)
        got = [torch.empty(sh, dtype=torch_type(dt), device=dev) for dt, sh in results]
        ws = torch.empty(max(256, plan.workspace_bytes()), dtype=torch.uint8, device=dev)
        plan.run({v: t.data_ptr() for v, t in zip(ids + outs, [t for t, _ in operands] + got)}, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        return got

    torch.manual_seed(3)
    # logits of 40000 x 60001, the last rows
    print("logits", flush=True)
    m, v, n = 40000, 60001, 3
    x = torch.zeros((m, v), dtype=torch.bfloat16, device=dev)
    x[-n:] = torch.randn((n, v), device=dev).bfloat16()
    tok = torch.randint(0, v, (m,), dtype=torch.int32, device=dev)
    one = torch.ones((m,), device=dev)
    lp, ent, top_lp, top_id = run("token_logprobs", [(x, "bf16"), (tok, "i32")], [("f32", (m,)), ("f32", (m,)), ("f32", (m, 2)), ("i32", (m, 2))], top=2)
    tail, tt = x[-n:].double().cpu().numpy(), tok[-n:].cpu().numpy()
    check_logprobs([o[-n:].double().cpu().numpy() for o in (lp, ent, top_lp, top_id)], tail, tt, 2, "last rows")
    assert bool((top_id[:-n] == torch.tensor([0, 1], device=dev)).all())
    dx, = run("token_logprobs_grad", [(x, "bf16"), (tok, "i32"), (one, "f32"), (one, "f32")], [("bf16", (m, v))])
    ref = L.token_logprobs_grad(tail, tt, np.ones(n), np.ones(n))
    within(dx[-n:].double().cpu().numpy(), ref, 2 * BF16 * np.abs(ref) + 1e-9, "last rows' gradient")
    del x, dx
    # a sequence of 300000 x 4096, padding but for its last rows
    print("sequence", flush=True)
    t, d, n = 300000, 4096, 5
    z = torch.zeros((t, 2 * d), dtype=torch.bfloat16, device=dev)
    z[-n:] = torch.randn((n, 2 * d), device=dev).bfloat16()
    keep = torch.zeros((t,), dtype=torch.int8, device=dev)
    keep[-n:] = 1
    h0, dT = torch.randn((1, d), device=dev), torch.randn((1, d), device=dev)
    h, hT = run("linear_scan", [(z, "bf16"), (h0, "f32"), (keep, "i8")], [("bf16", (t, d)), ("f32", (1, d))])
    zt, h0n = z[-n:].double().cpu().numpy(), h0.double().cpu().numpy()
    check_scan([h[-n:].double().cpu().numpy(), hT.double().cpu().numpy()], zt, h0n, None, "bf16", "last rows")
    assert not bool(h[:-n].any())
    dh = torch.zeros((t, d), dtype=torch.bfloat16, device=dev)
    dh[-n:] = torch.randn((n, d), device=dev).bfloat16()
    dz, dh0 = run("linear_scan_grad", [(z, "bf16"), (h0, "f32"), (dh, "bf16"), (dT, "f32"), (keep, "i8")], [("bf16", (t, 2 * d)), ("f32", (1, d))])
    check_grad([dz[-n:].double().cpu().numpy(), dh0.double().cpu().numpy()], zt, h0n, dh[-n:].double().cpu().numpy(), dT.double().cpu().numpy(), None, "bf16", "last rows")
    assert not bool(dz[:-n].any())
    del z, h, dh, dz
    # 1100000 rows of 2048
    print("rows", flush=True)
    m, d, n = 1100000, 2048, 4
    x = torch.zeros((m, d), dtype=torch.bfloat16, device=dev)
    x[-n:] = torch.randn((n, d), device=dev).bfloat16()
    g = torch.rand((d,), device=dev) + 0.5
    q, s = run("rms_norm_q8", [(x, "bf16"), (g, "f32")], [("i8", (m, d)), ("f32", (m,))], eps=1e-5)
    check_norm([q[-n:].double().cpu().numpy(), s[-n:].double().cpu().numpy()], x[-n:].double().cpu().numpy(), None, g.double().cpu().numpy(), "bf16", "last rows")
    assert not bool(q[:-n].any())
    for cols in (40, 300):
        w = torch.randint(-127, 128, (cols, d), dtype=torch.int8, device=dev)
        sw = torch.rand((cols,), device=dev)
        y, = run("dense_q8", [(q, "i8"), (s, "f32"), (w, "i8"), (sw, "f32")], [("f32", (m, cols))], out_dtype="f32")
        num = lambda a: a.double().cpu().numpy()  # noqa: E731
        check_q8(num(y[-n:]), (num(q[-n:]), num(s[-n:]), num(w), num(sw), None), "f32", "last rows")
        assert not bool(y[:-n].any())
