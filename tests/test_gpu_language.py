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


def test_scan_step_in_place():
    """A decoding step's new state over its old one."""
    for b, d, dtype in ((64, 1024, "f32"), (3, 77, "bf16")):
        call, z, h0, keep = scan_case(b, 1, d, dtype, "some", in_place={1: 1})
        check_scan(call.run().numbers(), z, h0, keep, dtype, "step in place")


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
