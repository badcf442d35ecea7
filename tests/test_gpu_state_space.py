"""The operators of a selective state-space language model on the GPU against their definitions in 64 bits."""
import numpy as np
import pytest

from oracle import language as L
from language_helpers import Call, tensor, within
from state_space_helpers import F, conv_bounds, conv_case, loss_bounds, loss_case, scan_bounds, scan_case

pytestmark = pytest.mark.gpu


# ---- causal_conv -----------------------------------------------------------------------------------------------------------
def conv_call(operands, b, t, d, k, dtype, silu, **more):
    return Call("causal_conv", operands[:4] + operands[6:], [(dtype, (b * t, d)), (dtype, (b, k - 1, d))], silu=silu, **more)


def conv_grad_call(operands, b, t, d, k, dtype, silu):
    return Call("causal_conv_grad", operands, [(dtype, (b * t, d)), ("f32", (d, k)), ("f32", (d,)), (dtype, (b, k - 1, d))], silu=silu)


CONVS = [(1, 1, 1, 2), (3, 1, 64, 4), (2, 2, 5, 4), (2, 9, 8, 8), (1, 33, 515, 3), (4, 64, 72, 4), (3, 65, 40, 5), (2, 200, 1000, 2), (1, 700, 96, 7), (5, 130, 9, 6),
         (70, 3, 24, 4), (2, 97, 4100, 4)]


@pytest.mark.parametrize("how", [None, "some", "ends"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,t,d,k", CONVS)
def test_causal_conv(b, t, d, k, dtype, how):
    for silu in (False, True):
        for w_dtype in {"f32", dtype}:
            what = f"conv {b}x{t}x{d} k={k} {dtype} {how} silu={silu} w={w_dtype}"
            print(what, flush=True)
            operands, v = conv_case(b, t, d, k, dtype, w_dtype, how, seed=b + t + d + k)
            x, w, bias, s0, dy, dsT, keep = v
            ey, ex, ew, eb, es = conv_bounds(*v, silu, dtype)
            y, sT = conv_call(operands, b, t, d, k, dtype, silu).run().numbers()
            ref = L.causal_conv(x, w, bias, s0, keep, silu)
            within(y, ref[0], ey, what)
            np.testing.assert_array_equal(sT, ref[1], err_msg=what)
            out = conv_grad_call(operands, b, t, d, k, dtype, silu).run().numbers()
            for name, got, want, tol in zip(("dx", "dw", "db", "ds0"), out, L.causal_conv_grad(*v, silu=silu), (ex, ew, eb, es)):
                within(got, want, tol, f"{what} {name}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_conv_padding_is_as_if_it_were_not_there(dtype):
    """Rows among padding give the same bits as the same rows alone; hundreds of rows of padding lie between tokens."""
    rng = np.random.default_rng(5)
    t, d, k, n = 1500, 48, 4, 37
    at = np.sort(rng.choice(t, size=n, replace=False))
    keep = np.zeros(t)
    keep[at] = np.where(rng.uniform(size=n) < 0.2, 2, 1)
    operands, v = conv_case(1, t, d, k, dtype, "f32", None, seed=6)
    tk, _ = tensor(keep, "i8")
    alone = [(tt[at].contiguous() if i in (0, 4) else tt, dt) for i, (tt, dt) in enumerate(operands)]
    ta, _ = tensor(keep[at], "i8")
    for call, shape in ((conv_call, 0), (conv_grad_call, 0)):
        wide = call(operands + [(tk, "i8")], 1, t, d, k, dtype, True).run().numbers()
        short = call(alone + [(ta, "i8")], 1, n, d, k, dtype, True).run().numbers()
        np.testing.assert_array_equal(wide[0][at], short[0])
        assert not wide[0][keep == 0].any()
        if call is conv_call:
            np.testing.assert_array_equal(wide[1], short[1])
        else:
            np.testing.assert_array_equal(wide[3], short[3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_conv_steps_continue_a_sequence_in_place(dtype):
    """T single steps, the state over the old one, give the bits of the sequence; a step without a token leaves the state."""
    b, t, d, k = 5, 9, 72, 4
    operands, v = conv_case(b, t, d, k, dtype, "f32", "some", seed=8)
    y, sT = conv_call(operands, b, t, d, k, dtype, True).run().numbers()
    state = operands[3][0].clone()
    keep = operands[6][0].view(b, t)
    for i in range(t):
        step = [(operands[0][0].view(b, t, d)[:, i].contiguous(), dtype), operands[1], operands[2], (state, dtype), None, None, (keep[:, i].contiguous(), "i8")]
        call = conv_call(step, b, 1, d, k, dtype, True, in_place={1: 3})
        out = call.run().numbers()
        np.testing.assert_array_equal(out[0], y.reshape(b, t, d)[:, i])
    np.testing.assert_array_equal(state.double().cpu().numpy(), sT)


# ---- selective_scan --------------------------------------------------------------------------------------------------------
def scan_call(operands, b, t, d, n, dtype, **more):
    x, dt, bc, a, skip, h0, dy, dhT, z, keep = operands
    return Call("selective_scan", [x, dt, bc, a, skip, h0] + [o for o in (z, keep) if o], [(dtype, (b * t, d)), ("f32", (b, d, n))], **more)


def scan_grad_call(operands, b, t, d, n, dtype):
    results = [(dtype, (b * t, d)), (dtype, (b * t, d)), (dtype, (b * t, 2 * n)), ("f32", (d, n)), ("f32", (d,)), ("f32", (b, d, n))]
    return Call("selective_scan_grad", [o for o in operands if o], results + ([(dtype, (b * t, d))] if operands[8] else []))


SCANS = [(1, 1, 1, 1), (3, 1, 66, 16), (2, 2, 5, 3), (2, 17, 64, 4), (3, 33, 70, 16), (2, 40, 30, 24), (1, 65, 130, 8), (2, 31, 17, 64), (1, 700, 33, 16), (5, 20, 9, 33),
         (1, 400, 600, 2), (40, 19, 70, 5)]
NAMES = ("dx", "ddt", "dbc", "da", "dskip", "dh0", "dz")


@pytest.mark.parametrize("how", [None, "some", "ends"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,t,d,n", SCANS)
def test_selective_scan(b, t, d, n, dtype, how):
    for gated in (False, True):
        what = f"scan {b}x{t}x{d} n={n} {dtype} {how} gated={gated}"
        print(what, flush=True)
        operands, v = scan_case(b, t, d, n, dtype, gated, how, seed=b + t + d + n)
        x, dt, bc, a, skip, h0, dy, dhT, z, keep = v
        ahead, back = scan_bounds(*v, dtype)
        got = scan_call(operands, b, t, d, n, dtype).run().numbers()
        for name, g, want, tol in zip(("y", "hT"), got, L.selective_scan(x, dt, bc, a, skip, h0, z, keep), ahead):
            within(g, want, tol, f"{what} {name}")
        got = scan_grad_call(operands, b, t, d, n, dtype).run().numbers()
        for name, g, want, tol in zip(NAMES, got, L.selective_scan_grad(x, dt, bc, a, skip, h0, dy, dhT, z, keep), back):
            within(g, want, tol, f"{what} {name}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,t,d,n", [(2, 9, 3, 3), (2, 200, 66, 16), (1, 3001, 40, 8), (300, 33, 64, 4)])
def test_documents_are_apart(b, t, d, n, dtype):
    """NaN and infinities of a document's tokens and of the old state reach nothing of the other documents."""
    operands, v = scan_case(b, t, d, n, dtype, True, None, seed=t)
    keep = np.ones((b, t))
    cut, end = t // 3, t - t // 3
    keep[:, [0, cut, end]] = 2
    dirty = [np.array(a) for a in v[:9]] + [keep.reshape(-1)]
    rng = np.random.default_rng(t)
    inside = np.zeros((b, t), bool)
    inside[:, cut:end] = True
    for i in (0, 1, 2, 6, 8):                                  # the middle document is of NaN, and so is the state before the first
        dirty[i][inside.reshape(-1)] = rng.choice([np.nan, np.inf], size=(inside.sum(), 1))
    dirty[5][:] = np.nan
    types = [dtype, dtype, dtype, "f32", "f32", "f32", dtype, "f32", dtype, "i8"]
    clean = [np.array(a) for a in v[:9]] + [keep.reshape(-1)]
    clean[5][:] = 0.0
    runs = []
    for values in (clean, dirty):
        device = [(tensor(a, ty)[0], ty) for a, ty in zip(values, types)]
        runs.append((scan_call(device, b, t, d, n, dtype).run().numbers(), scan_grad_call(device, b, t, d, n, dtype).run().numbers()))
    out = ~inside.reshape(-1)
    for (cy, chT), (dy_, dhT_) in [(runs[0][0], runs[1][0])]:
        np.testing.assert_array_equal(cy[out], dy_[out])
        np.testing.assert_array_equal(chT, dhT_)
    for i in (0, 1, 2, 6):
        np.testing.assert_array_equal(runs[0][1][i][out], runs[1][1][i][out], err_msg=NAMES[i])
    np.testing.assert_array_equal(runs[1][1][5], 0.0)
    for kind in ("causal_conv", "causal_conv_grad"):
        k = 4
        cop, cv = conv_case(b, t, d, k, dtype, "f32", None, seed=t)
        got = []
        for nan in (False, True):
            vals = [np.array(a) for a in cv[:6]] + [keep.reshape(-1)]
            if nan:
                vals[0][inside.reshape(-1)] = vals[4][inside.reshape(-1)] = np.nan
            vals[3][:] = np.nan if nan else 0.0
            device = [(tensor(a, ty)[0], ty) for a, ty in zip(vals, (dtype, "f32", "f32", dtype, dtype, dtype, "i8"))]
            got.append((conv_call if kind == "causal_conv" else conv_grad_call)(device, b, t, d, k, dtype, True).run().numbers())
        np.testing.assert_array_equal(got[0][0][out], got[1][0][out], err_msg=kind)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [3, 16, 64])
def test_scan_steps_continue_a_sequence_in_place(n, dtype):
    b, t, d = 3, 9, 70
    operands, v = scan_case(b, t, d, n, dtype, True, "some", seed=n)
    x, dt, bc, a, skip, h0, dy, dhT, z, keep = v
    ref = L.selective_scan(x, dt, bc, a, skip, h0, z, keep)
    ahead, _ = scan_bounds(*v, dtype)
    state = operands[5][0].clone()
    for i in range(t):
        row = lambda o: (o[0].view(b, t, -1)[:, i].contiguous(), o[1])
        step = [row(operands[0]), row(operands[1]), row(operands[2]), operands[3], operands[4], (state, "f32"), None, None, row(operands[8]),
                (operands[9][0].view(b, t)[:, i].contiguous(), "i8")]
        before = state.clone()
        got = scan_call(step, b, 1, d, n, dtype, in_place={1: 5}).run().numbers()
        within(got[0], ref[0].reshape(b, t, d)[:, i], ahead[0].reshape(b, t, d)[:, i], f"step {i}")
        none = keep.reshape(b, t)[:, i] == 0
        np.testing.assert_array_equal(state.cpu().numpy()[none], before.cpu().numpy()[none])
    within(state.double().cpu().numpy(), ref[1], ahead[1], "last state")


def test_scan_steps_at_their_ends():
    """Steps from 0 to far: softplus of -infinity is 0, which holds the state, of 60 it is 60; a decay of 2^-126 and less leaves nothing a state of f32 could show."""
    dt = np.array([-np.inf, -200.0, -87.0, -30.0, -16.0, 0.0, 15.0, 20.0, 30.0, 60.0])
    t, n, d = len(dt), 2, 3
    ops, v = scan_case(1, t, d, n, "f32", False, None, seed=1)
    v[1] = np.repeat(dt[:, None], d, 1)
    v[3] = np.array([[-1.0, -0.5], [-2.0, 0.0], [-1e-3, -4.0]])
    ops[1], ops[3] = (tensor(v[1], "f32")[0], "f32"), (tensor(v[3], "f32")[0], "f32")
    v[3] = ops[3][0].double().cpu().numpy()
    x, dts, bc, a, skip, h0, dy, dhT, z, keep = v
    finite = [np.where(np.isfinite(q), q, -1e3) if i == 1 else q for i, q in enumerate(v)]
    ahead, back = scan_bounds(*finite, "f32")
    for g, want, tol in zip(scan_call(ops, 1, t, d, n, "f32").run().numbers(), L.selective_scan(x, dts, bc, a, skip, h0), ahead):
        within(g, want, tol + 1e-37, "far steps")
    for name, g, want, tol in zip(NAMES, scan_grad_call(ops, 1, t, d, n, "f32").run().numbers(), L.selective_scan_grad(x, dts, bc, a, skip, h0, dy, dhT), back):
        within(g, want, tol + 1e-37, "far steps " + name)


# ---- dense_logprobs --------------------------------------------------------------------------------------------------------
def loss_call(operands, m, v, k, dtype, **more):
    return Call("dense_logprobs", operands[:3], [("f32", (m,)), ("f32", (m,))], **more)


def loss_grad_call(operands, lse, m, v, k, dtype, **more):
    t, _ = tensor(lse, "f32")
    return Call("dense_logprobs_grad", operands[:3] + [(t, "f32")] + operands[3:], [(dtype, (m, k)), (dtype, (v, k))], **more)


LOSSES = [(1, 1, 1), (1, 700, 64), (3, 2, 5), (5, 129, 17), (17, 1000, 40), (33, 333, 128), (64, 4097, 8), (128, 128, 130), (129, 257, 33), (300, 5003, 96), (1030, 70, 64),
          (8, 20000, 24), (2, 70001, 16), (700, 2000, 200),
          (1100, 16000, 40), (200, 12000, 1000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,v,k", LOSSES)
def test_dense_logprobs(m, v, k, dtype):
    operands, (x, w, tok, dlp, dlse) = loss_case(m, v, k, dtype, seed=m + v + k)
    ref = L.dense_logprobs(x, w, tok)
    ahead, back = loss_bounds(x, w, tok, ref[1], dlp, dlse, dtype)
    what = f"loss {m}x{v}x{k} {dtype}"
    print(what, flush=True)
    got = loss_call(operands, m, v, k, dtype).run().numbers()
    for name, g, want, tol in zip(("lp", "lse"), got, ref, ahead):
        within(g, want, tol, f"{what} {name}")
    got = loss_grad_call(operands, got[1], m, v, k, dtype, params=(1,)).run().numbers()
    for name, g, want, tol in zip(("dx", "dw"), got, L.dense_logprobs_grad(x, w, tok, ref[1], dlp, dlse), back):
        within(g, want, tol, f"{what} {name}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,v,k", [(40, 30000, 16), (700, 9000, 40), (129, 20001, 72)])
def test_dense_logprobs_by_pieces_of_the_vocabulary(m, v, k, dtype):
    """With the library's own workspace dl is there by pieces: the rows' derivatives are added up over them."""
    import torch
    from paper_1810_00952_amd import binding as B
    operands, (x, w, tok, dlp, dlse) = loss_case(m, v, k, dtype, seed=m + v)
    lse = L.dense_logprobs(x, w, tok)[1]
    _, back = loss_bounds(x, w, tok, lse, dlp, dlse, dtype)
    call = loss_grad_call(operands, lse, m, v, k, dtype)
    call.plan.run_static(call.bound, torch.cuda.current_stream().cuda_stream)
    for name, g, want, tol in zip(("dx", "dw"), call.numbers(), L.dense_logprobs_grad(x, w, tok, lse, dlp, dlse), back):
        within(g, want, tol, f"pieces {m}x{v}x{k} {dtype} {name}")
    assert call.plan.workspace_bytes() > B.STATIC_WORKSPACE_BYTES or m < 700


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,v,k", [(9, 700, 24), (300, 3000, 64)])
def test_rows_that_take_no_part(m, v, k, dtype):
    """NaN and infinities in rows whose derivatives are 0 (padding behind a batch's last token) reach neither dw nor the other rows."""
    operands, (x, w, tok, dlp, dlse) = loss_case(m, v, k, dtype, seed=m)
    lse = L.dense_logprobs(x, w, tok)[1]
    given = (tok >= 0) & (tok < v)
    out = (dlse == 0) & ((dlp == 0) | ~given)
    out[-1] = True
    dlse[out], dlp[out & given] = 0.0, 0.0
    dlp[out & ~given] = np.nan                                 # without a target it is not looked at
    ops = list(operands)
    ops[3], ops[4] = (tensor(dlp, "f32")[0], "f32"), (tensor(dlse, "f32")[0], "f32")
    clean = loss_grad_call(ops, lse, m, v, k, dtype).run().numbers()
    x2, lse2 = x.copy(), lse.copy()
    x2[out], lse2[out] = np.nan, np.inf
    x2[np.flatnonzero(out)[0], 0] = np.inf
    ops[0] = (tensor(x2, dtype)[0], dtype)
    dirty = loss_grad_call(ops, lse2, m, v, k, dtype).run().numbers()
    np.testing.assert_array_equal(clean[0], dirty[0])
    np.testing.assert_array_equal(clean[1], dirty[1])
    assert not dirty[0][out].any()
    lp, _ = loss_call(ops, m, v, k, dtype).run().numbers()
    assert np.isnan(lp[out & given]).all() and not lp[out & ~given].any() and np.isfinite(lp[~out]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("v", [5, 300, 5000])
def test_logits_that_are_no_numbers(v, dtype):
    rng = np.random.default_rng(v)
    x = np.array([[1.0, 0.0], [1.0, 1.0], [-1.0, 0.0], [0.0, 1.0]])
    w = np.stack([np.full(v, -np.inf), rng.normal(size=v)], 1)   # logits of -inf, -inf, +inf and, of 0 times -inf, NaN
    tok = np.array([0, 1, 2, 3])
    ops = [(tensor(x, dtype)[0], dtype), (tensor(w, dtype)[0], dtype), (tensor(tok, "i32")[0], "i32")]
    lp, lse = loss_call(ops, 4, v, 2, dtype).run().numbers()
    assert np.isneginf(lse[:2]).all() and np.isneginf(lp[:2]).all() and np.isnan(lse[2:]).all() and np.isnan(lp[2:]).all()
    x1, w1 = np.array([[1.0], [-1.0], [0.5]]), np.full((v, 1), -np.inf)
    ops = [(tensor(x1, dtype)[0], dtype), (tensor(w1, dtype)[0], dtype), (tensor(np.array([0, 1, -1]), "i32")[0], "i32")]
    lp, lse = loss_call(ops, 3, v, 1, dtype).run().numbers()
    assert np.isneginf(lse[[0, 2]]).all() and np.isneginf(lp[0]) and lp[2] == 0      # nothing but -inf
    assert np.isnan(lse[1]) and np.isnan(lp[1])                                       # +inf
    # some of -inf: they have no probability
    big = np.array([[3e4]])
    half = np.where(np.arange(v) % 2 == 0, -3e38, 0.0)[:, None]
    ops = [(tensor(big, dtype)[0], dtype), (tensor(half, dtype)[0], dtype), (tensor(np.array([1]), "i32")[0], "i32")]
    lp, lse = loss_call(ops, 1, v, 1, dtype).run().numbers()
    assert abs(lse[0] - np.log(v // 2)) < 8 * F * (1 + np.log(v)) + (v / 16 + 60) * F
    g = loss_grad_call(ops + [(tensor(np.array([1.0]), "f32")[0], "f32"), (tensor(np.array([0.0]), "f32")[0], "f32")], lse, 1, v, 1, dtype).run().numbers()
    assert not g[1][0::2].any()
