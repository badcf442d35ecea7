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


@pytest.mark.parametrize("gap", [255, 256, 700, 1999])
def test_conv_over_long_padding(gap):
    """Tokens far apart are neighbours; a sequence that is padding in front, or at its end, or at all."""
    b, t, d, k = 4, 2000, 24, 4
    operands, v = conv_case(b, t, d, k, "f32", "f32", None, seed=gap)
    keep = np.zeros((b, t))
    keep[0, [0, 1, t - 1 - (1999 - gap) // 2 if gap < 1999 else t - 1]] = 1
    keep[1, gap:gap + 70] = 1
    keep[2, :max(1, t - gap)] = 1
    x, w, bias, s0, dy, dsT = [np.array(a) for a in v[:6]]
    tk, keep = tensor(keep.reshape(-1), "i8")
    operands = operands + [(tk, "i8")]
    ey, ex, ew, eb, es = conv_bounds(x, w, bias, s0, dy, dsT, keep, True, "f32")
    y, sT = conv_call(operands, b, t, d, k, "f32", True).run().numbers()
    ref = L.causal_conv(x, w, bias, s0, keep, True)
    within(y, ref[0], ey, "long padding")
    np.testing.assert_array_equal(sT, ref[1])
    for got, want, tol in zip(conv_grad_call(operands, b, t, d, k, "f32", True).run().numbers(), L.causal_conv_grad(x, w, bias, s0, dy, dsT, keep, True), (ex, ew, eb, es)):
        within(got, want, tol, "long padding's gradient")


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


@pytest.mark.parametrize("state", [np.nan, np.inf, 1e30])
@pytest.mark.parametrize("b,t,d,n", [(2, 70, 66, 16), (1, 900, 40, 8), (3, 40, 5, 33)])
def test_padding_in_front_of_a_document_holds_a_state_that_reaches_nothing(b, t, d, n, state):
    """Left-padded sequences whose old state is that of something else: nothing of it is in the gradients, not even in sums over all rows."""
    operands, v = scan_case(b, t, d, n, "f32", True, None, seed=t)
    keep = np.ones((b, t))
    for i in range(b):
        first = t // 3 + 5 * i
        keep[i, :first], keep[i, first] = 0, 2
    values = [np.array(a) for a in v[:9]] + [keep.reshape(-1)]
    values[5][:] = state
    values[7][:, 0] = state if np.isfinite(state) else 1.0
    types = ["f32"] * 9 + ["i8"]
    device = [(tensor(a, ty)[0], ty) for a, ty in zip(values, types)]
    x, dt, bc, a, skip, h0, dy, dhT, z, keep = values
    clean = x, dt, bc, a, skip, np.zeros_like(h0), dy, dhT, z, keep
    ahead, back = scan_bounds(*clean, "f32")
    for g, want, tol in zip(scan_call(device, b, t, d, n, "f32").run().numbers(), L.selective_scan(*clean[:6], z, keep), ahead):
        within(g, want, tol, "left-padded")
    for name, g, want, tol in zip(NAMES, scan_grad_call(device, b, t, d, n, "f32").run().numbers(), L.selective_scan_grad(*clean[:8], z, keep), back):
        within(g, want, tol, "left-padded " + name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,t,d,n", [(1, 5, 3, 3), (2, 17, 66, 16), (1, 700, 33, 16), (3, 30, 20, 40)])
def test_a_last_state_past_f32_is_in_no_sum_over_rows(b, t, d, n, dtype):
    """The last token makes every state infinite, in sequences of no whole number of tiles and without padding: the gradient of a is of the states before it."""
    operands, v = scan_case(b, t, d, n, dtype, True, None, seed=t)
    values = [np.array(a) for a in v[:9]]
    last = np.arange(b) * t + t - 1
    values[1][last] = 1.0
    values[0][last], values[2][last, :n] = 1e20, 1e20          # their product leaves f32
    types = [dtype, dtype, dtype, "f32", "f32", "f32", dtype, "f32", dtype]
    both = [tensor(a, ty) for a, ty in zip(values, types)]
    device, v = [(tt, ty) for (tt, _), ty in zip(both, types)] + [None], [a for _, a in both] + [None]
    y, hT = scan_call(device, b, t, d, n, dtype).run().numbers()
    assert np.isposinf(hT).all()
    _, back = scan_bounds(*v, dtype)
    got = scan_grad_call(device, b, t, d, n, dtype).run().numbers()
    rows = np.setdiff1d(np.arange(b * t), last)
    for name, g, want, tol in zip(NAMES, got, L.selective_scan_grad(*v[:8], v[8]), back):
        if name in ("da", "dskip", "dh0"):
            within(g, want, tol, f"infinite last state {name}")
        else:
            within(g[rows], want[rows], tol[rows], f"infinite last state {name}")


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf, 1e30])
@pytest.mark.parametrize("b,t,d,n", [(3, 5, 5, 33), (3, 40, 66, 16), (2, 900, 40, 8), (40, 19, 70, 5)])
def test_a_sequence_of_padding_reaches_nothing(b, t, d, n, value):
    """Its states and derivatives go through as they are, whatever they are, and are in no sum over the batch: the other results have the bits they have beside zeros there."""
    operands, v = scan_case(b, t, d, n, "f32", True, "ends", seed=t)       # the last sequence is without a token
    runs = []
    for held in (0.0, value):
        h0, dhT = np.array(v[5]), np.array(v[7])
        h0[-1], dhT[-1] = held, held
        ops = list(operands)
        ops[5], ops[7] = (tensor(h0, "f32")[0], "f32"), (tensor(dhT, "f32")[0], "f32")
        runs.append(scan_call(ops, b, t, d, n, "f32").run().numbers() + scan_grad_call(ops, b, t, d, n, "f32").run().numbers())
    for i, (name, clean, got) in enumerate(zip(("y", "hT") + NAMES, *runs)):
        if name in ("hT", "dh0"):
            np.testing.assert_array_equal(got[-1], np.full_like(got[-1], np.float32(value)), err_msg=name)
            clean, got = clean[:-1], got[:-1]
        np.testing.assert_array_equal(got, clean, err_msg=name)
        assert np.isfinite(got).all(), name


@pytest.mark.parametrize("value", [np.nan, np.inf])
def test_conv_of_a_sequence_of_padding_reaches_nothing(value):
    b, t, d, k = 3, 130, 72, 4
    operands, v = conv_case(b, t, d, k, "f32", "f32", "ends", seed=2)
    runs = []
    for held in (0.0, value):
        ops = list(operands)
        for i in (3, 5):
            a = np.array(v[i])
            a[-1] = held
            ops[i] = (tensor(a, "f32")[0], "f32")
        runs.append(conv_call(ops, b, t, d, k, "f32", True).run().numbers() + conv_grad_call(ops, b, t, d, k, "f32", True).run().numbers())
    for name, clean, got in zip(("y", "sT", "dx", "dw", "db", "ds0"), *runs):
        if name in ("sT", "ds0"):
            np.testing.assert_array_equal(got[-1], np.full_like(got[-1], value), err_msg=name)
            clean, got = clean[:-1], got[:-1]
        np.testing.assert_array_equal(got, clean, err_msg=name)


@pytest.mark.parametrize("how", [None, "some", "ends"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,t,d,n", [(3, 1, 5, 3), (2, 37, 66, 16), (1, 200, 9, 40), (1, 700, 33, 4)])
def test_a_state_that_forgets_everything(b, t, d, n, dtype, how):
    """exp(s a) of an a of -infinity, or of one whose multiples leave f32, is 0 for a token, and rows that are none hold the state all the same.  The
    definition's 0 times infinity is its limit, which any a far below 0 gives."""
    operands, v = scan_case(b, t, d, n, dtype, True, how, seed=t + n)
    a = np.array(v[3])
    rng = np.random.default_rng(t)
    forgets = rng.uniform(size=a.shape) < 0.5
    forgets[0, 0] = True
    a[forgets] = rng.choice([-np.inf, -3e38], size=forgets.sum())
    operands[3] = (tensor(a, "f32")[0], "f32")
    v[3] = np.where(forgets, -1e30, v[3])
    ahead, back = scan_bounds(*v, dtype)
    z, keep = v[8], v[9]
    for name, g, want, tol in zip(("y", "hT"), scan_call(operands, b, t, d, n, dtype).run().numbers(), L.selective_scan(*v[:6], z, keep), ahead):
        within(g, want, tol, f"forgets {name}")
    for name, g, want, tol in zip(NAMES, scan_grad_call(operands, b, t, d, n, dtype).run().numbers(), L.selective_scan_grad(*v[:8], z, keep), back):
        within(g, want, tol, f"forgets {name}")


@pytest.mark.parametrize("b,t,d,n", [(1, 5000, 3, 2), (1, 2500, 64, 16), (2, 1300, 5, 40)])
def test_scan_of_many_chunks(b, t, d, n):
    """Few channels: every chunk of rows adds up those before it."""
    operands, v = scan_case(b, t, d, n, "f32", True, "some", seed=t)
    x, dt, bc, a, skip, h0, dy, dhT, z, keep = v
    a[-1, -1] = -0.01                                          # (a state that grows over thousands of rows leaves f32)
    operands[3] = (tensor(a, "f32")[0], "f32")
    a = operands[3][0].double().cpu().numpy()
    ahead, back = scan_bounds(x, dt, bc, a, skip, h0, dy, dhT, z, keep, "f32")
    for g, want, tol in zip(scan_call(operands, b, t, d, n, "f32").run().numbers(), L.selective_scan(x, dt, bc, a, skip, h0, z, keep), ahead):
        within(g, want, tol, "many chunks")
    for name, g, want, tol in zip(NAMES, scan_grad_call(operands, b, t, d, n, "f32").run().numbers(), L.selective_scan_grad(x, dt, bc, a, skip, h0, dy, dhT, z, keep), back):
        within(g, want, tol, "many chunks " + name)


@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("dtype,n", [("f32", 3), ("f32", 16), ("bf16", 8), ("f32", 40)])
def test_a_chunk_of_rows_in_which_states_grow_past_f32(dtype, n, padded):
    """A chunk of 64 rows between two that hold makes a state some e^100 times what it was, more than f32 reaches: what was small enough before is a number behind it, zero is zero."""
    b, t, d = 1, 192, 40
    operands, v = scan_case(b, t, d, n, dtype, True, None, seed=n)
    values = [np.array(a) for a in v[:9]] + [np.ones(b * t)]
    small = 1e-28
    for i in (0, 5, 6, 7):
        values[i] *= small
    values[1][:] = -10.0                                       # steps of some 5e-5, in the middle of 1
    values[1][64:128] = np.log(np.e - 1)
    values[3] = np.random.default_rng(n).uniform(1.5, 1.6, size=(d, n))
    values[5][0, 0], values[7][0, 0], values[0][:, 0], values[6][:, 0] = 0.0, 0.0, 0.0, 0.0      # a channel that stays zero
    if padded:
        for i in (0, 1, 2, 6, 8):
            values[i][5:20] = values[i][150:190] = np.nan
        values[9][5:20] = values[9][150:190] = 0
    types = [dtype, dtype, dtype, "f32", "f32", "f32", dtype, "f32", dtype, "i8"]
    both = [tensor(a, ty) for a, ty in zip(values, types)]
    device, v = [(tt, ty) for (tt, _), ty in zip(both, types)], [a for _, a in both]
    if not padded:
        device[9], v[9] = None, None
    x, dt, bc, a, skip, h0, dy, dhT, z, keep = v
    ahead, back = scan_bounds(*v, dtype)
    got = scan_call(device, b, t, d, n, dtype).run().numbers()
    for name, g, want, tol in zip(("y", "hT"), got, L.selective_scan(*v[:6], z, keep), ahead):
        within(g, want, tol, f"growth {name}")
    assert np.abs(got[1]).max() > 1e10 and not got[1][0, 0].any()
    got = scan_grad_call(device, b, t, d, n, dtype).run().numbers()
    for name, g, want, tol in zip(NAMES, got, L.selective_scan_grad(*v[:8], z, keep), back):
        within(g, want, tol, f"growth {name}")
    assert np.abs(got[5]).max() > 1e10 and not got[5][0, 0].any()


def test_chunks_of_a_growing_state_that_is_zero():
    """Hundreds of rows with gates of e^2: a state and a derivative of zero stay so, as in a scan of one chunk."""
    b, t, d, n = 1, 600, 64, 4
    operands, v = scan_case(b, t, d, n, "f32", False, None, seed=3)
    for i, value in ((0, 0.0), (1, np.log(np.e - 1)), (3, 2.0), (5, 0.0), (6, 0.0), (7, 0.0)):
        operands[i][0].fill_(value)
    for g in scan_call(operands, b, t, d, n, "f32").run().numbers() + scan_grad_call(operands, b, t, d, n, "f32").run().numbers():
        np.testing.assert_array_equal(g, 0.0)


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
          (1100, 16000, 40), (200, 12000, 1000), (6000, 130, 40)]


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
@pytest.mark.parametrize("m,v,k", [(40, 100001, 16), (129, 40001, 72), (17, 300007, 8)])
def test_gradients_by_several_pieces_of_the_vocabulary(m, v, k, dtype):
    """More than sixteen rows by pieces, the last of them short: in the library's own workspace dl has less than its whole size."""
    import torch
    from paper_1810_00952_amd import binding as B
    operands, (x, w, tok, dlp, dlse) = loss_case(m, v, k, dtype, seed=m + v)
    lse = L.dense_logprobs(x, w, tok)[1]
    _, back = loss_bounds(x, w, tok, lse, dlp, dlse, dtype)
    call = loss_grad_call(operands, lse, m, v, k, dtype)
    assert call.plan.workspace_bytes() > B.STATIC_WORKSPACE_BYTES
    call.plan.run_static(call.bound, torch.cuda.current_stream().cuda_stream)
    for name, g, want, tol in zip(("dx", "dw"), call.numbers(), L.dense_logprobs_grad(x, w, tok, lse, dlp, dlse), back):
        within(g, want, tol, f"pieces {m}x{v}x{k} {dtype} {name}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,v,k", [(1, 3, 2), (2, 1030, 260), (4, 63, 700), (5, 65, 513), (8, 2500, 1100), (9, 5000, 515), (12, 129, 1024), (15, 257, 2049), (16, 2600, 72)])
def test_gradient_of_few_rows(m, v, k, dtype):
    """Up to sixteen rows: their derivatives from the vocabulary's rows as they lie, run twice to the same bits."""
    operands, (x, w, tok, dlp, dlse) = loss_case(m, v, k, dtype, seed=7 * m + v + k)
    lse = L.dense_logprobs(x, w, tok)[1]
    _, back = loss_bounds(x, w, tok, lse, dlp, dlse, dtype)
    call = loss_grad_call(operands, lse, m, v, k, dtype)
    once = call.run().numbers()
    for name, g, want, tol in zip(("dx", "dw"), once, L.dense_logprobs_grad(x, w, tok, lse, dlp, dlse), back):
        within(g, want, tol, f"few rows {m}x{v}x{k} {dtype} {name}")
    for g, want in zip(call.run().numbers(), once):
        np.testing.assert_array_equal(g, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,v,k", [(3, 270001, 5), (16, 300000, 8)])
def test_gradient_of_few_rows_by_pieces(m, v, k, dtype):
    """Pieces of the vocabulary of which the last is short, in the library's own workspace."""
    import torch
    from paper_1810_00952_amd import binding as B
    operands, (x, w, tok, dlp, dlse) = loss_case(m, v, k, dtype, seed=m)
    lse = L.dense_logprobs(x, w, tok)[1]
    _, back = loss_bounds(x, w, tok, lse, dlp, dlse, dtype)
    call = loss_grad_call(operands, lse, m, v, k, dtype)
    assert call.plan.workspace_bytes() > B.STATIC_WORKSPACE_BYTES
    call.plan.run_static(call.bound, torch.cuda.current_stream().cuda_stream)
    for name, g, want, tol in zip(("dx", "dw"), call.numbers(), L.dense_logprobs_grad(x, w, tok, lse, dlp, dlse), back):
        within(g, want, tol, f"few rows by pieces {m}x{v}x{k} {dtype} {name}")


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


# ---- operators together, streams, graphs, large sizes ------------------------------------------------------------------------
def some_calls():
    operands, _ = conv_case(5, 70, 72, 4, "bf16", "f32", "some", seed=1)
    yield conv_call(operands, 5, 70, 72, 4, "bf16", True)
    yield conv_grad_call(operands, 5, 70, 72, 4, "bf16", True)
    for b, t, d, n in ((2, 150, 70, 16), (1, 700, 33, 24), (3, 1, 66, 5)):
        operands, _ = scan_case(b, t, d, n, "bf16", True, "some", seed=2)
        yield scan_call(operands, b, t, d, n, "bf16")
        yield scan_grad_call(operands, b, t, d, n, "bf16")
    for m, v, k, dtype in ((40, 3000, 72, "bf16"), (300, 500, 33, "f32"), (8, 20000, 24, "bf16")):
        operands, (x, w, tok, dlp, dlse) = loss_case(m, v, k, dtype, seed=3)
        yield loss_call(operands, m, v, k, dtype)
        yield loss_grad_call(operands, L.dense_logprobs(x, w, tok)[1], m, v, k, dtype)


def test_other_streams_graphs_and_the_same_bits_twice():
    import torch
    for call in some_calls():
        want = call.run().numbers()
        side = torch.cuda.Stream()
        for t in call.results:
            t.view(torch.uint8).fill_(0x5a)
        torch.cuda.synchronize()
        for a, b in zip(call.run(side).numbers(), want):
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


def test_one_plan_on_two_streams_at_once():
    """A plan's runs on different streams, each with a workspace and results of its own."""
    import torch
    for make in (lambda: loss_grad_call(*loss_args), lambda: scan_grad_call(scan_operands, 2, 300, 130, 16, "bf16")):
        operands, (x, w, tok, dlp, dlse) = loss_case(500, 3000, 64, "bf16", seed=4)
        loss_args = (operands, L.dense_logprobs(x, w, tok)[1], 500, 3000, 64, "bf16")
        scan_operands, _ = scan_case(2, 300, 130, 16, "bf16", True, "some", seed=5)
        calls = [make(), make()]
        want = make().run().numbers()
        streams = [torch.cuda.Stream() for _ in calls]
        torch.cuda.synchronize()
        for _ in range(4):
            for c, s in zip(calls, streams):
                c.run(s)
        for c in calls:
            for a, b in zip(c.numbers(), want):
                np.testing.assert_array_equal(a, b)


def test_one_plan_run_on_two_streams_at_once():
    """One plan, its operands shared, the runs that are under way at a time each with results and a workspace of its own."""
    import torch
    loss, (x, w, tok, dlp, dlse) = loss_case(500, 3000, 64, "bf16", seed=4)
    scan, _ = scan_case(2, 300, 130, 16, "bf16", True, "some", seed=5)
    for call in (loss_grad_call(loss, L.dense_logprobs(x, w, tok)[1], 500, 3000, 64, "bf16"), scan_grad_call(scan, 2, 300, 130, 16, "bf16")):
        want = call.run().numbers()
        ids = [next(v for v, p in call.bound.items() if p == t.data_ptr()) for t in call.results]
        streams, runs = [torch.cuda.Stream() for _ in range(2)], []
        for _ in streams:
            results = [torch.zeros_like(t) for t in call.results]
            workspace = torch.full((max(256, call.workspace_bytes),), 0xa5, dtype=torch.uint8, device="cuda:0")
            runs.append((results, workspace, {**call.bound, **{v: t.data_ptr() for v, t in zip(ids, results)}}))
        torch.cuda.synchronize()
        for _ in range(4):
            for (results, workspace, bound), s in zip(runs, streams):
                call.plan.run(bound, workspace.data_ptr(), workspace.numel(), s.cuda_stream)
        torch.cuda.synchronize()
        for results, workspace, bound in runs:
            for got, ref in zip(results, want):
                np.testing.assert_array_equal(got.double().cpu().numpy(), ref)


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
        if op.kind.startswith("causal_conv"):
            n = 6 if op.kind.endswith("grad") else 4
            keep = a[n] if len(a) > n else None
            zero = np.zeros_like(a[0]), np.zeros_like(a[3])
            ey, ex, ew, eb, es = conv_bounds(*a[:4], *(a[4:6] if n == 6 else zero), keep, True, dtype)
            ref = L.causal_conv_grad(*a[:6], keep, True) if n == 6 else L.causal_conv(*a[:4], keep, True)
            for got, want, tol in zip(out, ref, (ex, ew, eb, es) if n == 6 else (ey, 0)):
                within(got, want, tol, what)
        elif op.kind.startswith("selective_scan"):
            n = 8 if op.kind.endswith("grad") else 6
            z, keep = a[n], a[n + 1] if len(a) > n + 1 else None
            zero = np.zeros_like(a[0]), np.zeros_like(a[5])
            ahead, behind = scan_bounds(*a[:6], *(a[6:8] if n == 8 else zero), z, keep, dtype)
            ref = getattr(L, op.kind)(*a[:n], z=z, keep=keep)
            for got, want, tol in zip(out, ref, behind if n == 8 else ahead):
                within(got, want, tol, what)
        elif op.kind == "dense_logprobs":
            zero = np.zeros(len(a[0]))
            ref = L.dense_logprobs(*a)
            for got, want, tol in zip(out, ref, loss_bounds(*a, ref[1], zero, zero, dtype)[0]):
                within(got, want, tol, what)
        elif op.kind == "dense_logprobs_grad":
            for got, want, tol in zip(out, L.dense_logprobs_grad(*a), loss_bounds(*a, dtype)[1]):
                within(got, want, tol, what)
        else:                                       # what was there: its own gate, where it is a group of its own
            f = {"dense": O.dense, "dense_grad_x": O.dense_grad_x, "dense_grad_w": O.dense_grad_w, "add": lambda p, q: p + q, "bias_add": lambda p, q: p + q}[op.kind]
            assert_close(out[0], f(a[0], a[1]), dtype, what)
    return s


@pytest.mark.parametrize("args", [dict(), dict(batch=3, steps=37, dim=72, vocab=1001, states=7, packed=True), dict(batch=9, steps=1, dim=128), dict(batch=2, steps=70, dim=50, dtype="f32", taps=3)])
def test_state_space_lm(args):
    import workloads as W
    spec, data = W.state_space_lm(**args)
    spec.groups = [[i] for i in range(len(spec.ops))]          # every value leaves, so none is fused away
    check_graph(spec, data, args.get("dtype", "bf16"))


@pytest.mark.parametrize("args", [dict(), dict(batch=2, steps=150, dim=96, vocab=333, states=24, packed=True), dict(batch=3, steps=40, dim=40, dtype="f32", taps=2)])
def test_state_space_lm_train(args):
    import workloads as W
    s = check_graph(*W.state_space_lm_train(**args), args.get("dtype", "bf16"))
    names = [k["kernel"] for k in s.plan.describe()["steps"]]
    assert sum("selective_scan" in n for n in names) == 2 and sum("dense_logprobs" in n for n in names) == 2


@pytest.mark.parametrize("packed", [False, True])
def test_values_of_a_training_step_share_the_workspace(packed):
    """The step with all its values in memory of their own, and with those between its calls in the workspace: the same bits."""
    import torch
    import workloads as W
    from paper_1810_00952_amd import harness
    got = []
    for everything in (True, False):
        spec, data = W.state_space_lm_train(3, 90, 72, 16, 700, packed=packed)
        names = list(spec.outputs)
        if everything:
            for op in spec.ops:
                for v in op.outputs:
                    if v not in spec.outputs:
                        spec.output(v)
        s = harness.Session(spec)
        s.load(data)
        s.run()
        torch.cuda.synchronize()
        got.append(([s.tensors[v].clone() for v in names], s.plan.workspace_bytes()))
    for a, b in zip(got[0][0], got[1][0]):
        assert torch.equal(a, b) and bool(torch.isfinite(a.float()).all())
    assert got[0][1] < got[1][1]


def test_generation_continues_a_prompt():
    """A prompt, then the same tokens one at a time on the states each step left."""
    import torch
    import workloads as W
    from paper_1810_00952_amd import harness
    b, t, d, layers = 3, 12, 64, 2
    spec, data = W.state_space_lm(b, t, d, 8, layers, 300, dtype="f32")
    whole = harness.Session(spec)
    whole.load(data)
    whole.run()
    step_spec, _ = W.state_space_lm(b, 1, d, 8, layers, 300, dtype="f32")
    step = harness.Session(step_spec)
    state = {k: data[k] for l in range(layers) for k in (f"c{l}", f"h{l}")}
    lps = []
    for i in range(t):
        step.tensors = {}
        step.load({**data, "x": data["x"].reshape(b, t, d)[:, i], "tok": data["tok"].reshape(b, t)[:, i], **state})
        step.alloc()
        step.run()
        torch.cuda.synchronize()
        lps.append(step.output(0).cpu().numpy())
        for l in range(layers):
            state[f"c{l}"], state[f"h{l}"] = (step.tensors[step_spec.outputs[2 + 2 * l + j]].cpu().numpy() for j in range(2))
    # values of some 1 to 10 through 2 layers of five sums of at most 64 terms each, every one off by a few hundred F of itself; a state gathers those of 12 rows
    tol = 2 * 5 * 64 * 12 * 8 * F * 10
    want = whole.output(0).cpu().numpy().reshape(b, t)
    assert np.abs(np.stack(lps, 1) - want).max() < tol
    for l in range(layers):
        for j, name in enumerate(("c", "h")):
            assert np.abs(state[f"{name}{l}"] - whole.tensors[spec.outputs[2 + 2 * l + j]].cpu().numpy()).max() < tol


def test_past_32_bits():
    """Rows behind the first 4 GB of each operator's largest operand."""
    import torch
    from language_helpers import plan_of, torch_type
    dev = "cuda:0"

    def run(kind, operands, results, **attrs):
        plan, ids, outs = plan_of(kind, [(dt, t.shape) for t, dt in operands], results, **attrs)
        got = [torch.empty(sh, dtype=torch_type(dt), device=dev) for dt, sh in results]
        ws = torch.empty(max(256, plan.workspace_bytes()), dtype=torch.uint8, device=dev)
        plan.run({v: t.data_ptr() for v, t in zip(ids + outs, [t for t, _ in operands] + got)}, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        return got

    num = lambda a: a.double().cpu().numpy()  # noqa: E731
    torch.manual_seed(3)
    # a sequence of 600000 x 4096, padding but for its last rows
    print("sequence", flush=True)
    t, d, n, k, states = 600000, 4096, 5, 4, 2
    keep = torch.zeros((t,), dtype=torch.int8, device=dev)
    keep[-n:] = 1

    def wide(cols=d):
        a = torch.zeros((t, cols), dtype=torch.bfloat16, device=dev)
        a[-n:] = torch.randn((n, cols), device=dev).bfloat16()
        return a

    x, dy = wide(), wide()
    w, bias = torch.rand((d, k), device=dev) - 0.5, torch.randn((d,), device=dev)
    s0, dsT = (torch.randn((1, k - 1, d), device=dev).bfloat16() for _ in range(2))
    tail = [num(a) for a in (x[-n:], w, bias, s0, dy[-n:], dsT)]
    ey, ex, ew, eb, es = conv_bounds(*tail, None, True, "bf16")
    y, sT = run("causal_conv", [(x, "bf16"), (w, "f32"), (bias, "f32"), (s0, "bf16"), (keep, "i8")], [("bf16", (t, d)), ("bf16", (1, k - 1, d))], silu=1)
    ref = L.causal_conv(*tail[:4], None, True)
    within(num(y[-n:]), ref[0], ey, "last rows")
    np.testing.assert_array_equal(num(sT), ref[1])
    assert not bool(y[:-n].any())
    del y
    got = run("causal_conv_grad", [(x, "bf16"), (w, "f32"), (bias, "f32"), (s0, "bf16"), (dy, "bf16"), (dsT, "bf16"), (keep, "i8")],
              [("bf16", (t, d)), ("f32", (d, k)), ("f32", (d,)), ("bf16", (1, k - 1, d))], silu=1)
    ref = L.causal_conv_grad(*tail, None, True)
    assert not bool(got[0][:-n].any())
    for g, want, tol in zip([got[0][-n:]] + got[1:], ref, (ex, ew, eb, es)):
        within(num(g), want, tol, "last rows' gradient")
    del got
    print("scan", flush=True)
    dt, bc = wide() - 1.0, wide(2 * states)
    dt[:-n] = 0
    a, skip = -torch.rand((d, states), device=dev), torch.rand((d,), device=dev)
    h0, dhT = torch.randn((1, d, states), device=dev), torch.randn((1, d, states), device=dev)
    tail = [num(v) for v in (x[-n:], dt[-n:], bc[-n:], a, skip, h0, dy[-n:], dhT)]
    ahead, back = scan_bounds(*tail, None, None, "bf16")
    got = run("selective_scan", [(x, "bf16"), (dt, "bf16"), (bc, "bf16"), (a, "f32"), (skip, "f32"), (h0, "f32"), (keep, "i8")], [("bf16", (t, d)), ("f32", (1, d, states))])
    assert not bool(got[0][:-n].any())
    for g, want, tol in zip((got[0][-n:], got[1]), L.selective_scan(*tail[:6]), ahead):
        within(num(g), want, tol, "last rows of the scan")
    del got
    got = run("selective_scan_grad", [(x, "bf16"), (dt, "bf16"), (bc, "bf16"), (a, "f32"), (skip, "f32"), (h0, "f32"), (dy, "bf16"), (dhT, "f32"), (keep, "i8")],
              [("bf16", (t, d)), ("bf16", (t, d)), ("bf16", (t, 2 * states)), ("f32", (d, states)), ("f32", (d,)), ("f32", (1, d, states))])
    for i, (g, want, tol) in enumerate(zip(got, L.selective_scan_grad(*tail), back)):
        if i < 3:
            assert not bool(g[:-n].any())
        within(num(g[-n:] if i < 3 else g), want, tol, "last rows' gradient of the scan")
    del x, dy, dt, bc, got
    # a vocabulary of 1200000 x 2048, all logits but the last ones 0; then 1000000 rows
    print("vocabulary", flush=True)
    m, v, k, n = 3, 1200000, 2048, 4
    w = torch.zeros((v, k), dtype=torch.bfloat16, device=dev)
    w[-n:] = (torch.randn((n, k), device=dev) / 16).bfloat16()
    x = torch.randn((m, k), device=dev).bfloat16()
    tok = torch.tensor([v - 1, 5, v - n], dtype=torch.int32, device=dev)
    lp, lse = run("dense_logprobs", [(x, "bf16"), (w, "bf16"), (tok, "i32")], [("f32", (m,))] * 2)
    some = num(torch.cat([w[:1], w[-n:]]))
    logits = num(x) @ some.T
    total = np.log(v - n + np.exp(logits[:, 1:]).sum(1))
    size = 2 * k * F * (np.abs(num(x)) @ np.abs(some).T).max() + (v / 16 + 100) * F
    within(num(lse), total, size, "lse of a long vocabulary")
    at = np.array([logits[0, n], 0.0, logits[2, 1]])
    within(num(lp), at - total, size, "lp of a long vocabulary")
    one, half = torch.ones((m,), device=dev), torch.full((m,), 0.5, device=dev)
    dx, dw = run("dense_logprobs_grad", [(x, "bf16"), (w, "bf16"), (tok, "i32"), (lse, "f32"), (one, "f32"), (half, "f32")], [("bf16", (m, k)), ("bf16", (v, k))])
    dl = -0.5 * np.exp(logits - total[:, None])
    dl[0, n] += 1
    dl[2, 1] += 1
    want = dl[:, 1:].T @ num(x)
    within(num(dw[-n:]), want, 2.0 ** -6 * (np.abs(dl[:, 1:]).T @ np.abs(num(x))) + 1e-7, "last rows of dw")
    within(num(dx), dl[:, 1:] @ some[1:], 2.0 ** -6 * (np.abs(dl[:, 1:]) @ np.abs(some[1:])) + 1e-7, "dx of a long vocabulary")
    del w, dw
    print("rows", flush=True)
    m, v, k = 1000000, 70, 2400
    x = torch.zeros((m, k), dtype=torch.bfloat16, device=dev)
    x[-n:] = torch.randn((n, k), device=dev).bfloat16()
    w = (torch.randn((v, k), device=dev) / 24).bfloat16()
    tok = torch.randint(0, v, (m,), dtype=torch.int32, device=dev)
    dlp, dlse = torch.zeros((m,), device=dev), torch.zeros((m,), device=dev)
    dlp[-n:], dlse[-n:] = -1.0, 0.25
    lp, lse = run("dense_logprobs", [(x, "bf16"), (w, "bf16"), (tok, "i32")], [("f32", (m,))] * 2)
    last = num(x[-n:]), num(w), num(tok[-n:])
    ref = L.dense_logprobs(*last)
    ahead, back = loss_bounds(*last, ref[1], num(dlp[-n:]), num(dlse[-n:]), "bf16")
    for g, want, tol in zip((lp, lse), ref, ahead):
        within(num(g[-n:]), want, tol, "last rows' loss")
    dx, dw = run("dense_logprobs_grad", [(x, "bf16"), (w, "bf16"), (tok, "i32"), (lse, "f32"), (dlp, "f32"), (dlse, "f32")], [("bf16", (m, k)), ("bf16", (v, k))])
    ref = L.dense_logprobs_grad(*last, ref[1], num(dlp[-n:]), num(dlse[-n:]))
    within(num(dx[-n:]), ref[0], back[0], "last rows of dx")
    within(num(dw), ref[1], back[1], "dw of many rows")
    assert not bool(dx[:-n].any())
