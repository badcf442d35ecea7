"""The operators of a selective state-space language model without a GPU: typing rules and refusals in the oracle and in the library, states in
place, and the oracle's definitions pinned by hand, by brute force and by differences."""
import numpy as np
import pytest

from oracle import graph as OG
from oracle import language as L
from paper_1810_00952_amd import binding as B
from language_helpers import plan_of

X, W, BIAS, S0, KEEP = ("bf16", (12, 5)), ("f32", (5, 4)), ("f32", (5,)), ("bf16", (3, 3, 5)), ("i8", (12,))
CONV, CONV_OUT = [X, W, BIAS, S0], [X, S0]
CONV_GRAD_OUT = [X, W, BIAS, S0]
BC, A, H = ("bf16", (12, 14)), ("f32", (5, 7)), ("f32", (3, 5, 7))
SCAN, SCAN_OUT = [X, X, BC, A, BIAS, H], [X, H]
SCAN_GRAD, SCAN_GRAD_OUT = SCAN + [X, H], [X, X, BC, A, BIAS, H]
F4, TOK, LX, LW = ("f32", (4,)), ("i32", (4,)), ("bf16", (4, 9)), ("bf16", (30, 9))
LOSS, LOSS_GRAD = [LX, LW, TOK], [LX, LW, TOK, F4, F4, F4]


def but(operands, i, other):
    return operands[:i] + [other] + operands[i + 1:]


# kind, operands, results, attributes, category of the refusal (None: well typed)
CALLS = [
    ("causal_conv", CONV, CONV_OUT, {}, None),
    ("causal_conv", CONV + [KEEP], CONV_OUT, {"silu": 1}, None),
    ("causal_conv", but(CONV, 1, ("bf16", (5, 4))), CONV_OUT, {}, None),
    ("causal_conv", CONV, CONV_OUT, {"silu": 2}, "kind"),
    ("causal_conv", CONV[:3], CONV_OUT, {}, "type"),
    ("causal_conv", CONV + [KEEP, KEEP], CONV_OUT, {}, "type"),
    ("causal_conv", CONV + [("i8", (3, 4))], CONV_OUT, {}, "type"),
    ("causal_conv", CONV, CONV_OUT[:1], {}, "type"),
    ("causal_conv", but(CONV, 2, ("bf16", (5,))), CONV_OUT, {}, "type"),
    ("causal_conv", but(CONV, 3, ("f32", (3, 3, 5))), CONV_OUT, {}, "type"),
    ("causal_conv", but(CONV, 3, ("bf16", (3, 4, 5))), CONV_OUT, {}, "type"),
    ("causal_conv", but(CONV, 3, ("bf16", (5, 3, 5))), CONV_OUT, {}, "type"),
    ("causal_conv", but(CONV, 3, ("bf16", (9, 5))), CONV_OUT, {}, "type"),
    ("causal_conv", but(CONV, 1, ("i8", (5, 4))), CONV_OUT, {}, "type"),
    ("causal_conv", but(CONV, 0, ("i8", (12, 5))), CONV_OUT, {}, "type"),
    ("causal_conv", but(but(CONV, 1, ("f32", (5, 1))), 3, ("bf16", (3, 1, 5))), CONV_OUT, {}, "unsupported"),
    ("causal_conv", but(but(CONV, 1, ("f32", (5, 9))), 3, ("bf16", (3, 8, 5))), [X, ("bf16", (3, 8, 5))], {}, "unsupported"),
    ("causal_conv", [("f32", (12, 5)), ("bf16", (5, 4)), BIAS, ("f32", (3, 3, 5))], [("f32", (12, 5)), ("f32", (3, 3, 5))], {}, "type"),
    ("causal_conv_grad", CONV + [X, S0], CONV_GRAD_OUT, {}, None),
    ("causal_conv_grad", CONV + [X, S0, KEEP], CONV_GRAD_OUT, {"silu": 1}, None),
    ("causal_conv_grad", CONV + [X], CONV_GRAD_OUT, {}, "type"),
    ("causal_conv_grad", CONV + [X, X], CONV_GRAD_OUT, {}, "type"),
    ("causal_conv_grad", CONV + [("f32", (12, 5)), S0], CONV_GRAD_OUT, {}, "type"),
    ("causal_conv_grad", CONV + [X, S0], but(CONV_GRAD_OUT, 1, ("bf16", (5, 4))), {}, "type"),
    ("selective_scan", SCAN, SCAN_OUT, {}, None),
    ("selective_scan", SCAN + [X], SCAN_OUT, {}, None),
    ("selective_scan", SCAN + [KEEP], SCAN_OUT, {}, None),
    ("selective_scan", SCAN + [X, KEEP], SCAN_OUT, {}, None),
    ("selective_scan", SCAN + [KEEP, X], SCAN_OUT, {}, "type"),
    ("selective_scan", SCAN + [X, X], SCAN_OUT, {}, "type"),
    ("selective_scan", SCAN + [KEEP, KEEP], SCAN_OUT, {}, "type"),
    ("selective_scan", SCAN[:5], SCAN_OUT, {}, "type"),
    ("selective_scan", SCAN + [X, KEEP, KEEP], SCAN_OUT, {}, "type"),
    ("selective_scan", but(SCAN, 1, ("f32", (12, 5))), SCAN_OUT, {}, "type"),
    ("selective_scan", but(SCAN, 2, ("bf16", (12, 13))), SCAN_OUT, {}, "type"),
    ("selective_scan", but(SCAN, 3, ("bf16", (5, 7))), SCAN_OUT, {}, "type"),
    ("selective_scan", but(SCAN, 4, ("f32", (7,))), SCAN_OUT, {}, "type"),
    ("selective_scan", but(SCAN, 5, ("f32", (5, 5, 7))), SCAN_OUT, {}, "type"),
    ("selective_scan", but(SCAN, 5, ("f32", (15, 7))), SCAN_OUT, {}, "type"),
    ("selective_scan", but(SCAN, 5, ("bf16", (3, 5, 7))), SCAN_OUT, {}, "type"),
    ("selective_scan", [X, X, ("bf16", (12, 130)), ("f32", (5, 65)), BIAS, ("f32", (3, 5, 65))], [X, ("f32", (3, 5, 65))], {}, "unsupported"),
    ("selective_scan_grad", SCAN_GRAD, SCAN_GRAD_OUT, {}, None),
    ("selective_scan_grad", SCAN_GRAD + [KEEP], SCAN_GRAD_OUT, {}, None),
    ("selective_scan_grad", SCAN_GRAD + [X, KEEP], SCAN_GRAD_OUT + [X], {}, None),
    ("selective_scan_grad", SCAN_GRAD + [X], SCAN_GRAD_OUT, {}, "type"),
    ("selective_scan_grad", SCAN_GRAD, SCAN_GRAD_OUT + [X], {}, "type"),
    ("selective_scan_grad", but(SCAN_GRAD, 7, ("f32", (3, 5))), SCAN_GRAD_OUT, {}, "type"),
    ("selective_scan_grad", SCAN_GRAD[:7], SCAN_GRAD_OUT, {}, "type"),
    ("dense_logprobs", LOSS, [F4, F4], {}, None),
    ("dense_logprobs", but(LOSS, 1, ("f32", (30, 9))), [F4, F4], {}, "type"),
    ("dense_logprobs", but(LOSS, 1, ("bf16", (30, 8))), [F4, F4], {}, "type"),
    ("dense_logprobs", but(LOSS, 2, F4), [F4, F4], {}, "type"),
    ("dense_logprobs", LOSS[:2], [F4, F4], {}, "type"),
    ("dense_logprobs", LOSS, [F4], {}, "type"),
    ("dense_logprobs", [("i8", (4, 9)), ("i8", (30, 9)), TOK], [F4, F4], {}, "type"),
    ("dense_logprobs_grad", LOSS_GRAD, [LX, LW], {}, None),
    ("dense_logprobs_grad", but(LOSS_GRAD, 4, ("bf16", (4,))), [LX, LW], {}, "type"),
    ("dense_logprobs_grad", but(LOSS_GRAD, 5, ("f32", (5,))), [LX, LW], {}, "type"),
    ("dense_logprobs_grad", LOSS_GRAD[:5], [LX, LW], {}, "type"),
    ("dense_logprobs_grad", LOSS_GRAD, [LX, ("f32", (30, 9))], {}, "type"),
]


@pytest.mark.parametrize("i", range(len(CALLS)))
def test_typing_in_oracle_and_library(i):
    kind, operands, results, attrs, category = CALLS[i]
    if category is None:
        assert OG.infer(kind, operands, attrs) == results
        plan_of(kind, operands, results, **attrs)
        return
    with pytest.raises((B.RelayError, OG.IllTyped)) as e:
        got = OG.infer(kind, operands, attrs)
        if got != results:
            raise OG.IllTyped("type", "declared otherwise")
    assert e.value.category == category
    with pytest.raises(B.RelayError) as e:
        plan_of(kind, operands, results, **attrs)
    assert e.value.category == category, str(e.value)


@pytest.mark.parametrize("kind,operands,results", [
    ("causal_conv", [("f32", (1, (1 << 20) + 1)), ("f32", ((1 << 20) + 1, 2)), ("f32", ((1 << 20) + 1,)), ("f32", (1, 1, (1 << 20) + 1))],
     [("f32", (1, (1 << 20) + 1)), ("f32", (1, 1, (1 << 20) + 1))]),
    ("dense_logprobs", [("bf16", ((1 << 20) + 1, 8)), ("bf16", (9, 8)), ("i32", ((1 << 20) + 1,))], [("f32", ((1 << 20) + 1,))] * 2),
    ("dense_logprobs", [("bf16", (4, (1 << 20) + 1)), ("bf16", (9, (1 << 20) + 1)), ("i32", (4,))], [("f32", (4,))] * 2),
    ("selective_scan", [("f32", (1, (1 << 20) + 1))] * 2 + [("f32", (1, 2)), ("f32", ((1 << 20) + 1, 1)), ("f32", ((1 << 20) + 1,)), ("f32", (1, (1 << 20) + 1, 1))],
     [("f32", (1, (1 << 20) + 1)), ("f32", (1, (1 << 20) + 1, 1))]),
])
def test_sizes_past_the_kernels_are_refused(kind, operands, results):
    with pytest.raises(B.RelayError) as e:
        plan_of(kind, operands, results)
    assert e.value.category == "unsupported", str(e.value)


def test_too_many_operands():
    g = B.Graph(B.Context())
    v = [g.input("f32", (2, 2)) for _ in range(13)]
    with pytest.raises(B.RelayError) as e:
        g.op("selective_scan_grad", v, [("f32", (2, 2))])
    assert e.value.category == "type"
    with pytest.raises(B.RelayError) as e:
        g.op("relu", v[:1], [("f32", (2, 2))] * 9)
    assert e.value.category == "type"


@pytest.mark.parametrize("conv", [True, False])
@pytest.mark.parametrize("steps,others", [(1, ["grad"]), (1, ["again"]), (2, []), (40, [])])
def test_a_state_in_place_has_no_other_reader(conv, steps, others):
    b, d, n = 3, 8, 5
    x_t, s_t = ("f32", (b * steps, d)), ("f32", (b, 3, d) if conv else (b, d, n))
    g = B.Graph(B.Context())
    x, s0, dy, dsT = g.input(*x_t), g.input(*s_t), g.input(*x_t), g.input(*s_t)
    if conv:
        used = [x, g.input("f32", (d, 4)), g.input("f32", (d,)), s0]
        kind, grads = "causal_conv", [x_t, ("f32", (d, 4)), ("f32", (d,)), s_t]
    else:
        used = [x, g.input(*x_t), g.input("f32", (b * steps, 2 * n)), g.input("f32", (d, n)), g.input("f32", (d,)), s0]
        kind, grads = "selective_scan", [x_t, x_t, ("f32", (b * steps, 2 * n)), ("f32", (d, n)), ("f32", (d,)), s_t]
    outs = list(g.op(kind, used, [x_t, s_t])[1])
    for other in others:
        outs += g.op(kind + "_grad", used + [dy, dsT], grads)[1] if other == "grad" else g.op(kind, used, [x_t, s_t])[1]
    for v in outs:
        g.output(v)
    plan = g.plan()
    names = used + ([dy, dsT] if "grad" in others else []) + outs
    bound = {v: 4096 * (i + 1) for i, v in enumerate(names)}
    bound[outs[1]] = bound[s0]
    with pytest.raises(B.RelayError) as e:
        plan.run(bound, 1 << 20, max(256, plan.workspace_bytes()))
    assert e.value.category == "binding", str(e.value)


def test_gradient_takes_states_from_the_forward_pass():
    """One step of a plan finds the states between where the forward operator is there, another where it is not."""
    def steps(forward):
        g = B.Graph(B.Context())
        v = [g.input(*t) for t in SCAN_GRAD]
        outs = list(g.op("selective_scan", v[:6], SCAN_OUT)[1]) if forward else []
        for o in outs + g.op("selective_scan_grad", v, SCAN_GRAD_OUT)[1]:
            g.output(o)
        return [s["kernel"] for s in g.plan().describe()["steps"]]

    assert steps(True) == ["selective_scan", "selective_scan_grad"]
    assert steps(False) == ["selective_scan_states", "selective_scan_grad"]


@pytest.mark.parametrize("k", [33, 64])
@pytest.mark.parametrize("other", ["dense_logprobs", "dense_logprobs_grad", "dense_grad_x", "add"])
def test_a_packed_param_has_no_reader_that_wants_it_as_it_lies(other, k):
    """A head's matrix that a contraction reads too: packed where its rows are no whole vectors (33), and then for the contraction alone; declared twice it serves both."""
    m, v = 20, 300
    x_t, w_t, tok_t, row = ("bf16", (m, k)), ("bf16", (v, k)), ("i32", (m,)), ("f32", (m,))

    def plan(first, twice):
        g = B.Graph(B.Context())
        x, w, tok, dy = g.input(*x_t), g.param(*w_t), g.input(*tok_t), g.input("bf16", (m, v))
        rows = [g.input(*row) for _ in range(3)]
        w2 = g.param(*w_t) if twice else w
        calls = [lambda: g.op("dense", [x, w], [("bf16", (m, v))]),
                 lambda: {"dense_logprobs": lambda: g.op(other, [x, w2, tok], [row, row]), "dense_logprobs_grad": lambda: g.op(other, [x, w2, tok] + rows, [x_t, w_t]),
                          "dense_grad_x": lambda: g.op(other, [dy, w2], [x_t]), "add": lambda: g.op(other, [w2, w2], [w_t])}[other]()]
        for call in calls if first == "dense" else calls[::-1]:
            for o in call()[1]:
                g.output(o)
        return g.plan(), w

    for first in ("dense", "other"):
        p, w = plan(first, True)
        assert bool(p.packed_bytes(w)) == (k == 33)
        if k == 64:
            plan(first, False)
            continue
        with pytest.raises(B.RelayError) as e:
            plan(first, False)
        assert e.value.category == "unsupported" and "two different" in str(e.value)


@pytest.mark.parametrize("b,t,cut", [(8, 512, True), (10, 512, True), (11, 512, False), (12, 512, False), (15, 512, False), (16, 512, False), (2, 191, True), (2, 176, False), (2, 128, False)])
def test_a_scan_is_cut_into_three_chunks_or_not_at_all(b, t, cut):
    """Sixteen workgroups a sequence: two chunks would do half of the rows twice and fill no more CUs.  A chunk has four tiles of 16 rows and more.  The
    chunks' states are workspace."""
    d, n = 1024, 16
    x, h = ("bf16", (b * t, d)), ("f32", (b, d, n))
    p, _, _ = plan_of("selective_scan", [x, x, ("bf16", (b * t, 2 * n)), ("f32", (d, n)), ("f32", (d,)), h], [x, h])
    assert (p.workspace_bytes() > 0) == cut


# ---- the oracle ------------------------------------------------------------------------------------------------------------
def _differences(f, at, step=1e-6):
    got = np.zeros(at.size)
    for i in range(at.size):
        for sign in (1, -1):
            v = at.copy().reshape(-1)
            v[i] += sign * step
            got[i] += sign * f(v.reshape(at.shape)) / (2 * step)
    return got.reshape(at.shape)


KEEPS = np.array([1, 2, 1, 0, 1, 0, 0, 1, 1, 2, 0, 1])


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("keep", [None, KEEPS, np.zeros(12)])
def test_conv_gradient_is_that_of_its_result(keep, silu):
    rng = np.random.default_rng(3)
    b, t, d, k = 2, 6, 2, 3
    v = [rng.normal(size=s) for s in ((b * t, d), (d, k), (d,), (b, k - 1, d))]
    dy, dsT = rng.normal(size=(b * t, d)), rng.normal(size=(b, k - 1, d))

    def loss(*v):
        y, sT = L.causal_conv(*v, keep, silu)
        return (y * dy).sum() + (sT * dsT).sum()

    for i, got in enumerate(L.causal_conv_grad(*v, dy, dsT, keep, silu)):
        # central differences of step 1e-6: 1e-12 of the third derivative, 1e-16 / 1e-6 of rounding
        np.testing.assert_allclose(got, _differences(lambda a: loss(*v[:i], a, *v[i + 1:]), v[i]), atol=1e-8)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("keep", [None, KEEPS, np.zeros(12)])
def test_scan_gradient_is_that_of_its_result(keep, gated):
    rng = np.random.default_rng(4)
    b, t, d, n = 2, 6, 2, 3
    v = [rng.normal(size=s) for s in ((b * t, d), (b * t, d), (b * t, 2 * n), (d, n), (d,), (b, d, n))] + ([rng.normal(size=(b * t, d))] if gated else [])
    v[3] = -np.abs(v[3])
    dy, dhT = rng.normal(size=(b * t, d)), rng.normal(size=(b, d, n))

    def loss(*v):
        y, hT = L.selective_scan(*v[:6], z=v[6] if gated else None, keep=keep)
        return (y * dy).sum() + (hT * dhT).sum()

    got = L.selective_scan_grad(*v[:6], dy, dhT, z=v[6] if gated else None, keep=keep)
    assert len(got) == len(v)
    for i, g in enumerate(got):
        np.testing.assert_allclose(g, _differences(lambda a: loss(*v[:i], a, *v[i + 1:]), v[i]), atol=1e-8)


def test_loss_gradient_is_that_of_its_result():
    rng = np.random.default_rng(5)
    x, w, tok = rng.normal(size=(4, 3)), rng.normal(size=(6, 3)), np.array([2, -1, 5, 6])
    dlp, dlse = rng.normal(size=4), rng.normal(size=4)

    def loss(x, w):
        lp, lse = L.dense_logprobs(x, w, tok)
        return (lp * dlp).sum() + (lse * dlse).sum()

    dx, dw = L.dense_logprobs_grad(x, w, tok, L.dense_logprobs(x, w, tok)[1], dlp, dlse)
    np.testing.assert_allclose(dx, _differences(lambda t: loss(t, w), x), atol=1e-8)
    np.testing.assert_allclose(dw, _differences(lambda t: loss(x, t), w), atol=1e-8)


def test_loss_without_logits_is_that_of_the_logits():
    rng = np.random.default_rng(6)
    x, w, tok = rng.normal(size=(5, 3)), rng.normal(size=(7, 3)), np.array([0, 6, -1, 3, 7])
    lp, lse = L.dense_logprobs(x, w, tok)
    want, _ = L.token_logprobs(x @ w.T, tok)
    np.testing.assert_allclose(lp, want, atol=1e-13)
    np.testing.assert_allclose(lse, np.log(np.exp(x @ w.T).sum(1)), atol=1e-13)


def test_conv_by_hand():
    x = np.array([[1.0], [2.0], [np.nan], [3.0], [4.0]])
    y, sT = L.causal_conv(x, [[100.0, 10.0, 1.0]], [0.5], [[[7.0], [8.0]]], np.array([1, 1, 0, 2, 1]))
    assert y[:, 0].tolist() == [781.5, 812.5, 0.0, 3.5, 34.5] and sT[0, :, 0].tolist() == [3.0, 4.0]
    y, sT = L.causal_conv(x[:1], [[100.0, 10.0, 1.0]], [0.0], [[[7.0], [8.0]]])
    assert y.tolist() == [[781.0]] and sT[0, :, 0].tolist() == [8.0, 1.0]
    y, sT = L.causal_conv(x[:1], [[1.0, 1.0]], [0.0], [[[7.0]]], np.zeros(1))
    assert y.tolist() == [[0.0]] and sT.tolist() == [[[7.0]]]


def test_scan_by_hand():
    # softplus(ln(e - 1)) = 1: a step of 1, gates exp(a) = 1/2 and 1
    dt = np.full((3, 1), np.log(np.e - 1))
    y, hT = L.selective_scan([[2.0], [np.nan], [4.0]], dt, [[1.0, 10.0, 1.0, 1.0]] * 3, [[-np.log(2.0), 0.0]], [3.0], [[[8.0, 5.0]]], keep=np.array([1, 0, 1]))
    np.testing.assert_allclose(y[:, 0], [4 + 2 + 5 + 20 + 6, 0, 3 + 4 + 25 + 40 + 12])
    np.testing.assert_allclose(hT[0, 0], [7, 65])
