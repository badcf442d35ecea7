"""The operators of a recurrent language model without a GPU: their typing rules in the oracle and in the library, refusals, and the
oracle's definitions pinned by brute force and by differences."""
import math

import numpy as np
import pytest

from oracle import graph as OG
from oracle import language as L
from paper_1810_00952_amd import binding as B
from language_helpers import plan_of

Z, S, T = ("f32", (12, 10)), ("f32", (3, 5)), ("i32", (4,))
X = ("bf16", (4, 9))

# kind, operands, results, attributes, category of the refusal (None: well typed)
CALLS = [
    ("rms_norm_q8", [X, X, ("f32", (9,))], [("i8", (4, 9)), ("f32", (4,)), X], {}, None),
    ("rms_norm_q8", [X, ("bf16", (9,))], [("i8", (4, 9)), ("f32", (4,))], {"eps": 1e-6}, None),
    ("rms_norm_q8", [("f32", (4, 9)), ("f32", (9,))], [("i8", (4, 9)), ("f32", (4,))], {}, None),
    ("rms_norm_q8", [("f32", (4, 9)), ("bf16", (9,))], [("i8", (4, 9)), ("f32", (4,))], {}, "type"),
    ("rms_norm_q8", [X, ("f32", (4, 9)), ("f32", (9,))], [("i8", (4, 9)), ("f32", (4,)), X], {}, "type"),
    ("rms_norm_q8", [X, X, ("f32", (8,))], [("i8", (4, 9)), ("f32", (4,)), X], {}, "type"),
    ("rms_norm_q8", [X, X, ("f32", (9,))], [("i8", (4, 9)), ("f32", (4,))], {}, "type"),
    ("rms_norm_q8", [X, ("f32", (9,))], [("bf16", (4, 9)), ("f32", (4,))], {}, "type"),
    ("rms_norm_q8", [X], [("i8", (4, 9)), ("f32", (4,))], {}, "type"),
    ("rms_norm_q8", [("i8", (4, 9)), ("f32", (9,))], [("i8", (4, 9)), ("f32", (4,))], {}, "type"),
    ("rms_norm_q8", [("bf16", (4, 9, 1)), ("f32", (9,))], [("i8", (4, 9)), ("f32", (4,))], {}, "type"),
    ("rms_norm_q8", [X, ("f32", (9,))], [("i8", (4, 9)), ("f32", (4,))], {"eps": 0.0}, "kind"),
    ("rms_norm_q8", [X, ("f32", (9,))], [("i8", (4, 9)), ("f32", (4,))], {"eps": math.inf}, "kind"),
    ("rms_norm_q8", [X, ("f32", (9,))], [("i8", (4, 9)), ("f32", (4,))], {"eps": math.nan}, "kind"),
    ("dense_q8", [("i8", (4, 9)), ("f32", (4,)), ("i8", (7, 9)), ("f32", (7,))], [("f32", (4, 7))], {}, None),
    ("dense_q8", [("i8", (4, 9)), ("f32", (4,)), ("i8", (7, 9)), ("f32", (7,)), ("f32", (7,))], [("bf16", (4, 7))], {"out_dtype": "bf16"}, None),
    ("dense_q8", [("i8", (4, 9)), ("f32", (4,)), ("i8", (7, 8)), ("f32", (7,))], [("f32", (4, 7))], {}, "type"),
    ("dense_q8", [("i8", (4, 9)), ("f32", (7,)), ("i8", (7, 9)), ("f32", (7,))], [("f32", (4, 7))], {}, "type"),
    ("dense_q8", [("i8", (4, 9)), ("f32", (4,)), ("i8", (7, 9)), ("f32", (4,))], [("f32", (4, 7))], {}, "type"),
    ("dense_q8", [("i8", (4, 9)), ("f32", (4,)), ("i8", (7, 9)), ("f32", (7,)), ("bf16", (7,))], [("f32", (4, 7))], {}, "type"),
    ("dense_q8", [("bf16", (4, 9)), ("f32", (4,)), ("i8", (7, 9)), ("f32", (7,))], [("f32", (4, 7))], {}, "type"),
    ("dense_q8", [("i8", (4, 9)), ("f32", (4,)), ("i8", (7, 9)), ("f32", (7,))], [("i32", (4, 7))], {"out_dtype": "i32"}, "type"),
    ("linear_scan", [Z, S], [("f32", (12, 5)), S], {}, None),
    ("linear_scan", [Z, S, ("i8", (12,))], [("f32", (12, 5)), S], {}, None),
    ("linear_scan", [("bf16", (3, 10)), S], [("bf16", (3, 5)), S], {}, None),
    ("linear_scan", [("f32", (11, 10)), S], [("f32", (11, 5)), S], {}, "type"),
    ("linear_scan", [("f32", (12, 9)), S], [("f32", (12, 5)), S], {}, "type"),
    ("linear_scan", [Z, ("bf16", (3, 5))], [("f32", (12, 5)), ("bf16", (3, 5))], {}, "type"),
    ("linear_scan", [Z, S, ("i32", (12,))], [("f32", (12, 5)), S], {}, "type"),
    ("linear_scan", [Z, S, ("i8", (3,))], [("f32", (12, 5)), S], {}, "type"),
    ("linear_scan", [Z, S], [("bf16", (12, 5)), S], {}, "type"),
    ("linear_scan_grad", [Z, S, ("f32", (12, 5)), S], [Z, S], {}, None),
    ("linear_scan_grad", [Z, S, ("f32", (12, 5)), S, ("i8", (12,))], [Z, S], {}, None),
    ("linear_scan_grad", [Z, S, ("bf16", (12, 5)), S], [Z, S], {}, "type"),
    ("linear_scan_grad", [Z, S, ("f32", (12, 5)), ("f32", (5, 3))], [Z, S], {}, "type"),
    ("linear_scan_grad", [Z, S, ("f32", (12, 5))], [Z, S], {}, "type"),
    ("token_logprobs", [X, T], [("f32", (4,)), ("f32", (4,))], {}, None),
    ("token_logprobs", [X, T], [("f32", (4,)), ("f32", (4,)), ("f32", (4, 9)), ("i32", (4, 9))], {"top": 9}, None),
    ("token_logprobs", [X, T], [("f32", (4,)), ("f32", (4,)), ("f32", (4, 10)), ("i32", (4, 10))], {"top": 10}, "kind"),
    ("token_logprobs", [("f32", (4, 99)), T], [("f32", (4,)), ("f32", (4,)), ("f32", (4, 33)), ("i32", (4, 33))], {"top": 33}, "kind"),
    ("token_logprobs", [X, T], [("f32", (4,)), ("f32", (4,))], {"top": -1}, "kind"),
    ("token_logprobs", [X, T], [("f32", (4,)), ("f32", (4,))], {"top": 1}, "type"),
    ("token_logprobs", [X, ("i8", (4,))], [("f32", (4,)), ("f32", (4,))], {}, "type"),
    ("token_logprobs", [X, ("i32", (9,))], [("f32", (4,)), ("f32", (4,))], {}, "type"),
    ("token_logprobs_grad", [X, T, ("f32", (4,)), ("f32", (4,))], [X], {}, None),
    ("token_logprobs_grad", [X, T, ("f32", (4,)), ("bf16", (4,))], [X], {}, "type"),
    ("token_logprobs_grad", [X, T, ("f32", (4,)), ("f32", (4,))], [("f32", (4, 9))], {}, "type"),
    # whole numbers go to no other operator
    ("add", [("i8", (4, 9)), ("i8", (4, 9))], [("i8", (4, 9))], {}, "type"),
    ("relu", [("i32", (4, 9))], [("i32", (4, 9))], {}, "type"),
    ("flatten", [("i8", (4, 9))], [("i8", (4, 9))], {}, "type"),
    ("layout_transform", [("i8", (4, 9))], [("i8", (9, 4))], {"perm": (1, 0)}, "type"),
    ("dense", [("i8", (4, 9)), ("i8", (7, 9))], [("f32", (4, 7))], {"out_dtype": "f32"}, "type"),
    ("cast", [("f32", (4, 9))], [("i8", (4, 9))], {"to": "i8"}, "kind"),
    ("lstm_gates", [("f32", (2, 16)), ("f32", (2, 4))], [("f32", (2, 4)), ("i8", (2, 4))], {}, "type"),
]


@pytest.mark.parametrize("kind,operands,results,attrs,refused", CALLS)
def test_typing(kind, operands, results, attrs, refused):
    import workloads as W
    spec = W.GraphSpec("t")
    ids = [spec.input(f"x{i}", *o) for i, o in enumerate(operands)]
    _, outs = spec.op(kind, ids, results, **attrs)
    for v in outs:
        spec.output(v)
    if refused is None:
        OG.check(spec)
        plan = plan_of(kind, operands, results, **attrs)[0]
        assert plan.describe()["steps"]
        return
    with pytest.raises(OG.IllTyped) as e:
        OG.check(spec)
    assert e.value.category == refused
    with pytest.raises(B.RelayError) as e:
        plan_of(kind, operands, results, **attrs)
    assert e.value.category == refused, str(e.value)


def test_a_sum_past_32_bits_is_refused():
    def of(k):
        return plan_of("dense_q8", [("i8", (4, k)), ("f32", (4,)), ("i8", (7, k)), ("f32", (7,))], [("f32", (4, 7))])
    of(131071)                                   # 131071 * 128 * 128 < 2^31
    with pytest.raises(B.RelayError) as e:
        of(131072)
    assert e.value.category == "unsupported"


BIG = 1 << 27


@pytest.mark.parametrize("kind,operands,results", [
    ("rms_norm_q8", [("f32", (BIG, 4)), ("f32", (4,))], [("i8", (BIG, 4)), ("f32", (BIG,))]),
    ("dense_q8", [("i8", (16 * BIG - 1, 16)), ("f32", (16 * BIG - 1,)), ("i8", (1, 16)), ("f32", (1,))], [("f32", (16 * BIG - 1, 1))]),
    ("linear_scan", [("f32", (BIG, 2)), ("f32", (BIG, 1))], [("f32", (BIG, 1)), ("f32", (BIG, 1))]),
    ("linear_scan", [("f32", (4 * BIG, 128)), ("f32", (4 * BIG, 64))], [("f32", (4 * BIG, 64)), ("f32", (4 * BIG, 64))]),
    ("linear_scan", [("f32", (2 * BIG, 2)), ("f32", (BIG, 1))], [("f32", (2 * BIG, 1)), ("f32", (BIG, 1))]),
    ("linear_scan_grad", [("f32", (2 * BIG, 2)), ("f32", (BIG, 1)), ("f32", (2 * BIG, 1)), ("f32", (BIG, 1))], [("f32", (2 * BIG, 2)), ("f32", (BIG, 1))]),
    ("token_logprobs", [("f32", (BIG // 8 - 1, 4100)), ("i32", (BIG // 8 - 1,))], [("f32", (BIG // 8 - 1,)), ("f32", (BIG // 8 - 1,))]),
    ("token_logprobs_grad", [("f32", (BIG // 8 - 1, 4100)), ("i32", (BIG // 8 - 1,)), ("f32", (BIG // 8 - 1,)), ("f32", (BIG // 8 - 1,))], [("f32", (BIG // 8 - 1, 4100))])])
def test_more_threads_than_a_launch_has_are_refused(kind, operands, results):
    """A launch has fewer than 2^32 threads: a call that wants more is refused as its plan is made, not as it runs."""
    if operands[0][1] == (BIG, 2):                 # one token a sequence, a thread a channel: this many are there
        assert plan_of(kind, operands, results)[0].describe()["steps"]
        return
    with pytest.raises(B.RelayError) as e:
        plan_of(kind, operands, results)
    assert e.value.category == "unsupported", str(e.value)


def test_they_are_groups_of_their_own():
    g = B.Graph(B.Context())
    z, h0 = g.input("f32", (12, 10)), g.input("f32", (3, 5))
    a, (h, hT) = g.op("linear_scan", [z, h0], [("f32", (12, 5)), ("f32", (3, 5))])
    b, (y,) = g.op("relu", [h], [("f32", (12, 5))])
    with pytest.raises(B.RelayError) as e:
        g.group([a, b])
    assert e.value.category == "group"
    g.output(y)
    assert g.autogroup() == 2
    g.plan()


def test_run_refuses_bad_bindings():
    plan, ids, outs = plan_of("token_logprobs", [X, T], [("f32", (4,)), ("f32", (4,))])
    good = {v: 4096 * (i + 1) for i, v in enumerate(ids + outs)}
    for broken, category in (({**good, ids[1]: 4104}, "align"), ({k: v for k, v in good.items() if k != outs[1]}, "binding"), ({**good, 99: 64}, "binding"),
                             ({**good, ids[0]: 0}, "binding")):
        with pytest.raises(B.RelayError) as e:
            plan.run(broken)
        assert e.value.category == category
        with pytest.raises(B.RelayError) as e:
            plan.bind(broken).run()
        assert e.value.category == category


@pytest.mark.parametrize("steps,others", [(1, ["linear_scan_grad"]), (1, ["linear_scan"]), (2, []), (40, [])])
def test_a_state_in_place_has_no_other_reader(steps, others):
    """hT may lie over h0 where a sequence has one token and nothing behind the scan reads h0; elsewhere the bindings are refused."""
    b, d = 3, 8
    z_t, s_t, h_t = ("f32", (b * steps, 2 * d)), ("f32", (b, d)), ("f32", (b * steps, d))
    g = B.Graph(B.Context())
    z, h0, dh, dT = g.input(*z_t), g.input(*s_t), g.input(*h_t), g.input(*s_t)
    outs = list(g.op("linear_scan", [z, h0], [h_t, s_t])[1])
    for kind in others:
        outs += g.op(kind, [z, h0, dh, dT] if kind.endswith("grad") else [z, h0], [z_t, s_t] if kind.endswith("grad") else [h_t, s_t])[1]
    for v in outs:
        g.output(v)
    plan = g.plan()
    used = [z, h0] + ([dh, dT] if "linear_scan_grad" in others else []) + outs
    bound = {v: 4096 * (i + 1) for i, v in enumerate(used)}
    bound[outs[1]] = bound[h0]
    for run in (lambda: plan.run(bound, 1 << 20, max(256, plan.workspace_bytes())), lambda: plan.bind(bound, 1 << 20, max(256, plan.workspace_bytes())).run()):
        with pytest.raises(B.RelayError) as e:
            run()
        assert e.value.category == "binding", str(e.value)


# ---- the oracle ------------------------------------------------------------------------------------------------------------
def test_norm_by_hand():
    q, s, y = L.rms_norm_q8([[3.0, -4.0], [0.0, 0.0], [1.0, np.inf]], None, [1.0, 0.5], 1e-12, "f32")
    # mean square 12.5; the largest of 3 / sqrt(12.5), 2 / sqrt(12.5) is 127 steps
    assert np.isclose(s[0], 3 / np.sqrt(12.5) / 127) and s[1] == 0 and np.isnan(s[2])
    assert q.tolist() == [[127.0, -85.0], [0.0, 0.0], [0.0, 0.0]]


def _loss_by_differences(f, at, step=1e-6):
    got = np.zeros(at.size)
    for i in range(at.size):
        for sign in (1, -1):
            x = at.copy().reshape(-1)
            x[i] += sign * step
            got[i] += sign * f(x.reshape(at.shape)) / (2 * step)
    return got.reshape(at.shape)


@pytest.mark.parametrize("packed", [False, True])
def test_scan_gradient_is_that_of_its_result(packed):
    rng = np.random.default_rng(3)
    B_, T_, D = 2, 5, 3
    z, h0 = rng.normal(size=(B_ * T_, 2 * D)), rng.normal(size=(B_, D))
    dh, dhT = rng.normal(size=(B_ * T_, D)), rng.normal(size=(B_, D))
    keep = np.array([1, 2, 1, 0, 1, 0, 1, 1, 2, 0]) if packed else None
    if packed:                                  # rows of padding, whose result does not depend on the loss
        dh[keep == 0] = 0.0

    def loss(z, h0):
        h, hT = L.linear_scan(z, h0, keep)
        return (h * dh).sum() + (hT * dhT).sum()

    dz, dh0 = L.linear_scan_grad(z, h0, dh, dhT, keep)
    # central differences of step 1e-6: 1e-12 of the third derivative, 1e-16 / 1e-6 of rounding
    np.testing.assert_allclose(dz, _loss_by_differences(lambda t: loss(t, h0), z), atol=1e-8)
    np.testing.assert_allclose(dh0, _loss_by_differences(lambda t: loss(z, t), h0), atol=1e-8)


def test_scan_by_hand():
    z = np.array([[0.0, 2.0], [0.0, 4.0], [0.0, np.nan], [0.0, 6.0]])
    h, hT = L.linear_scan(z, [[8.0]], np.array([1, 2, 0, 1]))
    assert h[:, 0].tolist() == [5.0, 2.0, 0.0, 4.0] and hT.tolist() == [[4.0]]
    h, hT = L.linear_scan(z, [[8.0]], np.zeros(4))
    assert not h.any() and hT.tolist() == [[8.0]]


def test_logprob_gradient_is_that_of_its_result():
    rng = np.random.default_rng(4)
    x, tok = rng.normal(size=(4, 6)), np.array([2, -1, 5, 6])
    x[0, 3] = -np.inf
    dlp, dent = rng.normal(size=4), rng.normal(size=4)

    def loss(x):
        lp, ent = L.token_logprobs(x, tok)
        return (lp * dlp).sum() + (ent * dent).sum()

    dx = L.token_logprobs_grad(x, tok, dlp, dent)
    want = _loss_by_differences(loss, x)
    assert dx[0, 3] == 0
    np.testing.assert_allclose(np.delete(dx.reshape(-1), 3), np.delete(want.reshape(-1), 3), atol=1e-8)


def test_logprobs_by_hand():
    inf = np.inf
    x = np.array([[0.0, math.log(3.0), -inf], [-inf, -inf, -inf], [1.0, inf, 0.0], [2.0, 2.0, 2.0], [np.nan, 1.0, inf]])
    lp, ent, top_lp, ids = L.token_logprobs(x, [1, 0, 0, 9, 1], top=2)
    assert np.isclose(lp[0], math.log(0.75)) and lp[1] == -inf and np.isnan(lp[2]) and lp[3] == 0 and np.isnan(lp[4])
    assert np.isclose(ent[0], -0.75 * math.log(0.75) - 0.25 * math.log(0.25)) and ent[1] == 0 and np.isclose(ent[3], math.log(3.0))
    assert ids.tolist() == [[1, 0], [0, 1], [1, 0], [0, 1], [0, 2]]
    assert np.isneginf(top_lp[1]).all() and np.isnan(top_lp[2]).all()
    assert not L.token_logprobs_grad(x[1:2], [0], [1.0], [1.0]).any()
