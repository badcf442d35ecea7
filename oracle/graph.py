"""Oracle-side type checker and op-by-op graph runner -- TEST INFRASTRUCTURE ONLY.

Typing follows the paper's rules (figures "Rules for constructing types" and
"Rules for deriving types of expressions"):
  * Shape-T / Tensor-T: a tensor type is one base type and one shape of
    natural-number constants (here every dim >= 1, rank <= 6);
  * Type-UnaryOp: a unary operator keeps Tensor(b, s);
  * Type-Noncomp-BinaryOp: + - * / need both operands of the *same* b and s
    (so: no implicit broadcast, no implicit promotion) and return that type;
  * Type-Call: a call of a declared operator is well typed only when each
    argument has exactly the parameter type of the operator's arrow type; the
    result is the arrow's result type.  Here an operator's arrow type is
    instantiated from its argument types and attributes (the figure's caption
    notes quantified variables are already instantiated), and the caller's
    declared result type must equal it.

A change of layout is typed like any declared operator: its arrow type
permutes the Shape (the paper's types carry no layout; its section on
extensions proposes tracking it in types, and with row-major storage the
order of the Shape is the layout).

Execution evaluates one operator at a time in float64 and materialises every
intermediate.  A value leaving a fusion group is rounded once (nearest-even)
to its declared dtype; inside a group nothing is rounded.
"""
from __future__ import annotations

from typing import Dict, List, Tuple

import numpy as np

import oracle as O
from oracle import language as L

DTYPES = ("f32", "bf16", "i8", "i32")
FLOATS = ("f32", "bf16")
MAX_RANK = 6


class IllTyped(Exception):
    """category in {"kind", "shape", "type", "group", "unsupported"}"""

    def __init__(self, category: str, msg: str):
        super().__init__(f"[{category}] {msg}")
        self.category = category


def _check_tensor_type(t) -> None:
    if t.dtype not in DTYPES:
        raise IllTyped("kind", f"unknown base type {t.dtype!r}")
    if len(t.shape) > MAX_RANK:
        raise IllTyped("kind", f"rank {len(t.shape)} > {MAX_RANK}")
    for d in t.shape:
        if not isinstance(d, (int, np.integer)) or d < 1:
            raise IllTyped("shape", f"dimension {d!r} is not a positive constant")


def _pair(v, name):
    if not (isinstance(v, (tuple, list)) and len(v) == 2):
        raise IllTyped("kind", f"attribute {name} must be a pair")
    return int(v[0]), int(v[1])


def _out_dtype(attrs, in_dtype):
    od = attrs.get("out_dtype", in_dtype)
    if od not in (in_dtype, "f32"):
        raise IllTyped("type", f"out_dtype {od} not allowed for {in_dtype} operands")
    return od


def infer(kind: str, ins: List[Tuple[str, Tuple[int, ...]]], attrs: Dict) -> List[Tuple[str, Tuple[int, ...]]]:
    """Result type(s) of operator `kind` applied to argument types `ins`."""
    def need(n):
        if len(ins) != n:
            raise IllTyped("type", f"{kind} takes {n} arguments, got {len(ins)}")

    if kind in LANGUAGE:
        return _infer_language(kind, ins, attrs)
    for dt, _ in ins:
        if dt not in FLOATS:
            raise IllTyped("type", f"{kind} is of the float types, not of {dt}")
    if kind in ("neg", "sq", "relu", "sigmoid", "tanh"):
        need(1)
        return [ins[0]]
    if kind in ("add", "sub", "mul", "div"):
        need(2)
        if ins[0] != ins[1]:
            raise IllTyped("type", f"{kind}: operands {ins[0]} and {ins[1]} differ")
        return [ins[0]]
    if kind == "bias_add":
        need(2)
        (dx, sx), (db, sb) = ins
        axis = int(attrs.get("axis", 1))
        if not 0 <= axis < len(sx):
            raise IllTyped("type", "bias_add axis out of range")
        if sb != (sx[axis],):
            raise IllTyped("type", f"bias shape {sb} != ({sx[axis]},)")
        if not (db == dx or (dx == "bf16" and db == "f32")):
            raise IllTyped("type", f"bias dtype {db} not allowed with {dx}")
        return [ins[0]]
    if kind == "dense":
        need(2)
        (dx, sx), (dw, sw) = ins
        if len(sx) != 2 or len(sw) != 2:
            raise IllTyped("type", "dense wants rank-2 operands")
        if dx != dw:
            raise IllTyped("type", "dense operands differ in base type")
        if sx[1] != sw[1]:
            raise IllTyped("type", f"dense inner dims {sx[1]} vs {sw[1]}")
        return [(_out_dtype(attrs, dx), (sx[0], sw[0]))]
    if kind == "conv2d":
        need(2)
        (dx, sx), (dw, sw) = ins
        if len(sx) != 4 or len(sw) != 4:
            raise IllTyped("type", "conv2d wants rank-4 operands")
        if dx != dw:
            raise IllTyped("type", "conv2d operands differ in base type")
        if sx[1] != sw[1]:
            raise IllTyped("type", f"conv2d channels {sx[1]} vs {sw[1]}")
        (s0, s1), (p0, p1) = _pair(attrs.get("stride", (1, 1)), "stride"), _pair(attrs.get("pad", (0, 0)), "pad")
        if s0 < 1 or s1 < 1 or p0 < 0 or p1 < 0:
            raise IllTyped("kind", "bad stride/pad")
        if _pair(attrs.get("dilation", (1, 1)), "dilation") != (1, 1) or int(attrs.get("groups", 1)) != 1:
            raise IllTyped("unsupported", "dilation/groups")
        oh = (sx[2] + 2 * p0 - sw[2]) // s0 + 1
        ow = (sx[3] + 2 * p1 - sw[3]) // s1 + 1
        if sx[2] + 2 * p0 < sw[2] or sx[3] + 2 * p1 < sw[3]:
            raise IllTyped("shape", "kernel larger than padded input")
        return [(_out_dtype(attrs, dx), (sx[0], sw[0], oh, ow))]
    # partial derivatives of the contractions: the arrow types of the operators a reverse-mode gradient calls
    if kind == "dense_grad_x":              # (dy[M,N], W[N,K]) -> [M,K]
        need(2)
        (dy, sy), (dw, sw) = ins
        if len(sy) != 2 or len(sw) != 2:
            raise IllTyped("type", "dense_grad_x wants rank-2 operands")
        if dy != dw:
            raise IllTyped("type", "dense_grad_x operands differ in base type")
        if sy[1] != sw[0]:
            raise IllTyped("type", f"dense_grad_x: dy has {sy[1]} columns, W {sw[0]} rows")
        return [(_out_dtype(attrs, dy), (sy[0], sw[1]))]
    if kind == "dense_grad_w":              # (dy[M,N], x[M,K]) -> [N,K]
        need(2)
        (dy, sy), (dx, sx) = ins
        if len(sy) != 2 or len(sx) != 2:
            raise IllTyped("type", "dense_grad_w wants rank-2 operands")
        if dy != dx:
            raise IllTyped("type", "dense_grad_w operands differ in base type")
        if sy[0] != sx[0]:
            raise IllTyped("type", f"dense_grad_w: batch {sy[0]} vs {sx[0]}")
        return [(_out_dtype(attrs, dy), (sy[1], sx[1]))]
    if kind in ("conv2d_grad_x", "conv2d_grad_w"):
        # (dy[N,O,OH,OW], w[O,C,KH,KW]) -> [N,C,H,W]   /   (dy[N,O,OH,OW], x[N,C,H,W]) -> [O,C,KH,KW]
        # The forward output size floor((H + 2p - KH)/s) + 1 does not determine H (or KH) from the operands: the
        # declaration states the result's Shape and the forward relation is checked against it.
        need(2)
        (dy, sy), (d2, s2) = ins
        if len(sy) != 4 or len(s2) != 4:
            raise IllTyped("type", f"{kind} wants rank-4 operands")
        if dy != d2:
            raise IllTyped("type", f"{kind} operands differ in base type")
        (s0, s1), (p0, p1) = _pair(attrs.get("stride", (1, 1)), "stride"), _pair(attrs.get("pad", (0, 0)), "pad")
        if s0 < 1 or s1 < 1 or p0 < 0 or p1 < 0:
            raise IllTyped("kind", "bad stride/pad")
        decl = attrs.get("declared_shape")
        if decl is None or len(decl) != 4:
            raise IllTyped("type", f"{kind}: the declared result must be rank 4")
        if kind == "conv2d_grad_x":
            n, c, h, w = decl
            o, c2, kh, kw = s2
            x_shape = (sy[0], s2[1], h, w)
            ok = (n, c) == (sy[0], s2[1]) and sy[1] == o
        else:
            o, c, kh, kw = decl
            n, c2, h, w = s2
            x_shape = s2
            ok = (o, c) == (sy[1], s2[1]) and sy[0] == n
        if not ok:
            raise IllTyped("type", f"{kind}: batch / channel counts of operands and declared result disagree")
        if h + 2 * p0 < kh or w + 2 * p1 < kw:
            raise IllTyped("shape", "kernel larger than padded input")
        if ((h + 2 * p0 - kh) // s0 + 1, (w + 2 * p1 - kw) // s1 + 1) != tuple(sy[2:]):
            raise IllTyped("type", f"{kind}: the forward convolution of {x_shape} with a {kh}x{kw} kernel does not give dy's {sy[2:]}")
        return [(_out_dtype(attrs, dy), tuple(decl))]
    if kind == "maxpool2d":
        need(1)
        (dx, sx), = ins
        if len(sx) != 4:
            raise IllTyped("type", "maxpool2d wants rank 4")
        k, s, p = _pair(attrs["kernel"], "kernel"), _pair(attrs.get("stride", (1, 1)), "stride"), _pair(attrs.get("pad", (0, 0)), "pad")
        if min(k) < 1 or min(s) < 1 or min(p) < 0 or p[0] >= k[0] or p[1] >= k[1]:
            raise IllTyped("kind", "bad pool attributes")
        if sx[2] + 2 * p[0] < k[0] or sx[3] + 2 * p[1] < k[1]:
            raise IllTyped("shape", "window larger than padded input")
        return [(dx, (sx[0], sx[1], (sx[2] + 2 * p[0] - k[0]) // s[0] + 1, (sx[3] + 2 * p[1] - k[1]) // s[1] + 1))]
    if kind == "global_avgpool":
        need(1)
        (dx, sx), = ins
        if len(sx) != 4:
            raise IllTyped("type", "global_avgpool wants rank 4")
        return [(dx, (sx[0], sx[1], 1, 1))]
    if kind == "flatten":
        need(1)
        (dx, sx), = ins
        if len(sx) < 2:
            raise IllTyped("type", "flatten wants rank >= 2")
        return [(dx, (sx[0], int(np.prod(sx[1:], dtype=np.int64))))]
    if kind == "concat":
        need(2)
        (da, sa), (db, sb) = ins
        if int(attrs.get("axis", 1)) != 1 or len(sa) != 2 or len(sb) != 2:
            raise IllTyped("unsupported", "concat: rank 2, axis 1 only")
        if da != db or sa[0] != sb[0]:
            raise IllTyped("type", "concat operands disagree")
        return [(da, (sa[0], sa[1] + sb[1]))]
    if kind == "cast":
        need(1)
        to = attrs.get("to")
        if to not in FLOATS:
            raise IllTyped("kind", f"cast to {to!r}")
        return [(to, ins[0][1])]
    if kind == "layout_transform":
        need(1)
        (dx, sx), = ins
        perm = tuple(int(v) for v in attrs.get("perm", ()))
        if sorted(perm) != list(range(len(sx))):
            raise IllTyped("kind", f"perm {perm} is not a permutation of the {len(sx)} axes")
        return [(dx, tuple(sx[p] for p in perm))]
    if kind == "lstm_gates":
        need(2)
        (dz, sz), (dc, sc) = ins
        if dz != "f32" or dc != "f32":
            raise IllTyped("type", "lstm_gates wants f32 pre-activations and cell state")
        if len(sz) != 2 or len(sc) != 2 or sz[0] != sc[0] or sz[1] != 4 * sc[1]:
            raise IllTyped("type", f"lstm_gates shapes {sz} / {sc}")
        hd = attrs.get("h_dtype", None)
        if hd not in FLOATS + (None,):
            raise IllTyped("type", f"lstm_gates: h of {hd}")
        return [("f32", sc), (hd, sc)]   # h' dtype is taken from the declaration
    raise IllTyped("kind", f"unknown operator {kind!r}")


LANGUAGE = ("rms_norm_q8", "dense_q8", "linear_scan", "linear_scan_grad", "token_logprobs", "token_logprobs_grad",
            "causal_conv", "causal_conv_grad", "selective_scan", "selective_scan_grad", "dense_logprobs", "dense_logprobs_grad")
TOP_MAX = 32


def _infer_language(kind, ins, attrs):
    """The arrow types of a gated recurrent and of a selective state-space language model's operators."""
    def operand(i, *allowed):
        if ins[i] not in allowed:
            raise IllTyped("type", f"{kind}: operand {i} is {ins[i]}, not {allowed[0]}")

    def count(*allowed):
        if len(ins) not in allowed:
            raise IllTyped("type", f"{kind} takes {allowed} arguments, got {len(ins)}")

    def matrix(i, dtypes=FLOATS):
        if ins[i][0] not in dtypes or len(ins[i][1]) != 2:
            raise IllTyped("type", f"{kind}: operand {i} is {ins[i]}, not a matrix of {dtypes}")

    if kind == "rms_norm_q8":
        if not (0 < attrs.get("eps", 1e-5) < np.inf):
            raise IllTyped("kind", "eps is not a positive finite number")
        count(2, 3)
        matrix(0)
        e, (m, d) = ins[0]
        operand(len(ins) - 1, ("f32", (d,)), (e, (d,)))
        if len(ins) == 2:
            return [("i8", (m, d)), ("f32", (m,))]
        operand(1, ins[0])
        return [("i8", (m, d)), ("f32", (m,)), ins[0]]
    if kind == "dense_q8":
        count(4, 5)
        matrix(0, ("i8",)), matrix(2, ("i8",))
        (m, k), (n, k2) = ins[0][1], ins[2][1]
        if k != k2:
            raise IllTyped("type", f"dense_q8 inner dims {k} vs {k2}")
        operand(1, ("f32", (m,)))
        for i in range(3, len(ins)):
            operand(i, ("f32", (n,)))
        out = attrs.get("out_dtype", "f32")
        if out not in FLOATS:
            raise IllTyped("type", f"dense_q8: out_dtype {out}")
        return [(out, (m, n))]
    if kind in ("linear_scan", "linear_scan_grad"):
        n = 4 if kind.endswith("grad") else 2
        count(n, n + 1)
        matrix(0), matrix(1, ("f32",))
        (e, (rows, d2)), (b, d) = ins[0], ins[1][1]
        if d2 != 2 * d or rows % b:
            raise IllTyped("type", f"{kind}: z {ins[0]} is not [B*T,2D] for h0 {ins[1]}")
        if n == 4:
            operand(2, (e, (rows, d))), operand(3, ins[1])
        if len(ins) > n:
            operand(n, ("i8", (rows,)))
        return [ins[0] if n == 4 else (e, (rows, d)), ins[1]]
    if kind.startswith("causal_conv"):
        n = 6 if kind.endswith("grad") else 4
        if attrs.get("silu", 0) not in (0, 1):
            raise IllTyped("kind", "silu is neither 0 nor 1")
        count(n, n + 1)
        matrix(0), matrix(1)
        (e, (rows, d)), (wd, k), state = ins[0], ins[1][1], ins[3]
        operand(1, ("f32", (d, k)), (e, (d, k)))
        operand(2, ("f32", (d,)))
        if not 2 <= k <= 8:
            raise IllTyped("unsupported", f"{kind}: {k} taps")
        if len(state[1]) != 3 or rows % state[1][0]:
            raise IllTyped("type", f"{kind}: x {ins[0]} is not [B*T,D] for {state}")
        before = (e, (state[1][0], k - 1, d))
        operand(3, before)
        if n == 6:
            operand(4, ins[0]), operand(5, before)
        if len(ins) > n:
            operand(n, ("i8", (rows,)))
        return [ins[0], ("f32", (d, k)), ("f32", (d,)), before] if n == 6 else [ins[0], before]
    if kind.startswith("selective_scan"):
        n = 8 if kind.endswith("grad") else 6
        count(n, n + 1, n + 2)
        matrix(0)
        (e, (rows, d)), state = ins[0], ins[5]
        if len(state[1]) != 3 or rows % state[1][0]:
            raise IllTyped("type", f"{kind}: x {ins[0]} is not [B*T,D] for {state}")
        b, _, s = state[1]
        operand(1, ins[0]), operand(2, (e, (rows, 2 * s))), operand(3, ("f32", (d, s))), operand(4, ("f32", (d,))), operand(5, ("f32", (b, d, s)))
        if n == 8:
            operand(6, ins[0]), operand(7, state)
        rest = list(range(n, len(ins)))
        gated = bool(rest) and ins[n][0] != "i8"
        if gated:
            operand(rest.pop(0), ins[0])
        if rest:
            operand(rest.pop(0), ("i8", (rows,)))
        if rest:
            raise IllTyped("type", f"{kind}: too many operands")
        if s > 64:
            raise IllTyped("unsupported", f"{kind}: {s} states")
        return [ins[0], ins[0], ins[2], ins[3], ins[4], state] + ([ins[0]] if gated else []) if n == 8 else [ins[0], state]
    if kind.startswith("dense_logprobs"):
        count(6 if kind.endswith("grad") else 3)
        matrix(0), matrix(1)
        (e, (m, k)), (v, _) = ins[0], ins[1][1]
        operand(1, (e, (v, k))), operand(2, ("i32", (m,)))
        for i in range(3, len(ins)):
            operand(i, ("f32", (m,)))
        return [ins[0], ins[1]] if len(ins) > 3 else [("f32", (m,)), ("f32", (m,))]
    top = attrs.get("top", 0) if kind == "token_logprobs" else 0
    if not 0 <= top <= TOP_MAX:
        raise IllTyped("kind", "top out of range")
    count(2 if kind == "token_logprobs" else 4)
    matrix(0)
    m, v = ins[0][1]
    operand(1, ("i32", (m,)))
    if kind == "token_logprobs_grad":
        operand(2, ("f32", (m,))), operand(3, ("f32", (m,)))
        return [ins[0]]
    if top > v:
        raise IllTyped("kind", "more alternatives than columns")
    return [("f32", (m,)), ("f32", (m,))] + ([("f32", (m, top)), ("i32", (m, top))] if top else [])


def _run_language(kind, a, attrs, spec, op):
    if kind == "rms_norm_q8":
        r, g = (a[1], a[2]) if len(a) == 3 else (None, a[1])
        out = L.rms_norm_q8(a[0], r, g, float(np.float32(attrs.get("eps", 1e-5))), spec.values[op.inputs[0]].type.dtype)
        return out[:len(op.outputs)]
    if kind == "dense_q8":
        return [L.dense_q8(*a)]
    if kind == "linear_scan":
        return L.linear_scan(*a)
    if kind == "linear_scan_grad":
        return L.linear_scan_grad(*a)
    if kind == "token_logprobs":
        return L.token_logprobs(a[0], a[1], attrs.get("top", 0))
    if kind.startswith("causal_conv"):
        return getattr(L, kind)(*a, silu=bool(attrs.get("silu", 0)))
    if kind.startswith("selective_scan"):
        n = 8 if kind.endswith("grad") else 6
        gated = len(a) > n and spec.values[op.inputs[n]].type.dtype != "i8"
        return getattr(L, kind)(*a[:n], z=a[n] if gated else None, keep=a[-1] if len(a) > n + gated else None)
    if kind.startswith("dense_logprobs"):
        return getattr(L, kind)(*a)
    return [L.token_logprobs_grad(*a)]


INJECTIVE = {"neg", "sq", "relu", "sigmoid", "tanh", "add", "sub", "mul", "div", "bias_add", "cast"}
ANCHORS = {"dense", "conv2d"}


def check(spec) -> None:
    """Type-check a workloads.GraphSpec and validate its fusion groups."""
    for v in spec.values:
        _check_tensor_type(v.type)
    defined = {i for i, v in enumerate(spec.values) if v.role in ("input", "param")}
    producer = {}
    for oi, op in enumerate(spec.ops):
        for vid in op.inputs:
            if vid not in defined:
                raise IllTyped("type", f"op {oi} uses value {vid} before its definition")
        ins = [(spec.values[v].type.dtype, spec.values[v].type.shape) for v in op.inputs]
        attrs = dict(op.attrs)
        declared = [(spec.values[v].type.dtype, spec.values[v].type.shape) for v in op.outputs]
        if op.kind == "lstm_gates" and len(declared) == 2:
            attrs["h_dtype"] = declared[1][0]
        if op.kind in ("conv2d_grad_x", "conv2d_grad_w") and len(declared) == 1:
            attrs["declared_shape"] = tuple(declared[0][1])
        got = infer(op.kind, ins, attrs)
        if got != declared:
            raise IllTyped("type", f"op {oi} ({op.kind}): declared {declared}, inferred {got}")
        for v in op.outputs:
            defined.add(v)
            producer[v] = oi
    for vid in spec.outputs:
        if vid not in defined:
            raise IllTyped("type", f"output {vid} undefined")

    # ---- fusion groups: connected, one anchor at most and first, the rest
    # injective on the group's output shape, no intermediate escapes
    seen = set()
    consumers: Dict[int, List[int]] = {}
    for oi, op in enumerate(spec.ops):
        for v in op.inputs:
            consumers.setdefault(v, []).append(oi)
    for grp in spec.groups:
        if not grp:
            raise IllTyped("group", "empty group")
        for oi in grp:
            if not 0 <= oi < len(spec.ops) or oi in seen:
                raise IllTyped("group", f"op {oi} missing or in two groups")
            seen.add(oi)
        gset = set(grp)
        ops = [spec.ops[i] for i in sorted(grp)]
        kinds = [o.kind for o in ops]
        lead = 0
        if kinds[0] == "concat" and len(kinds) > 1 and kinds[1] == "dense":
            lead = 1        # concatenation of the GEMM's operand rows is part of the anchor's load
        anchors = [k for k in kinds if k in ANCHORS]
        if len(anchors) > 1:
            raise IllTyped("group", "more than one anchor")
        if anchors and kinds[lead] not in ANCHORS:
            raise IllTyped("group", "anchor is not the group's first operator")
        tail = ops[lead + 1:] if anchors else ops
        if len(ops) > 1:
            for idx, o in enumerate(tail):
                # the gate operator closes a group only as the epilogue of a dense contraction: its pre-activations
                # are the value the rest of the group computes and its cell state comes from outside
                last_gate = o.kind == "lstm_gates" and o is ops[-1] and bool(anchors) and kinds[lead] == "dense"
                if o.kind not in INJECTIVE and not last_gate:
                    raise IllTyped("group", f"{o.kind} cannot be fused")
                if last_gate:
                    prev = ops[-2]
                    if o.inputs[0] not in prev.outputs:
                        raise IllTyped("group", "lstm_gates must take the group's last result as its first operand")
                    if producer.get(o.inputs[1]) in gset:
                        raise IllTyped("group", "lstm_gates' cell state must come from outside the group")
        # connectivity + single escape
        for idx, o in enumerate(ops):
            if idx > 0 and not any(producer.get(v) in gset for v in o.inputs):
                raise IllTyped("group", "group is not connected")
        escaping_ops = set()
        for o in ops:
            for v in o.outputs:
                if v in spec.outputs or any(c not in gset for c in consumers.get(v, [])):
                    escaping_ops.add(id(o))
        if len(escaping_ops) > 1 or (escaping_ops and id(ops[-1]) not in escaping_ops):
            raise IllTyped("group", "an intermediate of the group is used outside it")
        if len(ops) > 1:
            out_shape = spec.values[ops[lead if anchors else 0].outputs[0]].type.shape
            for o in tail:
                if o.kind == "lstm_gates":
                    continue
                if spec.values[o.outputs[0]].type.shape != out_shape:
                    raise IllTyped("group", "fused operators differ in output shape")


def run(spec, data: Dict[str, np.ndarray], keep_all: bool = False, keep=()) -> Dict[int, np.ndarray]:
    """Evaluate the graph.  `data` maps the names of input/param values to
    stored arrays (float32, or uint16 bf16 bits).  Returns float64 arrays for
    the graph outputs (every value when keep_all; the outputs and the value ids
    in `keep` otherwise), each holding numbers exactly representable in that
    value's declared dtype if it crossed a group boundary."""
    check(spec)
    keep = set(keep)
    group_of = {}
    for gi, grp in enumerate(spec.groups):
        for oi in grp:
            group_of[oi] = gi
    nxt = len(spec.groups)
    for oi in range(len(spec.ops)):
        if oi not in group_of:
            group_of[oi] = nxt
            nxt += 1
    consumers: Dict[int, List[int]] = {}
    for oi, op in enumerate(spec.ops):
        for v in op.inputs:
            consumers.setdefault(v, []).append(oi)

    val: Dict[int, np.ndarray] = {}
    for i, v in enumerate(spec.values):
        if v.role in ("input", "param"):
            a = O.widen(data[v.name], v.type.dtype)
            if a.shape != v.type.shape:
                raise ValueError(f"{v.name}: data shape {a.shape} != declared {v.type.shape}")
            val[i] = a
    for oi, op in enumerate(spec.ops):
        a = [val[v] for v in op.inputs]
        k = op.kind
        if k == "dense":
            out = [O.dense(a[0], a[1])]
        elif k == "conv2d":
            out = [O.conv2d(a[0], a[1], tuple(op.attrs.get("stride", (1, 1))), tuple(op.attrs.get("pad", (0, 0))))]
        elif k == "dense_grad_x":
            out = [O.dense_grad_x(a[0], a[1])]
        elif k == "dense_grad_w":
            out = [O.dense_grad_w(a[0], a[1])]
        elif k == "conv2d_grad_x":
            out = [O.conv2d_grad_x(a[0], a[1], spec.values[op.outputs[0]].type.shape, tuple(op.attrs.get("stride", (1, 1))),
                                   tuple(op.attrs.get("pad", (0, 0))))]
        elif k == "conv2d_grad_w":
            out = [O.conv2d_grad_w(a[0], a[1], spec.values[op.outputs[0]].type.shape[2:], tuple(op.attrs.get("stride", (1, 1))),
                                   tuple(op.attrs.get("pad", (0, 0))))]
        elif k == "bias_add":
            out = [O.bias_add(a[0], a[1], int(op.attrs.get("axis", 1)))]
        elif k in ("add", "sub", "mul", "div"):
            out = [O.binary(k, a[0], a[1])]
        elif k in ("neg", "sq", "relu", "sigmoid", "tanh"):
            out = [O.unary(k, a[0])]
        elif k == "maxpool2d":
            out = [O.maxpool2d(a[0], tuple(op.attrs["kernel"]), tuple(op.attrs.get("stride", (1, 1))),
                               tuple(op.attrs.get("pad", (0, 0))))]
        elif k == "global_avgpool":
            out = [O.global_avgpool(a[0])]
        elif k == "flatten":
            out = [a[0].reshape(a[0].shape[0], -1)]
        elif k == "concat":
            out = [np.concatenate([a[0], a[1]], axis=1)]
        elif k == "layout_transform":
            # result[i0, i1, ...] = operand[j] with j[perm[k]] = i[k]: the library routine for exactly that
            out = [np.ascontiguousarray(np.transpose(a[0], tuple(int(v) for v in op.attrs["perm"])))]
        elif k == "cast":
            out = [a[0]]
        elif k == "lstm_gates":
            out = list(O.lstm_gates(a[0], a[1]))
        elif k in LANGUAGE:
            out = _run_language(k, a, op.attrs, spec, op)
        else:
            raise IllTyped("kind", k)
        for vid, arr in zip(op.outputs, out):
            crosses = vid in spec.outputs or any(group_of[c] != group_of[oi] for c in consumers.get(vid, []))
            if crosses or k == "cast":
                arr = O.round_to(arr, spec.values[vid].type.dtype)
            val[vid] = arr
        if not keep_all:
            # free operands no later op needs
            for v in op.inputs:
                if v in val and all(c <= oi for c in consumers.get(v, [])) and v not in spec.outputs and v not in keep:
                    del val[v]
    if keep_all:
        return val
    return {v: val[v] for v in list(spec.outputs) + [k for k in keep if k not in spec.outputs]}
