"""Performance cases of the operators of a selective state-space language model: the short causal convolution and the selective scan
that mix its tokens, for prompts, single tokens and training, and the token log probabilities of a large vocabulary that are found
from the last layer's rows without the logits in memory, with the gradients.

`run` computes each of them in its plain form, from elementary torch operations in 32 bits rounded once at the end, or, where `own`
is true, through the library: a typed graph declared and planned once, whose bound plan every pass runs.  `exact` computes the same
from the definitions in 64 bits."""
import math

import torch

own = False

DEVICE = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "i8": torch.int8, "i32": torch.int32}


# ---- the cases ---------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one generated token of 64 sequences through a layer's convolution: latency
        dict(name="conv_bf16_step", op="conv", dtype="bf16", batch=64, steps=1, dim=2048, taps=4, packed=False, train=False),
        # a long packed row of documents: memory bandwidth
        dict(name="conv_bf16_long", op="conv", dtype="bf16", batch=1, steps=16384, dim=4096, taps=4, packed=True, train=False),
        # a training step of the convolution: forward and backward pass
        dict(name="conv_train_bf16", op="conv", dtype="bf16", batch=8, steps=4096, dim=2048, taps=4, packed=False, train=True),
        # the same on odd sizes in f32, with documents packed into the sequences and their ends padded
        dict(name="conv_train_f32_ragged", op="conv", dtype="f32", batch=5, steps=777, dim=515, taps=3, packed=True, train=True),
        # one generated token of 64 sequences through a layer's scan: the states are read and written
        dict(name="scan_bf16_step", op="scan", dtype="bf16", batch=64, steps=1, dim=2048, states=16, gated=True, packed=False, train=False),
        # one long packed row of documents, scored: few channels, many steps
        dict(name="scan_bf16_long", op="scan", dtype="bf16", batch=1, steps=16384, dim=2048, states=16, gated=True, packed=True, train=False),
        # a training step of the scan: forward and backward pass
        dict(name="scan_train_bf16", op="scan", dtype="bf16", batch=8, steps=2048, dim=2048, states=16, gated=True, packed=False, train=True),
        # the same on odd sizes in f32, with documents and padding, without the gate
        dict(name="scan_train_f32_ragged", op="scan", dtype="f32", batch=3, steps=777, dim=515, states=24, gated=False, packed=True, train=True),
        # eight generated tokens are scored against a long vocabulary: the weights are read once
        dict(name="logprobs_bf16_decode", op="logprobs", dtype="bf16", rows=8, vocab=131072, dim=1024, train=False),
        # a prompt's 4096 tokens scored over the vocabulary of the benchmark's recurrent language model
        dict(name="logprobs_bf16_prompt", op="logprobs", dtype="bf16", rows=4096, vocab=32000, dim=1024, train=False),
        # a training step's loss and gradients over an odd vocabulary in bf16, at training scale
        dict(name="logprobs_train_bf16", op="logprobs", dtype="bf16", rows=8192, vocab=50001, dim=1024, train=True),
        # the same in f32 on small odd sizes
        dict(name="logprobs_train_f32_odd", op="logprobs", dtype="f32", rows=777, vocab=10007, dim=515, train=True),
    ]


def _log_int(rng, lo, hi, multiple=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, max(1, round(v / multiple)) * multiple))


def draw(rng):
    """One more case of the listed kinds.  Half of the feature counts are multiples of 8 or 64, as layers are usually laid out; the
    rest are whatever comes."""
    def count(lo, hi):
        m = rng.choice([1, 1, 8, 64])
        return _log_int(rng, max(lo, m), hi, m)

    def rows(lo, hi):
        return _log_int(rng, lo, hi)

    def within(top, *ranges):
        while True:
            got = [f(lo, hi) for f, lo, hi in ranges]
            if math.prod(got) <= top:
                return got

    op = rng.choice(["conv", "scan", "scan", "logprobs", "logprobs"])
    dtype, train, packed = rng.choice(["f32", "bf16"]), rng.random() < 0.5, rng.random() < 0.5
    if op == "conv":
        b, t, d = within((1 << 25) if dtype == "f32" else (1 << 26), (rows, 1, 128), (rows, 1, 16384), (count, 64, 8192))
        return dict(op=op, dtype=dtype, batch=b, steps=t, dim=d, taps=rng.choice([2, 3, 4, 4, 4, 5, 8]), packed=packed, train=train)
    if op == "scan":
        n = rng.choice([4, 8, 16, 16, 16, 24, 32, 64, rng.randrange(1, 65)])
        b, t, d = within((1 << 29) // n, (rows, 1, 128), (rows, 1, 16384), (count, 64, 4096))
        return dict(op=op, dtype=dtype, batch=b, steps=t, dim=d, states=n, gated=rng.random() < 0.7, packed=packed, train=train)
    m, v, d = within((1 << 34) if dtype == "f32" else (1 << 38), (rows, 1, 8192), (count, 1000, 131072), (count, 64, 4096))
    return dict(op=op, dtype=dtype, rows=m, vocab=v, dim=d, train=train)


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _inputs(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)

    def normal(shape, dtype="f32", mean=0.0, std=1.0):
        return torch.empty(shape, device=DEVICE).normal_(mean, std, generator=g).to(TORCH[dtype])

    def uniform(shape, lo, hi):
        return torch.empty(shape, device=DEVICE).uniform_(lo, hi, generator=g)

    op, e = case["op"], case["dtype"]
    if op == "logprobs":
        m, n, d = case["rows"], case["vocab"], case["dim"]
        v = dict(x=normal((m, d), e), w=normal((n, d), e, std=2.0 / math.sqrt(d)),
                 tok=torch.randint(0, n, (m,), device=DEVICE, generator=g, dtype=torch.int32))
        v["tok"][uniform((m,), 0.0, 1.0) < 0.05] = -1             # positions without a target
        if case["train"]:                                         # of a mean loss, and of a small part of the squared normaliser
            v |= dict(dlp=uniform((m,), -2.0 / m, 0.0), dlse=uniform((m,), 0.0, 0.02 / m))
        return v
    b, t, d = case["batch"], case["steps"], case["dim"]
    v = dict(x=normal((b * t, d), e))
    if op == "conv":
        k = case["taps"]
        v |= dict(w=uniform((d, k), -1.0, 1.0) / math.sqrt(k), b=normal((d,), std=0.1), s0=normal((b, k - 1, d), e))
        if case["train"]:
            v |= dict(dy=normal((b * t, d), e), dsT=normal((b, k - 1, d), e))
    else:
        n = case["states"]
        # steps of some 0.02 to 0.2, decays from 1 to the number of states
        v |= dict(dt=normal((b * t, d), e, mean=-3.0), bc=normal((b * t, 2 * n), e),
                  a=-torch.arange(1, n + 1, device=DEVICE) * uniform((d, n), 0.8, 1.2), skip=uniform((d,), 0.5, 1.5), h0=normal((b, d, n)))
        if case["gated"]:
            v["z"] = normal((b * t, d), e)
        if case["train"]:
            v |= dict(dy=normal((b * t, d), e), dhT=normal((b, d, n)))
    if case["packed"]:                                            # documents of some 400 tokens, the last quarter at most of a sequence padded
        keep = 1 + (uniform((b, t), 0.0, 1.0) < 1 / 400).to(torch.int8)
        keep[torch.arange(t, device=DEVICE)[None, :] >= t - uniform((b, 1), 0.0, t / 4.0).floor()] = 0
        v["keep"] = keep.reshape(-1).contiguous()
    return v


# ---- the library's operators -------------------------------------------------------------------------------------------
KEPT = ("w", "b", "a", "skip")                                    # constants of the model, the rest comes with every call


def _declare(graph, case, v):
    """The typed graph of one pass: {name: value id} of its operands, [(name, value id, dtype, shape)] of its results."""
    names = {torch.float32: "f32", torch.bfloat16: "bf16", torch.int8: "i8", torch.int32: "i32"}
    ids = {k: (graph.param if k in KEPT else graph.input)(names[t.dtype], tuple(t.shape)) for k, t in v.items()}
    made, op, e = [], case["op"], case["dtype"]

    def call(kind, operands, results, **attrs):
        _, outs = graph.op(kind, [ids[k] for k in operands if k in ids], [(dt, sh) for _, dt, sh in results], **attrs)
        for (name, dt, sh), vid in zip(results, outs):
            graph.output(vid)
            ids[name] = vid
            made.append((name, vid, dt, sh))

    if op == "logprobs":
        m, n, d = case["rows"], case["vocab"], case["dim"]
        call("dense_logprobs", ("x", "w", "tok"), [("lp", "f32", (m,)), ("lse", "f32", (m,))])
        if case["train"]:
            call("dense_logprobs_grad", ("x", "w", "tok", "lse", "dlp", "dlse"), [("dx", e, (m, d)), ("dw", e, (n, d))])
        return ids, made
    b, t, d = case["batch"], case["steps"], case["dim"]
    if op == "conv":
        k = case["taps"]
        call("causal_conv", ("x", "w", "b", "s0", "keep"), [("y", e, (b * t, d)), ("sT", e, (b, k - 1, d))], silu=True)
        if case["train"]:
            call("causal_conv_grad", ("x", "w", "b", "s0", "dy", "dsT", "keep"),
                 [("dx", e, (b * t, d)), ("dw", "f32", (d, k)), ("db", "f32", (d,)), ("ds0", e, (b, k - 1, d))], silu=True)
        return ids, made
    n = case["states"]
    call("selective_scan", ("x", "dt", "bc", "a", "skip", "h0", "z", "keep"), [("y", e, (b * t, d)), ("hT", "f32", (b, d, n))])
    if case["train"]:
        call("selective_scan_grad", ("x", "dt", "bc", "a", "skip", "h0", "dy", "dhT", "z", "keep"),
             [("dx", e, (b * t, d)), ("ddt", e, (b * t, d)), ("dbc", e, (b * t, 2 * n)), ("da", "f32", (d, n)), ("dskip", "f32", (d,)),
              ("dh0", "f32", (b, d, n))] + ([("dz", e, (b * t, d))] if case["gated"] else []))
    return ids, made


class _Planned:
    """One case as a program of the library keeps it: the plan, its weights as the plan wants them, its results and workspace."""

    def __init__(self, case, v):
        from paper_1810_00952_amd import Context, Graph

        graph = Graph(Context())
        ids, made = _declare(graph, case, v)
        plan = graph.plan()
        bound, self.kept = {}, []
        for name in v:
            vid = ids[name]
            bound[vid] = v[name].data_ptr()
            size = plan.packed_bytes(vid) if name in KEPT else 0
            if size:
                packed = torch.empty(size, dtype=torch.uint8, device=DEVICE)
                plan.prepack(vid, v[name].data_ptr(), packed.data_ptr(), torch.cuda.current_stream().cuda_stream)
                self.kept.append(packed)
                bound[vid] = packed.data_ptr()
        self.out = {name: torch.empty(shape, dtype=TORCH[dt], device=DEVICE) for name, _, dt, shape in made}
        for name, vid, _, _ in made:
            bound[vid] = self.out[name].data_ptr()
        space = torch.empty(max(256, plan.workspace_bytes()), dtype=torch.uint8, device=DEVICE)
        self.kept.append(space)
        self.bound = plan.bind(bound, space.data_ptr(), space.numel())

    def run(self):
        self.bound.run(torch.cuda.current_stream().cuda_stream)
        return self.out


def prepare(case, seed):
    v = _inputs(case, seed)
    state = dict(case=case, v=v)
    if own:
        state["planned"] = _Planned(case, v)
    return state


def run(state):
    if own:
        return state["planned"].run()
    case, v = state["case"], state["v"]
    return {"conv": _conv, "scan": _scan, "logprobs": _logprobs}[case["op"]](case, v)


# ---- plain forms -------------------------------------------------------------------------------------------------------
def _conv(case, v):
    b, t, d, k = case["batch"], case["steps"], case["dim"], case["taps"]
    e = v["x"].dtype
    x, s0, w = v["x"].float().view(b, t, d), v["s0"].float(), v["w"].float()
    at = torch.arange(t, device=x.device).expand(b, t)
    keep = v["keep"].view(b, t) if "keep" in v else torch.ones_like(at)
    # the tokens of a sequence one behind the other, padding behind them; the old state's tokens stand before them
    order = torch.argsort((keep == 0).to(torch.int8), dim=1, stable=True)
    flags = keep.gather(1, order)
    token = (flags != 0)[:, :, None]
    rows = order[:, :, None].expand(b, t, d)
    ext = torch.cat([s0, torch.where(token, x.gather(1, rows), 0.0)], 1)
    start = torch.cummax(torch.where(flags == 2, at + k - 1, 0), 1).values        # where a token's document begins in ext
    u = v["b"].expand(b, t, d)
    windows = []
    for j in range(k):                                            # tap j reads the token k - 1 - j before
        seen = (at + j >= start)[:, :, None]
        windows.append(torch.where(seen, ext[:, j:j + t], 0.0))
        u = u + w[:, j] * windows[j]
    gate = torch.sigmoid(u)
    y = torch.zeros_like(x).scatter(1, rows, torch.where(token, u * gate, 0.0))
    count = (flags != 0).sum(1)
    last = torch.where(count > 0, start.gather(1, (count - 1).clamp(min=0)[:, None])[:, 0], 0)
    tail = count[:, None] + torch.arange(k - 1, device=x.device)                  # the last k - 1 rows of ext that are tokens or state
    alive = (tail >= last[:, None])[:, :, None]
    tails = tail[:, :, None].expand(b, k - 1, d)
    out = {"y": y.reshape(b * t, d).to(e), "sT": torch.where(alive, ext.gather(1, tails), 0.0).to(e)}
    if case["train"]:
        dy = v["dy"].float().view(b, t, d).gather(1, rows)
        g = torch.where(token, dy * gate * (1 + u * (1 - gate)), 0.0)
        dext = torch.zeros_like(ext).scatter_add(1, tails, torch.where(alive, v["dsT"].float(), 0.0))
        dw = []
        for j in range(k):
            seen = (at + j >= start)[:, :, None]
            dext[:, j:j + t] += torch.where(seen, w[:, j] * g, 0.0)
            dw.append((g * windows[j]).sum((0, 1)))
        dx = torch.zeros_like(x).scatter(1, rows, torch.where(token, dext[:, k - 1:], 0.0))
        out |= {"dx": dx.reshape(b * t, d).to(e), "dw": torch.stack(dw, 1), "db": g.sum((0, 1)), "ds0": dext[:, :k - 1].to(e)}
    return out


def _prefixes(a, u):
    """h_t = a_t h_(t-1) + u_t along dimension 1 from zero, by doubling: after the pass of `step`, a and u are of 2 step tokens."""
    step, steps = 1, a.shape[1]
    while step < steps:
        u = torch.cat([u[:, :step], u[:, step:] + a[:, step:] * u[:, :-step]], 1)
        a = torch.cat([a[:, :step], a[:, step:] * a[:, :-step]], 1)
        step *= 2
    return u


def _scan(case, v):
    b, t, d, n = case["batch"], case["steps"], case["dim"], case["states"]
    e = v["x"].dtype
    x, dt = v["x"].float().view(b, t, d), v["dt"].float().view(b, t, d)
    bc = v["bc"].float().view(b, t, 2, n)
    step = torch.where(dt > 20, dt, torch.log1p(torch.exp(torch.clamp(dt, max=20))))
    keep = v["keep"].view(b, t, 1) if "keep" in v else None
    if case["gated"]:
        z = v["z"].float().view(b, t, d)
        sig = torch.sigmoid(z)
    if case["train"]:
        dy = v["dy"].float().view(b, t, d)
        du = dy * z * sig if case["gated"] else dy
        if keep is not None:
            du = torch.where(keep == 0, 0.0, du)
        dx, dstep = du * v["skip"], torch.zeros_like(x)
        dbc, da, dh0 = torch.empty_like(bc), torch.empty_like(v["a"]), torch.empty_like(v["h0"])
    u = x * v["skip"]
    hT = torch.empty_like(v["h0"])
    for i in range(n):                                            # one state of every channel after the other
        decay = torch.exp(step * v["a"][:, i])
        came = step * x * bc[:, :, 0, i, None]
        if keep is not None:                                      # padding holds the state, a document's first token forgets it
            decay = torch.where(keep == 0, 1.0, torch.where(keep == 2, 0.0, decay))
            came = torch.where(keep == 0, 0.0, came)
        first = torch.addcmul(came[:, :1], decay[:, :1], v["h0"][:, None, :, i])
        h = _prefixes(decay, torch.cat([first, came[:, 1:]], 1))
        hT[:, :, i] = h[:, -1]
        u = u + bc[:, :, 1, i, None] * h
        if case["train"]:
            before = torch.cat([v["h0"][:, None, :, i], h[:, :-1]], 1)
            after = torch.cat([decay[:, 1:], torch.ones_like(decay[:, :1])], 1)
            own_part = du * bc[:, :, 1, i, None]
            own_part[:, -1] += v["dhT"][:, :, i]
            G = _prefixes(after.flip(1), own_part.flip(1)).flip(1)
            dh0[:, :, i] = decay[:, 0] * G[:, 0]
            by = G if keep is None else torch.where(keep == 0, 0.0, G)
            dexp = by * before * decay
            if keep is not None:
                dexp = torch.where(keep == 1, dexp, 0.0)
            da[:, i] = (dexp * step).sum((0, 1))
            dstep += dexp * v["a"][:, i] + by * x * bc[:, :, 0, i, None]
            dx += by * step * bc[:, :, 0, i, None]
            dbc[:, :, 0, i] = (by * step * x).sum(2)
            dbc[:, :, 1, i] = (du * h).sum(2)
    y = u * z * sig if case["gated"] else u
    if keep is not None:
        y = torch.where(keep == 0, 0.0, y)
    out = {"y": y.reshape(b * t, d).to(e), "hT": hT}
    if case["train"]:
        out |= {"dx": dx.reshape(b * t, d).to(e), "ddt": (dstep * torch.sigmoid(dt)).reshape(b * t, d).to(e),
                "dbc": dbc.reshape(b * t, 2 * n).to(e), "da": da, "dskip": (du * x).sum((0, 1)), "dh0": dh0}
        if case["gated"]:
            dz = dy * u * sig * (1 + z * (1 - sig))
            if keep is not None:
                dz = torch.where(keep == 0, 0.0, dz)
            out["dz"] = dz.reshape(b * t, d).to(e)
    return out


def _logprobs(case, v):
    m, n = case["rows"], case["vocab"]
    tok = v["tok"].long()
    here = (tok >= 0) & (tok < n)
    at = torch.where(here, tok, 0)[:, None]
    x, w = v["x"].float(), v["w"].float()
    logits = torch.mm(x, w.t())
    top = logits.amax(1, keepdim=True)
    lse = (top + torch.log(torch.exp(logits - top).sum(1, keepdim=True)))
    out = {"lp": torch.where(here, (logits.gather(1, at) - lse)[:, 0], 0.0), "lse": lse[:, 0]}
    if case["train"]:
        dlp = (v["dlp"] * here)[:, None]
        dl = (v["dlse"][:, None] - dlp) * torch.exp(logits - lse)
        dl.scatter_add_(1, at, dlp)
        out |= {"dx": torch.mm(dl, w).to(v["x"].dtype), "dw": torch.mm(dl.t(), x).to(v["w"].dtype)}
    return out


# ---- what a pass cannot do without -------------------------------------------------------------------------------------
def work(case):
    size = {"f32": 4, "bf16": 2}[case["dtype"]]
    op, train = case["op"], case["train"]
    if op == "logprobs":
        m, n, d = case["rows"], case["vocab"], case["dim"]
        return dict(bytes=(m + n) * d * size * (2 if train else 1) + m * (20 if train else 12), flops=2 * m * n * d * (4 if train else 1))
    b, t, d = case["batch"], case["steps"], case["dim"]
    elements, flags = b * t * d, b * t if case["packed"] else 0
    if op == "conv":
        k = case["taps"]
        state, weights = b * (k - 1) * d * size, 4 * d * (k + 1)
        return dict(bytes=elements * size * (4 if train else 2) + state * (4 if train else 2) + weights * (2 if train else 1) + flags,
                    flops=elements * ((6 * k + 20) if train else (2 * k + 6)))
    n = case["states"]
    wide = 3 + (1 if case["gated"] else 0)                        # x, dt, y and z
    if train:
        wide += 3 + (1 if case["gated"] else 0)                   # dy, dx, ddt and dz
    state, weights, bc = 4 * b * d * n, 4 * d * (n + 1), b * t * 2 * n * size
    # an exponential, its argument, the update, its addend, the read-out; backward the state once more, its derivative, five sums
    return dict(bytes=elements * size * wide + state * (4 if train else 2) + weights * (2 if train else 1) + bc * (2 if train else 1) + flags,
                flops=elements * n * (24 if train else 7))


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------
def exact(case, seed):
    v = _inputs(case, seed)
    return {"conv": _exact_conv, "scan": _exact_scan, "logprobs": _exact_logprobs}[case["op"]](case, v)


def _flags(case, v):
    b, t = case["batch"], case["steps"]
    return v["keep"].view(b, t) if "keep" in v else torch.ones((b, t), dtype=torch.int8, device=DEVICE)


def _exact_conv(case, v):
    """Token by token, with the window of the last tokens as a tensor."""
    b, t, d, k = case["batch"], case["steps"], case["dim"], case["taps"]
    x, w, keep = v["x"].view(b, t, d), v["w"].double().t().contiguous(), _flags(case, v)
    window = torch.cat([v["s0"].double(), torch.zeros((b, 1, d), dtype=torch.float64, device=DEVICE)], 1)
    y = torch.zeros((b, t, d), dtype=torch.float64, device=DEVICE)
    pre, seen = (torch.zeros((t, b, d), dtype=torch.float64, device=DEVICE), torch.zeros((t, b, k, d), dtype=torch.float64, device=DEVICE)) if case["train"] else (None, None)
    for i in range(t):
        flag = keep[:, i, None, None]
        # the window holds the k - 1 tokens before in its first rows, the present one last
        now = torch.cat([window[:, :k - 1].masked_fill(flag == 2, 0.0), x[:, i, None].double()], 1)
        u = v["b"].double() + (now * w).sum(1)
        y[:, i] = (u / (1 + (-u).exp())).masked_fill(flag[:, :, 0] == 0, 0.0)
        if pre is not None:
            pre[i], seen[i] = u, now
        moved = torch.cat([now[:, 1:], torch.zeros_like(now[:, :1])], 1)
        window = torch.where(flag == 0, window, moved)
    out = {"y": y.view(b * t, d), "sT": window[:, :k - 1].clone()}
    if case["train"]:
        dwindow = v["dsT"].double()                               # the derivative by the k - 1 tokens before the next one
        dx = torch.zeros((b, t, d), dtype=torch.float64, device=DEVICE)
        dw, db = torch.zeros_like(w), torch.zeros_like(w[0])
        dy = v["dy"].view(b, t, d)
        for i in range(t - 1, -1, -1):
            flag = keep[:, i, None, None]
            u = pre[i]
            s = 1 / (1 + (-u).exp())
            g = (dy[:, i].double() * (s + u * s * (1 - s))).masked_fill(flag[:, :, 0] == 0, 0.0)
            db += g.sum(0)
            dw += (g[:, None] * seen[i].masked_fill(flag == 0, 0.0)).sum(0)
            dnow = torch.cat([torch.zeros_like(dwindow[:, :1]), dwindow], 1) + g[:, None] * w
            dx[:, i] = dnow[:, k - 1].masked_fill(flag[:, :, 0] == 0, 0.0)
            dwindow = torch.where(flag == 0, dwindow, dnow[:, :k - 1].masked_fill(flag == 2, 0.0))
        out |= {"dx": dx.view(b * t, d), "dw": dw.t().contiguous(), "db": db, "ds0": dwindow}
    return out


def _exact_scan(case, v):
    """Token by token, the state as a tensor of [batch, channel, state]."""
    b, t, d, n = case["batch"], case["steps"], case["dim"], case["states"]
    keep, gated, train = _flags(case, v), case["gated"], case["train"]
    A, skip, state = v["a"].double(), v["skip"].double(), v["h0"].double()
    at = {k: v[k].view(b, t, -1) for k in ("x", "dt", "bc", "z", "dy") if k in v}
    y = torch.zeros((b, t, d), dtype=torch.float64, device=DEVICE)
    came = torch.zeros((t, b, d, n), dtype=torch.float64, device=DEVICE) if train else None

    def token(i):
        x, bc = at["x"][:, i].double(), at["bc"][:, i].double()
        raw = at["dt"][:, i].double()
        step = raw.clamp(min=0) + torch.log1p((-raw.abs()).exp())
        return x, bc[:, :n], bc[:, n:], raw, step, (step[:, :, None] * A).exp()

    for i in range(t):
        flag = keep[:, i, None, None]
        x, B, C, _, step, decay = token(i)
        before = state.masked_fill(flag == 2, 0.0)
        if train:
            came[i] = before
        new = before * decay + (step * x)[:, :, None] * B[:, None, :]
        state = torch.where(flag == 0, state, new)
        r = (new * C[:, None, :]).sum(2) + skip * x
        if gated:
            z = at["z"][:, i].double()
            r = r * z / (1 + (-z).exp())
        y[:, i] = r.masked_fill(flag[:, :, 0] == 0, 0.0)
    out = {"y": y.view(b * t, d), "hT": state}
    if not train:
        return out
    G = v["dhT"].double()
    made = {k: torch.zeros((b, t, d), dtype=torch.float64, device=DEVICE) for k in ("dx", "ddt") + (("dz",) if gated else ())}
    dbc = torch.zeros((b, t, 2 * n), dtype=torch.float64, device=DEVICE)
    dA, dskip = torch.zeros_like(A), torch.zeros_like(skip)
    for i in range(t - 1, -1, -1):
        flag = keep[:, i, None, None]
        flat = flag[:, :, 0] == 0
        x, B, C, raw, step, decay = token(i)
        du = at["dy"][:, i].double()
        before = came[i]
        new = before * decay + (step * x)[:, :, None] * B[:, None, :]
        if gated:
            z = at["z"][:, i].double()
            s = 1 / (1 + (-z).exp())
            r = (new * C[:, None, :]).sum(2) + skip * x
            made["dz"][:, i] = (du * r * (s + z * s * (1 - s))).masked_fill(flat, 0.0)
            du = du * z * s
        du = du.masked_fill(flat, 0.0)
        now = G + du[:, :, None] * C[:, None, :]
        use = now.masked_fill(flag == 0, 0.0)
        arg = use * before * decay                                # the derivative by step times A
        dstep = (arg * A).sum(2) + x * (use * B[:, None, :]).sum(2)
        made["dx"][:, i] = du * skip + step * (use * B[:, None, :]).sum(2)
        made["ddt"][:, i] = dstep / (1 + (-raw).exp())
        dbc[:, i, :n] = (use * (step * x)[:, :, None]).sum(1)
        dbc[:, i, n:] = (du[:, :, None] * new).sum(1)
        dA += (arg * step[:, :, None]).sum(0)
        dskip += (du * x).sum(0)
        G = torch.where(flag == 0, G, (now * decay).masked_fill(flag == 2, 0.0))
    out |= {k: g.view(b * t, d) for k, g in made.items()}
    return out | {"dbc": dbc.view(b * t, 2 * n), "da": dA, "dskip": dskip, "dh0": G}


def _exact_logprobs(case, v):
    found = {"lp": [], "lse": [], "dx": []}
    w = v["w"].double()
    wt = w.t().contiguous()
    dw = torch.zeros_like(w) if case["train"] else None
    m, n = case["rows"], case["vocab"]
    block = max(1, (1 << 27) // n)
    for i in range(0, m, block):                                  # rows by blocks, to bound the 64-bit logits
        x, tok = v["x"][i:i + block].double(), v["tok"][i:i + block].long()
        r = torch.arange(x.shape[0], device=DEVICE)
        logs = torch.mm(x, wt)
        lse = torch.logsumexp(logs, 1)
        given = (tok >= 0) & (tok < n)
        hit = tok.clamp(0, n - 1)
        found["lp"].append(torch.where(given, logs[r, hit] - lse, 0.0))
        found["lse"].append(lse)
        if case["train"]:
            dlp = torch.where(given, v["dlp"][i:i + block].double(), 0.0)
            dl = logs.sub_(lse[:, None]).exp_() * (v["dlse"][i:i + block].double() - dlp)[:, None]
            dl[r, hit] += dlp
            found["dx"].append(torch.mm(dl, w))
            dw += torch.mm(dl.t().contiguous(), x)
    out = {k: torch.cat(t) for k, t in found.items() if t}
    if case["train"]:
        out["dw"] = dw
    return out
