"""The local half of Algorithm 1 on resident replicas, as a program meets it: products with a model's matrices in both
directions, the norm of each worker's gradients with clipping, and the local update.

``own`` False: every operator in elementary torch operations, in 32 bits, rounded once at the end.
``own`` True: the same through ``paper_1909_09010_amd.binding``.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
ACTS = ("none", "relu", "gelu", "silu", "sigmoid", "tanh")
BLOCK = 8192                      # floats per block of a blocked state, the library's advice
DEV = "cuda:0"


# ---------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------
def _forward(name, dtype, workers, rows, outs, ins, act="none", bias=True, residual="none", pre=False):
    c = {"op": "forward", "dtype": dtype, "workers": workers, "rows": rows, "outs": outs, "ins": ins, "act": act,
         "bias": bias, "residual": residual, "pre": pre}
    return dict(c, name=name) if name else c


def _backward(name, dtype, workers, rows, outs, ins, act="none", bias=True, residual="none"):
    c = {"op": "backward", "dtype": dtype, "workers": workers, "rows": rows, "outs": outs, "ins": ins, "act": act,
         "bias": bias, "residual": residual}
    return dict(c, name=name) if name else c


def _grads(name, op, dtype, workers, vocab, embed, hidden, layers, **more):
    c = {"op": op, "dtype": dtype, "workers": workers, "vocab": vocab, "embed": embed, "hidden": hidden, "layers": layers,
         **more}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of each of the 4 tiny models: an LSTM layer's gates, the input's share being the residual
        _forward("token_gates_f32", "f32", 4, 1, 256, 64, act="sigmoid", residual="before"),
        # 8 hypotheses against a vocabulary of 50,000 words: one model that answers
        _forward("beams_vocabulary_bf16", "bf16", 1, 8, 50000, 1024),
        # a time step of training, 128 sequences, the 8 medium models' recurrent gates (650 is no multiple of 4)
        _forward("step_gates_f32", "f32", 8, 128, 2600, 650, act="tanh", residual="before", pre=True),
        # the projection of the paper's LSTMP layer over its batch of 5120 tokens, 16 workers
        _forward("projection_f32", "f32", 16, 5120, 512, 2048, residual="after"),
        # the head of its adaptive softmax, 8192 words and 5 tails: rows of an odd length
        _forward("softmax_head_bf16", "bf16", 8, 5120, 8197, 512),
        # the gradients of that layer's gates for the same batch
        _backward("gates_bf16", "bf16", 4, 5120, 8192, 1024, act="tanh"),
        # of the medium models' gates, 20 sequences of 35 tokens
        _backward("medium_gates_f32", "f32", 8, 700, 2600, 650, act="sigmoid", residual="before"),
        # of a small layer, 40 tokens
        _backward("small_layer_f16", "f16", 4, 40, 256, 64, act="relu"),
        # 36 small tensors: what launches cost
        _grads("clip_tiny_f32", "clip", "f32", 4, 1000, 64, 64, 2, max_norm=10.0),
        # 16 workers' gradients of the medium model
        _grads("clip_medium_f32", "clip", "f32", 16, 10000, 650, 650, 2, max_norm=10.0),
        # the local update, gradients in 16 bits, of the tiny models in rows and of medium ones in blocks
        _grads("step_tiny_bf16", "step", "bf16", 4, 1000, 64, 64, 2, max_norm=10.0, layout="rows", rule="adagrad"),
        _grads("step_medium_f32", "step", "f32", 16, 10000, 650, 650, 2, max_norm=10.0, layout="blocked", rule="adagrad"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Rows from a token to a batch, widths from the tiny model's to the vocabulary's, 1 to 16 workers."""
    op = rng.choice(("forward", "forward", "backward", "backward", "clip", "step"))
    dtype = rng.choice(("f32", "bf16", "f16"))
    if op in ("forward", "backward"):
        while True:
            workers, rows = _log(rng, 1, 16), _log(rng, 1, 5120)
            outs, ins = _log(rng, 64, 50000), _log(rng, 64, 2048)
            if rng.random() < 0.5:                     # models' widths are mostly round
                outs, ins = -(-outs // 64) * 64, -(-ins // 64) * 64
            size = workers * (rows * ins + outs * ins + 3 * rows * outs)
            if workers * rows * outs * ins <= (1.7e11 if op == "forward" else 8.5e10) and size <= 1.5e9:
                break
        act, bias = rng.choice(ACTS), rng.random() < 0.7
        residual = rng.choice(("none", "before", "after"))
        if op == "forward":
            return _forward(None, dtype, workers, rows, outs, ins, act, bias, residual, rng.random() < 0.4)
        return _backward(None, dtype, workers, rows, outs, ins, act, bias, residual)
    embed, hidden = _log(rng, 20, 650), _log(rng, 20, 650)
    shape = dict(workers=_log(rng, 1, 16), vocab=_log(rng, 50, 10000), embed=embed, hidden=hidden, layers=rng.randint(1, 2))
    max_norm = rng.choice((0.5, 10.0, 1e4))
    if op == "clip":
        return _grads(None, op, dtype, max_norm=max_norm, **shape)
    return _grads(None, op, dtype, max_norm=max_norm, layout=rng.choice(("rows", "blocked")),
                  rule=rng.choice(("adagrad", "adagrad", "sgd")), **shape)


def _shapes(c):
    """The tensors of an LSTM language model, in the order of the flat parameter vector."""
    h, out = c["hidden"], [(c["vocab"], c["embed"])]
    for layer in range(c["layers"]):
        out += [(4 * h, c["embed"] if layer == 0 else h), (4 * h, h), (4 * h,)]
    return out + [(c["vocab"], h), (c["vocab"],)]


def _params(c):
    return sum(math.prod(s) for s in _shapes(c))


def work(case):
    b, w = BYTES[case["dtype"]], case["workers"]
    if case["op"] in ("forward", "backward"):
        m, n, k = case["rows"], case["outs"], case["ins"]
        values = m * k + n * k + (n if case["bias"] else 0) + m * n
        if case["op"] == "forward":
            values += (m * n if case["residual"] != "none" else 0) + (m * n if case["pre"] else 0)
            return {"bytes": w * b * values, "flops": 2 * w * m * n * k}
        values += m * k + n * k + (m * n if case["act"] != "none" else 0) + (m * n if case["residual"] == "before" else 0)
        return {"bytes": w * b * values, "flops": 4 * w * m * n * k}
    n = w * _params(case)
    if case["op"] == "clip":
        return {"bytes": 2 * b * n + 4 * w, "flops": 3 * n}
    adagrad = case["rule"] == "adagrad"
    return {"bytes": (b + (16 if adagrad else 8)) * n + 4 * w, "flops": (9 if adagrad else 5) * n}


# ---------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------
def _randn(g, shape, scale, dtype):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt, G = TYPES[case["dtype"]], case["workers"]
    s = {"case": case}
    if case["op"] in ("forward", "backward"):
        m, n, k = case["rows"], case["outs"], case["ins"]
        # every worker's matrix and bias lie in its row of the replicas, padded to 1024 values
        row = torch.zeros((G, -(-(n * k + n) // 1024) * 1024), device=DEV, dtype=dt)
        row[:, : n * k + n] = _randn(g, (G, n * k + n), k ** -0.5, dt)
        s["w"] = row[:, : n * k].view(G, n, k)
        s["bias"] = row[:, n * k: n * k + n] if case["bias"] else None
        s["x"] = _randn(g, (G, m, k), 1.0, dt)
        if case["op"] == "forward":
            s["residual"] = _randn(g, (G, m, n), 1.0, dt) if case["residual"] != "none" else None
            s["y"] = torch.empty((G, m, n), device=DEV, dtype=dt)
            s["pre"] = torch.empty((G, m, n), device=DEV, dtype=dt) if case["pre"] else None
        else:
            s["dy"] = _randn(g, (G, m, n), 0.1, dt)
            s["pre"] = _randn(g, (G, m, n), 1.0, dt) if case["act"] != "none" else None
            s["dx"] = torch.empty((G, m, k), device=DEV, dtype=dt)
            grad = torch.zeros_like(row)                # gradients lie as the parameters do
            s["dw"] = grad[:, : n * k].view(G, n, k)
            s["dbias"] = grad[:, n * k: n * k + n] if case["bias"] else None
            s["dresidual"] = torch.empty((G, m, n), device=DEV, dtype=dt) if case["residual"] == "before" else None
        if own:
            _prepare_linear(s)
        return s
    shapes, P = _shapes(case), _params(case)
    s["grads"] = [[_randn(g, sh, 0.05, dt) for sh in shapes] for _ in range(G)]
    s["norms"] = torch.zeros(G, device=DEV)
    if case["op"] == "clip":
        # clipped gradients go into one row for each worker, in the order of the parameters
        s["rows"] = torch.empty((G, P), device=DEV, dtype=dt)
        s["out"] = []
        for w in range(G):
            parts = torch.split(s["rows"][w], [math.prod(sh) for sh in shapes])
            s["out"].append([p.view(sh) for p, sh in zip(parts, shapes)])
    else:
        if case["layout"] == "rows":
            width = -(-P // 1024) * 1024
            s["theta"] = torch.zeros((G, width), device=DEV)
            s["sums"] = torch.zeros((G, width), device=DEV)
            theta, sums = s["theta"], s["sums"]
        else:
            blocks = -(-P // BLOCK)                     # [block][theta, omega, delta][worker][floats]
            s["arena"] = torch.zeros((blocks, 3, G, BLOCK), device=DEV)
            s["theta"] = s["arena"][:, 0]
            s["sums"] = torch.zeros((blocks, G, BLOCK), device=DEV)
        for w in range(G):
            v = torch.randn(P, generator=g, device=DEV) * 0.05
            h = torch.rand(P, generator=g, device=DEV) * 0.2 + 0.1
            if case["layout"] == "rows":
                theta[w, :P], sums[w, :P] = v, h
            else:
                pad = torch.zeros(s["theta"].shape[0] * BLOCK - P, device=DEV)
                s["theta"][:, w] = torch.cat([v, pad]).view(-1, BLOCK)
                s["sums"][:, w] = torch.cat([h, pad]).view(-1, BLOCK)
    if own:
        _prepare_grads(s)
    return s


def _prepare_linear(s):
    from paper_1909_09010_amd import binding as B
    c = s["case"]
    lin = B.Linear(c["rows"], c["outs"], c["ins"], batch=c["workers"], dtype=TYPES[c["dtype"]],
                   activation=getattr(B, "ACT_" + c["act"].upper()),
                   residual=getattr(B, "RESIDUAL_" + c["residual"].upper()))
    s["linear"] = lin
    if c["op"] == "forward":
        s["io"] = lin.forward_io(s["x"], s["w"], s["y"], bias=s["bias"], residual=s["residual"], pre=s["pre"])
        need = lin.workspace_bytes()
    else:
        s["io"] = lin.backward_io(s["dy"], s["x"], s["w"], pre=s["pre"], dx=s["dx"], dw=s["dw"], dbias=s["dbias"],
                                  dresidual=s["dresidual"])
        need = lin.workspace_bytes(backward=True)
    s["workspace"] = torch.empty(max(need, 16), device=DEV, dtype=torch.uint8)


def _prepare_grads(s):
    from paper_1909_09010_amd import binding as B
    c = s["case"]
    s["handle"] = B.Grads(s["grads"])
    if c["op"] == "clip":
        s["handle_out"] = B.Grads(s["out"])
        return
    G = c["workers"]
    if c["layout"] == "rows":
        s["at"] = B.make_state(s["theta"], None, None, s["theta"].stride(0))
        s["sums_at"] = B.make_state(s["sums"], None, None, s["sums"].stride(0))
    else:
        s["at"] = B.make_state(s["theta"], None, None, BLOCK, BLOCK, 3 * G * BLOCK)
        s["sums_at"] = B.make_state(s["sums"], None, None, BLOCK, BLOCK, G * BLOCK)


# ---------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------
RATE, EPS = 0.1, 1e-7


def _act(z, kind):
    if kind == "none":
        return z
    if kind == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if kind == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if kind == "silu":
        return z / (1.0 + torch.exp(-z))
    if kind == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-z))
    return torch.tanh(z)


def _slope(z, kind):
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if kind == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    if kind == "sigmoid":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 - p)
    t = torch.tanh(z)
    return 1.0 - t * t


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    c, stream = s["case"], torch.cuda.current_stream()
    if c["op"] == "forward":
        s["linear"].forward(s["io"], s["workspace"], stream)
        return [t for t in (s["y"], s["pre"]) if t is not None]
    if c["op"] == "backward":
        s["linear"].backward(s["io"], s["workspace"], stream)
        return [t for t in (s["dx"], s["dw"], s["dbias"], s["dresidual"]) if t is not None]
    if c["op"] == "clip":
        s["handle"].clip(c["max_norm"], s["norms"], out=s["handle_out"], stream=stream)
        return [s["norms"], s["rows"]]
    adagrad = c["rule"] == "adagrad"
    s["handle"].local_step(s["at"], s["sums_at"] if adagrad else None, _params(c), RATE, EPS, c["max_norm"], s["norms"],
                           stream=stream)
    return [s["norms"], s["theta"]] + ([s["sums"]] if adagrad else [])


def _run_plain(s):
    c = s["case"]
    dt = TYPES[c["dtype"]]
    if c["op"] == "forward":
        z = torch.bmm(s["x"].float(), s["w"].float().transpose(1, 2).contiguous())
        if s["bias"] is not None:
            z = z + s["bias"].float()[:, None, :]
        if c["residual"] == "before":
            z = z + s["residual"].float()
        y = _act(z, c["act"])
        if c["residual"] == "after":
            y = y + s["residual"].float()
        return [y.to(dt)] + ([z.to(dt)] if c["pre"] else [])
    if c["op"] == "backward":
        dz = s["dy"].float()
        if c["act"] != "none":
            dz = dz * _slope(s["pre"].float(), c["act"])
        out = [torch.bmm(dz, s["w"].float()).to(dt), torch.bmm(dz.transpose(1, 2).contiguous(), s["x"].float()).to(dt)]
        if c["bias"]:
            out.append(dz.sum(1).to(dt))
        if c["residual"] == "before":
            out.append(dz.to(dt))
        return out
    scales = []
    for w, ts in enumerate(s["grads"]):
        total = torch.zeros((), device=DEV)
        for t in ts:
            f = t.float()
            total = total + (f * f).sum()
        s["norms"][w] = torch.sqrt(total)
        scales.append(torch.clamp(c["max_norm"] / s["norms"][w], max=1.0))
    if c["op"] == "clip":
        for w, ts in enumerate(s["grads"]):
            for t, o in zip(ts, s["out"][w]):
                if c["dtype"] == "f32":
                    torch.mul(t, scales[w], out=o)
                else:
                    o.copy_(t.float() * scales[w])
        return [s["norms"], s["rows"]]
    P = _params(c)
    for w, ts in enumerate(s["grads"]):
        flat = torch.cat([t.reshape(-1).float() for t in ts]) * scales[w]
        if c["layout"] == "rows":
            theta, sums = s["theta"][w, :P], s["sums"][w, :P]
        else:
            theta, sums = s["theta"][:, w], s["sums"][:, w]
            flat = torch.cat([flat, torch.zeros(theta.shape[0] * BLOCK - P, device=DEV)]).view(-1, BLOCK)
        if c["rule"] == "adagrad":
            sums += flat * flat
            theta -= RATE * flat / (torch.sqrt(sums) + EPS)
        else:
            theta -= RATE * flat
    return [s["norms"], s["theta"]] + ([s["sums"]] if c["rule"] == "adagrad" else [])


# ---------------------------------------------------------------------------------------------
# The definitions in 64 bits, worker by worker
# ---------------------------------------------------------------------------------------------
_EXACT = {
    "none": (lambda z: z, lambda z: torch.ones_like(z)),
    "relu": (lambda z: z.clamp(min=0), lambda z: (z > 0).double()),
    "gelu": (lambda z: z * (1 - 0.5 * torch.erfc(z / 2 ** 0.5)),
             lambda z: 1 - 0.5 * torch.erfc(z / 2 ** 0.5) + z * torch.exp(-z ** 2 / 2) / (2 * math.pi) ** 0.5),
    "silu": (lambda z: z * torch.sigmoid(z), lambda z: torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)),
    "sigmoid": (torch.sigmoid, lambda z: torch.sigmoid(z) * torch.sigmoid(-z)),
    "tanh": (torch.tanh, lambda z: torch.cosh(z) ** -2),
}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    G = case["workers"]
    if case["op"] in ("forward", "backward"):
        f, df = _EXACT[case["act"]]
        parts = []
        for g in range(G):
            x, w = s["x"][g].double(), s["w"][g].double()
            if case["op"] == "forward":
                z = x @ w.T.contiguous()
                z = z + s["bias"][g].double() if case["bias"] else z
                z = z + s["residual"][g].double() if case["residual"] == "before" else z
                y = f(z) + s["residual"][g].double() if case["residual"] == "after" else f(z)
                parts.append([y] + ([z] if case["pre"] else []))
            else:
                dz = s["dy"][g].double()
                dz = dz * df(s["pre"][g].double()) if case["act"] != "none" else dz
                parts.append([dz @ w, dz.T.contiguous() @ x] + ([dz.sum(0)] if case["bias"] else []) +
                             ([dz] if case["residual"] == "before" else []))
        return [torch.stack(p) for p in zip(*parts)]
    norms = torch.stack([torch.stack([t.double().square().sum() for t in ts]).sum().sqrt() for ts in s["grads"]])
    clip = torch.minimum(torch.ones_like(norms), case["max_norm"] / norms)
    if case["op"] == "clip":
        return [norms, torch.stack([torch.cat([t.double().flatten() for t in ts]) * clip[w] for w, ts in enumerate(s["grads"])])]
    P, adagrad = _params(case), case["rule"] == "adagrad"
    theta, sums = s["theta"].double(), s["sums"].double()
    for w, ts in enumerate(s["grads"]):
        g = torch.cat([t.double().flatten() for t in ts]) * clip[w]
        if case["layout"] == "rows":
            where = (torch.full((P,), w, device=DEV), torch.arange(P, device=DEV))
        else:
            e = torch.arange(P, device=DEV)
            where = (e // BLOCK, torch.full_like(e, w), e % BLOCK)
        if adagrad:
            h = sums[where] + g ** 2
            sums[where] = h
            theta[where] -= RATE * g / (h.sqrt() + EPS)
        else:
            theta[where] -= RATE * g
    return [norms, theta] + ([sums] if adagrad else [])
