"""The losses that resident replicas train on, as a program meets them: the cross entropy of a softmax over a large vocabulary and
distillation from a teacher's top logits, each from the hidden rows and the models' output matrices, with gradients.

``own`` False: every operator in elementary torch operations, in 32 bits, rounded once at the end.
``own`` True: the same through ``paper_1909_09010_amd.binding``, which keeps no logits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
DEV = "cuda:0"


# ---------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------
def _case(name, op, dtype, workers, rows, vocab, ins, bias=True, ignored=0.0, weighted=False, top=0, temperature=1.0):
    c = {"op": op, "dtype": dtype, "workers": workers, "rows": rows, "vocab": vocab, "ins": ins, "bias": bias, "ignored": ignored,
         "weighted": weighted, "top": top, "temperature": temperature}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a token of each of the 4 tiny models, scored
        _case("score_token_f32", "entropy", "f32", 4, 1, 1000, 64),
        # 8 hypotheses of one model against 50,000 words: what rescoring takes
        _case("score_beams_bf16", "entropy", "bf16", 1, 8, 50000, 1024),
        # 20 sequences of 35 tokens of the 8 medium models (650 is no multiple of 4), the ends of sequences padded
        _case("entropy_medium_f32", "entropy", "f32", 8, 700, 10000, 650, ignored=0.1),
        # the head of the paper's adaptive softmax, 8192 words and 5 tails, over its batch of 5120 tokens
        _case("entropy_head_bf16", "entropy", "bf16", 8, 5120, 8197, 512),
        # the same batch against the whole vocabulary of 267,735 words
        _case("entropy_vocabulary_bf16", "entropy", "bf16", 1, 5120, 267735, 512, bias=False),
        # the gradients of a mini-batch of 4 tiny models: what launches cost
        _case("entropy_grads_tiny_f16", "entropy_grads", "f16", 4, 40, 1000, 64),
        # of the medium models' mini-batch
        _case("entropy_grads_medium_f32", "entropy_grads", "f32", 8, 700, 10000, 650, ignored=0.1),
        # of two of the models of 50,000 words and width 1024, tokens weighted
        _case("entropy_grads_words_bf16", "entropy_grads", "bf16", 2, 5120, 50000, 1024, weighted=True),
        # 64 tokens of small models learning from 8 words of a teacher each
        _case("distill_small_f32", "distill", "f32", 4, 64, 1000, 64, top=8, temperature=2.0),
        # the head again, 64 words of a teacher a token
        _case("distill_head_bf16", "distill", "bf16", 8, 5120, 8197, 512, ignored=0.1, top=64, temperature=2.0),
        # the gradients of the medium models' mini-batch, odd numbers throughout
        _case("distill_grads_medium_f16", "distill_grads", "f16", 8, 699, 10001, 650, ignored=0.1, top=19, temperature=1.5),
        # and of the head's batch
        _case("distill_grads_head_bf16", "distill_grads", "bf16", 8, 5120, 8197, 512, top=64, temperature=2.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """From a token to a batch of them, from a small vocabulary to the whole one, 1 to 16 workers."""
    op = rng.choice(("entropy", "entropy_grads", "distill", "distill_grads"))
    dtype = rng.choice(("f32", "bf16", "f16"))
    grads = op.endswith("grads")
    while True:
        workers, rows = _log(rng, 1, 16), _log(rng, 1, 5120)
        vocab, ins = _log(rng, 200, 267735), _log(rng, 32, 1024)
        if rng.random() < 0.5:                          # models' widths are mostly round
            vocab, ins = -(-vocab // 64) * 64, -(-ins // 64) * 64
        logits, weights = workers * rows * vocab, workers * vocab * ins
        if logits <= (5e8 if grads else 1.3e9) and logits * ins <= (5e11 if grads else 7e11) and weights <= 3e8:
            break
    distill = op.startswith("distill")
    return _case(None, op, dtype, workers, rows, vocab, ins, rng.random() < 0.7, rng.choice((0.0, 0.1, 0.4)), rng.random() < 0.3,
                 _log(rng, 1, 128) if distill else 0, rng.choice((1.0, 1.5, 4.0)) if distill else 1.0)


def _padded(c):
    """Rows of every worker that count for nothing."""
    return int(c["rows"] * c["ignored"])


def work(case):
    b, G, M, V, K, T = (BYTES[case["dtype"]], *(case[k] for k in ("workers", "rows", "vocab", "ins", "top")))
    live = M - _padded(case)
    inputs = b * (live * K + V * K + (V if case["bias"] else 0)) + (12 * live * T if T else 0) + (0 if T else 8 * M)
    if not case["op"].endswith("grads"):
        return {"bytes": G * (inputs + 8 * M), "flops": 2 * G * live * V * K}
    outputs = b * (M * K + V * K + (V if case["bias"] else 0))
    return {"bytes": G * (inputs + 8 * live + outputs), "flops": 6 * G * live * V * K}


# ---------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------
def _randn(g, shape, scale, dtype):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = TYPES[case["dtype"]]
    G, M, V, K, T = (case[k] for k in ("workers", "rows", "vocab", "ins", "top"))
    s = {"case": case}
    # every worker's matrix and bias lie in its row of the replicas, padded to 1024 values
    row = torch.zeros((G, -(-(V * K + V) // 1024) * 1024), device=DEV, dtype=dt)
    row[:, : V * K] = _randn(g, (G, V * K), 2.0 * K ** -0.5, dt)
    s["w"] = row[:, : V * K].view(G, V, K)
    # words in the order of their frequency, which falls as one over their rank
    frequency = -torch.log(torch.arange(1, V + 1, device=DEV, dtype=torch.float32))
    row[:, V * K: V * K + V] = (frequency + torch.randn((G, V), generator=g, device=DEV) * 0.3).to(dt)
    s["bias"] = row[:, V * K: V * K + V] if case["bias"] else None
    s["x"] = _randn(g, (G, M, K), 1.0, dt)
    word = (torch.exp(torch.rand((G, M), generator=g, device=DEV, dtype=torch.float64) * math.log(V + 1)).long() - 1).clamp(0, V - 1)
    padded = torch.zeros((G, M), device=DEV, dtype=torch.bool)
    if _padded(case):
        order = torch.argsort(torch.rand((G, M), generator=g, device=DEV), 1)
        padded.scatter_(1, order[:, : _padded(case)], True)
    if T == 0:
        s["target"] = torch.where(padded, torch.full_like(word, -100), word)
    else:
        T = min(T, V)
        # the teacher's words: the target and others at random distances from it, no word twice, in no order
        gaps = (torch.rand((G, M, T), generator=g, device=DEV) * (V // T)).long().clamp(max=V // T - 1) + 1
        gaps[:, :, 0] = 0
        ids = (word[:, :, None] + torch.cumsum(gaps, 2)) % V
        s["teacher"] = torch.cumsum(torch.rand((G, M, T), generator=g, device=DEV) * (-8.0 / T), 2)
        kept = torch.randint(1, 2 * T + 1, (G, M, 1), generator=g, device=DEV)         # half of the tokens have fewer words
        ids = torch.where((torch.arange(T, device=DEV) < kept) & ~padded[:, :, None], ids, torch.full_like(ids, -1))
        s["target"] = ids.contiguous()
    if not case["op"].endswith("grads"):
        s["loss"], s["lse"] = (torch.empty((G, M), device=DEV) for _ in range(2))
    else:
        live = (~padded).sum(1, keepdim=True).clamp(min=1)
        s["dloss"] = (1.0 / live.float()).expand(G, M)
        if case["weighted"]:
            s["dloss"] = s["dloss"] * (torch.rand((G, M), generator=g, device=DEV) + 0.5)
        s["lse"] = torch.zeros((G, M), device=DEV)       # as the forward left it
        for w in range(G):
            for i in range(0, M, 1024):
                z = s["x"][w, i: i + 1024].float() @ s["w"][w].float().T.contiguous()
                z = z + s["bias"][w].float() if case["bias"] else z
                s["lse"][w, i: i + 1024] = torch.logsumexp(z / case["temperature"], 1)
        s["lse"].masked_fill_(padded, 0.0)
        s["dx"] = torch.empty((G, M, K), device=DEV, dtype=dt)
        grad = torch.zeros_like(row)                      # gradients lie as the parameters do
        s["dw"] = grad[:, : V * K].view(G, V, K)
        s["dbias"] = grad[:, V * K: V * K + V] if case["bias"] else None
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    from paper_1909_09010_amd import binding as B
    c = s["case"]
    grads = c["op"].endswith("grads")
    if c["top"]:
        h = B.Distill(c["rows"], c["vocab"], c["ins"], s["target"].shape[2], c["temperature"], batch=c["workers"], dtype=TYPES[c["dtype"]])
        words = (s["target"], s["teacher"])
    else:
        h = B.CrossEntropy(c["rows"], c["vocab"], c["ins"], batch=c["workers"], dtype=TYPES[c["dtype"]])
        words = (s["target"],)
    if grads:
        s["io"] = h.backward_io(s["x"], s["w"], *words, s["lse"], s["dloss"], bias=s["bias"], dx=s["dx"], dw=s["dw"], dbias=s["dbias"])
    else:
        s["io"] = h.forward_io(s["x"], s["w"], *words, s["loss"], s["lse"], bias=s["bias"])
    s["operator"] = h
    s["workspace"] = torch.empty(max(h.workspace_bytes(backward=grads), 16), device=DEV, dtype=torch.uint8)


# ---------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    stream = torch.cuda.current_stream()
    if s["case"]["op"].endswith("grads"):
        s["operator"].backward(s["io"], s["workspace"], stream)
        return [t for t in (s["dx"], s["dw"], s["dbias"]) if t is not None]
    s["operator"].forward(s["io"], s["workspace"], stream)
    return [s["loss"], s["lse"]]


def _teacher(s):
    """Words that stand for nothing as 0, with no share; the shares of the others; which rows have any."""
    present = s["target"] >= 0
    t = torch.where(present, s["teacher"] / s["case"]["temperature"], torch.full_like(s["teacher"], -math.inf))
    most = t.amax(2, keepdim=True)
    e = torch.where(present, torch.exp(t - most), torch.zeros_like(t))
    total = e.sum(2, keepdim=True)
    return s["target"].clamp(min=0), e / torch.where(total > 0, total, torch.ones_like(total)), present.any(2)


def _run_plain(s):
    c = s["case"]
    tau, dt = c["temperature"], TYPES[c["dtype"]]
    x, w = s["x"].float(), s["w"].float()
    z = torch.bmm(x, w.transpose(1, 2).contiguous())
    if c["bias"]:
        z += s["bias"].float()[:, None, :]
    if c["top"]:
        ids, share, live = _teacher(s)
        z /= tau
    else:
        ids, live = s["target"].clamp(min=0)[:, :, None], s["target"] >= 0
        share = torch.ones_like(ids, dtype=torch.float32)
    nothing = torch.zeros((), device=DEV)
    if not c["op"].endswith("grads"):
        most = z.amax(2, keepdim=True)
        at = z.gather(2, ids)
        lse = torch.log(torch.exp(z.sub_(most)).sum(2)) + most[:, :, 0]
        if c["top"]:
            terms = torch.where(share > 0, share * (torch.log(share) - at + lse[:, :, None]), nothing)
            loss = tau * tau * terms.sum(2)
        else:
            loss = lse - at[:, :, 0]
        return [torch.where(live, loss, nothing), torch.where(live, lse, nothing)]
    dz = torch.exp(z.sub_(s["lse"][:, :, None]))
    dz.scatter_add_(2, ids, -share)
    dz = torch.where(live[:, :, None], dz * (tau * s["dloss"])[:, :, None], nothing)
    out = [torch.bmm(dz, w).to(dt)]
    s["dw"].copy_(torch.bmm(dz.transpose(1, 2).contiguous(), x))
    return out + [s["dw"]] + ([dz.sum(1).to(dt)] if c["bias"] else [])


# ---------------------------------------------------------------------------------------------
# The definitions in 64 bits, worker by worker, some rows at a time
# ---------------------------------------------------------------------------------------------
def _exact_rows(c, s, g, rows):
    """Logits over the temperature, and the distribution that they are held to, zero for rows that count for nothing."""
    z = s["x"][g, rows].double() @ s["w"][g].double().T.contiguous()
    if c["bias"]:
        z += s["bias"][g].double()
    z /= c["temperature"]
    word = s["target"][g, rows]
    if c["top"]:
        t = (s["teacher"][g, rows].double() / c["temperature"]).masked_fill(word < 0, -math.inf)
        p = torch.softmax(t, 1).masked_fill(word < 0, 0.0)          # rows without a word: NaN, masked
        live = (word >= 0).any(1)
        return z, word.clamp(min=0), p, live
    return z, word.clamp(min=0)[:, None], (word >= 0).double()[:, None], word >= 0


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    G, M, tau = case["workers"], case["rows"], case["temperature"]
    step = max(1, min(M, 200_000_000 // case["vocab"]))
    parts = []
    for g in range(G):
        loss, lse, dx, dw, db = [], [], [], 0.0, 0.0
        for i in range(0, M, step):
            rows = slice(i, min(i + step, M))
            z, word, p, live = _exact_rows(case, s, g, rows)
            if not case["op"].endswith("grads"):
                n = torch.logsumexp(z, 1)
                logq = z.gather(1, word) - n[:, None]
                loss.append(tau ** 2 * (torch.special.xlogy(p, p) - torch.where(p > 0, p * logq, 0.0 * p)).sum(1) * live)
                lse.append(torch.where(live, n, torch.zeros_like(n)))
                continue
            dz = torch.exp(z - s["lse"][g, rows].double()[:, None])
            dz.scatter_add_(1, word, -p)
            dz *= torch.where(live, tau * s["dloss"][g, rows].double(), torch.zeros_like(s["lse"][g, rows]).double())[:, None]
            dx.append(dz @ s["w"][g].double())
            dw = dw + dz.T.contiguous() @ s["x"][g, rows].double()
            db = db + dz.sum(0)
        if case["op"].endswith("grads"):
            parts.append([torch.cat(dx), dw] + ([db] if case["bias"] else []))
        else:
            parts.append([torch.cat(loss), torch.cat(lse)])
    return [torch.stack(p) for p in zip(*parts)]
