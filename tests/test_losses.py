"""Cross entropy over a vocabulary and distillation from a teacher's top logits, against the formulas in 64 bits.

Bounds, derived before any run (u = 2^-24, S = the sum of the magnitudes of what is added up):
  a logit: a sum of K products in f32, whatever its order: 2 (K + 16) u S (matrix instructions may round by cutting); f32 operands taken apart: 2^-21 S
  and 2^-39 of the largest of each row against the other operand's sum of magnitudes;
  lse: the largest error of the row's logits over tau (the derivatives are probabilities); an exponential of d is off by (4 |d| + 8) u, weighted by the
  probabilities again; adding up 400 u, since no value passes more additions on its way; a few roundings of lse itself;
  a share q of the teacher: (8 |s - most| / tau + top + 16) u;
  dz = weight (p - q): p as lse's terms, the rest roundings; 16-bit types in large sizes: half a unit of dz (f16: and 2^-25 of what its largest weight
  is below 2^15, 2^-39 of that weight);
  dx, dw: sums as of logits over dz and its errors; rounding to the type at the end: half a unit, 2^-8 (bf16), 2^-11 (f16, and 2^-25 below its normal range).
Errors of many roundings do not add up all one way: their root mean square is held to 2^-21 of S's and the roundings' own.  Those of dz: p is off by what its
logit is off, 2^-21 S, by half a unit of each of d = z / tau - lse, d log2 e (u |d| p both), the exponential (2 u p) and the product with the weight (u p), and
q by u for that product and the subtraction: where p is near q, dz itself says nothing of its error.
"""
import ctypes
import math

import pytest
import torch

from paper_1909_09010_amd import binding as B

DEV = "cuda:0"
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
U = 2.0 ** -24
gpu = pytest.mark.gpu
INF = float("inf")


def mm(a, b):
    """a b' for every worker, in 64 bits."""
    return torch.stack([x.double() @ y.double().T.contiguous() for x, y in zip(a, b)]) if a.shape[0] else torch.zeros(0, a.shape[1], b.shape[1], dtype=torch.float64,
                                                                                                                       device=a.device)


def spread(a, b):
    """2^-39 of a row's largest meets every value of the other operand."""
    if a.shape[-1] == 0 or a.numel() == 0 or b.numel() == 0:
        return torch.zeros(a.shape[0], a.shape[1], b.shape[1], dtype=torch.float64, device=a.device)
    a, b = a.double().abs(), b.double().abs()
    return a.amax(2)[:, :, None] * b.sum(2)[:, None, :] + a.sum(2)[:, :, None] * b.amax(2)[:, None, :]


def sum_bound(a, b, dtype):
    S = mm(a.abs(), b.abs())
    bound = (2 * a.shape[2] + 32) * U * S
    if dtype == torch.float32:
        bound = bound + 2.0 ** -21 * S + 2.0 ** -39 * spread(a, b)
    return bound, S


def check(got, want, bound, rms, what):
    """Element by element within `bound`, the root mean square of the errors within `rms`."""
    got, want = got.detach().double(), want.double()
    assert got.shape == want.shape, what
    if got.numel() == 0:
        return
    assert torch.isfinite(got).all(), what
    err = (got - want).abs()
    worst = (err - bound).max().item()
    assert worst <= 0, f"{what}: {worst:.3g} beyond the bound, error {err.max().item():.3g}"
    e, r = err.square().mean().sqrt().item(), rms.square().mean().sqrt().item()
    assert e <= r, f"{what}: rms error {e:.3g}, bound {r:.3g}"


class Case:
    """Inputs on the device, and what 64 bits make of them."""

    def __init__(self, G, M, V, K, dtype, top=0, tau=1.0, bias=True, ignored=0.2, seed=0, place=None, weighted=True, shared=()):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.size, self.dtype, self.top, self.tau = (G, M, V, K), dtype, top, tau
        place = place or {}
        put = lambda name, t: place.get(name, lambda v: v)(t)
        randn = lambda *s: torch.randn(s, generator=g, device=DEV)
        rand = lambda *s: torch.rand(s, generator=g, device=DEV)
        self.x = put("x", randn(G, M, K).to(dtype))
        self.w = put("w", (randn(G, V, K) * 2 * max(K, 1) ** -0.5).to(dtype))
        if "x" in shared:
            self.x = self.x[:1].expand(G, -1, -1)
        if "w" in shared:
            self.w = self.w[:1].expand(G, -1, -1)
        self.bias = put("bias", randn(G, V).to(dtype)) if bias else None
        dead = rand(G, M) < ignored
        if top == 0:
            t = (rand(G, M).square() * V).long().clamp(max=max(V - 1, 0))
            self.words, self.teacher = put("words", torch.where(dead, torch.full_like(t, -100), t)), None
        else:
            ids = (rand(G, M, top) * V).long().clamp(max=max(V - 1, 0))                    # the same word twice now and then
            gone = (rand(G, M, top) < 0.2) | dead[:, :, None]
            self.words = put("words", torch.where(gone, torch.full_like(ids, -1), ids))
            self.teacher = put("teacher", randn(G, M, top) * 2)
        d = rand(G, M) + 0.5 if weighted else torch.ones(G, 1, device=DEV).expand(G, M)
        self.dloss = put("dloss", d / max(M, 1))

    def operator(self, **k):
        G, M, V, K = self.size
        if self.top:
            return B.Distill(M, V, K, self.top, self.tau, G, self.dtype, **k)
        return B.CrossEntropy(M, V, K, G, self.dtype, **k)

    def held(self):
        return (self.words, self.teacher) if self.top else (self.words,)

    def solve(self):
        """z / tau, lse, loss, dz and their bounds, in 64 bits."""
        G, M, V, K = self.size
        tau = self.tau
        bz, S = sum_bound(self.x, self.w, self.dtype)
        z = mm(self.x, self.w)
        if self.bias is not None:
            z, S = z + self.bias.double()[:, None], S + self.bias.double().abs()[:, None]
        z, bz, S = z / tau, (bz + 4 * U * S) / tau, S / tau
        if self.top:
            there = (self.words >= 0) & (self.teacher > -INF)
            s = self.teacher.double().masked_fill(~there, -INF) / tau
            q = torch.softmax(s, 2).masked_fill(~there, 0.0)
            off = (s - s.amax(2, keepdim=True)).abs().masked_fill(~there, 0.0)
            eq = q * (8 * off + self.top + 16) * U
        else:
            there = (self.words >= 0)[:, :, None]
            q = there.double()
            eq = torch.zeros_like(q)
        words = (self.words if self.top else self.words[:, :, None]).clamp(min=0)
        live = there.any(2)
        self.live = live
        lse = torch.logsumexp(z, 2)
        p = torch.exp(z - lse[:, :, None])
        d = (z - lse[:, :, None]).abs()
        elogit = bz.amax(2) if V else torch.zeros_like(lse)
        self.e_lse = elogit + U * ((p * (4 * d + 8)).sum(2) + 400 + 8 * lse.abs())
        self.r_lse = 2.0 ** -21 * (S.amax(2) if V else lse) + U * (32 + 4 * lse.abs() + (p * d).sum(2))
        self.lse = torch.where(live, lse, torch.zeros_like(lse))
        at, eat = z.gather(2, words) if V else torch.zeros_like(q), bz.gather(2, words) if V else torch.zeros_like(q)
        logq = torch.where(q > 0, torch.log(q.clamp(min=1e-300)), torch.zeros_like(q))
        term = torch.where(q > 0, logq - at + lse[:, :, None], torch.zeros_like(q))
        self.loss = tau ** 2 * (q * term).sum(2)
        size = logq.abs() + at.abs() + lse.abs()[:, :, None] + 1
        self.e_loss = tau ** 2 * (q * (self.e_lse[:, :, None] + eat + 8 * U * size) + 2 * eq * (term.abs() + 1) + U * (self.top + 8) * q * term.abs()).sum(2)
        self.r_loss = tau ** 2 * (self.r_lse + (q * (2.0 ** -21 * (S.gather(2, words) if V else q) + 4 * U * size)).sum(2))
        # gradients: from the lse that the library is handed, which is this one rounded to f32
        self.lse32 = self.lse.float()
        lse = self.lse32.double()[:, :, None]
        p = torch.exp(z - lse)
        weight = torch.where(live, tau * self.dloss.double(), torch.zeros_like(self.lse))[:, :, None]
        share = torch.zeros_like(z).scatter_add_(2, words, q) if V else torch.zeros_like(z)
        dz = torch.where(live[:, :, None], weight * (p - share), torch.zeros_like(p))
        more = torch.zeros_like(z).scatter_add_(2, words, eq) if V else torch.zeros_like(z)
        edz = weight.abs() * (p * (bz + U * (4 * (z - lse).abs() + 16)) + more + (self.top + 4) * U * share)
        edz = torch.where(live[:, :, None], edz, torch.zeros_like(edz))
        self.rdz = weight.abs() * (p * (2.0 ** -21 * S + U * (2 * (z - lse).abs() + 4)) + more + 2 * U * share)
        self.rdz = torch.where(live[:, :, None], self.rdz, torch.zeros_like(edz))
        return dz, edz


def run_forward(c, op=None, lse=True, workspace=None, stream=None):
    G, M = c.size[:2]
    op = op or c.operator()
    loss, n = torch.full((G, M), 7.0, device=DEV), torch.full((G, M), 7.0, device=DEV) if lse else None
    ws = workspace if workspace is not None else torch.empty(max(op.workspace_bytes(), 256), dtype=torch.uint8, device=DEV)
    op.forward(op.forward_io(c.x, c.w, *c.held(), loss, n, bias=c.bias), ws, stream)
    return loss, n


def grad_outputs(c, want, gt, place=None):
    G, M, V, K = c.size
    place = place or {}
    new = {"dx": lambda: torch.full((G, M, K), 7.0, dtype=c.dtype, device=DEV), "dw": lambda: torch.full((G, V, K), 7.0, dtype=gt, device=DEV),
           "dbias": lambda: torch.full((G, V), 7.0, dtype=gt, device=DEV)}
    return {n: place.get(n, lambda v: v)(new[n]()) for n in want}


def run_case(c, want=("dx", "dw", "dbias"), f32_grads=False, accumulate=False, place=None):
    """Forward and backward of a case, checked."""
    G, M, V, K = c.size
    dz, edz = c.solve()
    op = c.operator(weight_grad_f32=f32_grads, accumulate=accumulate)
    loss, lse = run_forward(c, op)
    torch.cuda.synchronize()
    zero = torch.zeros_like(c.lse)
    check(lse, c.lse, torch.where(c.live, c.e_lse, zero), c.r_lse + U, "lse")
    check(loss, torch.where(c.live, c.loss, zero), torch.where(c.live, c.e_loss, zero), c.r_loss + U, "loss")
    assert (loss[~c.live] == 0).all() and (lse[~c.live] == 0).all()
    gt = torch.float32 if f32_grads else c.dtype
    out = grad_outputs(c, want, gt, place)
    ws = torch.empty(max(op.workspace_bytes(True), 256), dtype=torch.uint8, device=DEV)
    op.backward(op.backward_io(c.x, c.w, *c.held(), c.lse32, c.dloss, bias=c.bias, **out), ws)
    torch.cuda.synchronize()
    h = HALF[c.dtype]
    rounded = torch.zeros_like(dz)
    if c.dtype != torch.float32:
        rounded = h * dz.abs()
        if c.dtype == torch.float16 and M:
            rounded = rounded + 2.0 ** -39 * (c.tau * c.dloss.double().abs()).amax(1)[:, None, None]
    was = 7.0 if accumulate else 0.0
    if "dx" in out:
        live = c.live[:, :, None]
        want_dx = mm(dz, c.w.transpose(1, 2))
        b, S = sum_bound(dz, c.w.double().transpose(1, 2), c.dtype)
        b = b + mm(edz + rounded, c.w.abs().transpose(1, 2))
        r = 2.0 ** -21 * S + mm(rounded ** 2 + c.rdz ** 2, c.w.double().transpose(1, 2) ** 2).sqrt()
        b = torch.where(live, b + h * (want_dx.abs() + b) + 2.0 ** -25, torch.zeros_like(b))
        check(out["dx"], want_dx, b, r + h * want_dx.abs() + 2.0 ** -25, "dx")
    hg = HALF[gt]
    x = torch.where(c.live[:, :, None], c.x.double(), torch.zeros((), dtype=torch.float64, device=DEV))
    if "dw" in out:
        want_dw = mm(dz.transpose(1, 2), x.transpose(1, 2))
        b, S = sum_bound(dz.transpose(1, 2), x.transpose(1, 2), c.dtype)
        b = b + mm((edz + rounded).transpose(1, 2), x.abs().transpose(1, 2))
        r = 2.0 ** -21 * (S + was) + mm((rounded ** 2 + c.rdz ** 2).transpose(1, 2), (x ** 2).transpose(1, 2)).sqrt()
        want_dw = want_dw + was
        check(out["dw"], want_dw, b + U * was + hg * (want_dw.abs() + b) + 2.0 ** -25, r + hg * want_dw.abs() + 2.0 ** -25, "dw")
    if "dbias" in out:
        want_db, S = dz.sum(1) + was, dz.abs().sum(1)
        b = edz.sum(1) + (2 * M + 32) * U * S + U * was
        check(out["dbias"], want_db, b + hg * (want_db.abs() + b) + 2.0 ** -25, 2.0 ** -20 * (S + was) + edz.sum(1) + hg * want_db.abs() + 2.0 ** -25, "dbias")
    return out


# workers, rows, vocabulary, features
SIZES = [(1, 1, 1, 1), (4, 1, 1000, 64), (2, 3, 5, 7), (1, 8, 5000, 1024), (3, 17, 33, 65), (2, 40, 300, 64), (2, 129, 257, 130), (1, 300, 130, 31),
         (1, 64, 64, 2050), (5, 2, 70, 200), (2, 33, 300, 72), (1, 700, 1001, 64), (2, 65, 4100, 2), (3, 256, 512, 128), (1, 1000, 8, 24), (2, 500, 2100, 40),
         (1, 5, 40009, 24), (1, 20, 33000, 64), (2, 50, 17000, 48)]


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES)
def test_cross_entropy(size, dtype):
    i = SIZES.index(size)
    run_case(Case(*size, dtype, bias=i % 3 != 1, seed=i), f32_grads=i % 4 == 2, accumulate=i % 2 == 1)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES)
def test_distill(size, dtype):
    i = SIZES.index(size)
    run_case(Case(*size, dtype, top=(1, 5, 64, 17, 130)[i % 5], tau=(1.0, 2.0, 0.7)[i % 3], bias=i % 3 != 1, seed=i), f32_grads=i % 4 == 2,
             accumulate=i % 2 == 1)


# tiles of 256 x 256 and of 128 x 128, operands laid out, sums cut between workgroups
LARGE = [(2, 2100, 8197, 520), (1, 1030, 20001, 130), (8, 700, 1500, 650), (1, 5120, 3000, 72), (3, 515, 2048, 1024), (16, 256, 1024, 264)]


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", LARGE)
@pytest.mark.parametrize("top", [0, 19])
def test_large(size, dtype, top):
    i = LARGE.index(size)
    run_case(Case(*size, dtype, top=top, tau=1.5 if top else 1.0, seed=i, weighted=i % 2 == 0), f32_grads=i % 2 == 1, accumulate=i % 3 == 1)


# more of the gradient than is held at a time: parts of a vocabulary, and some of the workers
PIECES = [(1, 2600, 160003, 40), (3, 2000, 120001, 24)]


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", PIECES)
def test_pieces(size, dtype):
    run_case(Case(*size, dtype, top=0 if size[0] == 1 else 7, seed=3, tau=1.0 if size[0] == 1 else 2.0))


@gpu
@pytest.mark.parametrize("top", [255, 256, 257, 1000, 1024])
def test_long_lists_of_words(top):
    run_case(Case(2, 30, 900, 40, torch.float32, top=top, tau=3.0, seed=top))
    run_case(Case(1, 200, 3000, 64, torch.bfloat16, top=top, tau=1.0, seed=top))


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(2, 0, 8, 8), (0, 8, 8, 8), (2, 8, 9, 0), (1, 300, 3, 0), (2, 70, 600, 0)])
@pytest.mark.parametrize("top", [0, 3])
def test_empty(size, dtype, top):
    run_case(Case(*size, dtype, top=top, seed=1))


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [3, 200])
def test_no_vocabulary(dtype, M):
    """Nothing to sum over: lse is -infinity and no row can name a word; what counts for nothing stays 0."""
    c = Case(2, M, 0, 8, dtype, ignored=2.0)
    loss, lse = run_forward(c)
    assert (loss == 0).all() and (lse == 0).all()
    op, out = c.operator(), grad_outputs(c, ("dx", "dw", "dbias"), dtype)
    ws = torch.empty(max(op.workspace_bytes(True), 256), dtype=torch.uint8, device=DEV)
    op.backward(op.backward_io(c.x, c.w, *c.held(), lse, c.dloss, bias=c.bias, **out), ws)
    assert (out["dx"] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(3, 60, 210, 40), (2, 600, 1300, 200)])
@pytest.mark.parametrize("top", [0, 4])
def test_each_output_alone(size, dtype, top):
    for want in (("dx",), ("dw",), ("dbias",), ("dx", "dbias"), ("dw", "dbias")):
        run_case(Case(*size, dtype, top=top, seed=5), want=want, accumulate="dw" in want)
    c = Case(*size, dtype, top=top, seed=5)
    a, _ = run_forward(c)
    b, _ = run_forward(c, lse=False)
    assert torch.equal(a, b)
    op = c.operator()
    op.backward(op.backward_io(c.x, c.w, *c.held(), a, c.dloss, bias=c.bias), torch.empty(op.workspace_bytes(True), dtype=torch.uint8, device=DEV))


# -- placements -----------------------------------------------------------------------------------
def in_rows(offset, stride):
    """Matrices in workers' rows of `stride` values from `offset` on, as tensors lie in theta."""
    def put(t):
        buf = torch.full((t.shape[0], stride), 5.0, dtype=t.dtype, device=DEV)
        v = buf[:, offset: offset + t[0].numel()].view(t.shape)
        v.copy_(t)
        return v
    return put


def columns_of(width, offset):
    def put(t):
        buf = torch.full((*t.shape[:2], width), 5, dtype=t.dtype, device=DEV)
        v = buf[:, :, offset: offset + t.shape[2]]
        v.copy_(t)
        return v
    return put


def tokens_first(t):
    v = torch.empty((t.shape[1], t.shape[0], *t.shape[2:]), dtype=t.dtype, device=DEV).transpose(0, 1)
    v.copy_(t)
    return v


def every_third(t):
    v = torch.full((*t.shape, 3), 5, dtype=t.dtype, device=DEV)[..., 1]
    v.copy_(t)
    return v


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(3, 3, 77, 136), (3, 40, 300, 136), (3, 200, 77, 136), (2, 700, 1500, 264)])
@pytest.mark.parametrize("top", [0, 6])
def test_placements(size, dtype, top):
    G, M, V, K = size
    for place in ({"w": in_rows(5, V * K + 11), "bias": in_rows(3, V + 5), "dw": in_rows(1, V * K + 3), "dbias": in_rows(7, V + 9)},
                  {"x": columns_of(K + 14, 3), "w": columns_of(K + 24, 16), "dx": columns_of(K + 5, 1), "dloss": every_third},
                  {"x": tokens_first, "dx": tokens_first, "words": tokens_first, "dloss": tokens_first, "w": columns_of(K + 8, 8)}):
        if top:
            place = {**place, "words": columns_of(top + 3, 2), "teacher": columns_of(top + 1, 1)}
        else:
            place = {**place, "words": place.get("words", every_third)}
        run_case(Case(*size, dtype, top=top, seed=2, place=place), place=place)
    run_case(Case(*size, dtype, top=top, seed=2, shared=("x",)))
    run_case(Case(*size, dtype, top=top, seed=2, shared=("w",)))
    run_case(Case(*size, dtype, top=top, seed=2, shared=("x", "w"), bias=False))


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [1, 30, 64, 130, 520])
@pytest.mark.parametrize("top", [0, 5])
def test_nothing_beside_the_outputs_is_written(dtype, M, top):
    G, V, K = 2, 1067, 72
    c = Case(G, M, V, K, dtype, top=top, seed=M)
    op = c.operator()
    for backward in (False, True):
        need = op.workspace_bytes(backward)
        ws = torch.full((need + 512,), 17, dtype=torch.uint8, device=DEV)
        wide = lambda *s, t=dtype: torch.full(s, 3.0, dtype=t, device=DEV)
        if backward:
            bx, bw, bb = wide(G, M + 2, K + 6), wide(G, V + 2, K + 6), wide(G, V + 6)
            c.solve()
            op.backward(op.backward_io(c.x, c.w, *c.held(), c.lse32, c.dloss, bias=c.bias, dx=bx[:, 1: M + 1, 3: K + 3], dw=bw[:, 1: V + 1, 3: K + 3],
                                       dbias=bb[:, 3: V + 3]), ws[:need])
            torch.cuda.synchronize()
            bx[:, 1: M + 1, 3: K + 3], bw[:, 1: V + 1, 3: K + 3], bb[:, 3: V + 3] = 3.0, 3.0, 3.0
            assert (bx == 3).all() and (bw == 3).all() and (bb == 3).all()
        else:
            bl, bn = wide(G, M + 2, t=torch.float32), wide(G, M + 2, t=torch.float32)
            op.forward(op.forward_io(c.x, c.w, *c.held(), bl[:, 1: M + 1], bn[:, 1: M + 1], bias=c.bias), ws[:need])
            torch.cuda.synchronize()
            bl[:, 1: M + 1], bn[:, 1: M + 1] = 3.0, 3.0
            assert (bl == 3).all() and (bn == 3).all()
        assert (ws[need:] == 17).all()


# -- rows that do not count, words that are not there, values that are no numbers ----------------------
def gradients(c, lse, out=None):
    op = c.operator()
    out = out or grad_outputs(c, ("dx", "dw", "dbias"), c.dtype)
    ws = torch.full((max(op.workspace_bytes(True), 256),), 255, dtype=torch.uint8, device=DEV)          # NaN, whatever the type
    op.backward(op.backward_io(c.x, c.w, *c.held(), lse, c.dloss, bias=c.bias, **out), ws)
    torch.cuda.synchronize()
    return out


ROWS = [(2, 5, 90, 40), (2, 60, 210, 40), (2, 150, 400, 72), (2, 600, 1300, 200), (1, 4, 9000, 64)]


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", ROWS)
@pytest.mark.parametrize("top", [0, 4])
def test_rows_that_do_not_count_may_hold_anything(size, dtype, top):
    c = Case(*size, dtype, top=top, seed=8, ignored=0.5)
    loss, lse = run_forward(c)
    want = gradients(c, lse)
    dead = (c.words < 0).all(2) if top else c.words < 0
    assert dead.any() and not dead.all()
    for k, bad in enumerate((float("nan"), INF)):
        c.x = torch.where(dead[:, :, None], torch.full_like(c.x, bad), c.x)
        c.dloss = torch.where(dead, torch.full_like(c.dloss, bad), c.dloss)
        if top:
            c.teacher = torch.where(dead[:, :, None], torch.full_like(c.teacher, bad), c.teacher)
        a, b = run_forward(c)
        assert torch.equal(a, loss) and torch.equal(b, lse)
        got = gradients(c, torch.where(dead, torch.full_like(lse, bad), lse))
        for n in want:
            assert torch.equal(got[n], want[n]), n
        assert (got["dx"][dead] == 0).all()


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", ROWS)
@pytest.mark.parametrize("top", [0, 4])
def test_no_row_counts(size, dtype, top):
    c = Case(*size, dtype, top=top, ignored=2.0)
    c.x = torch.full_like(c.x, float("nan"))
    loss, lse = run_forward(c)
    assert (loss == 0).all() and (lse == 0).all()
    got = gradients(c, lse)
    assert all((t == 0).all() for t in got.values())


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", ROWS)
@pytest.mark.parametrize("top", [0, 4])
def test_words_beyond_the_vocabulary(size, dtype, top):
    """Loss, lse and the row's gradients are NaN; other rows and workers keep theirs."""
    c = Case(*size, dtype, top=top, ignored=0.0, seed=4)
    loss, lse = run_forward(c)
    want = gradients(c, lse)
    for bad in (size[2], 2 ** 31 + 1, 2 ** 62):
        words = c.words
        c.words = words.clone()
        if top:
            c.words[0, 1, 2] = bad
        else:
            c.words[0, 1] = bad
        a, b = run_forward(c)
        assert torch.isnan(a[0, 1]) and torch.isnan(b[0, 1])
        a[0, 1], b[0, 1] = loss[0, 1], lse[0, 1]
        assert torch.equal(a, loss) and torch.equal(b, lse)
        got = gradients(c, lse)
        assert torch.isnan(got["dx"][0, 1]).all() and torch.isnan(got["dw"][0]).all() and torch.isnan(got["dbias"][0]).all()
        got["dx"][0, 1] = want["dx"][0, 1]
        assert torch.equal(got["dx"], want["dx"])
        if size[0] > 1:
            assert torch.equal(got["dw"][1], want["dw"][1]) and torch.equal(got["dbias"][1], want["dbias"][1])
        c.words = words


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", ROWS)
def test_teachers_words_in_any_order_absent_and_twice(size, dtype):
    G, M, V, K = size
    c = Case(*size, dtype, top=6, tau=2.0, seed=6, ignored=0.0)
    c.words = c.words.clamp(min=0)
    c.words[:, :, 3] = c.words[:, :, 0]                     # twice
    c.words[:, :, 5] = -1
    c.teacher[:, 0, 1:] = -INF                              # all of one word
    c.teacher[:, 2] = -INF                                  # no word
    c.words[:, 3] = c.words[:, 3, :1]                       # six times the same
    c.words[:, 3, 5] = c.words[:, 3, 0]
    run_case(c)
    loss, lse = run_forward(c)
    want = gradients(c, lse)
    order = torch.tensor([4, 0, 5, 2, 1, 3], device=DEV)
    c.words, c.teacher = c.words[:, :, order].contiguous(), c.teacher[:, :, order].contiguous()
    a, b = run_forward(c)
    got = gradients(c, lse)
    assert torch.equal(b, lse) and torch.allclose(a, loss, rtol=1e-5, atol=1e-6)
    assert all(torch.allclose(got[n].float(), want[n].float(), rtol=2e-2, atol=1e-5) for n in got)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", ROWS)
@pytest.mark.parametrize("top", [0, 3])
@pytest.mark.parametrize("low", ["-inf", "lowest"])
def test_forbidden_words(size, dtype, top, low):
    """A bias of -infinity, or of the type's lowest value, takes its word out: as in the vocabulary without it."""
    G, M, V, K = size
    c = Case(*size, dtype, top=top, seed=9, ignored=0.1)
    c.words = torch.where(c.words >= 0, c.words // 2 * 2, c.words).clamp(max=(V - 1) // 2 * 2)
    kept = torch.arange(0, V, 2, device=DEV)
    c.bias[:, 1::2] = -INF if low == "-inf" else torch.finfo(dtype).min
    small = Case(G, M, len(kept), K, dtype, top=top, seed=9)
    small.x, small.w, small.bias, small.teacher, small.dloss = c.x, c.w[:, kept].contiguous(), c.bias[:, kept].contiguous(), c.teacher, c.dloss
    small.words = torch.where(c.words >= 0, c.words // 2, c.words)
    dz, edz = small.solve()
    loss, lse = run_forward(c)
    assert ((lse - small.lse).abs() <= small.e_lse).all() and ((loss - torch.where(small.live, small.loss, 0.0)).abs() <= small.e_loss).all()
    got, want = gradients(c, lse), gradients(small, lse)
    assert (got["dw"][:, 1::2] == 0).all() and (got["dbias"][:, 1::2] == 0).all()
    # the same sums in other orders, each within its bound
    b = mm((edz + 4 * HALF[dtype] * dz.abs()).transpose(1, 2), torch.where(small.live[:, :, None], c.x.double().abs(), 0.0).transpose(1, 2))
    assert ((got["dw"][:, kept].double() - want["dw"].double()).abs() <= 2 * b + 2 * HALF[dtype] * want["dw"].double().abs() + 2.0 ** -24).all()


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", ROWS)
def test_infinities_and_nan(size, dtype):
    G, M, V, K = size
    c = Case(*size, dtype, seed=10, ignored=0.0)
    loss, lse = run_forward(c)
    x = c.x
    c.x = x.clone()
    c.x[0, 1, 2] = float("nan")
    a, b = run_forward(c)
    assert torch.isnan(a[0, 1]) and torch.isnan(b[0, 1])
    a[0, 1], b[0, 1] = loss[0, 1], lse[0, 1]
    assert torch.equal(a, loss) and torch.equal(b, lse)
    c.x, bias = x, c.bias
    c.words[0, 0], c.words[0, 1] = 0, 1
    c.bias = bias.clone()
    c.bias[0, 1] = -INF                                     # row 1 is held to a word that cannot be
    a, b = run_forward(c)
    assert a[0, 1] == INF and torch.isfinite(a[0, 0]) and torch.isfinite(b).all()
    c.bias[0, 1] = INF
    a, b = run_forward(c)
    assert (b[0] == INF).all() and a[0, 0] == INF and torch.isnan(a[0, 1])
    c.bias[0] = -INF
    a, b = run_forward(c)
    assert (b[0] == -INF).all() and torch.isnan(a[0]).all()


# up to 8 rows of more than 64 features, and 33 rows, which are more than half of what a workgroup has
FEW = [(2, 5, 300, 72), (1, 8, 1067, 200), (3, 1, 130, 129), (2, 33, 300, 50)]


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", FEW)
@pytest.mark.parametrize("top", [0, 4])
def test_few_rows(size, dtype, top):
    for f32_grads, accumulate in ((False, False), (True, False), (False, True), (True, True)):
        run_case(Case(*size, dtype, top=top, tau=1.0 if top == 0 else 1.5, seed=4, ignored=0.1), f32_grads=f32_grads, accumulate=accumulate)
    for want in (("dx",), ("dw",), ("dbias",), ("dw", "dbias")):
        run_case(Case(*size, dtype, top=top, seed=5), want=want)
    test_no_row_counts(size, dtype, top)
    test_forbidden_words(size, dtype, top, "-inf")
    if size[1] < 4:                                         # the others write into rows 0 to 3
        return
    test_words_beyond_the_vocabulary(size, dtype, top)
    test_infinities_and_nan(size, dtype)
    if top:
        test_teachers_words_in_any_order_absent_and_twice(size, dtype)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(2, 5, 300, 72), (1, 8, 1067, 200), (2, 32, 300, 50)])
@pytest.mark.parametrize("top", [0, 4])
def test_few_rows_that_do_not_count(size, dtype, top):
    test_rows_that_do_not_count_may_hold_anything(size, dtype, top)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("top", [5, 90])
def test_windows_of_more_than_a_tile(dtype, top):
    """So large a vocabulary that a window of the lists holds the columns of two waves."""
    run_case(Case(1, 70, 600001, 16, dtype, top=top, tau=2.0, seed=6))


@gpu
@pytest.mark.parametrize("dtype", DTYPES[1:])
def test_equal_weights_are_not_rounded_one_way(dtype):
    """The mean's weights are one number, of which each row's own word has -(1 - p): rounded as it is, all rows' errors would be the same.  A rounding of half a unit h is off
    by 0.43 h of a value in the root mean square (ulp^2 / 12 over the value's square, averaged over a binade's logarithm); two of them, of dz and of the result, by 0.6 of the
    most that one can be; 2 / 3 leaves a tenth for how values lie."""
    c = Case(1, 895, 6000, 200, dtype, weighted=False, ignored=0.0, seed=12)
    dz, _ = c.solve()
    out = gradients(c, c.lse32)
    for got, want in ((out["dx"], mm(dz, c.w.transpose(1, 2))), (out["dw"], mm(dz.transpose(1, 2), c.x.transpose(1, 2)))):
        assert (got.double() - want).norm() <= 2 / 3 * HALF[dtype] * want.norm()


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_all_rows_are_held_to_the_same_words(dtype):
    """Lists that lie in one window each: more words of a wave's rows and columns than are held at hand."""
    c = Case(1, 300, 700, 40, dtype, top=9, seed=7)
    c.words = torch.where(c.words < 0, c.words, 130 + torch.arange(9, device=DEV) * 2)
    run_case(c)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(1, 40, 500, 64), (1, 700, 1500, 200)])
@pytest.mark.parametrize("scale", [0.0, 1e-30, 1e-6, 1024.0, 1e30])
def test_weights_of_any_size(size, dtype, scale):
    """dx and dw are linear in dloss; f16 holds what its results can hold.  The weights of some rows are 2^12 times those of others."""
    G, M, V, K = size
    c = Case(*size, dtype, seed=11, ignored=0.1)
    _, lse = run_forward(c)
    c.dloss = (torch.rand(G, M, device=DEV) + 0.5) * scale * torch.where(torch.arange(M, device=DEV) % 2 == 0, 1.0, 2.0 ** -12)
    dz, edz = c.solve()
    op = c.operator(weight_grad_f32=True)
    out = {"dw": torch.empty(G, V, K, device=DEV), "dx": torch.empty(G, M, K, dtype=dtype, device=DEV)}
    ws = torch.empty(max(op.workspace_bytes(True), 256), dtype=torch.uint8, device=DEV)
    op.backward(op.backward_io(c.x, c.w, *c.held(), c.lse32, c.dloss, bias=c.bias, **out), ws)
    x = torch.where(c.live[:, :, None], c.x.double(), 0.0)
    want = mm(dz.transpose(1, 2), x.transpose(1, 2))
    b, _ = sum_bound(dz.transpose(1, 2), x.transpose(1, 2), torch.float32)
    rounded = HALF[dtype] * dz.abs() + 2.0 ** -39 * c.dloss.double().abs().amax()
    b = b + mm((edz + rounded).transpose(1, 2), x.abs().transpose(1, 2)) + U * want.abs() + 2.0 ** -126
    assert ((out["dw"].double() - want).abs() <= b).all()
    want = mm(dz, c.w.transpose(1, 2))
    b, _ = sum_bound(dz, c.w.double().transpose(1, 2), torch.float32)
    b = b + mm(edz + rounded, c.w.abs().transpose(1, 2))
    fits = want.abs() + b <= torch.finfo(dtype).max * 0.99
    tiny = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -126
    assert ((out["dx"].double() - want).abs() <= b + HALF[dtype] * (want.abs() + b) + tiny)[fits].all()


# -- gradients against differences ---------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("size", [(2, 30, 90, 20), (1, 200, 600, 40), (1, 600, 2000, 72)])
@pytest.mark.parametrize("top", [0, 5])
def test_gradients_against_differences(size, top):
    """The library's own forward along a random direction, f32: the step h leaves h^2 of the third derivative, and the losses' rounding over h."""
    G, M, V, K = size
    c = Case(*size, torch.float32, top=top, tau=1.5 if top else 1.0, seed=12)
    _, lse = run_forward(c)
    got = gradients(c, lse)
    g = torch.Generator(device=DEV).manual_seed(1)
    for name, grad in (("x", "dx"), ("w", "dw"), ("bias", "dbias")):
        was = getattr(c, name)
        way = torch.randn(was.shape, generator=g, device=DEV)
        way /= way.flatten(1).norm(dim=1).view(-1, *[1] * (way.dim() - 1)) / math.sqrt(M)
        h, losses = 2.0 ** -6, []
        for sign in (1, -1):
            setattr(c, name, was + sign * h * way)
            losses.append((run_forward(c)[0].double() * c.dloss.double()).sum(1))
        setattr(c, name, was)
        want = (losses[0] - losses[1]) / (2 * h)
        have = (got[grad].double() * way.double()).flatten(1).sum(1)
        # a logit moves by at most a few units along the way; its third derivative over 6 is below 1 then
        assert ((want - have).abs() <= 8 * h * h + 2.0 ** -20 / h).all(), (name, want, have)


# -- order, streams, graphs -----------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(2, 5, 900, 64), (2, 60, 210, 40), (2, 700, 3000, 136)])
@pytest.mark.parametrize("top", [0, 6])
def test_equal_calls_give_equal_bits_and_nothing_is_kept(size, dtype, top):
    c, other = Case(*size, dtype, top=top, seed=13), Case(*size, dtype, top=top, seed=14)
    op = c.operator()
    ws = torch.empty(max(op.workspace_bytes(), op.workspace_bytes(True), 256), dtype=torch.uint8, device=DEV)
    first = None
    for k in range(3):
        ws.fill_(255 * k & 255)
        run_forward(other, op, workspace=ws)
        loss, lse = run_forward(c, op, workspace=ws)
        out = grad_outputs(c, ("dx", "dw", "dbias"), dtype)
        op.backward(op.backward_io(c.x, c.w, *c.held(), lse, c.dloss, bias=c.bias, **out), ws)
        now = [loss, lse, *out.values()]
        first = first or [t.clone() for t in now]
        assert all(torch.equal(a, b) for a, b in zip(now, first))


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(2, 5, 900, 64), (2, 60, 210, 40), (2, 700, 3000, 136)])
@pytest.mark.parametrize("top", [0, 6])
def test_captured_calls_replayed(size, dtype, top):
    """Two graphs of forward and backward share a workspace; between their replays the program changes the inputs and calls eagerly."""
    c = Case(*size, dtype, top=top, seed=15)
    op = c.operator()
    ws = torch.empty(max(op.workspace_bytes(), op.workspace_bytes(True), 256), dtype=torch.uint8, device=DEV)
    G, M = c.size[:2]
    results = []
    for _ in range(2):
        loss, lse = torch.empty(G, M, device=DEV), torch.empty(G, M, device=DEV)
        results.append((loss, lse, grad_outputs(c, ("dx", "dw", "dbias"), dtype)))
    ios = [(op.forward_io(c.x, c.w, *c.held(), l, n, bias=c.bias), op.backward_io(c.x, c.w, *c.held(), n, c.dloss, bias=c.bias, **o)) for l, n, o in results]
    graphs = []
    side = torch.cuda.Stream()
    for f, b in ios:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            op.forward(f, ws, side)
            op.backward(b, ws, side)
        graphs.append(g)
    for turn in range(3):
        fresh = Case(*size, dtype, top=top, seed=20 + turn)
        for name in ("x", "w", "bias", "words", "teacher", "dloss"):
            if getattr(c, name) is not None:
                getattr(c, name).copy_(getattr(fresh, name))
        loss, lse = run_forward(c, op)
        want = [loss, lse, *gradients(c, lse).values()]
        torch.cuda.synchronize()
        for g, (l, n, o) in zip(graphs, results):
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip([l, n, *o.values()], want))


@gpu
def test_two_streams_at_once():
    sizes = [(2, 700, 3000, 136), (1, 900, 2000, 200)]
    cases = [Case(*s, torch.bfloat16, top=t, seed=30 + t) for s, t in zip(sizes, (0, 9))]
    ops = [c.operator() for c in cases]
    want = []
    for c in cases:
        loss, lse = run_forward(c)
        want.append([loss, lse, *gradients(c, lse).values()])
    streams = [torch.cuda.Stream() for _ in cases]
    spaces = [torch.empty(max(o.workspace_bytes(), o.workspace_bytes(True)), dtype=torch.uint8, device=DEV) for o in ops]
    outs = [grad_outputs(c, ("dx", "dw", "dbias"), c.dtype) for c in cases]
    losses = [torch.empty(2, *c.size[:2], device=DEV) for c in cases]
    torch.cuda.synchronize()
    for _ in range(4):
        for c, o, s, ws, out, l in zip(cases, ops, streams, spaces, outs, losses):
            o.forward(o.forward_io(c.x, c.w, *c.held(), l[0], l[1], bias=c.bias), ws, s)
            o.backward(o.backward_io(c.x, c.w, *c.held(), l[1], c.dloss, bias=c.bias, **out), ws, s)
    torch.cuda.synchronize()
    for w, l, out in zip(want, losses, outs):
        assert all(torch.equal(a, b) for a, b in zip(w, [l[0], l[1], *out.values()]))


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_both_losses_then_the_local_step(dtype):
    """A step as a trainer takes it: both losses' gradients into one dw, the norm with clipping, and SGD on theta in place."""
    G, M, V, K, rate, most = 3, 130, 1000, 64, 0.5, 0.05
    a = Case(G, M, V, K, dtype, seed=16)
    b = Case(G, M, V, K, dtype, top=8, tau=2.0, seed=16)
    b.x, b.w, b.bias = a.x, a.w, a.bias
    theta = torch.cat([a.w.float().flatten(1), a.bias.float()], 1).contiguous()
    want = theta.double().clone()
    grads = torch.zeros(G, V * K + V, device=DEV)
    dw, db = grads[:, : V * K].view(G, V, K), grads[:, V * K:]
    for c in (a, b):
        op = c.operator(weight_grad_f32=True, accumulate=True)
        ws = torch.empty(max(op.workspace_bytes(), op.workspace_bytes(True)), dtype=torch.uint8, device=DEV)
        loss, lse = run_forward(c, op, workspace=ws)
        op.backward(op.backward_io(c.x, c.w, *c.held(), lse, c.dloss, bias=c.bias, dw=dw, dbias=db), ws)
    handle, norms = B.Grads([[dw[g], db[g]] for g in range(G)]), torch.empty(G, device=DEV)
    handle.local_step(B.make_state(theta, None, None, theta.stride(0)), None, V * K + V, rate, 0.0, most, norms)
    torch.cuda.synchronize()
    total = torch.zeros_like(want)
    for c in (a, b):
        dz, _ = c.solve()
        x = torch.where(c.live[:, :, None], c.x.double(), 0.0)
        total += torch.cat([mm(dz.transpose(1, 2), x.transpose(1, 2)).flatten(1), dz.sum(1)], 1)
    n = total.norm(dim=1)
    assert torch.allclose(norms.double(), n, rtol=4 * HALF[dtype] if dtype != torch.float32 else 1e-5)
    want -= rate * total * (most / n).clamp(max=1.0)[:, None]
    # each step is at most rate * most in norm, its error that times a few half units
    assert ((theta.double() - want).norm(dim=1) <= rate * most * (4 * HALF[dtype] + 2.0 ** -16) + U * want.norm(dim=1)).all()
    handle.destroy()


# -- refusals, on any machine ----------------------------------------------------------------------------
def desc(**k):
    d = dict(struct_size=ctypes.sizeof(B.LossDesc), dtype=B.F32, batch=2, top=0, rows=4, vocab=6, in_features=8, temperature=1.0)
    d.update(k)
    return B.LossDesc(**d)


def workspace_status(d, bytes_out=True):
    n = ctypes.c_int64(-1)
    rc = B.lib().gbmuf_loss_workspace(ctypes.byref(d) if d is not None else None, 0, ctypes.byref(n) if bytes_out else None)
    return rc, n.value


def test_descriptions():
    assert workspace_status(desc())[0] == B.GBMUF_OK and workspace_status(desc())[1] > 0
    assert workspace_status(desc(), False)[0] == B.GBMUF_EINVAL
    assert workspace_status(None)[0] == B.GBMUF_EINVAL
    for bad in (dict(struct_size=8), dict(dtype=3), dict(dtype=-1), dict(batch=-1), dict(rows=-1), dict(vocab=-1), dict(in_features=-1), dict(top=-1),
                dict(top=3, temperature=0.0), dict(top=3, temperature=-1.0), dict(top=3, temperature=float("nan")), dict(top=3, temperature=INF)):
        assert workspace_status(desc(**bad)) == (B.GBMUF_EINVAL, 0), bad
    for far in (dict(batch=65536), dict(rows=2 ** 31), dict(vocab=2 ** 31), dict(in_features=2 ** 31), dict(top=1025), dict(top=2, temperature=2.0 ** 41),
                dict(top=2, temperature=2.0 ** -41), dict(rows=2 ** 25, vocab=2 ** 25), dict(rows=2 ** 29, vocab=8, batch=2)):
        assert workspace_status(desc(**far)) == (B.GBMUF_EUNSUPPORTED, 0), far
    assert workspace_status(desc(temperature=float("nan")))[0] == B.GBMUF_OK                 # cross entropy has none
    # the other loss's entry points refuse the description
    io, grad = B.LossIo(), B.LossGradIo()
    L = B.lib()
    assert L.gbmuf_cross_entropy(ctypes.byref(desc(top=2)), ctypes.byref(io), None, 0, None) == B.GBMUF_EINVAL
    assert L.gbmuf_distill(ctypes.byref(desc()), ctypes.byref(io), None, 0, None) == B.GBMUF_EINVAL
    assert L.gbmuf_cross_entropy_backward(ctypes.byref(desc(top=2)), ctypes.byref(grad), None, 0, None) == B.GBMUF_EINVAL
    assert L.gbmuf_distill_backward(ctypes.byref(desc()), ctypes.byref(grad), None, 0, None) == B.GBMUF_EINVAL
    for k in (dict(dtype=torch.int32), dict(batch=-1)):
        with pytest.raises(B.GbmufError):
            B.CrossEntropy(4, 6, 8, **k)
    for k in (dict(top=0), dict(top=2, temperature=0.0), dict(top=2000)):
        with pytest.raises(B.GbmufError):
            B.Distill(4, 6, 8, **k)


def test_more_rows_than_launches_have():
    assert workspace_status(desc(rows=2 ** 20, vocab=8, batch=2 ** 7, in_features=8))[0] == B.GBMUF_OK
    assert workspace_status(desc(rows=2 ** 18 + 1, vocab=0, batch=2 ** 10)) == (B.GBMUF_EUNSUPPORTED, 0)
    assert workspace_status(desc(rows=2 ** 20, vocab=8, batch=2 ** 5, in_features=8, top=2, temperature=1.0))[0] == B.GBMUF_OK
    assert workspace_status(desc(rows=2 ** 20 + 1, vocab=8, batch=2 ** 5, in_features=8, top=2, temperature=1.0)) == (B.GBMUF_EUNSUPPORTED, 0)


def test_workspaces_of_any_sizes():
    for batch in (0, 1, 3):
        for rows in (0, 1, 40, 70, 700):
            for vocab in (0, 1, 1000, 70000):
                for features in (0, 1, 200):
                    for dtype in (B.F32, B.BF16, B.F16):
                        d = desc(batch=batch, rows=rows, vocab=vocab, in_features=features, dtype=dtype)
                        n = ctypes.c_int64(-1)
                        for backward in (0, 1):
                            assert B.lib().gbmuf_loss_workspace(ctypes.byref(d), backward, ctypes.byref(n)) == B.GBMUF_OK and n.value >= 0


def test_workspaces_stay_bounded():
    """Of 16 times 5120 rows against 267,735 words the logits' gradient alone would be 44 GB in 16 bits."""
    for dtype in DTYPES:
        assert B.CrossEntropy(5120, 267735, 512, 1, dtype).workspace_bytes(True) < 1.8e9
        assert B.CrossEntropy(5120, 267735, 512, 16, dtype).workspace_bytes(True) < 2.5e9
        assert B.CrossEntropy(5120, 267735, 512, 1, dtype).workspace_bytes() < 0.4e9


def host(size=(2, 4, 6, 8), dtype=torch.float32, top=0):
    G, M, V, K = size
    t = {"x": torch.zeros(G, M, K, dtype=dtype), "w": torch.zeros(G, V, K, dtype=dtype), "bias": torch.zeros(G, V, dtype=dtype),
         "target": torch.zeros((G, M, top) if top else (G, M), dtype=torch.int64), "loss": torch.zeros(G, M), "lse": torch.zeros(G, M), "dloss": torch.zeros(G, M),
         "dx": torch.zeros(G, M, K, dtype=dtype), "dw": torch.zeros(G, V, K, dtype=dtype), "dbias": torch.zeros(G, V, dtype=dtype)}
    if top:
        t["teacher"] = torch.zeros(G, M, top)
    return t


def matrix(t):
    if t is None:
        return B.Matrix()
    return B.Matrix(t.data_ptr(), t.stride(1) if t.dim() > 1 else 0, t.stride(0))


def status(t, backward=False, top=0, workspace="enough", **k):
    """The C entry point on host addresses, which it must refuse before it looks at them."""
    d = desc(top=top, **k)
    rc, need = workspace_status(d)
    L = B.lib()
    n = ctypes.c_int64()
    L.gbmuf_loss_workspace(ctypes.byref(d), int(backward), ctypes.byref(n))
    io = (B.LossGradIo if backward else B.LossIo)(**{f: (t[f] if isinstance(t.get(f), B.Matrix) else matrix(t.get(f))) if f not in ("bias", "dbias")
                                                    else (B.Matrix(t[f].data_ptr(), 0, t[f].stride(0)) if isinstance(t.get(f), torch.Tensor) else t.get(f) or B.Matrix())
                                                    for f, _ in (B.LossGradIo if backward else B.LossIo)._fields_})
    space = torch.zeros(n.value + 512, dtype=torch.uint8)
    at = (space.data_ptr() + 255) // 256 * 256
    ws, size = {"enough": (at, n.value), "none": (None, 0), "short": (at, n.value - 1), "crooked": (at + 16, n.value)}.get(workspace, (workspace, n.value))
    fn = getattr(L, ("gbmuf_distill" if top else "gbmuf_cross_entropy") + ("_backward" if backward else ""))
    return fn(ctypes.byref(d), ctypes.byref(io), ws, size, None)


@pytest.mark.parametrize("top", [0, 3])
@pytest.mark.parametrize("backward", [False, True])
def test_calls_that_are_refused(top, backward):
    t = host(top=top)
    bad = lambda **k: status({**t, **k}, backward, top)
    L = B.lib()
    fn = getattr(L, ("gbmuf_distill" if top else "gbmuf_cross_entropy") + ("_backward" if backward else ""))
    assert fn(None, None, None, 0, None) == B.GBMUF_EINVAL and fn(ctypes.byref(desc(top=top)), None, None, 0, None) == B.GBMUF_EINVAL
    needed = ["x", "w", "target"] + (["teacher"] if top else []) + (["lse", "dloss"] if backward else ["loss"])
    for n in needed:
        assert bad(**{n: None}) == B.GBMUF_EINVAL, n
        m = matrix(t[n])
        assert bad(**{n: B.Matrix(m.data + 1, m.ld, m.batch_stride)}) == B.GBMUF_EINVAL, n
        assert bad(**{n: B.Matrix(m.data, -1, m.batch_stride)}) == B.GBMUF_EINVAL, n
        assert bad(**{n: B.Matrix(m.data, m.ld, -1)}) == B.GBMUF_EINVAL, n
        assert bad(**{n: B.Matrix(m.data, 2 ** 50, m.batch_stride)}) == B.GBMUF_EINVAL, n
    outs = ["dx", "dw"] if backward else ["loss", "lse"]
    for n in outs:
        m = matrix(t[n])
        assert bad(**{n: B.Matrix(m.data, 0, m.batch_stride)}) == B.GBMUF_EINVAL, n                     # elements that are not apart
        assert bad(**{n: B.Matrix(m.data, m.ld, 0)}) == B.GBMUF_EINVAL, n
        for other in needed + ["bias"]:
            if other != n:
                assert bad(**{n: B.Matrix(t[other].data_ptr(), m.ld, m.batch_stride)}) == B.GBMUF_EINVAL, (n, other)
    a, b = outs
    assert bad(**{a: B.Matrix(t[b].data_ptr(), matrix(t[a]).ld, matrix(t[a]).batch_stride)}) == B.GBMUF_EINVAL
    for w in ("none", "short", "crooked"):
        assert status(t, backward, top, workspace=w) == B.GBMUF_EINVAL, w
    big = torch.zeros(1 << 22, dtype=torch.uint8)
    at = (big.data_ptr() + 255) // 256 * 256
    inside = B.Matrix(at + 64, 8, 4 * 8)
    assert status({**t, "x": inside}, backward, top, workspace=at) == B.GBMUF_EINVAL


@pytest.mark.parametrize("top", [0, 3])
def test_the_binding_refuses(top):
    t = host(top=top)
    op = B.Distill(4, 6, 8, top, 1.0, 2) if top else B.CrossEntropy(4, 6, 8, 2)
    held = (t["target"], t["teacher"]) if top else (t["target"],)
    ok = op.forward_io(t["x"], t["w"], *held, t["loss"], t["lse"], bias=t["bias"])
    with pytest.raises(B.GbmufError):
        op.forward(ok, torch.empty(op.workspace_bytes(), dtype=torch.uint8))                            # tensors of the host
    with pytest.raises(B.GbmufError):
        op.forward_io(t["x"].double(), t["w"], *held, t["loss"], t["lse"])
    with pytest.raises(B.GbmufError):
        op.forward_io(t["x"], t["w"][:, :5], *held, t["loss"], t["lse"])
    with pytest.raises(B.GbmufError):
        op.forward_io(t["x"], t["w"].transpose(1, 2).contiguous().transpose(1, 2), *held, t["loss"], t["lse"])
    with pytest.raises(B.GbmufError):
        op.forward_io(t["x"], t["w"], t["target"].int(), *held[1:], t["loss"], t["lse"])
    with pytest.raises(B.GbmufError):
        op.forward_io(t["x"], t["w"], *held, t["loss"].half(), t["lse"])
    with pytest.raises(B.GbmufError):
        op.backward_io(t["x"], t["w"], *held, t["lse"], t["dloss"], dw=t["dw"].bfloat16())
    if top:
        with pytest.raises(B.GbmufError):
            op.forward_io(t["x"], t["w"], t["target"], t["teacher"].half(), t["loss"], t["lse"])


# -- as many rows, and as many words, as descriptions may have -------------------------------------------
@gpu
@pytest.mark.parametrize("size", [(2 ** 20, 2 ** 5), (2 ** 17 - 1, 2 ** 8)])
def test_as_many_rows_of_a_teacher_as_there_may_be(size):
    """2^25, and some fewer: one word of a teacher has the whole share, so the loss is cross entropy's."""
    M, G = size
    V, K = 8, 8
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(G, M, K, generator=g, device=DEV).bfloat16()
    w = torch.randn(G, V, K, generator=g, device=DEV).bfloat16()
    words = torch.randint(-1, V, (G, M, 1), generator=g, device=DEV)
    teacher = torch.randn(G, M, 1, generator=g, device=DEV)
    op = B.Distill(M, V, K, 1, 1.0, G, torch.bfloat16)
    loss, lse = torch.full((G, M), 7.0, device=DEV), torch.full((G, M), 7.0, device=DEV)
    dx, dw, dloss = torch.empty_like(x), torch.empty_like(w), torch.ones(1, 1, device=DEV).expand(G, M)
    ws = torch.empty(max(op.workspace_bytes(), op.workspace_bytes(True)), dtype=torch.uint8, device=DEV)
    op.forward(op.forward_io(x, w, words, teacher, loss, lse), ws)
    op.backward(op.backward_io(x, w, words, teacher, lse, dloss, dx=dx, dw=dw), ws)
    torch.cuda.synchronize()
    for i in (0, G // 2, G - 1):
        xs, ws_ = x[i].double(), w[i].double()
        z, S = xs @ ws_.T.contiguous(), xs.abs() @ ws_.abs().T.contiguous()
        live, word = words[i, :, 0] >= 0, words[i].clamp(min=0)
        n = torch.logsumexp(z, 1, keepdim=True)
        p, d = torch.exp(z - n), (z - n).abs()
        # as derived above: a logit, lse (every logit's, and adding up), and p with lse rounded to f32
        bz = (2 * K + 32) * U * S
        e_lse = bz.amax(1) + U * ((p * (4 * d + 8)).sum(1) + 400 + 8 * n[:, 0].abs())
        want = torch.where(live, n[:, 0] - z.gather(1, word)[:, 0], 0.0)
        assert ((loss[i] - want).abs() <= e_lse + bz.gather(1, word)[:, 0] + 8 * U * (n[:, 0].abs() + z.abs().amax(1) + 1)).all()
        share = torch.zeros_like(z).scatter_(1, word, 1.0)
        dz = torch.where(live[:, None], p - share, 0.0)
        edz = p * (bz + e_lse[:, None] + U * (4 * d + 16)) + 8 * U * share
        want, size = dz @ ws_, dz.abs() @ ws_.abs()
        bound = (edz + 2.0 ** -8 * (dz.abs() + edz)) @ ws_.abs() + (2 * V + 32) * U * size               # dz is rounded once
        worst = ((dx[i].double() - want).abs() - (bound + 2.0 ** -8 * (want.abs() + bound))).amax().item()
        assert worst <= 0, worst
        assert torch.isfinite(dw[i]).all()


@gpu
def test_as_many_rows_as_there_may_be():
    """2^28 of a vocabulary of none: half of them do not count, the others name words that there are not."""
    M, G = 2 ** 21, 2 ** 7
    x, w = torch.empty(G, M, 0, device=DEV), torch.empty(G, 0, 0, device=DEV)
    target = (torch.arange(M, device=DEV) % 2 - 1).expand(G, M)
    loss, lse = torch.full((G, M), 7.0, device=DEV), torch.full((G, M), 7.0, device=DEV)
    op = B.CrossEntropy(M, 0, 0, G)
    op.forward(op.forward_io(x, w, target, loss, lse), torch.empty(max(op.workspace_bytes(), 256), dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    for t in (loss, lse):
        assert (t[:, ::2] == 0).all() and torch.isnan(t[:, 1::2]).all()


@gpu
@pytest.mark.parametrize("accumulate", [False, True])
def test_as_many_words_as_there_may_be(accumulate):
    """Sums over no rows, of 2^29 words: more workgroups of 64 than a grid's first dimension holds."""
    V = 2 ** 29 + 70
    op = B.CrossEntropy(0, V, 0, 1, torch.bfloat16, accumulate=accumulate)
    db = torch.full((1, V), 3.0, dtype=torch.bfloat16, device=DEV)
    none = lambda *s, t=torch.float32: torch.empty(s, dtype=t, device=DEV)
    op.backward(op.backward_io(none(1, 0, 0, t=torch.bfloat16), none(1, V, 0, t=torch.bfloat16), none(1, 0, t=torch.int64), none(1, 0), none(1, 0), dbias=db),
                torch.empty(max(op.workspace_bytes(True), 256), dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    assert (db == (3.0 if accumulate else 0.0)).all()


# -- rows that do not count, whatever the logits are -----------------------------------------------------
# few rows, up to 64 features, small sizes, many rows; f32 of more rows than small sizes have
ROUTES = [*ROWS, (2, 6, 300, 200), (1, 2600, 300, 72), (1, 900, 3000, 64)]


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", ROUTES)
@pytest.mark.parametrize("top", [0, 4])
@pytest.mark.parametrize("bad", [float("nan"), INF, "most"])
def test_rows_that_do_not_count_have_no_gradient_whatever_the_logits_are(size, dtype, top, bad):
    """A bias that is no number, infinite or the type's largest value; the last worker has no row that counts."""
    c = Case(*size, dtype, top=top, seed=8, ignored=0.5)
    c.words[-1] = -1
    c.bias = c.bias.clone()
    c.bias[:, [1, size[2] - 1]] = torch.finfo(dtype).max if bad == "most" else bad
    loss, lse = run_forward(c)
    dead = (c.words < 0).all(2) if top else c.words < 0
    assert dead.any()
    assert (loss[dead] == 0).all() and (lse[dead] == 0).all()
    got = gradients(c, lse)
    assert (got["dx"][dead] == 0).all()
    assert (got["dw"][-1] == 0).all() and (got["dbias"][-1] == 0).all()


# -- temperatures, and logits far from 0 -----------------------------------------------------------------
def test_temperatures():
    """What one f32 of lse can carry: beyond, exp(z / tau - lse) would keep fewer than 8 bits for logits of 64."""
    for t in (2.0 ** -10, 0.01, 1.0, 2.0 ** 10):
        assert workspace_status(desc(top=2, temperature=t))[0] == B.GBMUF_OK, t
    for t in (2.0 ** -11, 2.0 ** -20, 2.0 ** -40, 2.0 ** 11, 2.0 ** 20, 2.0 ** 40):
        assert workspace_status(desc(top=2, temperature=t)) == (B.GBMUF_EUNSUPPORTED, 0), t


class Exact(Case):
    """Logits that every type holds exactly: products of eighths, few enough for 24 bits; `far` is added to those of every second row."""

    def __init__(self, G, M, V, K, dtype, far=0.0, **k):
        super().__init__(G, M, V, K, dtype, **k)
        eighths = lambda t, most: ((t.float() * 8).round().clamp(-8 * most, 8 * most) / 8).to(dtype)
        self.x, self.w, self.bias = eighths(self.x, 2), eighths(self.w, 2), eighths(self.bias, 2)
        self.w[:, :, 0] = 1.0
        self.x[:, ::2, 0] = far
        self.x[:, 1::2, 0] = 0.0

    def compare(self):
        """Loss and gradients, those from the forward's own lse, against 64 bits."""
        G, M, V, K = self.size
        tau = self.tau
        z = (mm(self.x, self.w) + self.bias.double()[:, None]) / tau
        words = (self.words if self.top else self.words[:, :, None]).clamp(min=0)
        there = self.words >= 0 if self.top else (self.words >= 0)[:, :, None]
        if self.top:
            s = self.teacher.double().masked_fill(~there, -INF) / tau
            q = torch.softmax(s, 2).masked_fill(~there, 0.0)
            off = (s - s.amax(2, keepdim=True)).abs().masked_fill(~there, 0.0)
            eq = q * (8 * off + self.top + 16) * U
        else:
            q, eq = there.double(), torch.zeros_like(there, dtype=torch.float64)
        live = there.any(2)
        n = torch.logsumexp(z, 2)
        p, d = torch.exp(z - n[:, :, None]), (z - n[:, :, None]).abs()
        # as at the head of this file, of logits that are exact
        e_lse = U * ((p * (4 * d + 8)).sum(2) + 400 + 8 * n.abs())
        loss, lse = run_forward(self)
        out = gradients(self, lse)
        assert (loss[~live] == 0).all() and (lse[~live] == 0).all()
        assert ((lse.double() - n).abs() <= e_lse)[live].all()
        logq = torch.where(q > 0, torch.log(q.clamp(min=1e-300)), torch.zeros_like(q))
        at = z.gather(2, words)
        term = torch.where(q > 0, logq - at + n[:, :, None], torch.zeros_like(q))
        want = tau ** 2 * (q * term).sum(2)
        size = logq.abs() + at.abs() + n.abs()[:, :, None] + 1
        e_loss = tau ** 2 * (q * (e_lse[:, :, None] + 8 * U * size) + 2 * eq * (term.abs() + 1) + U * (self.top + 8) * q * term.abs()).sum(2)
        assert ((loss.double() - want).abs() <= e_loss)[live].all()
        weight = torch.where(live, tau * self.dloss.double(), 0.0)[:, :, None]
        share, more = (torch.zeros_like(z).scatter_add_(2, words, v) for v in (q, eq))
        dz = weight * (p - share)
        edz = weight * (p * torch.expm1(e_lse[:, :, None] + U * (4 * d + 16 + 4 * n.abs()[:, :, None])) + more + (self.top + 4) * U * share)
        h = HALF[self.dtype]
        if self.dtype != torch.float32:                     # rounded once, where sizes are large
            edz = edz + h * (dz.abs() + edz) + 2.0 ** -39 * (tau * self.dloss.double().abs()).amax(1)[:, None, None]
        x = torch.where(live[:, :, None], self.x.double(), 0.0)
        for got, a, e, b in ((out["dx"], dz, edz, self.w.double().transpose(1, 2)), (out["dw"], dz.transpose(1, 2), edz.transpose(1, 2), x.transpose(1, 2))):
            want = mm(a, b)
            bound = mm(e, b.abs()) + sum_bound(a, b, self.dtype)[0]
            bound = bound + h * (want.abs() + bound) + 2.0 ** -25
            worst = ((got.double() - want).abs() - bound).amax().item()
            assert worst <= 0, worst


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", ROUTES)
@pytest.mark.parametrize("tau", [2.0 ** -10, 2.0 ** -3, 2.0 ** 10])
def test_temperatures_at_their_ends(size, dtype, tau):
    Exact(*size, dtype, top=5, tau=tau, seed=17).compare()


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", ROUTES)
def test_logits_far_from_0(size, dtype):
    """100 / tau is more than what exponents are formed of in one multiply-add, for every second row."""
    Exact(*size, dtype, top=5, tau=2.0 ** -10, far=100.0, seed=18).compare()
    Exact(*size, dtype, top=5, tau=2.0 ** -10, far=-100.0, seed=19).compare()
    if dtype != torch.float16:
        Exact(*size, dtype, far=2.0 ** 17, seed=20).compare()
        Exact(*size, dtype, far=-(2.0 ** 17), seed=21).compare()


# -- wide rows -------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(1, 300, 2100, 2050), (2, 140, 1000, 4100), (1, 1100, 700, 1536)])
@pytest.mark.parametrize("top", [0, 20])
def test_wide_rows(size, dtype, top):
    """More than 16 steps a tile."""
    run_case(Case(*size, dtype, top=top, tau=1.5 if top else 1.0, seed=22), accumulate=size[0] == 2)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(1, 300, 70000, 2050), (3, 80, 30000, 2050)])
def test_pieces_of_wide_words(size, dtype):
    """w lies on no 16 bytes and is more than is laid out at a time: parts of the vocabulary, and some of the workers."""
    G, M, V, K = size
    crooked = {"w": in_rows(5, V * K + 11)}
    run_case(Case(*size, dtype, top=0 if G == 1 else 6, tau=1.0 if G == 1 else 2.0, seed=23, place=crooked))
    c = Case(*size, dtype, seed=24, place={**crooked, "x": in_rows(3, M * K + 5)})
    loss, lse = run_forward(c)
    c.x, c.w = columns_of(K + 6, 0)(c.x), columns_of(K + 6, 0)(c.w)
    assert all(t.data_ptr() % 16 == 0 and t.stride(1) % 8 == 0 and t.stride(0) % 8 == 0 for t in (c.x, c.w))
    a, b = run_forward(c)                                   # 16-bit types take them as they lie: other tiles, the same sums
    c.solve()
    assert ((a - loss).abs().double() <= 2 * c.e_loss)[c.live].all() and ((b - lse).abs().double() <= 2 * c.e_lse)[c.live].all()


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [3, 200])
def test_words_of_no_vocabulary(M, dtype):
    """A row that names one gets NaN; its dx is a sum of nothing."""
    c = Case(2, M, 0, 8, dtype, ignored=2.0)
    c.words[:, 1] = 0
    loss, lse = run_forward(c)
    assert torch.isnan(loss[:, 1]).all() and torch.isnan(lse[:, 1]).all()
    assert (loss[:, 0] == 0).all() and (lse[:, 0] == 0).all()
    assert (gradients(c, lse)["dx"] == 0).all()
