"""Products with a model's matrices and their gradients, against the formulas in 64 bits.

Bounds, derived before any run (u = 2^-24, S = the sum of the magnitudes of what is added up):
  a sum of n products in f32, whatever its order: 2 n u S (twice the textbook's n u S: matrix instructions may round by cutting);
  f32 operands taken apart: 2^-23 each and 2^-22 for the product that is left out: 2^-21 S, and 2^-39 of the largest of
  each row against the other operand's sum of magnitudes;
  rounding to the type at the end: half a unit, 2^-8 (bf16, 8 bits) or 2^-11 (f16, 11 bits, and 2^-25 below its normal range) of the result;
  16-bit backward: dz rounded to the type before the products, half a unit of each term;
  activations: slope at most 1.2, and 16 u of |z| + |y| for the functions themselves.
Errors of many roundings do not add up all one way: their root mean square is held to 2^-21 of S's (and the roundings above).
"""
import ctypes
import gc
import math
import weakref

import numpy as np
import pytest
import torch

from paper_1909_09010_amd import binding as B

DEV = "cuda:0"
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
U = 2.0 ** -24
ACTS = [B.ACT_NONE, B.ACT_RELU, B.ACT_GELU, B.ACT_SILU, B.ACT_SIGMOID, B.ACT_TANH]
gpu = pytest.mark.gpu


def act64(z, kind):
    if kind == B.ACT_RELU:
        return z.clamp(min=0)
    if kind == B.ACT_GELU:
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2))
    if kind == B.ACT_SILU:
        return z * torch.sigmoid(z)
    if kind == B.ACT_SIGMOID:
        return torch.sigmoid(z)
    if kind == B.ACT_TANH:
        return torch.tanh(z)
    return z


def slope64(z, kind):
    if kind == B.ACT_NONE:
        return torch.ones_like(z)
    if kind == B.ACT_RELU:
        return (z > 0).double()
    z = z.clone().requires_grad_(True)
    with torch.enable_grad():
        (d,) = torch.autograd.grad(act64(z, kind).sum(), z)
    return d


def check(got, want, bound, rms, what):
    """Element by element within `bound`, the root mean square of the errors within `rms`."""
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape, what
    if got.numel() == 0:
        return
    err = (got - want).abs()
    assert torch.isfinite(got).all(), what
    worst = (err - bound).max().item()
    assert worst <= 0, f"{what}: {worst:.3g} beyond the bound, error {err.max().item():.3g}"
    e, r = err.square().mean().sqrt().item(), rms.square().mean().sqrt().item()
    assert e <= r, f"{what}: rms error {e:.3g}, bound {r:.3g}"


def sum_bound(n, S, dtype, rows=None):
    """Of a sum of n products with magnitudes summing to S; rows: (row maxima of a) x (sums of |b|) both ways, f32 only."""
    b = (2 * n + 16) * U * S
    if dtype == torch.float32:
        b = b + 2.0 ** -21 * S + 2.0 ** -39 * rows
    return b


def spread(a, b):
    """2^-39 of a row's largest meets every value of the other operand: max|a| sum|b| + max|b| sum|a|."""
    if a.shape[-1] == 0:
        return torch.zeros(a.shape[0], a.shape[1], b.shape[1], dtype=torch.float64)
    a, b = a.abs(), b.abs()
    return a.amax(2)[:, :, None] * b.sum(2)[:, None, :] + a.sum(2)[:, :, None] * b.amax(2)[:, None, :]


def mm(a, b):
    return torch.matmul(a, b.transpose(1, 2))


def make(shape, dtype, g, scale=1.0):
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def forward_case(G, M, N, K, dtype, act, residual, bias, pre, seed=0, place=None):
    """Runs one forward and checks y and z.  place: how tensors lie on the device, by name."""
    g = torch.Generator().manual_seed(seed)
    x, w = make((G, M, K), dtype, g), make((G, N, K), dtype, g, max(K, 1) ** -0.5)
    b = make((G, N), dtype, g) if bias else None
    r = make((G, M, N), dtype, g) if residual else None
    place = place or {}
    put = lambda name, t: None if t is None else place.get(name, lambda v: v.to(DEV))(t)
    dx, dw, dbv, dr = put("x", x), put("w", w), put("bias", b), put("residual", r)
    y = put("y", torch.full((G, M, N), float("nan"), dtype=dtype))
    z = put("pre", torch.full((G, M, N), float("nan"), dtype=dtype)) if pre else None
    lin = B.Linear(M, N, K, G, dtype, act, residual)
    io = lin.forward_io(dx, dw, y, bias=dbv, residual=dr, pre=z)
    ws = torch.empty(max(lin.workspace_bytes(), 256), dtype=torch.uint8, device=DEV)
    lin.forward(io, ws, torch.cuda.current_stream())
    torch.cuda.synchronize()
    X, W = x.double(), w.double()
    s, S = mm(X, W), mm(X.abs(), W.abs())
    if bias:
        s, S = s + b.double()[:, None], S + b.double().abs()[:, None]
    if residual == B.RESIDUAL_BEFORE:
        s, S = s + r.double(), S + r.double().abs()
    bz, rz = sum_bound(K, S, dtype, spread(X, W)), 2.0 ** -21 * S
    h = HALF[dtype]
    if pre:
        check(z, s, bz + h * (s.abs() + bz) + 2.0 ** -25, rz + h * s.abs() + 2.0 ** -25, "pre")
    out = act64(s, act)
    by, ry = 1.2 * bz + 16 * U * (s.abs() + out.abs()), 1.2 * rz + 16 * U * (s.abs() + out.abs())
    if residual == B.RESIDUAL_AFTER:
        out = out + r.double()
        by, ry = by + U * out.abs(), ry + U * out.abs()
    check(y, out, by + h * (out.abs() + by) + 2.0 ** -25, ry + h * out.abs() + 2.0 ** -25, "y")
    return y, z


SIZES = [(1, 1, 1, 1), (4, 1, 256, 64), (2, 3, 5, 7), (1, 8, 1000, 1024), (3, 17, 33, 65), (2, 128, 128, 64), (2, 129, 257, 650),
         (1, 300, 130, 31), (1, 64, 64, 2050), (5, 2, 70, 200), (1, 16, 32, 8192), (1, 257, 640, 96), (2, 33, 300, 72),
         (1, 5, 4099, 130), (1, 1, 50, 5000), (3, 64, 20, 1), (1, 1000, 8, 24)]


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES)
def test_forward(size, dtype):
    i = SIZES.index(size)
    forward_case(*size, dtype, ACTS[i % 6], (i // 2) % 3, i % 3 != 1, i % 2 == 0, seed=i)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("residual", [0, 1, 2])
def test_forward_every_activation_and_residual(dtype, act, residual):
    forward_case(2, 37, 45, 50, dtype, act, residual, True, True, seed=act + 10 * residual)
    forward_case(2, 3, 45, 50, dtype, act, residual, True, False, seed=act + 10 * residual)


@gpu
@pytest.mark.parametrize("size", [(2, 0, 8, 8), (2, 8, 0, 8), (0, 8, 8, 8), (2, 8, 9, 0), (1, 1, 3, 0)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_forward_empty(size, dtype):
    forward_case(*size, dtype, B.ACT_TANH, B.RESIDUAL_AFTER, True, True)


# -- placements -----------------------------------------------------------------------------------
def in_rows(offset, stride):
    """Matrices in workers' rows of `stride` values from `offset` on, as tensors lie in theta."""
    def put(t):
        buf = torch.full((t.shape[0], stride), 7.0, dtype=t.dtype, device=DEV)
        n = t[0].numel()
        assert offset + n <= stride
        v = buf[:, offset: offset + n].view(t.shape)
        v.copy_(t)
        return v
    return put


def columns_of(width, offset):
    def put(t):
        buf = torch.full((*t.shape[:2], width), 7.0, dtype=t.dtype, device=DEV)
        v = buf[:, :, offset: offset + t.shape[2]]
        v.copy_(t)
        return v
    return put


def tokens_first(t):
    """[rows, workers, columns]: a worker's row lies inside each token's."""
    buf = torch.empty((t.shape[1], t.shape[0], t.shape[2]), dtype=t.dtype, device=DEV)
    v = buf.transpose(0, 1)
    v.copy_(t)
    return v


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [3, 40, 200])
def test_forward_placements(dtype, rows):
    G, M, N, K = 3, rows, 77, 136
    for place in ({"w": in_rows(5, 12000), "bias": in_rows(3, 90)}, {"x": columns_of(150, 3), "y": columns_of(83, 1)},
                  {"x": columns_of(144, 8), "w": columns_of(160, 16)}, {"x": tokens_first, "y": tokens_first, "pre": tokens_first},
                  {"residual": columns_of(99, 11), "pre": columns_of(80, 2)}):
        forward_case(G, M, N, K, dtype, B.ACT_GELU, B.RESIDUAL_BEFORE, True, True, place=place)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [2, 70])
def test_forward_shared_inputs_and_in_place_residual(dtype, rows):
    G, N, K = 4, 50, 64
    g = torch.Generator().manual_seed(1)
    x1, w, r = make((1, rows, K), dtype, g).to(DEV), make((G, N, K), dtype, g, 0.1).to(DEV), make((G, rows, N), dtype, g).to(DEV)
    lin = B.Linear(rows, N, K, G, dtype, B.ACT_NONE, B.RESIDUAL_AFTER)
    ws = torch.empty(max(lin.workspace_bytes(), 256), dtype=torch.uint8, device=DEV)
    a, b = torch.empty_like(r), r.clone()
    lin.forward(lin.forward_io(x1.expand(G, -1, -1), w, a, residual=r), ws)
    lin.forward(lin.forward_io(x1.repeat(G, 1, 1), w, b, residual=b), ws)                    # y is the residual
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    w1, c, d = w[:1], torch.empty_like(r), torch.empty_like(r)                               # one matrix for all workers
    x = x1.repeat(G, 1, 1)
    lin.forward(lin.forward_io(x, w1.expand(G, -1, -1), c, residual=r[:, :1].expand(-1, rows, -1)), ws)
    lin.forward(lin.forward_io(x, w1.repeat(G, 1, 1), d, residual=r[:, :1].repeat(1, rows, 1)), ws)
    torch.cuda.synchronize()
    assert torch.equal(c, d)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [1, 5, 31, 64, 130])
def test_nothing_beside_the_outputs_is_written(dtype, M):
    G, N, K = 2, 67, 72
    buf = torch.full((G, M + 2, N + 6), 3.0, dtype=dtype, device=DEV)
    y = buf[:, 1: M + 1, 3: N + 3]
    x, w = torch.ones(G, M, K, dtype=dtype, device=DEV), torch.ones(G, N, K, dtype=dtype, device=DEV)
    lin = B.Linear(M, N, K, G, dtype)
    need = lin.workspace_bytes()
    ws = torch.full((need + 512,), 17, dtype=torch.uint8, device=DEV)
    lin.forward(lin.forward_io(x, w, y), ws[:need] if need else None)
    torch.cuda.synchronize()
    assert (y == K).all() and (ws[need:] == 17).all()
    y.fill_(3.0)
    assert (buf == 3.0).all()


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [4, 100])
def test_infinities_and_nan_stay_where_they_belong(dtype, M):
    G, N, K = 2, 40, 100
    g = torch.Generator().manual_seed(2)
    x, w = make((G, M, K), dtype, g).to(DEV), make((G, N, K), dtype, g, 0.1).to(DEV)
    lin = B.Linear(M, N, K, G, dtype)
    ws = torch.empty(max(lin.workspace_bytes(), 256), dtype=torch.uint8, device=DEV)
    clean, got = torch.empty(G, M, N, dtype=dtype, device=DEV), torch.empty(G, M, N, dtype=dtype, device=DEV)
    lin.forward(lin.forward_io(x, w, clean), ws)
    x[0, 1, 3], x[1, 2, K - 1], w[1, 7, 0] = float("nan"), float("inf"), -float("inf")
    lin.forward(lin.forward_io(x, w, got), ws)
    torch.cuda.synchronize()
    bad = torch.zeros(G, M, N, dtype=torch.bool, device=DEV)
    bad[0, 1], bad[1, 2], bad[1, :, 7] = True, True, True
    assert not torch.isfinite(got[bad]).any()
    assert torch.equal(got[~bad], clean[~bad])


@gpu
def test_f32_rows_of_very_different_sizes():
    # every row of x and of w has a scale of its own
    G, M, N, K = 1, 90, 70, 130
    g = torch.Generator().manual_seed(3)
    x = torch.randn(G, M, K, generator=g) * 10.0 ** torch.linspace(-30, 30, M)[None, :, None]
    w = torch.randn(G, N, K, generator=g) * 10.0 ** torch.linspace(-7, 7, N)[None, :, None]
    lin = B.Linear(M, N, K, G)
    ws = torch.empty(lin.workspace_bytes(), dtype=torch.uint8, device=DEV)
    y = torch.empty(G, M, N, device=DEV)
    lin.forward(lin.forward_io(x.to(DEV), w.to(DEV), y), ws)
    X, W = x.double(), w.double()
    S = mm(X.abs(), W.abs())
    check(y / 1.0, mm(X, W), sum_bound(K, S, torch.float32, spread(X, W)) + 2.0 ** -126, 2.0 ** -21 * S, "y")
    x.fill_(1.5e38)                                         # near the end of the range; and below its normal part
    w.zero_()
    w[0, :, 0] = 1.0
    w[0, 1, 0] = 1e-39
    lin.forward(lin.forward_io(x.to(DEV), w.to(DEV), y), ws)
    torch.cuda.synchronize()
    assert torch.allclose(y[0, :, 0].cpu().double(), x[0, :, 0].double(), rtol=2 ** -20)
    assert torch.allclose(y[0, :, 1].cpu().double(), (x.double()[0, :, 0] * w.double()[0, 1, 0]), rtol=2 ** -20)


# -- backward -------------------------------------------------------------------------------------
def matmul64(a, b):
    return torch.matmul(a, b)


def backward_case(G, M, N, K, dtype, act, residual, f32_grads=False, accumulate=False, seed=0, place=None, want=("dx", "dw", "dbias")):
    g = torch.Generator().manual_seed(100 + seed)
    x, w = make((G, M, K), dtype, g), make((G, N, K), dtype, g, max(K, 1) ** -0.5)
    dy, z = make((G, M, N), dtype, g, 0.3), make((G, M, N), dtype, g)
    gt = torch.float32 if f32_grads else dtype
    old_w, old_b = make((G, N, K), gt, g), make((G, N), gt, g)
    place = place or {}
    put = lambda name, t: place.get(name, lambda v: v.to(DEV))(t)
    lin = B.Linear(M, N, K, G, dtype, act, residual, weight_grad_f32=f32_grads, accumulate=accumulate)
    ws = torch.empty(max(lin.workspace_bytes(True), 256), dtype=torch.uint8, device=DEV)
    outs = {}
    if "dx" in want:
        outs["dx"] = put("dx", torch.full((G, M, K), float("nan"), dtype=dtype))
    if "dw" in want:
        outs["dw"] = put("dw", old_w if accumulate else torch.full((G, N, K), float("nan"), dtype=gt))
    if "dbias" in want:
        outs["dbias"] = put("dbias", old_b if accumulate else torch.full((G, N), float("nan"), dtype=gt))
    if "dresidual" in want:
        outs["dresidual"] = put("dresidual", torch.full((G, M, N), float("nan"), dtype=dtype))
    io = lin.backward_io(put("dy", dy), put("x", x), put("w", w), pre=put("pre", z) if act else None, **outs)
    lin.backward(io, ws, torch.cuda.current_stream())
    torch.cuda.synchronize()
    X, W, Z, DY = x.double(), w.double(), z.double(), dy.double()
    dz = DY * slope64(Z, act)
    bz = DY.abs() * 16 * U * (1 + Z.abs())                      # of dz itself
    h, hg = HALF[dtype], HALF[gt]
    r = bz + (h * dz.abs() + 2.0 ** -25 if dtype != torch.float32 else 0 * bz)       # as the products take it
    if "dx" in want:
        WT = W.transpose(1, 2)
        want_v, S = matmul64(dz, W), matmul64(dz.abs(), W.abs())
        b = sum_bound(N, S, dtype, spread(dz, WT)) + matmul64(r, W.abs())
        rms = 2.0 ** -21 * S + matmul64(r.square(), W.square()).sqrt()
        check(outs["dx"], want_v, b + h * (want_v.abs() + b) + 2.0 ** -25, rms + h * want_v.abs() + 2.0 ** -25, "dx")
    if "dw" in want:
        DT, XT = dz.transpose(1, 2), X.transpose(1, 2)
        want_v, S = matmul64(DT, X), matmul64(DT.abs(), X.abs())
        b = sum_bound(M, S, dtype, spread(DT, XT)) + matmul64(r.transpose(1, 2), X.abs())
        rms = 2.0 ** -21 * S + matmul64(r.transpose(1, 2).square(), X.square()).sqrt()
        if accumulate:
            want_v = want_v + old_w.double()
            b, rms = b + U * want_v.abs(), rms + U * want_v.abs()
        check(outs["dw"], want_v, b + hg * (want_v.abs() + b) + 2.0 ** -25, rms + hg * want_v.abs() + 2.0 ** -25, "dw")
    if "dbias" in want:
        want_v, S = dz.sum(1), dz.abs().sum(1)
        b = (M + 16) * U * S + bz.sum(1)
        rms = 2.0 ** -21 * S + bz.sum(1)
        if accumulate:
            want_v = want_v + old_b.double()
            b, rms = b + U * want_v.abs(), rms + U * want_v.abs()
        check(outs["dbias"], want_v, b + hg * (want_v.abs() + b) + 2.0 ** -25, rms + hg * want_v.abs() + 2.0 ** -25, "dbias")
    if "dresidual" in want:
        check(outs["dresidual"], dz, bz + h * (dz.abs() + bz) + 2.0 ** -25, bz + h * dz.abs() + 2.0 ** -25, "dresidual")
    return outs


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES)
def test_backward(size, dtype):
    i = SIZES.index(size)
    residual = B.RESIDUAL_BEFORE if i % 2 else B.RESIDUAL_NONE
    backward_case(*size, dtype, ACTS[(i + 1) % 6], residual, seed=i, want=("dx", "dw", "dbias") + (("dresidual",) if i % 2 else ()))


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ACTS)
def test_backward_every_activation(dtype, act):
    backward_case(2, 70, 45, 50, dtype, act, B.RESIDUAL_BEFORE, want=("dx", "dw", "dbias", "dresidual"), seed=act)
    backward_case(2, 70, 48, 64, dtype, act, B.RESIDUAL_NONE, f32_grads=True, accumulate=True, seed=act)
    backward_case(1, 2, 48, 64, dtype, act, B.RESIDUAL_AFTER, accumulate=True, seed=act)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("want", [("dx",), ("dw",), ("dbias",), ("dresidual",), ("dx", "dbias"), ("dw", "dresidual")])
@pytest.mark.parametrize("act", [B.ACT_NONE, B.ACT_TANH])
def test_backward_any_outputs(dtype, want, act):
    backward_case(3, 50, 72, 40, dtype, act, B.RESIDUAL_BEFORE, want=want)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("size", [(2, 0, 8, 9), (2, 8, 0, 9), (2, 8, 9, 0), (0, 8, 8, 8)])
def test_backward_empty(size, dtype, accumulate):
    backward_case(*size, dtype, B.ACT_SILU, B.RESIDUAL_NONE, accumulate=accumulate)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_backward_placements(dtype):
    for place in ({"w": in_rows(5, 12000), "dw": in_rows(5, 12000), "dbias": in_rows(3, 90)},
                  {"x": columns_of(150, 3), "dx": columns_of(150, 3), "dy": columns_of(83, 1)},
                  {"dy": columns_of(88, 8), "pre": columns_of(79, 1), "w": columns_of(144, 8)},
                  {"x": tokens_first, "dx": tokens_first, "dy": tokens_first, "dresidual": tokens_first}):
        for act in (B.ACT_NONE, B.ACT_RELU):
            backward_case(3, 90, 77, 136, dtype, act, B.RESIDUAL_BEFORE, place=place, want=("dx", "dw", "dbias", "dresidual"))


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_backward_of_shared_inputs_is_each_workers_own(dtype):
    G, M, N, K = 3, 40, 24, 56
    g = torch.Generator().manual_seed(5)
    x, w, dy, z = (make(s, dtype, g).to(DEV) for s in ((1, M, K), (1, N, K), (1, M, N), (G, M, N)))
    for act in (B.ACT_NONE, B.ACT_TANH):
        lin = B.Linear(M, N, K, G, dtype, act)
        ws = torch.empty(lin.workspace_bytes(True), dtype=torch.uint8, device=DEV)
        res = []
        for spread_out in (lambda t: t.expand(G, -1, -1), lambda t: t.repeat(G, 1, 1)):
            dx, dw, db = (torch.empty(s, dtype=dtype, device=DEV) for s in ((G, M, K), (G, N, K), (G, N)))
            lin.backward(lin.backward_io(spread_out(dy), spread_out(x), spread_out(w), pre=z if act else None, dx=dx, dw=dw, dbias=db), ws)
            res.append((dx, dw, db))
        torch.cuda.synchronize()
        for a, b in zip(*res):
            assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences(act):
    """<grad, v> against (L(+h v) - L(-h v)) / 2h with L = sum(c * y), both by the library, f32.  Error of the quotient: h^2 / 6
    times the third derivative (below 3 |c| |dz|^3 here) and the roundings of L over h."""
    G, M, N, K, h = 2, 33, 29, 47, 2.0 ** -6
    g = torch.Generator().manual_seed(6)
    x, w, b, r, c = (torch.randn(s, generator=g).to(DEV) for s in ((G, M, K), (G, N, K), (G, N), (G, M, N), (G, M, N)))
    w = w * K ** -0.5
    lin = B.Linear(M, N, K, G, torch.float32, act, B.RESIDUAL_BEFORE)
    ws = torch.empty(max(lin.workspace_bytes(), lin.workspace_bytes(True)), dtype=torch.uint8, device=DEV)

    def loss(x, w, b, r):
        y, z = torch.empty(G, M, N, device=DEV), torch.empty(G, M, N, device=DEV)
        lin.forward(lin.forward_io(x, w, y, bias=b, residual=r, pre=z), ws, torch.cuda.current_stream())
        return (y.double() * c.double()).sum().item(), z, y
    L0, z, _ = loss(x, w, b, r)
    if act == B.ACT_RELU:                                    # away from its corner: differences see no slope there
        c = torch.where(z.abs() < 0.25, torch.zeros_like(c), c)
    grads = [torch.empty_like(t) for t in (x, w, b, r)]
    lin.backward(lin.backward_io(c, x, w, pre=z, dx=grads[0], dw=grads[1], dbias=grads[2], dresidual=grads[3]), ws, torch.cuda.current_stream())
    for i in range(4):
        v = torch.randn(grads[i].shape, generator=g).to(DEV)
        v = v / (8 if i < 2 else 4)
        args = [x, w, b, r]
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + h * v, args[i] - h * v
        (lu, _, yu), (ld, _, yd) = loss(*up), loss(*down)
        want = (lu - ld) / (2 * h)
        got = (grads[i].double() * v.double()).sum().item()
        move = (yu - yd).double().abs().max().item() / (2 * h)          # the largest |d y| along v
        tol = h * h / 6 * 3 * (c.double().abs().sum().item()) * max(move, 1.0) ** 3 * 0.05 + 2.0 ** -20 * (c.abs() * yu.abs()).double().sum().item() / h * 0.05
        assert abs(got - want) <= tol + 1e-3 * abs(want), (i, got, want, tol)


@gpu
@pytest.mark.parametrize("act", ACTS[1:])
def test_activations_and_slopes_over_the_range(act):
    """z = x * 1, f32: the exponentials and reciprocals are within 2 units and 1, a handful of roundings around them: 16 half units of
    the value itself, of 1 + |z| where a slope's two terms cancel.  Nothing is asked below 2^-120."""
    z = torch.cat([torch.linspace(-12, 12, 4001), torch.tensor([0.0, 1e-30, -1e-30, 0.25, -0.25, 0.2499999, -0.2499999, 3e-5, 19.0, -30.0, 31.0, 86.0, -86.0,
                                                               1e4, -1e4, 1e20, -1e20, 3e38, -3e38])])
    M = z.numel()
    lin = B.Linear(M, 1, 1, 1, torch.float32, act, B.RESIDUAL_BEFORE)
    ws = torch.empty(max(lin.workspace_bytes(), lin.workspace_bytes(True), 256), dtype=torch.uint8, device=DEV)
    one, r = torch.ones(1, 1, device=DEV), torch.zeros(M, 1, device=DEV)
    x, y, d = z.view(M, 1).to(DEV), torch.empty(M, 1, device=DEV), torch.empty(M, 1, device=DEV)
    lin.forward(lin.forward_io(x, one, y, residual=r), ws)
    lin.backward(lin.backward_io(torch.ones(M, 1, device=DEV), x, one, pre=x, dresidual=d), ws)
    got, slope = y.cpu().double().view(-1), d.cpu().double().view(-1)
    Z = z.double()
    want = act64(Z, act)
    finite = torch.isfinite(got)
    assert finite.all() and ((got - want).abs() <= 16 * U * want.abs() + 2.0 ** -120).all(), (got - want).abs().max()
    inside = Z.abs() <= 100
    w = slope64(Z, act)[inside]
    if act == B.ACT_SIGMOID:                               # y (1 - y) has no bits left in 64 where y is near 1
        w = 1 / (2 * torch.cosh(Z[inside] / 2)) ** 2
    if act == B.ACT_TANH:
        w = 1 / torch.cosh(Z[inside]) ** 2
    size = w.abs() if act in (B.ACT_RELU, B.ACT_SIGMOID, B.ACT_TANH) else 1 + Z[inside].abs()
    assert ((slope[inside] - w).abs() <= 16 * U * size + 2.0 ** -120).all()
    far = {B.ACT_SIGMOID: (0.0, 0.0), B.ACT_TANH: (0.0, 0.0)}.get(act, (0.0, 1.0))
    assert (slope[Z < -100] == far[0]).all() and (slope[Z > 100] == far[1]).all()
    x[:] = float("nan")
    lin.forward(lin.forward_io(x, one, y, residual=r), ws)
    lin.backward(lin.backward_io(torch.ones(M, 1, device=DEV), x, one, pre=x, dresidual=d), ws)
    assert torch.isnan(y).all() and torch.isnan(d).all()
    for value, wanted in ((float("inf"), {B.ACT_SIGMOID: 1.0, B.ACT_TANH: 1.0}.get(act, float("inf"))), (float("-inf"), {B.ACT_TANH: -1.0}.get(act, 0.0))):
        x[:] = value
        lin.forward(lin.forward_io(x, one, y, residual=r), ws)
        if value > 0 or act in (B.ACT_RELU, B.ACT_SIGMOID, B.ACT_TANH):             # -inf * 0 is NaN in the others' formulas
            assert (y == wanted).all()


# -- sizes that take the larger tiles, operands laid out, split sums ---------------------------------
LARGE = [(16, 1030, 1031, 1029), (16, 1024, 1040, 1032), (2, 4100, 2056, 136), (1, 2049, 4104, 3001), (1, 200, 6000, 2500), (3, 300, 128, 9000),
         (1, 70, 3000, 10240), (16, 1024, 776, 1016), (16, 1021, 775, 1013)]


def product64(a, b):
    """a b' for every worker, in 64 bits on the GPU."""
    return torch.stack([(x.to(DEV) @ y.to(DEV).T.contiguous()).cpu() for x, y in zip(a, b)])


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", LARGE)
@pytest.mark.parametrize("kind", [(B.ACT_NONE, B.RESIDUAL_NONE), (B.ACT_GELU, B.RESIDUAL_AFTER)])
def test_forward_large(size, dtype, kind, monkeypatch):
    monkeypatch.setitem(globals(), "mm", product64)
    forward_case(*size, dtype, kind[0], kind[1], True, kind[0] != 0, seed=7)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", LARGE)
@pytest.mark.parametrize("act", [B.ACT_NONE, B.ACT_TANH])
def test_backward_large(size, dtype, act, monkeypatch):
    monkeypatch.setitem(globals(), "matmul64", lambda a, b: product64(a, b.transpose(1, 2)))
    backward_case(*size, dtype, act, B.RESIDUAL_BEFORE, f32_grads=act == 0, accumulate=act == 0, seed=7,
                  want=("dx", "dw", "dbias") + (("dresidual",) if act else ()))


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_large_placements_and_each_output_alone(dtype, monkeypatch):
    monkeypatch.setitem(globals(), "mm", product64)
    monkeypatch.setitem(globals(), "matmul64", lambda a, b: product64(a, b.transpose(1, 2)))
    G, M, N, K = 4, 1100, 1030, 520
    aligned = {"x": columns_of(528, 8), "y": columns_of(1048, 0), "w": in_rows(8, N * K + 16), "dy": columns_of(1048, 16), "dx": columns_of(533, 1)}
    odd = {"x": columns_of(531, 3), "y": columns_of(1037, 1), "w": in_rows(5, N * K + 7), "dy": tokens_first, "dx": tokens_first, "dw": in_rows(3, N * K + 9)}
    for place in (aligned, odd):
        forward_case(G, M, N, K, dtype, B.ACT_SILU, B.RESIDUAL_BEFORE, True, True, place=place)
        backward_case(G, M, N, K, dtype, B.ACT_NONE, B.RESIDUAL_BEFORE, place=place, want=("dx", "dw", "dbias", "dresidual"))
    for want in (("dx",), ("dw",), ("dbias",), ("dresidual",)):
        backward_case(G, M, N, K, dtype, B.ACT_RELU, B.RESIDUAL_BEFORE, want=want)


# -- sizes whose gradients' sums are cut between few and many workgroups, with ragged edges -----------
MIDDLE = [(1, 64, 20000, 64), (4, 128, 2600, 66), (3, 100, 513, 301), (2, 66, 1030, 3), (8, 128, 650, 650), (2, 70, 2, 1500), (1, 65, 4100, 2)]


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", MIDDLE)
def test_middle_sizes(size, dtype):
    forward_case(*size, dtype, B.ACT_TANH, B.RESIDUAL_BEFORE, True, True, seed=9)
    backward_case(*size, dtype, B.ACT_GELU, B.RESIDUAL_BEFORE, seed=9, want=("dx", "dw", "dbias", "dresidual"))
    backward_case(*size, dtype, B.ACT_NONE, B.RESIDUAL_BEFORE, f32_grads=True, accumulate=True, seed=10)


@gpu
@pytest.mark.parametrize("size", [(1, 900, 1100, 2050), (1, 700, 750, 4500)])
def test_f32_rows_of_very_different_sizes_in_large_products(size):
    """Rows and columns over 60 and 14 powers of ten: each has a scale of its own, in both directions."""
    G, M, N, K = size
    g = torch.Generator().manual_seed(12)
    over = lambda e, n: 10.0 ** torch.linspace(-e, e, n)
    x, w = torch.randn(G, M, K, generator=g) * over(15, M)[None, :, None], torch.randn(G, N, K, generator=g) * over(7, N)[None, :, None]
    lin = B.Linear(M, N, K, G)
    ws = torch.empty(max(lin.workspace_bytes(), lin.workspace_bytes(True)), dtype=torch.uint8, device=DEV)
    y = torch.empty(G, M, N, device=DEV)
    lin.forward(lin.forward_io(x.to(DEV), w.to(DEV), y), ws)
    X, W = x.double(), w.double()
    S = product64(X.abs(), W.abs())
    check(y, product64(X, W), sum_bound(K, S, torch.float32, spread(X, W)) + 2.0 ** -126, 2.0 ** -21 * S, "y")
    # dx sums over n, dw over the rows: dz has a scale for each of its rows, then for each of its columns
    dy = torch.randn(G, M, N, generator=g)
    for d, b, what in ((dy * over(15, M)[None, :, None], torch.randn(G, N, K, generator=g) * over(7, K)[None, None], "dx"),
                       (dy * over(15, N)[None, None], torch.randn(G, M, K, generator=g) * over(7, K)[None, None], "dw")):
        out = torch.empty(G, M if what == "dx" else N, K, device=DEV)
        io = lin.backward_io(d.to(DEV), w=b.to(DEV), dx=out) if what == "dx" else lin.backward_io(d.to(DEV), x=b.to(DEV), dw=out)
        lin.backward(io, ws)
        p, q = (d if what == "dx" else d.transpose(1, 2)).double(), b.transpose(1, 2).double()
        S = product64(p.abs(), q.abs())
        check(out, product64(p, q), sum_bound(p.shape[2], S, torch.float32, spread(p, q)) + 2.0 ** -126, 2.0 ** -21 * S, what)


@gpu
def test_infinities_in_large_f32_products_reach_only_their_rows():
    G, M, N, K = 2, 800, 900, 3001
    g = torch.Generator().manual_seed(13)
    x, w = (torch.randn(s, generator=g).to(DEV) for s in ((G, M, K), (G, N, K)))
    lin = B.Linear(M, N, K, G)
    ws = torch.empty(lin.workspace_bytes(), dtype=torch.uint8, device=DEV)
    clean, got = torch.empty(G, M, N, device=DEV), torch.empty(G, M, N, device=DEV)
    lin.forward(lin.forward_io(x, w, clean), ws)
    x[0, 5, 7], x[1, 700, 3000], w[1, 899, 0] = float("inf"), float("nan"), float("-inf")
    lin.forward(lin.forward_io(x, w, got), ws)
    torch.cuda.synchronize()
    bad = torch.zeros(G, M, N, dtype=torch.bool, device=DEV)
    bad[0, 5], bad[1, 700], bad[1, :, 899] = True, True, True
    assert not torch.isfinite(got[bad]).any() and torch.equal(got[~bad], clean[~bad])


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act,N", [(B.ACT_NONE, 4104), (B.ACT_GELU, 4099)])
def test_results_above_what_the_caches_hold_are_those_of_their_rows(dtype, act, N):
    """Every element's sum has one order, so a call gives the bits of calls on its rows, whose results are small (but whose
    products are large enough for f32 to be taken apart)."""
    G, M, K = 2, 8232, 160
    g = torch.Generator().manual_seed(15)
    x, w, b, r = (make(s, dtype, g).to(DEV) for s in ((G, M, K), (G, N, K), (G, N), (G, 1, N)))
    r = r.expand(G, M, N)

    def run(x, r):
        lin = B.Linear(x.shape[1], N, K, G, dtype, act, B.RESIDUAL_AFTER)
        y = torch.empty(G, x.shape[1], N, dtype=dtype, device=DEV)
        z = torch.empty_like(y) if act else None
        ws = torch.empty(max(lin.workspace_bytes(), 256), dtype=torch.uint8, device=DEV)
        lin.forward(lin.forward_io(x, w, y, bias=b, residual=r, pre=z), ws, torch.cuda.current_stream())
        torch.cuda.synchronize()
        return y, z
    y, z = run(x, r)
    for i in range(0, M, 2058):
        part = [t.contiguous() for t in (x[:, i: i + 2058], r[:, i: i + 2058])]
        py, pz = run(*part)
        assert torch.equal(y[:, i: i + 2058], py) and (z is None or torch.equal(z[:, i: i + 2058], pz))
    X, W, rows = x[:, 4000:4050].cpu().double(), w.cpu().double(), slice(4000, 4050)
    s, S = mm(X, W) + b.cpu().double()[:, None], mm(X.abs(), W.abs()) + b.cpu().double().abs()[:, None]
    out, h = act64(s, act) + r[:, rows].cpu().double(), HALF[dtype]
    bound = 1.2 * sum_bound(K, S, dtype, spread(X, W)) + 16 * U * (s.abs() + out.abs() + 1)
    assert ((y[:, rows].cpu().double() - out).abs() <= bound + h * (out.abs() + bound) + 2.0 ** -25).all()


# -- streams, graphs, equal bits ------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(2, 1, 300, 600), (2, 150, 130, 2048)])
def test_equal_calls_give_equal_bits_on_any_stream_and_in_graphs(dtype, size):
    G, M, N, K = size
    g = torch.Generator().manual_seed(8)
    x, w, dy = (make(s, dtype, g).to(DEV) for s in ((G, M, K), (G, N, K), (G, M, N)))
    lin = B.Linear(M, N, K, G, dtype, B.ACT_SIGMOID)
    ws = torch.empty(max(lin.workspace_bytes(), lin.workspace_bytes(True)), dtype=torch.uint8, device=DEV)
    bufs = [[torch.zeros(s, dtype=dtype, device=DEV) for s in ((G, M, N), (G, M, N), (G, M, K), (G, N, K), (G, N))] for _ in range(2)]

    def both(o, stream):
        lin.forward(lin.forward_io(x, w, o[0], pre=o[1]), ws, stream)
        lin.backward(lin.backward_io(dy, x, w, pre=o[1], dx=o[2], dw=o[3], dbias=o[4]), ws, stream)
    torch.cuda.synchronize()
    both(bufs[0], None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both(bufs[1], side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*bufs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both(bufs[1], torch.cuda.current_stream())
    for replay in range(3):
        x.copy_(make((G, M, K), dtype, g))
        for t in bufs[1]:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        both(bufs[0], None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*bufs)), replay
        assert torch.randn(1 << 18, device=DEV).sum().item() != 0.5         # eager work between the replays


# -- refusals (no GPU needed: they come before the device is asked) ---------------------------------
def code_of(fn):
    with pytest.raises(B.GbmufError) as e:
        fn()
    return e.value.code


def test_descriptions_that_are_refused():
    for kw in (dict(rows=-1, out_features=4, in_features=4), dict(rows=4, out_features=-1, in_features=4),
               dict(rows=4, out_features=4, in_features=-1), dict(rows=4, out_features=4, in_features=4, batch=-1),
               dict(rows=4, out_features=4, in_features=4, activation=6), dict(rows=4, out_features=4, in_features=4, activation=-1),
               dict(rows=4, out_features=4, in_features=4, residual=3), dict(rows=4, out_features=4, in_features=4, dtype=torch.float64)):
        assert code_of(lambda: B.Linear(**kw)) == B.GBMUF_EINVAL, kw
    for kw in (dict(rows=2 ** 31, out_features=4, in_features=4), dict(rows=4, out_features=2 ** 31, in_features=4),
               dict(rows=4, out_features=4, in_features=2 ** 31), dict(rows=4, out_features=4, in_features=4, batch=65536)):
        assert code_of(lambda: B.Linear(**kw)) == B.GBMUF_EUNSUPPORTED, kw
    d = B.LinearDesc(ctypes.sizeof(B.LinearDesc) - 8, 0, 1, 0, 0, 0, 0, 0, 4, 4, 4)
    n = ctypes.c_int64()
    assert B.lib().gbmuf_linear_workspace(ctypes.byref(d), 0, ctypes.byref(n)) == B.GBMUF_EINVAL
    assert B.lib().gbmuf_linear_workspace(None, 0, ctypes.byref(n)) == B.GBMUF_EINVAL


def test_matrices_that_are_refused():
    G, M, N, K = 2, 6, 8, 5
    lin = B.Linear(M, N, K, G, torch.float32, B.ACT_TANH, B.RESIDUAL_BEFORE)
    x, w, r, y, z = (torch.zeros(s) for s in ((G, M, K), (G, N, K), (G, M, N), (G, M, N), (G, M, N)))
    ws = torch.zeros(lin.workspace_bytes() + 256, dtype=torch.uint8)
    ws = ws[-ws.data_ptr() % 256:][: lin.workspace_bytes()]
    for bad in (dict(x=torch.zeros(G, M, K + 1)), dict(w=torch.zeros(G, N, K, dtype=torch.float16)), dict(y=torch.zeros(G, N, M).transpose(1, 2)),
                dict(residual=torch.zeros(M, N)), dict(bias=torch.zeros(N))):
        kw = dict(dict(x=x, w=w, y=y, residual=r), **bad)
        assert code_of(lambda: lin.forward_io(**kw)) == B.GBMUF_EINVAL, list(bad)
    run = lambda space=ws, **kw: lin.forward(lin.forward_io(**dict(dict(x=x, w=w, y=y, residual=r), **kw)), space)
    assert code_of(lambda: run(residual=None)) == B.GBMUF_EINVAL                  # the residual is missing
    assert code_of(lambda: run(x=None)) == B.GBMUF_EINVAL
    assert code_of(lambda: run(y=None)) == B.GBMUF_EINVAL
    assert code_of(lambda: run(y=y[:1].expand(G, -1, -1))) == B.GBMUF_EINVAL      # elements on top of each other
    assert code_of(lambda: run(y=y[:, :1].expand(-1, M, -1))) == B.GBMUF_EINVAL
    assert code_of(lambda: run(pre=y)) == B.GBMUF_EINVAL
    assert code_of(lambda: run(pre=r)) == B.GBMUF_EINVAL
    big = torch.zeros(4 * G * M * N)
    assert code_of(lambda: run(y=big[: G * M * N].view(G, M, N), x=big[10: 10 + G * M * K].view(G, M, K))) == B.GBMUF_EINVAL
    assert code_of(lambda: run(y=big[: G * M * N].view(G, M, N), residual=big[1: 1 + G * M * N].view(G, M, N))) == B.GBMUF_EINVAL
    io = lin.forward_io(x, w, y, residual=r)
    io.x.ld = -5
    assert code_of(lambda: lin.forward(io, ws)) == B.GBMUF_EINVAL
    io = lin.forward_io(x, w, y, residual=r)
    io.y.data += 2
    assert code_of(lambda: lin.forward(io, ws)) == B.GBMUF_EINVAL
    dy, dx, dw = torch.zeros(G, M, N), torch.zeros(G, M, K), torch.zeros(G, N, K)
    need = lin.workspace_bytes(True)
    space = torch.zeros(need + 256, dtype=torch.uint8)
    space = space[-space.data_ptr() % 256:][:need]
    back = lambda **kw: lin.backward(lin.backward_io(**dict(dict(dy=dy, x=x, w=w, pre=z, dx=dx, dw=dw), **kw)), space)
    assert code_of(lambda: back(pre=None)) == B.GBMUF_EINVAL
    assert code_of(lambda: back(dy=None)) == B.GBMUF_EINVAL
    assert code_of(lambda: back(x=None)) == B.GBMUF_EINVAL
    assert code_of(lambda: back(w=None)) == B.GBMUF_EINVAL
    assert code_of(lambda: back(dx=x)) == B.GBMUF_EINVAL
    assert code_of(lambda: back(dresidual=dy)) == B.GBMUF_EINVAL
    after = B.Linear(M, N, K, G, torch.float32, B.ACT_NONE, B.RESIDUAL_AFTER)
    assert code_of(lambda: after.backward(after.backward_io(dy, dresidual=z), space)) == B.GBMUF_EINVAL


def test_workspaces_that_overlap_and_strides_beyond_any_memory_are_refused():
    G, M, N, K = 2, 1500, 1500, 1500                       # a size that takes a workspace
    lin = B.Linear(M, N, K, G)
    need = lin.workspace_bytes()
    assert need > 0
    at = lambda k: B.Matrix((1 << 40) + (k << 30), K, M * K)           # places that are only compared
    io = B.LinearIo()
    io.x, io.w, io.y = at(0), at(1), at(2)
    lib, d = B.lib(), lin.desc
    call = lambda space: lib.gbmuf_linear(ctypes.byref(d), ctypes.byref(io), space, need, None)
    for k in range(3):
        assert call((1 << 40) + (k << 30)) == B.GBMUF_EINVAL and call((1 << 40) + (k << 30) + 70312 * 256) == B.GBMUF_EINVAL
    for k in range(3):
        for field in ("ld", "batch_stride"):
            io = B.LinearIo()
            io.x, io.w, io.y = at(0), at(1), at(2)
            setattr((io.x, io.w, io.y)[k], field, (1 << 62) + 5)
            assert call(1 << 45) == B.GBMUF_EINVAL


def test_outputs_side_by_side_are_taken():
    """Views that interleave without sharing a value pass every check: without a GPU the call then ends at the device."""
    if torch.cuda.is_available():
        pytest.skip("host memory")
    G, M, N, K = 3, 4, 8, 8
    lin = B.Linear(M, N, K, G, torch.float32)
    need = lin.workspace_bytes()
    ws = torch.zeros(need + 256, dtype=torch.uint8)
    ws = ws[-ws.data_ptr() % 256:][:need]
    x, w = torch.zeros(G, M, K), torch.zeros(G, N, K)
    row = torch.zeros(G, M, 2 * N)
    for y, z in ((row[:, :, :N], row[:, :, N:]), (row.view(M, G, 2 * N).transpose(0, 1)[:, :, :N], row.view(M, G, 2 * N).transpose(0, 1)[:, :, N:])):
        assert code_of(lambda: lin.forward(lin.forward_io(x, w, y, pre=z), ws)) == B.GBMUF_EDEVICE
    grow = torch.zeros(G, N * K + N)
    back = torch.zeros(lin.workspace_bytes(True) + 256, dtype=torch.uint8)
    back = back[-back.data_ptr() % 256:][: lin.workspace_bytes(True)]
    io = lin.backward_io(torch.zeros(G, M, N), x, w, dw=grow[:, : N * K].view(G, N, K), dbias=grow[:, N * K:])
    assert code_of(lambda: lin.backward(io, back)) == B.GBMUF_EDEVICE


def test_workspace_that_is_missing_or_too_small_is_refused():
    """Sizes that lay operands out.  The matrices are addresses that no check follows."""
    if torch.cuda.is_available():
        pytest.skip("addresses of no memory")
    G, M, N, K = 1, 8192, 8192, 8192
    at = lambda i: B.Matrix((i + 1) << 40, K, 0)
    for dtype, item in ((torch.float32, 4), (torch.bfloat16, 2)):
        lin = B.Linear(M, N, K, G, dtype)
        need, back = lin.workspace_bytes(), lin.workspace_bytes(True)
        assert need >= G * (M * K + N * K) * item and back >= G * (M * N + N * K + M * K) * item     # one copy of each operand
        io = B.LinearIo(x=at(0), w=at(1), y=at(2))
        grad = B.LinearGradIo(x=at(0), w=at(1), dy=at(2), dx=at(3), dw=at(4))
        L, d = B.lib(), ctypes.byref(lin.desc)
        for p, n in ((None, need), (1 << 50, need - 1), ((1 << 50) + 128, need)):
            assert L.gbmuf_linear(d, ctypes.byref(io), p, n, None) == B.GBMUF_EINVAL
            assert L.gbmuf_linear_backward(d, ctypes.byref(grad), p, n - need + back, None) == B.GBMUF_EINVAL
        assert L.gbmuf_linear(d, ctypes.byref(io), 1 << 50, need, None) == B.GBMUF_EDEVICE
        assert L.gbmuf_linear_backward(d, ctypes.byref(grad), 1 << 50, back, None) == B.GBMUF_EDEVICE
    assert B.Linear(0, 8, 8, 1).workspace_bytes() < 1 << 20


# -- few rows against many outputs: the wide forms, tiles for 33 to 64 rows, and 16-bit rows that lie on 16 bytes or do not ------
WIDE = [(1, 8, 32801, 72), (1, 16, 32803, 66), (1, 17, 32771, 40), (1, 20, 32803, 136), (2, 32, 16400, 44), (1, 33, 32769, 24), (1, 64, 32801, 130),
        (16, 40, 2100, 264), (16, 17, 2050, 65)]


def whole_pieces(n):
    return (n + 7) // 8 * 8


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("size", WIDE)
def test_few_rows_against_many_outputs(size, aligned, dtype):
    """Every act and residual in turn; what lies beside the outputs stays."""
    G, M, N, K = size
    i = WIDE.index(size) + (3 if aligned else 0)
    if aligned:
        place = {"x": columns_of(whole_pieces(K) + 8, 8), "w": columns_of(whole_pieces(K), 0)}
    else:
        place = {"x": columns_of(K + 3, 1), "w": in_rows(5, N * K + 7)}
    place.update({"y": columns_of(N + 5, 3), "pre": columns_of(N + 4, 1), "residual": columns_of(N + 9, 2)})
    y, z = forward_case(*size, dtype, ACTS[i % 6], i % 3, True, i % 2 == 0, seed=20 + i, place=place)
    for t, first in ((y, 3), (z, 1)):
        if t is not None:
            buf = t._base
            assert buf.shape[2] > N and (buf[:, :, :first] == 7.0).all() and (buf[:, :, first + N:] == 7.0).all()


# -- f32 taken apart: what a wide range inside a row and infinities leave ------------------------------------------------
def wide_rows(shape, g):
    """Magnitudes from 1 down to 2^-35 along the last axis."""
    n = shape[-1]
    return torch.randn(shape, generator=g).sign() * (0.5 + 0.5 * torch.rand(shape, generator=g)) * 2.0 ** torch.linspace(0, -35, n)


def small_part_only(shape, g):
    """Zero where wide_rows is above 2^-28."""
    t = torch.randn(shape, generator=g)
    t[..., : shape[-1] * 4 // 5] = 0
    return t


@gpu
@pytest.mark.parametrize("swap", [False, True])
@pytest.mark.parametrize("size", [(1, 900, 1100, 2050), (1, 700, 750, 4500)])
def test_f32_values_far_below_their_rows_largest(size, swap):
    """Only values below 2^-28 of their row's largest meet anything but zeros: what is kept of them, 2^-39 of the largest, is all
    that results have.  Forward, dx and dw, the wide rows on either side."""
    G, M, N, K = size
    g = torch.Generator().manual_seed(31)
    f, h = (small_part_only, wide_rows) if swap else (wide_rows, small_part_only)
    lin = B.Linear(M, N, K, G)
    ws = torch.empty(max(lin.workspace_bytes(), lin.workspace_bytes(True)), dtype=torch.uint8, device=DEV)
    x, w = f((G, M, K), g), h((G, N, K), g)
    y = torch.empty(G, M, N, device=DEV)
    lin.forward(lin.forward_io(x.to(DEV), w.to(DEV), y), ws)
    results = [(y, x, w, "y")]
    dz, w = f((G, M, N), g), h((G, K, N), g)
    dx = torch.empty(G, M, K, device=DEV)
    lin.backward(lin.backward_io(dz.to(DEV), w=w.transpose(1, 2).contiguous().to(DEV), dx=dx), ws)
    results.append((dx, dz, w, "dx"))
    dz, x = f((G, N, M), g), h((G, K, M), g)
    dw = torch.empty(G, N, K, device=DEV)
    lin.backward(lin.backward_io(dz.transpose(1, 2).contiguous().to(DEV), x=x.transpose(1, 2).contiguous().to(DEV), dw=dw), ws)
    results.append((dw, dz, x, "dw"))
    for got, a, b, what in results:
        a, b = a.double(), b.double()
        S = product64(a.abs(), b.abs())
        bound = sum_bound(a.shape[2], S, torch.float32, spread(a, b))
        check(got, product64(a, b), bound, bound, what)
        assert (product64(a, b).abs() > 4 * bound).double().mean() > 0.3, what          # the bound is not the result itself


@gpu
@pytest.mark.parametrize("size", [(2, 800, 900, 3001), (1, 700, 750, 4500)])
def test_infinities_in_large_f32_products_are_those_of_the_definition(size):
    """Infinities against values, zeros, each other at the same place and at others, and NaN: the pattern that 64 bits give, and finite
    results as they are without."""
    G, M, N, K = size
    inf, nan = float("inf"), float("nan")
    g = torch.Generator().manual_seed(32)

    def spoil(a, b):                                         # a product over the last axis of both
        a[0, 5, 7], a[0, 6, 11], a[0, 9, 20], a[0, 30, 40], a[0, 31, 41], a[G - 1, 50, 60] = inf, -inf, inf, -inf, 1e6, nan
        b[0, 3, 9], b[0, 4, 11], b[0, 10, 7], b[0, 11, 20], b[0, 12, 40] = inf, inf, 0.0, -inf, -inf
        return a, b

    def same(got, clean, a, b, what):
        want = torch.matmul(a.double(), b.double().transpose(1, 2))
        got = got.cpu()
        finite = torch.isfinite(want)
        assert torch.equal(torch.isnan(got), torch.isnan(want)), what
        assert torch.equal(got == inf, want == inf) and torch.equal(got == -inf, want == -inf), what
        assert 500 < (~finite).sum() < finite.sum(), what
        rows = torch.ones(got.shape, dtype=torch.bool)
        rows[0, 31], rows[0, :, 10] = False, False           # other finite values than before
        assert torch.equal(got[finite & rows], clean.cpu()[finite & rows]), what
    lin = B.Linear(M, N, K, G)
    ws = torch.empty(max(lin.workspace_bytes(), lin.workspace_bytes(True)), dtype=torch.uint8, device=DEV)
    turn = lambda t: t.transpose(1, 2).contiguous().to(DEV)
    for what, rows, columns, over in (("y", M, N, K), ("dx", M, K, N), ("dw", N, K, M)):
        a, b = torch.randn((G, rows, over), generator=g), torch.randn((G, columns, over), generator=g)
        out = []
        for p, q in ((a, b), spoil(a.clone(), b.clone())):
            o = torch.empty(G, rows, columns, device=DEV)
            if what == "y":
                lin.forward(lin.forward_io(p.to(DEV), q.to(DEV), o), ws)
            elif what == "dx":
                lin.backward(lin.backward_io(p.to(DEV), w=turn(q), dx=o), ws)
            else:
                lin.backward(lin.backward_io(turn(p), x=turn(q), dw=o), ws)
            torch.cuda.synchronize()
            out.append((o, p, q))
        same(out[1][0], out[0][0], out[1][1], out[1][2], what)


@gpu
def test_more_rows_than_one_dimension_of_a_grid():
    """36 M rows of f32 that are taken apart, 9 M workgroups, 56 GB: every value is written, and rows are those of calls on few of them."""
    M, N, K, part = 36_000_000, 256, 64, 1_000_000
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("memory")
    lin, small = B.Linear(M, N, K), B.Linear(part, N, K)
    g = torch.Generator(device=DEV).manual_seed(33)
    x, y, w = torch.empty(M, K, device=DEV), torch.empty(M, N, device=DEV), torch.randn(N, K, generator=g, device=DEV)
    for i in range(0, M, part):
        x[i: i + part].normal_(generator=g)
        y[i: i + part].fill_(float("nan"))
    ws = torch.empty(lin.workspace_bytes(), dtype=torch.uint8, device=DEV)
    lin.forward(lin.forward_io(x, w, y), ws, torch.cuda.current_stream())
    torch.cuda.synchronize()
    few = torch.empty(part, N, device=DEV)
    for i in range(0, M, part):
        if i % (5 * part) == 0 or i in (33 * part, 34 * part, 16 * part, 17 * part):
            small.forward(small.forward_io(x[i: i + part], w, few), ws, torch.cuda.current_stream())
            assert torch.equal(y[i: i + part], few), i
        assert torch.isfinite(y[i: i + part]).all(), i
    X, W = x[None, -1000:].cpu().double(), w[None].cpu().double()
    S = mm(X.abs(), W.abs())
    check(y[None, -1000:], mm(X, W), sum_bound(K, S, torch.float32, spread(X, W)), 2.0 ** -21 * S, "y")


def test_tensors_of_the_host_and_of_several_devices_are_refused(monkeypatch):
    """Before the call: a kernel that read them would fault.  (Without a GPU the library says that one is missing, as before.)"""
    G, M, N, K = 2, 70, 80, 90
    lin = B.Linear(M, N, K, G)
    space = lambda n: (lambda t: t[-t.data_ptr() % 256:][:n])(torch.zeros(n + 256, dtype=torch.uint8))
    x, w, y, dw = torch.zeros(G, M, K), torch.zeros(G, N, K), torch.zeros(G, M, N), torch.zeros(G, N, K)
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    io, grad = lin.forward_io(x, w, y), lin.backward_io(y, x, dw=dw)
    assert code_of(lambda: lin.forward(io, space(lin.workspace_bytes()))) == B.GBMUF_EINVAL
    assert code_of(lambda: lin.backward(grad, space(lin.workspace_bytes(True)))) == B.GBMUF_EINVAL
    bare = B.LinearIo(x=B.Matrix(1 << 40, K, M * K), w=B.Matrix(1 << 41, K, N * K), y=B.Matrix(1 << 42, N, M * N))      # as if on the GPU
    assert code_of(lambda: lin.forward(bare, torch.zeros(1 << 20, dtype=torch.uint8))) == B.GBMUF_EINVAL
    elsewhere = torch.zeros(G, M, K, device="meta")
    assert code_of(lambda: lin.forward_io(elsewhere, w, y)) == B.GBMUF_EINVAL


def test_a_calls_tensors_live_as_long_as_it_can_be_made():
    lin = B.Linear(3, 4, 5)
    x, w, y, dw = torch.zeros(3, 5), torch.zeros(4, 5), torch.zeros(3, 4), torch.zeros(4, 5)
    seen = [weakref.ref(t) for t in (x, w, y, dw)]
    io, grad = lin.forward_io(x, w, y), lin.backward_io(y, x, dw=dw)
    del x, w, y, dw
    gc.collect()
    assert all(r() is not None for r in seen)
    del io, grad
    gc.collect()
    assert all(r() is None for r in seen)
