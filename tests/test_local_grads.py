"""Norms of workers' gradients, clipping and the local update, against 64 bits and, where the method fixes every rounding, bit for bit.

A norm is summed in 64 bits and rounded once: within 2^-23 of the exact one.  The clip factor is one f32 division of the norm and the
product one f32 multiply, then one rounding to the type of the output; the update rounds every operation by itself, so numpy's
f32 arithmetic gives the same bits.
"""
import math

import numpy as np
import pytest
import torch

from paper_1909_09010_amd import binding as B
from paper_1909_09010_amd import workloads as W

DEV = "cuda:0"
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
gpu = pytest.mark.gpu

SHAPES = [
    [(7,), (3, 5), (1,)],
    [(1000, 64), (256, 64), (256,)],
    [(129, 33)],
    [(0,), (4, 0), (70001,), (2, 2)],
    [],
]


def tensors(dtype, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [[(torch.randn(s, generator=g) * scale).to(dtype).to(DEV) for s in ss] for ss in SHAPES]


def norm64(ts):
    return math.sqrt(sum(float(t.cpu().double().square().sum()) for t in ts))


def factor(norm, most):
    n, m = np.float32(norm), np.float32(most)
    return np.float32(1.0) if n <= m else m / n


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_norms(dtype):
    ts = tensors(dtype)
    h, n = B.Grads(ts), torch.full((len(ts),), -1.0, device=DEV)
    h.norm(n, torch.cuda.current_stream())
    want = np.array([norm64(t) for t in ts])
    assert np.all(np.abs(n.cpu().double().numpy() - want) <= 2.0 ** -23 * want)
    again = torch.empty_like(n)
    h.norm(again)
    torch.cuda.synchronize()
    assert torch.equal(n, again)


@gpu
def test_norms_of_very_large_and_very_small_values():
    ts = [[torch.full((1000,), 1e30, device=DEV)], [torch.full((999,), 1e-35, device=DEV)], [torch.zeros(5, device=DEV)],
          [torch.tensor([float("inf"), 1.0], device=DEV)], [torch.tensor([float("nan"), 1.0], device=DEV)], [torch.full((4,), 3e38, device=DEV)]]
    h, n = B.Grads(ts), torch.empty(6, device=DEV)
    h.norm(n, torch.cuda.current_stream())
    n = n.cpu().numpy()
    assert abs(n[0] / (1e30 * math.sqrt(1000)) - 1) < 1e-6 and abs(n[1] / (float(np.float32(1e-35)) * math.sqrt(999)) - 1) < 1e-6
    assert n[2] == 0 and n[3] == np.inf and np.isnan(n[4]) and n[5] == np.inf


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("out_dtype", DTYPES)
@pytest.mark.parametrize("most", [0.0, 1.5, 1e9, math.inf])
def test_clip_into_other_tensors(dtype, out_dtype, most):
    ts = tensors(dtype)
    out = [[torch.full(t.shape, 9.0, dtype=out_dtype, device=DEV) for t in w] for w in ts]
    before = [[t.clone() for t in w] for w in ts]
    n = torch.empty(len(ts), device=DEV)
    B.Grads(ts).clip(most, n, out=B.Grads(out), stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    for w, (a, b, c) in enumerate(zip(ts, out, before)):
        f = torch.tensor(factor(n[w].item(), most))
        for s, d, o in zip(a, b, c):
            assert torch.equal(s, o)
            assert torch.equal(d.cpu(), (s.cpu().float() * f).to(out_dtype))


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_clip_in_place(dtype):
    ts = tensors(dtype, scale=0.01)
    before = [[t.cpu() for t in w] for w in ts]
    n = torch.empty(len(ts), device=DEV)
    h = B.Grads(ts)
    h.clip(1.0, n, stream=torch.cuda.current_stream())
    first = n.cpu()
    clipped = 0
    for w, (a, b) in enumerate(zip(ts, before)):
        f = factor(first[w].item(), 1.0)
        clipped += f < 1
        for s, o in zip(a, b):
            assert torch.equal(s.cpu(), (o.float() * torch.tensor(f)).to(dtype))
    assert 0 < clipped < len(ts)
    h.norm(n)
    torch.cuda.synchronize()
    assert (n.cpu() <= 1.0 + 2.0 ** -8).all()


@gpu
def test_clip_with_infinite_and_nan_gradients():
    ts = [[torch.tensor([1.0, float("inf"), -2.0], device=DEV)], [torch.tensor([1.0, float("nan")], device=DEV)], [torch.ones(4, device=DEV)]]
    n = torch.empty(3, device=DEV)
    B.Grads(ts).clip(0.5, n, stream=torch.cuda.current_stream())
    a, b, c = (t[0].cpu().numpy() for t in ts)
    assert a[0] == 0 and np.isnan(a[1]) and a[2] == 0 and np.isnan(b).all() and (c == 0.25).all()


@gpu
def test_clip_without_a_bound_copies_whatever_the_norm():
    ts = [[torch.tensor([1.0, float("inf"), -2.0], device=DEV)], [torch.tensor([1.0, float("nan")], device=DEV)], [torch.ones(4, device=DEV)]]
    out = [[torch.zeros_like(t) for t in tt] for tt in ts]
    n = torch.empty(3, device=DEV)
    B.Grads(ts).clip(math.inf, n, out=B.Grads(out), stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    for a, b in zip(ts, out):
        np.testing.assert_array_equal(a[0].cpu().numpy(), b[0].cpu().numpy())


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_strided_and_unaligned_tensors(dtype, shift):
    g = torch.Generator().manual_seed(4)
    flat = (torch.randn(50000, generator=g)).to(dtype).to(DEV)
    wide = (torch.randn(300, 41, generator=g)).to(dtype).to(DEV)
    ts = [[flat[shift: shift + 20003], flat[20010 + shift: 40000].view(-1)], [wide[:, 2: 39], wide[:, 40], flat[40001:49999:3]]]
    keep_flat, keep_wide = flat.clone(), wide.clone()
    n = torch.empty(2, device=DEV)
    out = [[torch.empty(t.shape, dtype=torch.float32, device=DEV) for t in w] for w in ts]
    out[1][0] = torch.full((300, 50), 5.0, device=DEV)[:, 7:44]
    # the vector with gaps is a matrix of one column: its output is given the same form
    out[1][1], out[1][2] = torch.full((300, 3), 5.0, device=DEV)[:, 1], torch.full((3333, 2), 5.0, device=DEV)[:, 0]
    assert out[1][2].shape == ts[1][2].shape
    B.Grads(ts).clip(2.0, n, out=B.Grads(out), stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(flat, keep_flat) and torch.equal(wide, keep_wide)
    want = np.array([norm64(t) for t in ts])
    assert np.all(np.abs(n.cpu().double().numpy() - want) <= 2.0 ** -23 * want)
    for w in range(2):
        f = torch.tensor(factor(n[w].item(), 2.0))
        for s, d in zip(ts[w], out[w]):
            assert torch.equal(d.cpu(), s.cpu().float() * f)
    assert (out[1][0]._base[:, :7] == 5.0).all() and (out[1][0]._base[:, 44:] == 5.0).all()
    B.Grads(ts).clip(2.0, n, stream=torch.cuda.current_stream())          # and in place, beside values that stay
    torch.cuda.synchronize()
    assert torch.equal(flat[20003 + shift: 20010 + shift], keep_flat[20003 + shift: 20010 + shift])
    assert torch.equal(wide[:, :2], keep_wide[:, :2]) and torch.equal(wide[:, 39], keep_wide[:, 39])
    assert torch.equal(flat[40002:49999:3], keep_flat[40002:49999:3])


# -- local update ---------------------------------------------------------------------------------
class Placed:
    """K x P values in rows, in blocks of B floats, or in blocks of an arena of three arrays."""

    def __init__(self, values, layout, block=8192):
        K, P = values.shape
        self.K, self.P, self.layout = K, P, layout
        if layout == "rows":
            self.buf = torch.full((K, P + 5), 42.0, device=DEV)
            self.view = self.buf[:, 3: P + 3]
            self.view.copy_(values)
            self.state = B.make_state(self.view, None, None, P + 5)
        else:
            nb, arrays = max(-(-P // block), 1), 3 if layout == "arena" else 1
            self.buf = torch.full((nb, arrays, K, block), 42.0, device=DEV)
            self.view = self.buf[:, arrays - 1]
            pad = torch.full((K, nb * block), 42.0, device=DEV)
            pad[:, :P] = values
            self.view.copy_(pad.view(K, nb, block).transpose(0, 1))
            self.state = B.make_state(self.view, None, None, block, block, arrays * K * block)

    def get(self):
        if self.layout == "rows":
            return self.view.cpu().numpy()
        return self.view.transpose(0, 1).reshape(self.K, -1)[:, : self.P].cpu().numpy()

    def rest(self):
        n = self.buf.numel() - self.K * self.P
        return int((self.buf == 42.0).sum().item()) >= n


def step_numpy(theta, sums, g, f, rate, eps):
    g = (g.astype(np.float32) * np.float32(f)).astype(np.float32)
    if sums is None:
        return theta - np.float32(rate) * g, None
    sums = sums + g * g
    return theta - (np.float32(rate) * g) / (np.sqrt(sums) + np.float32(eps)), sums


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout,block", [("rows", 0), ("blocked", 8192), ("blocked", 4), ("arena", 64)])
@pytest.mark.parametrize("adagrad", [True, False])
@pytest.mark.parametrize("most", [2.0, math.inf])
def test_local_step(dtype, layout, block, adagrad, most):
    K, shapes = 3, [(50, 13), (7,), (0,), (2500,), (1,), (33, 64)]
    P = sum(math.prod(s) for s in shapes) + 3            # the last 3 parameters have no gradient
    rng = np.random.default_rng(5)
    theta, sums = rng.standard_normal((K, P)).astype(np.float32), (rng.random((K, P)) + 0.1).astype(np.float32)
    grads = [[torch.tensor(rng.standard_normal(s) * (0.001 if w == 1 else 1.0)).to(dtype).to(DEV) for s in shapes] for w in range(K)]
    t, s = Placed(torch.tensor(theta), layout, block), Placed(torch.tensor(sums), "rows" if block == 4 else layout, block)
    h, n = B.Grads(grads), torch.empty(K, device=DEV)
    for _ in range(2):
        h.local_step(t.state, s.state if adagrad else None, P, 0.1, 1e-7, most, n, stream=torch.cuda.current_stream())
        torch.cuda.synchronize()
        norms = n.cpu().numpy()
        for w in range(K):
            assert abs(norms[w] - norm64(grads[w])) <= 2.0 ** -23 * norm64(grads[w])
            g = np.concatenate([x.float().cpu().numpy().ravel() for x in grads[w]])
            a, b = step_numpy(theta[w, :-3], sums[w, :-3] if adagrad else None, g, factor(norms[w], most), 0.1, 1e-7)
            theta[w, :-3] = a
            if adagrad:
                sums[w, :-3] = b
        assert np.array_equal(t.get(), theta) and np.array_equal(s.get(), sums)
        assert t.rest() and s.rest()
    assert (norms > 2.0).any() and (norms < 2.0).any()


@gpu
def test_local_step_by_offsets_and_without_norms():
    rng = np.random.default_rng(6)
    theta = rng.standard_normal((2, 100)).astype(np.float32)
    grads = [[torch.tensor(rng.standard_normal(n).astype(np.float32)).to(DEV) for n in (10, 20)] for _ in range(2)]
    t = Placed(torch.tensor(theta), "rows")
    B.Grads(grads, offsets=[[70, 5], [0, 51]]).local_step(t.state, None, 100, 0.5, stream=torch.cuda.current_stream())
    for w, offs in enumerate(((70, 5), (0, 51))):
        for g, o in zip(grads[w], offs):
            g = g.cpu().numpy()
            theta[w, o: o + len(g)] -= np.float32(0.5) * g
    assert np.array_equal(t.get(), theta)


@gpu
def test_a_worker_whose_gradients_are_not_finite_is_skipped_on_request():
    theta = np.ones((3, 8), dtype=np.float32)
    for skip in (True, False):
        grads = [[torch.ones(8, device=DEV)], [torch.tensor([float("inf")] + [1.0] * 7, device=DEV)], [torch.tensor([float("nan")] + [1.0] * 7, device=DEV)]]
        t, n = Placed(torch.tensor(theta), "rows"), torch.empty(3, device=DEV)
        B.Grads(grads).local_step(t.state, None, 8, 0.5, max_norm=math.inf if skip else 1.0, norms=n, skip_nonfinite=skip, stream=torch.cuda.current_stream())
        got = t.get()
        assert (got[0] < 1).all()
        if skip:
            assert (got[1:] == 1).all()
        else:
            assert np.isnan(got[1, 0]) and (got[1, 1:] == 1).all() and np.isnan(got[2]).all()


@gpu
def test_step_on_a_state_of_the_library_and_a_sync_after_it():
    """theta in the recommended arena, Adagrad's sums in their own; the sync that follows sees what the step wrote."""
    w = W.get("tiny")
    off = W.component_offsets(w)
    P = int(off[-1])
    pl = B.Plan(off, w.K, w.q, w.p, seed=w.seed)
    st = W.init_state(w, DEV, layout="blocked", plan=pl)
    rows = W.init_state(w, DEV, layout="rows", plan=pl)
    sums = [W.DeviceState(w.K, P, DEV, layout, plan=pl) for layout in ("blocked", "rows")]
    g = torch.Generator(device=DEV).manual_seed(1)
    grads = [[torch.randn(r, c, device=DEV, generator=g) for _, r, c in W.tensors(w)] for _ in range(w.K)]
    h, n, s = B.Grads(grads), torch.empty(w.K, device=DEV), torch.cuda.current_stream()
    for a, b in zip((st, rows), sums):
        b.zero_()
        for rnd in range(2):
            h.local_step(a.desc(), b.desc(), P, 0.1, 1e-7, 10.0, n, stream=s)
            pl.sync_state(a.desc(), w.eta, w.zeta, w.mode, rnd, s)
    torch.cuda.synchronize()
    for i in range(3):
        assert np.array_equal(st.to_host(i), rows.to_host(i))
    assert np.array_equal(sums[0].to_host(0), sums[1].to_host(0)) and float(np.abs(sums[0].to_host(0)).max()) > 0
    pl.destroy()


@gpu
def test_graph_replays_equal_eager_calls():
    K, P = 4, 30000
    g = torch.Generator(device=DEV).manual_seed(2)
    grads = [[torch.randn(100, 200, device=DEV, generator=g), torch.randn(10000, device=DEV, generator=g)] for _ in range(K)]
    theta = torch.randn(K, P, device=DEV, generator=g)
    other, sums, sums2 = theta.clone(), torch.zeros(K, P, device=DEV), torch.zeros(K, P, device=DEV)
    h, n = B.Grads(grads), torch.empty(K, device=DEV)
    a, b = B.make_state(theta, None, None, P), B.make_state(other, None, None, P)
    sa, sb = B.make_state(sums, None, None, P), B.make_state(sums2, None, None, P)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        h.local_step(a, sa, P, 0.1, 1e-7, 5.0, n, stream=torch.cuda.current_stream())
    for replay in range(3):
        for ts in grads:
            for t in ts:
                t.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        h.local_step(b, sb, P, 0.1, 1e-7, 5.0, n)
        torch.cuda.synchronize()
        assert torch.equal(theta, other) and torch.equal(sums, sums2), replay
        assert torch.randn(1 << 18, device=DEV).sum().item() != 0.5


# -- refusals ---------------------------------------------------------------------------------------
def raw(entries, workers=1):
    import ctypes
    table = (B.GradTensor * max(len(entries), 1))(*[B.GradTensor(*e) for e in entries])
    d = B.GradsDesc(ctypes.sizeof(B.GradsDesc), workers, len(entries), ctypes.addressof(table))
    h = ctypes.c_void_p()
    rc = B.lib().gbmuf_grads_create(ctypes.byref(h), ctypes.byref(d))
    if rc == B.GBMUF_OK:
        B.lib().gbmuf_grads_destroy(h)
    else:
        assert not h
    return rc


def test_handles_that_are_refused():
    p = 4096                                              # only looked at, never followed
    assert raw([(p, 1, 8, 8, -1, 0, 0)]) == B.GBMUF_OK
    assert raw([]) == B.GBMUF_OK
    assert raw([(0, 1, 0, 0, -1, 0, 0)]) == B.GBMUF_OK    # an empty tensor has no data
    for e in ((p, 1, 8, 8, -1, 1, 0), (p, 1, 8, 8, -1, -1, 0), (p, 1, 8, 8, -1, 0, 3), (p, 1, 8, 8, -1, 0, -1), (p, -1, 8, 8, -1, 0, 0),
              (p, 1, -8, 8, -1, 0, 0), (p, 2, 8, 7, -1, 0, 0), (p, 1, 8, 8, -2, 0, 0), (0, 1, 8, 8, -1, 0, 0), (p + 2, 1, 8, 8, -1, 0, 0),
              (p + 1, 1, 8, 8, -1, 0, 1)):
        assert raw([e]) == B.GBMUF_EINVAL, e
    assert raw([(p, 1, 8, 8, 0, 0, 0), (p, 1, 8, 8, 7, 0, 0)]) == B.GBMUF_EINVAL          # places overlap
    assert raw([(p, 1, 8, 8, 10, 0, 0), (p, 1, 8, 8, 0, 0, 0), (p, 1, 3, 3, 8, 0, 0)]) == B.GBMUF_EINVAL
    assert raw([(p, 1, 8, 8, 0, 0, 0), (p, 1, 8, 8, 7, 1, 0)], workers=2) == B.GBMUF_OK   # of different workers
    assert raw([], workers=0) == B.GBMUF_EINVAL
    assert raw([], workers=1025) == B.GBMUF_EUNSUPPORTED
    assert raw([(p, 1 << 40, 1 << 40, 1 << 40, -1, 0, 0)]) == B.GBMUF_EUNSUPPORTED
    assert B.lib().gbmuf_grads_create(None, None) == B.GBMUF_EINVAL
    assert B.lib().gbmuf_grads_destroy(None) == B.GBMUF_OK
    with pytest.raises(B.GbmufError):
        B.Grads([[torch.zeros(4, dtype=torch.float64)]])
    with pytest.raises(B.GbmufError):
        B.Grads([[torch.zeros(4, 5, 6)[:, :, 1:]]])


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", ["rows", "blocked"])
def test_more_than_the_caches_hold(dtype, layout):
    """26 M values of 2 workers, tensors of odd sizes, rows with gaps and unaligned views: norm, clipping apart and in place, the step."""
    K, P = 2, 13_000_040
    rng = np.random.default_rng(11)
    flat = torch.tensor(rng.standard_normal((K, P + 3), dtype=np.float32)).to(dtype)
    dev = flat.to(DEV)
    wide = torch.zeros(K, 1000, 40, dtype=dtype, device=DEV)
    wide[:, :, 1:34] = dev[:, 1: 33001].view(K, 1000, 33)
    ts = [[wide[w, :, 1:34], dev[w, 33001: 8_000_000], dev[w, 8_000_000: P + 1]] for w in range(K)]
    values = flat[:, 1: P + 1]
    h, n = B.Grads(ts), torch.empty(K, device=DEV)
    out = [[torch.empty(t.shape, dtype=torch.float32, device=DEV) for t in w] for w in ts]
    h.clip(3.0, n, out=B.Grads(out), stream=torch.cuda.current_stream())
    norms = n.cpu().numpy()
    want = np.array([math.sqrt(float(values[w].double().square().sum())) for w in range(K)])
    assert np.all(np.abs(norms - want) <= 2.0 ** -23 * want)
    clipped = [values[w].float() * torch.tensor(factor(norms[w], 3.0)) for w in range(K)]
    for w in range(K):
        assert torch.equal(torch.cat([t.reshape(-1) for t in out[w]]).cpu(), clipped[w])
    theta, sums = rng.standard_normal((K, P), dtype=np.float32), rng.random((K, P), dtype=np.float32) + np.float32(0.1)
    t, s = Placed(torch.tensor(theta), layout), Placed(torch.tensor(sums), layout)
    h.local_step(t.state, s.state, P, 0.1, 1e-7, 3.0, n, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert np.array_equal(n.cpu().numpy(), norms)
    got, got_sums = t.get(), s.get()
    for w in range(K):
        a, b = step_numpy(theta[w], sums[w], values[w].float().numpy(), factor(norms[w], 3.0), 0.1, 1e-7)
        assert np.array_equal(got[w], a) and np.array_equal(got_sums[w], b)
    assert t.rest() and s.rest()
    h.clip(3.0, n, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    for w in range(K):
        assert torch.equal(torch.cat([x.reshape(-1) for x in ts[w]]).cpu(), clipped[w].to(dtype))
    assert (wide[:, :, 0] == 0).all() and (wide[:, :, 34:] == 0).all() and torch.equal(dev[:, 0].cpu(), flat[:, 0])


def test_calls_that_are_refused():
    ts = [[torch.zeros(10), torch.zeros(4, 5)], [torch.zeros(30)]]
    h, n, theta, sums = B.Grads(ts) if not torch.cuda.is_available() else None, torch.zeros(2), torch.zeros(2, 30), torch.zeros(2, 30)
    if h is None:
        pytest.skip("host memory")
    st, su = B.make_state(theta, None, None, 30), B.make_state(sums, None, None, 30)

    def code(fn):
        with pytest.raises(B.GbmufError) as e:
            fn()
        return e.value.code
    E = B.GBMUF_EINVAL
    assert code(lambda: h.norm(None)) == E
    assert code(lambda: h.clip(-1.0, n)) == E and code(lambda: h.clip(float("nan"), n)) == E and code(lambda: h.clip(1.0, None)) == E
    for other in ([[torch.zeros(10), torch.zeros(4, 5)]], [[torch.zeros(10), torch.zeros(5, 4).t()], [torch.zeros(30)]],
                  [[torch.zeros(10), torch.zeros(21)], [torch.zeros(30)]], [[torch.zeros(10)], [torch.zeros(30)]]):
        assert code(lambda: h.clip(1.0, n, out=B.Grads(other))) == E
    step = lambda a=st, b=su, P=30, rate=0.1, eps=0.0, most=1.0, norms=n: h.local_step(a, b, P, rate, eps, most, norms)
    assert code(lambda: step(P=29)) == E and code(lambda: step(P=-1)) == E
    assert code(lambda: step(rate=float("nan"))) == E and code(lambda: step(eps=-1.0)) == E and code(lambda: step(eps=float("nan"))) == E
    assert code(lambda: step(most=-1.0)) == E and code(lambda: step(most=float("nan"))) == E and code(lambda: step(norms=None)) == E
    assert code(lambda: step(a=B.make_state(None, None, None, 30))) == E and code(lambda: step(b=B.make_state(None, None, None, 30))) == E
    assert code(lambda: step(a=B.make_state(theta, None, None, 29))) == E
    assert code(lambda: step(b=st)) == E and code(lambda: step(b=B.make_state(theta.data_ptr() + 40, None, None, 30))) == E
    assert code(lambda: step(a=B.make_state(theta.data_ptr() + 2, None, None, 30))) == E
    for B_, ws, bs in ((6, 6, 12), (2, 2, 4), (8, 7, 16), (8, 8, 15), (-8, 8, 16)):
        assert code(lambda: step(a=B.make_state(theta, None, None, ws, B_, bs))) == E
    for ws, bs in (((1 << 61) + 1, 0), (30, (1 << 61) + 1)):
        assert code(lambda: step(a=B.make_state(theta, None, None, ws, 0 if bs == 0 else 8, bs))) == E
    # side by side in one arena: the checks pass, and the device is what is missing
    arena = torch.zeros(2, 2, 32)
    assert code(lambda: step(a=B.make_state(arena[:, 0], None, None, 64), b=B.make_state(arena[:, 1], None, None, 64))) == B.GBMUF_EDEVICE
    assert code(lambda: step()) == B.GBMUF_EDEVICE and code(lambda: h.norm(n)) == B.GBMUF_EDEVICE and code(lambda: h.clip(1.0, n)) == B.GBMUF_EDEVICE


# -- clipping into tensors of other shapes: as many values, counted row by row ------------------------------------------------
def shaped(values, shape, dtype):
    """A view of `shape` = (rows, columns, pitch, first column) with 5.0 in the gaps; (n,): a vector."""
    if len(shape) == 1:
        return values.to(dtype).clone()
    rows, cols, pitch, first = shape
    buf = torch.full((rows, pitch), 5.0, dtype=dtype, device=DEV)
    v = buf[:, first: first + cols]
    v.copy_(values.view(rows, cols))
    return v


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("out_dtype", DTYPES)
@pytest.mark.parametrize("times", [1, 1250])             # 55 thousand values, and 69 million, which no cache holds
def test_clip_into_other_shapes(dtype, out_dtype, times):
    pairs = [((11100,), (300, 37, 50, 7)), ((60, 185, 200, 3), (300, 37, 41, 1)), ((300, 37, 40, 0), (100, 111, 120, 9)), ((300, 37, 41, 2), (11100,)),
             ((5550, 2, 3, 0), (3700, 3, 7, 1))]
    grow = lambda s: (s[0] * times, *s[1:])
    g = torch.Generator(device=DEV).manual_seed(21)
    values = [torch.randn(11100 * times, generator=g, device=DEV).to(dtype) for _ in pairs]
    src = [shaped(v, grow(a), dtype) for v, (a, _) in zip(values, pairs)]
    dst = [shaped(torch.zeros_like(v), grow(b), out_dtype) for v, (_, b) in zip(values, pairs)]
    n = torch.empty(2, device=DEV)
    B.Grads([src[:2], src[2:]]).clip(3.0, n, out=B.Grads([dst[:2], dst[2:]]), stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    for w, part in enumerate((slice(0, 2), slice(2, 5))):
        want = math.sqrt(sum(float(v.double().square().sum()) for v in values[part]))
        assert abs(n[w].item() - want) <= 2.0 ** -23 * want
        f = torch.tensor(factor(n[w].item(), 3.0), device=DEV)
        for v, d, (_, b) in zip(values[part], dst[part], pairs[part]):
            assert torch.equal(d.reshape(-1), (v.float() * f).to(out_dtype))
            if len(b) > 1:
                assert (d._base[:, :b[3]] == 5.0).all() and (d._base[:, b[3] + b[1]:] == 5.0).all()
    for v, s, (a, _) in zip(values, src, pairs):
        assert torch.equal(s.reshape(-1), v)
        if len(a) > 1:
            assert (s._base[:, :a[3]] == 5.0).all() and (s._base[:, a[3] + a[1]:] == 5.0).all()


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_clipped_values_are_the_same_wherever_they_lie(dtype):
    """In f16: an f32 product, then its rounding, for values taken side by side and one by one, zeros' signs among them."""
    g = torch.Generator(device=DEV).manual_seed(22)
    v = torch.randn(200001, generator=g, device=DEV).to(dtype)
    v[::1000] = -0.0
    n, out, column = torch.empty(2, device=DEV), torch.empty(200001, dtype=torch.float16, device=DEV), torch.empty(200001, 2, dtype=torch.float16, device=DEV)
    B.Grads([[v], [v]]).clip(3.0, n, out=B.Grads([[out], [column[:, 0]]]), stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    f = torch.tensor(factor(n[0].item(), 3.0))
    want = (v.cpu().float() * f).to(torch.float16).view(torch.int16)
    assert torch.equal(out.cpu().view(torch.int16), want) and torch.equal(column[:, 0].cpu().view(torch.int16), want)


@gpu
def test_zero_gradients_on_fresh_sums_leave_theta_as_it_is():
    """Embedding rows that a batch does not touch, before any step: the default eps makes 0 / eps of them.  An eps of 0 is the caller's word."""
    g = torch.randn(3, 1000, generator=torch.Generator().manual_seed(23))
    g[:, ::3] = 0
    theta = np.ones((3, 1000), dtype=np.float32)
    t, s, n = Placed(torch.tensor(theta), "rows"), Placed(torch.zeros(3, 1000), "rows"), torch.empty(3, device=DEV)
    h = B.Grads([[v.to(DEV)] for v in g])
    h.local_step(t.state, s.state, 1000, 0.1, max_norm=1.0, norms=n, stream=torch.cuda.current_stream())
    got = t.get()
    assert (got[:, ::3] == 1).all() and np.isfinite(got).all() and (got[:, 1::3] != 1).all()
    t, s = Placed(torch.tensor(theta), "rows"), Placed(torch.zeros(3, 1000), "rows")
    h.local_step(t.state, s.state, 1000, 0.1, 0.0, 1.0, n, stream=torch.cuda.current_stream())
    got = t.get()
    assert np.isnan(got[:, ::3]).all() and np.isfinite(got[:, 1::3]).all()


def test_tensors_of_the_host_and_norms_of_another_form_are_refused(monkeypatch):
    if torch.cuda.is_available():
        pytest.skip("host memory")
    h, theta = B.Grads([[torch.zeros(8)], [torch.zeros(8)]]), torch.zeros(2, 8)
    st = B.make_state(theta, None, None, 8)
    calls = (lambda n: h.norm(n), lambda n: h.clip(1.0, n), lambda n: h.local_step(st, None, 8, 0.1, max_norm=1.0, norms=n))
    for call in calls:
        for n, want in ((torch.zeros(2), B.GBMUF_EDEVICE), (torch.zeros(3), B.GBMUF_EDEVICE), (torch.zeros(1), B.GBMUF_EINVAL),
                        (torch.zeros(2, dtype=torch.float64), B.GBMUF_EINVAL), (torch.zeros(4)[::2], B.GBMUF_EINVAL)):
            with pytest.raises(B.GbmufError) as e:
                call(n)
            assert e.value.code == want
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    for call in (*(lambda c=c: c(torch.zeros(2)) for c in calls), lambda: B.Grads([[torch.zeros(8)]]),
                 lambda: B.Grads([[torch.zeros(8), torch.zeros(8, device="meta")]])):
        with pytest.raises(B.GbmufError) as e:
            call()
        assert e.value.code == B.GBMUF_EINVAL


def test_rows_that_span_more_than_any_memory_are_refused():
    """Their places would overflow 64 bits."""
    p = 4096
    for rows, cols, stride in ((2, 8, 1 << 62), (3, 8, 1 << 61), (2, 8, (1 << 63) - 1), (1 << 20, 8, 1 << 29), (1 << 30, 0, 1 << 40)):
        assert raw([(p, rows, cols, stride, -1, 0, 0)]) == B.GBMUF_EINVAL, (rows, cols, stride)
    assert raw([(p, 1, 8, 1 << 62, -1, 0, 0)]) == B.GBMUF_OK              # one row has no stride
    assert raw([(p, 1 << 20, 1, 1 << 28, -1, 0, 0)]) == B.GBMUF_OK


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_call_above_what_the_caches_hold_gives_the_bits_of_calls_for_each_worker(dtype):
    """200 M values of 20 workers, rows with gaps and unaligned views: norms, clipping apart and in place, both steps, against 20 handles of
    10 M values whose arrays the caches hold."""
    K, P = 20, 10_000_040
    gen = torch.Generator(device=DEV).manual_seed(24)
    flat = torch.empty(K, P + 3, dtype=dtype, device=DEV)
    for w in range(K):
        flat[w] = torch.randn(P + 3, generator=gen, device=DEV) * (0.001 if w % 3 == 0 else 1.0)
    wide = torch.zeros(K, 1000, 40, dtype=dtype, device=DEV)
    wide[:, :, 1:34] = flat[:, 1: 33001].view(K, 1000, 33)
    parts = lambda f, w, v: [w[v, :, 1:34], f[v, 33001: 8_000_000], f[v, 8_000_000: P + 1]]

    def calls(groups):
        """Every call for each group of workers in turn; what they leave, in the order of the workers."""
        f, v = flat.clone(), wide.clone()
        clipped = torch.full((K, P + 3), 5.0, dtype=dtype, device=DEV)
        theta, sums, sgd = torch.ones(K, P, device=DEV), torch.full((K, P), 0.1, device=DEV), torch.ones(K, P, device=DEV)
        n = torch.empty(4, K, device=DEV)
        at = lambda t, g: B.make_state(t[g.start:], None, None, P)
        for g in groups:
            h = B.Grads([parts(f, v, w) for w in g])
            out = B.Grads([[clipped[w, 1: 33001], clipped[w, 33001: 8_000_000], clipped[w, 8_000_000: P + 1]] for w in g])
            s, k = torch.cuda.current_stream(), slice(g.start, g.stop)
            h.norm(n[0, k], s)
            h.clip(3.0, n[1, k], out=out, stream=s)
            h.local_step(at(theta, g), at(sums, g), P, 0.1, 1e-7, 3.0, n[2, k], stream=s)
            h.local_step(at(sgd, g), None, P, 0.1, max_norm=3.0, norms=n[3, k], stream=s)
            h.clip(3.0, n[1, k], stream=s)
            torch.cuda.synchronize()
        return f, v, clipped, theta, sums, sgd, n
    for a, b in zip(calls([range(K)]), calls([range(w, w + 1) for w in range(K)])):
        assert torch.equal(a, b)
        del a, b
