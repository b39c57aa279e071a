"""Algorithm 1 whole, on one GPU: K workers train a small language model, each on its own text, and gossip.

The K replicas lie in rows of theta.  A mini-batch's forward and backward products read the matrices of all workers where they lie
(one call for all of them), Adagrad with clipping at the norm of each worker's gradients updates theta in place, and every
``period`` mini-batches the replicas are synchronised.  The model predicts a word from the two before it:

    h = tanh(W1 [e(a), e(b)] + b1),  u = h + (W2 h + b2),  logits = W3 u + b3

    python examples/resident_training.py [--steps 200] [--workers 4] [--layout rows|blocked]

With ``--layout blocked`` the state keeps the library's recommended placement between mini-batches; the local step writes it
there, and theta is copied to rows for the products.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1909_09010_amd import binding as B  # noqa: E402
from paper_1909_09010_amd import workloads as W  # noqa: E402

DEV = "cuda:0"


class Model:
    """Shapes of the parameters in the order of a worker's row, and one product per layer."""

    def __init__(self, workers: int, tokens: int, vocab: int = 200, embed: int = 32, hidden: int = 64):
        self.K, self.tokens, self.vocab, self.embed, self.hidden = workers, tokens, vocab, embed, hidden
        self.shapes = [("embedding", (vocab, embed)), ("w1", (hidden, 2 * embed)), ("b1", (hidden,)), ("w2", (hidden, hidden)),
                       ("b2", (hidden,)), ("w3", (vocab, hidden)), ("b3", (vocab,))]
        sizes = [math.prod(s) for _, s in self.shapes]
        self.offsets = [0]
        for n in sizes:
            self.offsets.append(self.offsets[-1] + n)
        self.P = self.offsets[-1]
        self.l1 = B.Linear(tokens, hidden, 2 * embed, workers, torch.float32, B.ACT_TANH)
        self.l2 = B.Linear(tokens, hidden, hidden, workers, torch.float32, B.ACT_NONE, B.RESIDUAL_AFTER)
        self.l3 = B.Linear(tokens, vocab, hidden, workers, torch.float32)
        need = max(max(l.workspace_bytes(), l.workspace_bytes(True)) for l in (self.l1, self.l2, self.l3))
        self.workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)

    def views(self, rows: torch.Tensor) -> dict:
        """The parameters (or gradients) of all workers as views of their rows."""
        return {n: rows[:, a:b].unflatten(1, s) for (n, s), a, b in zip(self.shapes, self.offsets, self.offsets[1:])}

    def step(self, p: dict, g: dict, context: torch.Tensor, target: torch.Tensor) -> torch.Tensor:
        """Mean loss of every worker for context [K, tokens, 2] and target [K, tokens]; gradients into g."""
        K, T, E, H, V = self.K, self.tokens, self.embed, self.hidden, self.vocab
        s, ws = torch.cuda.current_stream(), self.workspace
        worker = torch.arange(K, device=DEV)[:, None, None]
        x = p["embedding"][worker, context].reshape(K, T, 2 * E)
        z1, h, u, logits = (torch.empty(K, T, n, device=DEV) for n in (H, H, H, V))
        self.l1.forward(self.l1.forward_io(x, p["w1"], h, bias=p["b1"], pre=z1), ws, s)
        self.l2.forward(self.l2.forward_io(h, p["w2"], u, bias=p["b2"], residual=h), ws, s)
        self.l3.forward(self.l3.forward_io(u, p["w3"], logits, bias=p["b3"]), ws, s)
        logp = torch.log_softmax(logits, 2)
        loss = -logp.gather(2, target[:, :, None]).mean((1, 2))
        dlogits = (logp.exp() - torch.nn.functional.one_hot(target, V)) / T
        du, dh, dx = (torch.empty(K, T, n, device=DEV) for n in (H, H, 2 * E))
        self.l3.backward(self.l3.backward_io(dlogits, u, p["w3"], dx=du, dw=g["w3"], dbias=g["b3"]), ws, s)
        self.l2.backward(self.l2.backward_io(du, h, p["w2"], dx=dh, dw=g["w2"], dbias=g["b2"]), ws, s)
        dh += du                                          # the residual's way around the product
        self.l1.backward(self.l1.backward_io(dh, x, p["w1"], pre=z1, dx=dx, dw=g["w1"], dbias=g["b1"]), ws, s)
        g["embedding"].zero_()
        at = (worker.expand(K, T, 2).reshape(-1), context.reshape(-1))
        g["embedding"].index_put_(at, dx.reshape(-1, E), accumulate=True)
        return loss


def text(workers: int, length: int, vocab: int, seed: int) -> torch.Tensor:
    """Each worker's own stretch of one language, in which a word mostly follows from the one before it."""
    g = torch.Generator().manual_seed(seed)
    follows = torch.randint(0, vocab, (vocab,), generator=g)
    words = torch.randint(0, vocab, (workers, length), generator=g)
    surprise = torch.rand(workers, length, generator=g) < 0.2
    for t in range(2, length):
        words[:, t] = torch.where(surprise[:, t], words[:, t], follows[words[:, t - 1]])
    return words


def train(steps: int = 200, workers: int = 4, layout: str = "rows", tokens: int = 64, period: int = 16, rate: float = 0.1,
          max_norm: float = 1.0, seed: int = 0):
    """Returns the workers' losses, [steps, workers]."""
    m = Model(workers, tokens)
    # one component for each tensor, as the paper's deployment; 1 neighbour
    plan = B.Plan(m.offsets, workers, min(1, workers - 1), 0, seed=seed)
    state = W.DeviceState(workers, m.P, DEV, layout, plan=plan)
    state.zero_()
    g = torch.Generator(device=DEV).manual_seed(seed)
    first = torch.cat([torch.randn(math.prod(s), generator=g, device=DEV) * (s[-1] ** -0.5 if len(s) > 1 else 0.0) for _, s in m.shapes])
    for k in range(workers):
        state.set_row(0, k, first)
        state.set_row(1, k, first)
    sums = W.DeviceState(workers, m.P, DEV, layout, plan=plan)          # Adagrad's sums of squares lie as theta does
    sums.zero_()
    rows = state.view2d(0)[:, : m.P] if layout == "rows" else torch.empty(workers, m.P, device=DEV)
    rows_at = B.make_state(rows, None, None, rows.stride(0))
    grad_rows = torch.zeros(workers, m.P, device=DEV)
    p, grad = m.views(rows), m.views(grad_rows)
    grads = B.Grads([[grad[n][k] for n, _ in m.shapes] for k in range(workers)])
    norms = torch.empty(workers, device=DEV)
    words = text(workers, steps * tokens + 2, m.vocab, seed).to(DEV)
    losses = []
    for t in range(steps):
        part = words[:, t * tokens: (t + 1) * tokens + 2]
        context, target = torch.stack([part[:, :-2], part[:, 1:-1]], 2), part[:, 2:]
        if layout != "rows":
            plan.state_copy(rows_at, state.desc(gossip_ma=True), 1, torch.cuda.current_stream())
        losses.append(m.step(p, grad, context, target))
        grads.local_step(state.desc(gossip_ma=True), sums.desc(gossip_ma=True), m.P, rate, 1e-7, max_norm, norms, skip_nonfinite=True,
                         stream=torch.cuda.current_stream())
        if (t + 1) % period == 0:
            plan.sync_state(state.desc(), 0.5, 1.0, B.MODE_PAPER, t // period, torch.cuda.current_stream())
    torch.cuda.synchronize()
    out = torch.stack(losses).cpu()
    grads.destroy()
    plan.destroy()
    return out


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    a.add_argument("--steps", type=int, default=200)
    a.add_argument("--workers", type=int, default=4)
    a.add_argument("--layout", choices=("rows", "blocked"), default="rows")
    a = a.parse_args()
    losses = train(a.steps, a.workers, a.layout)
    for t in range(0, a.steps, max(1, a.steps // 10)):
        print(f"step {t:5d}  loss of each worker " + "  ".join(f"{v:.3f}" for v in losses[t].tolist()))
    print("last        loss of each worker " + "  ".join(f"{v:.3f}" for v in losses[-1].tolist()))
