"""The example that trains resident replicas: its gradients are those of the model it states, it learns, and the placement of
the state does not change what it computes."""
import importlib.util
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def example():
    spec = importlib.util.spec_from_file_location("resident_training", os.path.join(ROOT, "examples", "resident_training.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_gradients_of_the_example_against_autograd_in_64_bits():
    ex = example()
    m = ex.Model(3, 50)
    g = torch.Generator().manual_seed(0)
    rows = torch.randn(3, m.P, generator=g) * 0.2
    context, target = torch.randint(0, m.vocab, (3, 50, 2), generator=g), torch.randint(0, m.vocab, (3, 50), generator=g)
    dev = rows.to(ex.DEV)
    grad_rows = torch.empty_like(dev)
    loss = m.step(m.views(dev), m.views(grad_rows), context.to(ex.DEV), target.to(ex.DEV))
    torch.cuda.synchronize()
    r = rows.double().requires_grad_(True)
    p = m.views(r)
    want = []
    for k in range(3):
        x = p["embedding"][k][context[k]].reshape(50, -1)
        h = torch.tanh(x @ p["w1"][k].T + p["b1"][k])
        u = h + h @ p["w2"][k].T + p["b2"][k]
        want.append(torch.nn.functional.cross_entropy(u @ p["w3"][k].T + p["b3"][k], target[k]))
    torch.stack(want).sum().backward()
    # sums of at most 200 products of values of order one in f32: 1e-5 is far above their rounding, 1e-7 the gradients' floor
    assert torch.allclose(loss.cpu().double(), torch.stack(want).detach(), rtol=1e-5)
    assert torch.allclose(grad_rows.cpu().double(), r.grad, rtol=1e-4, atol=1e-6)


def test_the_example_learns_in_either_placement():
    ex = example()
    rows, blocked = (ex.train(steps=120, layout=layout) for layout in ("rows", "blocked"))
    assert torch.isfinite(rows).all()
    assert (rows[-10:].mean(0) < 0.75 * rows[:5].mean(0)).all()
    # embedding gradients are added by atomics, whose order may differ from run to run
    assert torch.allclose(rows[:8], blocked[:8], rtol=1e-4)
