"""The example network that names missing tokens: one step's updates, on given tokens and on a
teacher's saved answers, against automatic differentiation in float64; and that it runs."""

import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import token_distill as X  # noqa: E402


@pytest.mark.parametrize("what", ["tokens", "teacher"])
def test_step_against_float64(what):
    V, n, d, lr, k = 700, 12, 40, 0.25, 9
    rng = np.random.default_rng(2)
    net = X.TokenNetwork(V, 400, n, d, "f32", seed=4)
    ids = rng.integers(0, V, 300)
    tokens = torch.from_numpy(ids.astype(np.int32)).to(X.DEV)
    text = torch.arange(300, device=X.DEV) // 25
    missing = rng.integers(0, V, n)
    missing[3] = -1
    top, logp = rng.integers(0, V, (n, k)), np.log(rng.dirichlet(np.ones(k), n)).astype(np.float32)
    E, O = (p.detach().double().cpu().requires_grad_() for p in (net.E, net.O))
    before = E.detach().clone(), O.detach().clone()
    if what == "tokens":
        loss = net.step(tokens, text, torch.from_numpy(missing).to(X.DEV), lr)
    else:
        loss = net.learn(tokens, text, torch.from_numpy(top).to(X.DEV), torch.from_numpy(logp).to(X.DEV), lr)
    x = E[torch.from_numpy(ids)].view(n, 25, d).mean(1)
    z = (x / (x.square().mean(1, keepdim=True) + X.EPS).sqrt()) @ O
    lp = torch.log_softmax(z, 1)
    if what == "tokens":
        real = np.flatnonzero(missing >= 0)
        want = -lp[real, missing[real]].mean()
    else:
        q = torch.softmax(torch.from_numpy(logp).double(), 1)
        want = (q * (q.log() - lp.gather(1, torch.from_numpy(top)))).sum(1).mean()
    want.backward()
    # sums of at most 700 terms, each within some 1,000 u of its terms' sizes
    assert abs(float(loss) - float(want.detach())) <= 1e-4 * float(want.detach())
    for got, old, p in ((net.E, before[0], E), (net.O, before[1], O)):
        moved = (got.double().cpu() - old) / -lr
        rounding = float(old.norm() / p.grad.norm()) * 2.0 ** -23 / lr
        assert float((moved - p.grad).norm() / p.grad.norm()) <= 1e-4 + rounding


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_example_runs(kind):
    losses, distances, logp, top = X.train(steps=4, dim=32, small=16, kind=kind, n_batches=2)
    assert np.isfinite(losses).all() and np.isfinite(distances).all()
    assert bool((logp <= 0).all()) and top.shape == (len(logp), 3)
    assert bool((top[:, 0] != top[:, 1]).all()) and bool((top >= 0).all())


def test_hold_out():
    tokens = torch.tensor([7, 8, 9, 3, 1, 2], dtype=torch.int32, device=X.DEV)
    text = torch.tensor([0, 0, 0, 1, 3, 3], device=X.DEV)
    left, of, missing = X.hold_out(tokens, text, 4)
    assert left.tolist() == [7, 9, 3, 1] and of.tolist() == [0, 0, 1, 3] and missing.tolist() == [8, -1, -1, 2]
