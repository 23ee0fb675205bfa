"""The example network over decoded tokens: one step's updates against automatic
differentiation in float64 with the oracle's masks, and the loss of a short training."""

import math
import os
import sys

import numpy as np
import pytest

from oracle import rows as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import text_network as X  # noqa: E402


def test_step_against_float64():
    d, V, n, lr = 72, 400, 900, 0.5
    rng = np.random.default_rng(1)
    net = X.TextNetwork(V, n, d, "f32", p=0.2, seed=3)
    net.u += torch.from_numpy(rng.standard_normal(d)).to(net.u)
    net.w1 += 0.1 * torch.from_numpy(rng.standard_normal(d)).to(net.w1)
    ids = rng.integers(0, V, n)
    tokens = torch.from_numpy(ids.astype(np.int32)).to(X.DEV)
    text = torch.arange(n, device=X.DEV) // 30
    labels = torch.from_numpy(rng.choice([-1.0, 1.0], 30)).float().to(X.DEV)
    names = ("E", "A", "u", "w1", "w2")
    before = {k: getattr(net, k).detach().double().cpu().requires_grad_() for k in names}
    loss = net.step(tokens, text, labels, lr, 5)
    drops = [torch.from_numpy(R.dropout(np.ones((n, d)), (m.p, m.seed, m.mask))) for m in net.drops(5)]

    def norm(h, w):
        return h / (h.square().mean(1, keepdim=True) + X.EPS).sqrt() * w

    p = before
    x = math.sqrt(d) * p["E"][torch.from_numpy(ids)] * drops[0]
    h = x + drops[1] * (norm(x, p["w1"]) @ p["A"])
    v = drops[2] * norm(h, p["w2"])
    z = (v @ p["u"]).view(30, 30).mean(1)
    want = torch.nn.functional.softplus(-labels.double().cpu() * z).mean()
    want.backward()
    # sums of at most 900 terms, each within 1,000 u of its terms: 6e-5 at the worst
    assert abs(float(loss) - float(want.detach())) <= 1e-4 * float(want.detach())
    for k in names:
        moved = (getattr(net, k).double().cpu() - before[k].detach()) / -lr
        off = float((moved - before[k].grad).norm() / before[k].grad.norm())
        # and the update's own rounding, u of the parameter over the step
        rounding = float(before[k].detach().norm() / before[k].grad.norm()) * 2.0 ** -23 / lr
        assert off <= 1e-4 + rounding, (k, off)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_training_lowers_the_loss(kind):
    losses, served, whole = X.train(steps=40, dim=64, kind=kind, n_batches=2)
    assert abs(losses[0] - math.log(2)) < 1e-3                  # u starts at zero
    assert np.mean(losses[-4:]) < 0.8 * losses[0]
    # 8 bits: half a step of at most 1/16 of each element, errors of either sign
    assert abs(served - whole) < 0.1 * max(1.0, abs(whole))
