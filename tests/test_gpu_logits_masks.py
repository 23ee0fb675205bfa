"""Alternatives of rows of mostly equal logits: all equal, or a mask of the type's lowest value that leaves
fewer columns than alternatives are asked for.  Their values, and that such rows take the way that
ordinary ones do: k searches of the row, the way for rows whose largest logits are nearly all in a few
lanes' columns, take 5 to 50 times an ordinary row's time at these sizes."""

import numpy as np
import pytest

import paper_1702_06943_amd as T
from logits_cases import DEV, TYPES, torch, workspace

pytestmark = pytest.mark.gpu


def rows(n, d, kind, left):
    """Random rows; all columns but `left` of each at the type's lowest value (0: all equal)."""
    g = torch.Generator(DEV).manual_seed(n + d)
    Z = torch.randn((n, d), device=DEV, generator=g).to(TYPES[kind])
    if left is None:
        return Z
    if left == 0:
        return torch.full_like(Z, 1.5)
    at = torch.rand((n, d), device=DEV, generator=g).topk(left, 1).indices
    out = torch.full_like(Z, torch.finfo(TYPES[kind]).min)
    return out.scatter_(1, at, Z.gather(1, at))


class Call:
    def __init__(self, Z, k):
        self.Z, self.ws = Z, workspace(*Z.shape, k)
        self.top = torch.empty((len(Z), k), dtype=torch.int64, device=DEV)
        self.top_logp = torch.empty((len(Z), k), device=DEV)

    def __call__(self):
        T.toc_logprob(self.Z, top_ids=self.top, top_logp=self.top_logp, ws=self.ws)

    def time(self):
        """The shortest of five replays of 20 captured calls (ms)."""
        self()
        graph, best = torch.cuda.CUDAGraph(), float("inf")
        with torch.cuda.graph(graph):
            for _ in range(20):
                self()
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            graph.replay()
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        return best


@pytest.mark.parametrize("n,d,kind,k", [(1, 47236, "bf16", 5), (64, 47236, "bf16", 20), (64, 47236, "f32", 20),
                                        (600, 47236, "bf16", 64), (1001, 9973, "f16", 20), (300, 3000, "bf16", 64),
                                        (9, 88832, "f16", 20), (3, 300007, "bf16", 32)])
def test_mostly_equal(n, d, kind, k):
    ordinary = Call(rows(n, d, kind, None), k).time()
    for left in (0, 1, 3, k - 2):
        call = Call(rows(n, d, kind, left), k)
        took = call.time()
        at = np.unique([0, 1 % n, n // 2, n - 1])
        order = torch.sort(call.Z[at].float(), dim=1, descending=True, stable=True)
        assert torch.equal(call.top[at], order.indices[:, :k]), left
        # binary32 sums against 64 bits: d / 64 additions of positive numbers and the logarithm, 1e-4 at most,
        # and half a step of log p itself, which is 3e38 at the mask
        want = (order.values.double() - torch.logsumexp(order.values.double(), 1, keepdim=True))[:, :k]
        assert bool(((call.top_logp[at].double() - want).abs() <= 1e-4 + 2.0 ** -22 * want.abs()).all()), left
        assert took < 3 * ordinary, (left, took, ordinary)
