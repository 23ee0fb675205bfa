"""The operators on rows of logits as a program uses them together: a teacher's most probable
tokens saved and learnt from, a training step from lookup to gradient, all of it on another stream
and captured into graphs; and the binding's refusals."""

import numpy as np
import pytest

import paper_1702_06943_amd as T
from logits_cases import DEV, TYPES, L, host, logits, torch, vec, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", sorted(TYPES))
def test_teacher_to_student(kind):
    """The distance from a row's own saved alternatives is 0, and its gradient; from another's it is
    what the oracle says; a step along the gradient makes it smaller."""
    rng = np.random.default_rng(3)
    n, d, k = 40, 9001, 32
    own, own64 = logits(rng, n, d, kind)
    other, other64 = logits(rng, n, d, kind)
    ws = workspace(n, d, k)
    top, lp, lse = torch.empty((n, k), dtype=torch.int32, device=DEV), torch.empty((n, k), device=DEV), torch.empty(n, device=DEV)
    T.toc_logprob(own, lse=lse, top_ids=top, top_logp=lp, ws=ws)
    loss, dZ = torch.empty(n, device=DEV), torch.empty_like(own)
    zeros = torch.zeros(n, device=DEV)
    # saved log probabilities are logits whose whole row sums to 1
    T.toc_distill_grad(own, dZ, top, lp, torch.ones(n, device=DEV), loss, top_lse=zeros, ws=ws)
    assert float(loss.abs().max()) < 1e-5                     # log p of two calls, 32 times q <= 1
    T.toc_distill(own, top, own.float().gather(1, top.long()), loss, top_lse=lse, ws=ws)
    assert float(loss.abs().max()) < 1e-5
    T.toc_distill_grad(other, dZ, top, lp, torch.ones(n, device=DEV), loss, ws=ws)
    want = L.distill(other64, top.cpu().numpy(), host(lp))
    assert np.allclose(host(loss), want, rtol=1e-4, atol=1e-5)
    nearer = (other.float() - 0.5 * dZ.float()).to(other.dtype)
    after = torch.empty(n, device=DEV)
    T.toc_distill(nearer, top, lp, after, ws=ws)
    assert bool((after < loss).all())


class Step:
    """Rows of a table, a norm, logits over the whole vocabulary, their loss and the gradients back to
    the table; all buffers kept."""

    def __init__(self, n, V, d):
        g = torch.Generator(DEV).manual_seed(1)
        self.n, self.V, self.d = n, V, d
        self.E = torch.randn((V, d), generator=g, device=DEV) * 0.3
        self.out = torch.randn((d, V), generator=g, device=DEV) * 0.2
        self.w = torch.ones(d, device=DEV)
        self.x, self.y, self.dx = (torch.empty((n, d), device=DEV) for _ in range(3))
        self.z = torch.empty((n, V), device=DEV)
        self.dE = torch.empty_like(self.E)
        self.ids = torch.randint(0, V, (n,), generator=g, device=DEV)
        self.given = torch.randint(0, V, (n,), generator=g, device=DEV)
        self.dlogp = torch.full((n,), -1.0 / n, device=DEV)
        self.logp, self.h = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        self.top, self.top_logp = torch.empty((n, 5), dtype=torch.int64, device=DEV), torch.empty((n, 5), device=DEV)
        size = max(T.toc_embed_grad_workspace_size(n, V, d), T.toc_rmsnorm_grad_workspace_size(n, d),
                   T.toc_logits_workspace_size(n, V, 5))
        self.ws = torch.empty(size, dtype=torch.uint8, device=DEV)

    def __call__(self):
        T.toc_embed(self.ids, self.E, self.x)
        T.toc_rmsnorm(self.x, self.y, w=self.w)
        torch.matmul(self.y, self.out, out=self.z)
        T.toc_logprob(self.z, top_ids=self.top, top_logp=self.top_logp, ws=self.ws)
        T.toc_logprob_grad(self.z, self.z, self.given, self.dlogp, logp=self.logp, entropy=self.h, ws=self.ws)
        torch.matmul(self.z, self.out.t().contiguous(), out=self.y)
        T.toc_rmsnorm_grad(self.x, self.y, self.dx, None, w=self.w)
        T.toc_embed_grad(self.ids, self.dx, self.dE, self.ws)
        return [t.clone() for t in (self.logp, self.h, self.top, self.top_logp, self.z, self.dE)]


@pytest.mark.parametrize("n,V", [(50, 700), (30, 9001), (2, 140001)])
def test_step_and_graph(n, V):
    s = Step(n, V, 24)
    logp, h, top, top_logp, dz, dE = s()
    # the same in float64 with automatic differentiation
    E = s.E.double().cpu().requires_grad_()
    x = E[s.ids.cpu()]
    y = x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt()
    z = y @ s.out.double().cpu()
    lp = torch.log_softmax(z, 1)
    at = lp.gather(1, s.given.cpu()[:, None])[:, 0]
    (-at.mean()).backward()
    lp, at = lp.detach(), at.detach()
    assert float((logp.cpu() - at).abs().max()) < 1e-4          # logits of size 5 summed in binary32: 1e-5
    assert float((h.cpu() + (lp.exp() * lp).sum(1)).abs().max()) < 1e-4
    assert float((dE.cpu() - E.grad).abs().max()) < 1e-4 * float(E.grad.abs().max())
    assert torch.equal(top[:, 0].cpu(), lp.argmax(1)) and float((top_logp.cpu() - lp.gather(1, top.cpu())).abs().max()) < 1e-4
    # captured on another stream and replayed with other tokens, eager work of its own between
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            out = s()
    torch.cuda.current_stream().wait_stream(side)
    for seed in range(3):
        gen = torch.Generator(DEV).manual_seed(seed)
        s.ids.copy_(torch.randint(0, V, (n,), generator=gen, device=DEV))
        s.given.copy_(torch.randint(-1, V, (n,), generator=gen, device=DEV))
        want = s()
        s.ws.fill_(seed)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("n,d", [(9, 20000), (3, 300000)])
def test_two_streams_at_once(n, d):
    """Calls on two streams, each with its own workspace, as alone."""
    rng = np.random.default_rng(d)
    Z = [logits(rng, n, d, "bf16")[0] for _ in range(2)]
    ids = torch.arange(n, device=DEV)

    def buffers(i):
        return (Z[i], torch.empty(n, device=DEV), torch.empty((n, 9), dtype=torch.int64, device=DEV),
                torch.empty((n, 9), device=DEV), torch.empty_like(Z[i]), workspace(n, d, 9))

    def call(Z, logp, top, tl, dZ, ws, stream=None):
        T.toc_logprob(Z, ids, logp, top_ids=top, top_logp=tl, ws=ws, stream=stream)
        T.toc_logprob_grad(Z, dZ, ids, logp, ws=ws, stream=stream)

    alone, both = ([buffers(i) for i in range(2)] for _ in range(2))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for b in alone:
        call(*b)
    torch.cuda.synchronize()
    for _ in range(20):
        for b, s in zip(both, streams):
            call(*b, stream=s)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        assert all(torch.equal(x, y) for x, y in zip(a[1:5], b[1:5]))


def test_binding_refusals():
    n, d = 3, 8
    Z, v = torch.zeros((n, d), device=DEV), torch.zeros(n, device=DEV)
    ids = torch.zeros(n, dtype=torch.int64, device=DEV)
    top, tl = torch.zeros((n, 2), dtype=torch.int64, device=DEV), torch.zeros((n, 2), device=DEV)
    bad = [
        dict(ids=ids.float()), dict(ids=ids[:2]), dict(ids=ids.cpu()), dict(ids=None), dict(logp=v[:2]),
        dict(logp=v.double()), dict(lse=v.cpu()), dict(entropy=torch.zeros((n, 1), device=DEV)), dict(top_ids=top),
        dict(top_logp=tl), dict(top_ids=top.int(), top_logp=tl), dict(top_ids=top.float(), top_logp=tl),
        dict(top_ids=top, top_logp=tl[:, :1]), dict(top_ids=top.t().contiguous().t(), top_logp=tl),
        dict(top_ids=top, top_logp=tl.double()), dict(scale=0.0), dict(Z=Z.double()), dict(Z=Z.cpu()), dict(Z=Z.t()),
        dict(Z=Z[0]), dict(Z=Z[:1].expand(n, d)), dict(Z=Z.int()),
    ]
    for change in bad:
        a = dict(dict(Z=Z, ids=ids, logp=v), **change)
        with pytest.raises(T.TocError) as e:
            T.toc_logprob(**a)
        assert e.value.status == T.TOC_EINVAL, change
    for change in (dict(dZ=Z[:2]), dict(dZ=Z.half()), dict(dZ=Z.cpu()), dict(dlogp=v[:2]), dict(ids=None), dict(dlse=v.half()),
                   dict(dentropy=v.cpu()), dict(dZ=Z[:, :7])):
        a = dict(dict(Z=Z, dZ=Z, ids=ids, dlogp=v), **change)
        with pytest.raises(T.TocError) as e:
            T.toc_logprob_grad(**a)
        assert e.value.status == T.TOC_EINVAL, change
    for change in (dict(top_ids=top[:2]), dict(top_ids=top.float()), dict(top_ids=top[:, ::2], top_z=tl), dict(top_z=tl.double()),
                   dict(top_z=tl.half()), dict(top_z=tl[:, :1]), dict(top_ids=top[:1].expand(n, 2)), dict(top_ids=top[0]),
                   dict(loss=v[:1]), dict(top_lse=v[:1]), dict(top_scale=-1.0), dict(top_ids=top.cpu())):
        a = dict(dict(Z=Z, top_ids=top, top_z=tl, loss=v), **change)
        for grad in (False, True):
            with pytest.raises(T.TocError) as e:
                T.toc_distill_grad(dZ=Z, dloss=v, **a) if grad else T.toc_distill(**a)
            assert e.value.status == T.TOC_EINVAL, change
    with pytest.raises(T.TocError) as e:
        T.toc_distill_grad(Z, Z, top, tl, v[:1])
    assert e.value.status == T.TOC_EINVAL


def test_no_alternatives_asked_for():
    Z, v = torch.randn((3, 50), device=DEV), torch.empty(3, device=DEV)
    top, tl = torch.empty((3, 0), dtype=torch.int64, device=DEV), torch.empty((3, 0), device=DEV)
    T.toc_logprob(Z, lse=v, top_ids=top, top_logp=tl)
    assert torch.allclose(v, torch.logsumexp(Z, 1), atol=1e-5)
