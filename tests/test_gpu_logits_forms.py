"""Gradients for rows of logits in each shape of workgroup that their length and number choose: 130 rows
and more, so that none is dealt out in parts, each against the 64-bit oracle, in another place and in
the logits' own.  Lanes and chunks of a lane of each case stand beside it; "twice" names rows longer
than the registers, which are read again while they are written."""

import numpy as np
import pytest

import paper_1702_06943_amd as T
import test_gpu_distill
from logits_cases import DEV, TYPES, L, Soft, close, gaps_untouched, grad_tol, given, host, taught_tol, torch, vec, workspace

pytestmark = pytest.mark.gpu
FORMS = [
    (1100, 1200, "bf16"),     # 64 x 2
    (1100, 4003, "bf16"),     # 64 x 8
    (1100, 2003, "f32"),      # 64 x 8
    (200, 5001, "f16"),       # 256 x 2
    (600, 17001, "bf16"),     # 256 x 8
    (130, 27001, "f16"),      # 512 x 6
    (130, 13001, "f32"),      # 512 x 6
    (130, 50001, "f16"),      # 1,024 x 6
    (130, 27001, "f32"),      # 1,024 x 6
    (130, 60001, "bf16"),     # 512 x 20
    (130, 85001, "f16"),      # 512 x 20
    (130, 90001, "f16"),      # 1,024 x 12
    (250, 47236, "f32"),      # 1,024 x 12
    (130, 120001, "bf16"),    # 1,024 x 16
    (130, 60001, "f32"),      # 1,024 x 16
    (130, 140001, "bf16"),    # 1,024 x 6, twice
    (130, 80001, "f32"),      # 1,024 x 6, twice
]


def logits_of(n, d, kind):
    """Rows that begin at any element, most of them at odd ones; a row wholly masked, one all but, one in part."""
    g = torch.Generator(DEV).manual_seed(n + d)
    Z = torch.empty(n * (d + 1) + 1, dtype=TYPES[kind], device=DEV)[1:].view(n, d + 1)[:, :d]
    Z.copy_(torch.randn((n, d), device=DEV, generator=g).mul_(3))
    Z[1] = -float("inf")
    Z[1, d - 2] = 1.0
    Z[2, ::3] = -float("inf")
    Z[n - 2] = -float("inf")
    return Z


def ends(n):
    return np.r_[:3, n // 2, n - 3:n]


@pytest.mark.parametrize("parts", ["l", "lse"])
@pytest.mark.parametrize("n,d,kind", FORMS)
def test_score_gradient(n, d, kind, parts):
    rng = np.random.default_rng(n + d)
    Z = logits_of(n, d, kind)
    ids, idt = given(rng, n, d, 64)
    ids[n - 1], idt[n - 1] = d - 1, d - 1
    g = {p: rng.standard_normal(n).astype(np.float32) for p in parts}
    dev = [vec(g[p]) if p in g else None for p in "lse"]
    scale = float(np.float32(0.9))
    dZ = torch.full((n, d), 7.0, device=DEV).to(TYPES[kind])
    T.toc_logprob_grad(Z, dZ, idt, *dev, scale=scale, ws=workspace(n, d))
    at = ends(n)
    Z64, real = Z[at].double().cpu().numpy(), (ids >= 0) & (ids < d)
    g = {p: x[at] for p, x in g.items()}
    want = L.logprob_grad(Z64, ids[at], scale, g.get("l"), g.get("s"), g.get("e"))
    target = np.arange(d) == ids[at][:, None]
    tol = grad_tol(Soft(Z64, scale), want, kind, real[at] * g["l"], g.get("s", 0.0), g.get("e", 0.0), target)
    close(dZ[at], want, tol, "dZ")
    # in place, the numbers beside it asked for: the same bits
    out = [torch.full((n,), 7.0, device=DEV) for _ in range(3)]
    beside = [torch.full((n,), 7.0, device=DEV) for _ in range(3)]
    T.toc_logprob(Z, idt, *out, scale=scale, ws=workspace(n, d))
    T.toc_logprob_grad(Z, Z, idt, *dev, *(beside if "e" in parts else beside[:2]), scale=scale, ws=workspace(n, d))
    assert torch.equal(Z, dZ)
    for a, b in zip(out, beside if "e" in parts else beside[:2]):
        a, b = host(a), host(b)
        assert np.array_equal(np.isinf(a), np.isinf(b))
        a, b = np.where(np.isinf(a), 0, a), np.where(np.isinf(b), 0, b)
        assert np.all(np.abs(a - b) <= 1e-4 * (1 + np.abs(a)))      # two shapes' orders of one sum


@pytest.mark.parametrize("k", [9, 256])
@pytest.mark.parametrize("n,d,kind", FORMS)
def test_teacher_gradient(n, d, kind, k):
    """Entries anywhere, at both ends of a row, in neighbouring columns and the same column twice and more."""
    rng = np.random.default_rng(n + d + k)
    Z = logits_of(n, d, kind)
    ids = rng.integers(0, d, (n, k))
    ids[:, :4] = [0, d - 1, d - 2, 0]
    if k > 9:
        ids[:, 100:130] = np.arange(30) + d // 2
        ids[:, 130:136] = ids[:, 7:8]
        ids[:, 200:220] = ids[:, 20:40]
    ids[:, 5] = -1
    t64 = rng.standard_normal((n, k)).astype(np.float32).astype(np.float64)
    idt, t = torch.from_numpy(ids.astype(np.int32)).to(DEV), vec(t64)
    c = rng.standard_normal(n).astype(np.float32)
    loss, dZ = torch.full((n,), 7.0, device=DEV), torch.full((n, d), 7.0, device=DEV).to(TYPES[kind])
    T.toc_distill_grad(Z, dZ, idt, t, vec(c), ws=workspace(n, d))
    at = ends(n)
    Z64 = Z[at].double().cpu().numpy()
    s = Soft(Z64, 1.0)
    tol, rel = taught_tol(s, ids[at], t64[at], 1.0, None)
    want = L.distill_grad(Z64, ids[at], t64[at], c[at])
    close(dZ[at], want, test_gpu_distill.grad_tol(s, want, kind, c[at], ids[at], t64[at], 1.0, None, rel), "dZ")
    # in place, the loss beside it: the same bits
    T.toc_distill_grad(Z, Z, idt, t, vec(c), loss, ws=workspace(n, d))
    assert torch.equal(Z, dZ)
    with np.errstate(invalid="ignore"):
        want = L.distill(Z64, ids[at], t64[at])
    got, far = host(loss)[at], np.isinf(want)
    assert np.array_equal(got[far], want[far])
    close(np.where(far, 0, got), np.where(far, 0, want), tol, "loss")


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("d", [1, 7, 9, 127, 129, 300, 568, 569, 900, 1001, 1135, 1136, 1152])
def test_short_rows_in_place(d, kind):
    """So many short rows that 16 lanes have one (64 from 569 binary32 or 1,137 16-bit columns on): the same bits
    in the logits' own place, with the numbers beside them and without."""
    rng = np.random.default_rng(d)
    n, scale = 4096 + 5, 0.9
    buf = torch.full((n * (d + 3) + 1,), 7.0, device=DEV).to(TYPES[kind])
    Z = buf[1:].view(n, d + 3)[:, :d]
    Z.copy_(torch.from_numpy(rng.standard_normal((n, d)) * 3))
    Z[5], Z[n - 1, ::2] = -float("inf"), -float("inf")
    ids, idt = given(rng, n, d, 32)
    g = [vec(x) for x in rng.standard_normal((3, n))]
    for x in g:
        x[7] = 0
    dZ = torch.full((n, d), 7.0, device=DEV).to(TYPES[kind])
    out, beside = ([torch.full((n,), 7.0, device=DEV) for _ in range(3)] for _ in range(2))
    T.toc_logprob_grad(Z, dZ, idt, *g, *out, scale, workspace(n, d))
    again = buf.clone()[1:].view(n, d + 3)[:, :d]
    T.toc_logprob_grad(again, again, idt, *g, *beside, scale, workspace(n, d))
    T.toc_logprob_grad(Z, Z, idt, *g, scale=scale, ws=workspace(n, d))
    for x in (again, Z):
        assert torch.equal(x, dZ) and gaps_untouched(x)
    for a, b in zip(out, beside):
        assert torch.equal(a, b)
    assert not dZ[5].any() and not dZ[7].any()
