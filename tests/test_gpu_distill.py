"""Distance from a teacher's saved logits and its gradient on the GPU against the 64-bit oracle:
types, counts of saved logits, entries that are no token or equal, masks, strides, in place."""

import numpy as np
import pytest

import paper_1702_06943_amd as T
from logits_cases import (DEV, LEAST, TYPES, U, UNIT, L, Soft, blank, close, gaps_untouched, host, logits, saved,
                          taught_tol, torch, vec, workspace)

pytestmark = pytest.mark.gpu
INF = float("inf")


def grad_tol(s, want, kind, c, ids, t, scale, lse, rel):
    """p's error, the entries' errors where they are, and the rounding to the type."""
    tol = np.zeros(want.shape)
    for i in range(len(ids)):
        _, q = L.teacher(ids[i], t[i], s.d, scale, None if lse is None else float(lse[i]))
        tol[i] = s.p[i] * (q.sum() * (s.p_error()[i] + 40 * U) + (q * rel[i]).sum()) + 2.0 ** -120 * q.sum()
        for a in np.flatnonzero(q > 0):
            # equal entries are added one after the other
            tol[i, ids[i][a]] += q[a] * (rel[i][a] + (len(q) + 4) * U)
    return s.scale * np.abs(c)[:, None] * tol + UNIT[kind] * np.abs(want) + LEAST[kind]


def check(Z, Z64, ids, idt, t64, t, c, scale, t_scale, lse, kind, dz, what=""):
    n, d = Z.shape
    scale, t_scale = float(np.float32(scale)), float(np.float32(t_scale))
    c = c.astype(np.float32)
    lse = None if lse is None else lse.astype(np.float32)
    s = Soft(Z64, scale)
    loss, again = torch.full((n,), 7.0, device=DEV), torch.full((n,), 7.0, device=DEV)
    dl = None if lse is None else vec(lse)
    T.toc_distill(Z, idt, t, loss, scale, t_scale, dl, workspace(n, d))
    T.toc_distill_grad(Z, dz, idt, t, vec(c), again, scale, t_scale, dl, workspace(n, d))
    want = L.distill(Z64, ids, t64, scale, t_scale, lse)
    tol, rel = taught_tol(s, ids, t64, t_scale, lse)
    ends = np.isinf(want)
    for got in (loss, again):
        got = host(got)
        assert np.array_equal(got[ends], want[ends])
        close(np.where(ends, 0, got), np.where(ends, 0, want), tol, what + "loss")
    want = L.distill_grad(Z64, ids, t64, c, scale, t_scale, lse)
    close(dz, want, grad_tol(s, want, kind, c, ids, t64, t_scale, lse, rel), what + "dZ")
    assert gaps_untouched(dz)


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("d,k", [(1, 1), (1, 4), (3, 2), (8, 8), (9, 20), (65, 64), (300, 256), (513, 65), (1000, 7),
                                 (2049, 100), (5000, 256), (9001, 33), (33000, 64)])
def test_distill(d, k, kind):
    rng = np.random.default_rng(d + k)
    n = 21 if d < 3000 else 5
    for bits, gap, shift, whole, t_kind, repeats in ((64, 0, 0, False, kind, False), (32, 3, 1, True, "f32", False),
                                                     (64, 5, 3, False, "f32", True)):
        Z, Z64 = logits(rng, n, d, kind, gap, shift)
        ids, idt, t64, t = saved(rng, n, d, k, bits, t_kind, repeats)
        ids[0], idt[0] = -1, -1                               # a row without entries
        c = rng.standard_normal(n)
        c[1] = 0
        lse = np.log(np.exp(0.7 * t64).sum(1) * 1.2) if whole else None
        check(Z, Z64, ids, idt, t64, t, c, 0.6, 0.7, lse, kind, blank(n, d, kind, gap, shift), f"{bits}, {t_kind}: ")


@pytest.mark.parametrize("n,d,kind", [(1, 47236, "bf16"), (2, 70001, "f32"), (1, 262144, "f16"), (3, 140001, "bf16")])
def test_long_rows(n, d, kind):
    rng = np.random.default_rng(d)
    Z, Z64 = logits(rng, n, d, kind)
    ids, idt, t64, t = saved(rng, n, d, 64, 64, kind)
    check(Z, Z64, ids, idt, t64, t, rng.standard_normal(n), 1.0, 1.0, None, kind, blank(n, d, kind))


@pytest.mark.parametrize("n,d,kind", [(300, 140001, "bf16"), (1100, 8192, "f32"), (3000, 700, "f16"),
                                      (1000, 4003, "bf16"), (500, 9001, "f16"), (600, 9001, "bf16"), (1023, 1501, "f32"),
                                      (2051, 6001, "bf16")])
def test_many_rows(n, d, kind):
    """The first and the last of many rows are as they would be alone."""
    rng = np.random.default_rng(d)
    Z = torch.randn((n, d), device=DEV, generator=torch.Generator(DEV).manual_seed(d)).mul_(3).to(TYPES[kind])
    ids = rng.integers(0, d, (n, 9))
    idt, t = torch.from_numpy(ids).to(DEV), torch.randn((n, 9), device=DEV)
    c = rng.standard_normal(n).astype(np.float32)
    loss, dZ = torch.empty(n, device=DEV), torch.empty_like(Z)
    T.toc_distill_grad(Z, dZ, idt, t, vec(c), loss, ws=workspace(n, d))
    only = torch.empty(n, device=DEV)
    T.toc_distill(Z, idt, t, only, ws=workspace(n, d))
    at = np.r_[:3, n - 3:n]
    Z64, t64 = Z[at].double().cpu().numpy(), t[at].double().cpu().numpy()
    s = Soft(Z64, 1.0)
    tol, rel = taught_tol(s, ids[at], t64, 1.0, None)
    want = L.distill(Z64, ids[at], t64)
    close(loss[at], want, tol, "loss")
    close(only[at], want, tol, "loss alone")
    want = L.distill_grad(Z64, ids[at], t64, c[at])
    close(dZ[at], want, grad_tol(s, want, kind, c[at], ids[at], t64, 1.0, None, rel), "dZ")


@pytest.mark.parametrize("kind", sorted(TYPES))
def test_in_place(kind):
    rng = np.random.default_rng(4)
    for n, d, k in ((19, 70, 12), (9, 1500, 40), (5, 12000, 256), (2, 140001, 100)):
        Z, _ = logits(rng, n, d, kind)
        _, idt, _, t = saved(rng, n, d, k, 32, kind, repeats=True)
        c = vec(rng.standard_normal(n))
        dZ = torch.empty_like(Z)
        T.toc_distill_grad(Z, dZ, idt, t, c, ws=workspace(n, d))
        loss = torch.empty(n, device=DEV)
        T.toc_distill(Z, idt, t, loss, ws=workspace(n, d))
        again = torch.empty(n, device=DEV)
        T.toc_distill_grad(Z, Z, idt, t, c, again, ws=workspace(n, d))
        assert torch.equal(Z, dZ)
        assert float((loss - again).abs().max()) <= 1e-5 * (1 + float(loss.abs().max()))


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("d", [40, 3001, 20000])
def test_masked(d, kind):
    """The student's masked columns, with and without entries there, wholly masked rows, saved
    logits of minus infinity and the type's lowest value."""
    rng = np.random.default_rng(d)
    n, k = 8, 10
    Z, _ = logits(rng, n, d, kind, masked=0.4)
    ids, idt, t64, t = saved(rng, n, d, k, 64, kind, none=0.0)
    at = torch.arange(n, device=DEV)[:, None]
    Z[at[:5], idt[:5]] = 1.5                     # entries of rows 0 to 4 are not masked
    Z[5, idt[5, 0]] = -INF                       # an infinite loss
    Z[6] = -INF
    t[1, 3], t[2, :9], t[3, 2] = -INF, -INF, torch.finfo(TYPES[kind]).min
    t[7] = -INF                                  # a teacher's row of nothing
    Z64, t64 = Z.double().cpu().numpy(), t.double().cpu().numpy()
    lse = None
    check(Z, Z64, ids, idt, t64, t, rng.standard_normal(n), 1.0, 1.0, lse, kind, blank(n, d, kind))
    loss = torch.empty(n, device=DEV)
    T.toc_distill(Z, idt, t, loss, ws=workspace(n, d))
    assert host(loss)[5] == INF and host(loss)[6] == INF and host(loss)[7] == 0


def test_bad_rows_that_take_no_part():
    Z = torch.full((4, 900), float("nan"), device=DEV)
    Z[3] = 1.0
    ids = torch.tensor([[5, 6], [-1, 900], [5, 6], [5, 6]], device=DEV)
    t = torch.tensor([[1.0, 2.0]] * 4, device=DEV)
    dZ, loss = torch.full_like(Z, 7.0), torch.empty(4, device=DEV)
    T.toc_distill_grad(Z, dZ, ids, t, torch.tensor([0.0, 1.0, 1.0, 1.0], device=DEV), loss, ws=workspace(4, 900))
    assert not host(dZ)[:2].any() and np.isnan(host(dZ)[2]).all() and np.isfinite(host(dZ)[3]).all()
    assert np.isnan(host(loss)[[0, 2]]).all() and host(loss)[1] == 0
    again = torch.full_like(Z, 7.0)
    T.toc_distill_grad(Z, again, ids, t, torch.tensor([0.0, 1.0, 1.0, 1.0], device=DEV), ws=workspace(4, 900))
    assert np.array_equal(host(again), host(dZ), equal_nan=True)


def test_strided_teacher():
    """The first columns of wider saved matrices."""
    rng = np.random.default_rng(2)
    n, d = 7, 600
    Z, Z64 = logits(rng, n, d, "bf16")
    ids, idt, t64, t = saved(rng, n, d, 64, 64, "bf16")
    loss, want = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    T.toc_distill(Z, idt[:, :20], t[:, :20], loss, ws=workspace(n, d))
    T.toc_distill(Z, idt[:, :20].contiguous(), t[:, :20].contiguous(), want, ws=workspace(n, d))
    assert torch.equal(loss, want)


@pytest.mark.parametrize("d", [17, 2500, 50000])
def test_grad_is_the_difference(d):
    rng = np.random.default_rng(d)
    n, k, h = 3, 9, 2.0 ** -6
    Z, _ = logits(rng, n, d, "f32")
    _, idt, _, t = saved(rng, n, d, k, 64, "f32", repeats=True)
    c, ws = rng.standard_normal(n).astype(np.float32), workspace(n, d)
    way = torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32)).to(DEV)
    dZ = torch.empty_like(Z)
    T.toc_distill_grad(Z, dZ, idt, t, vec(c), ws=ws)

    def value(step):
        loss = torch.empty(n, device=DEV)
        T.toc_distill(Z + step * way, idt, t, loss, ws=ws)
        return c.astype(np.float64) * host(loss)

    got = (dZ.double() * way.double()).sum(1).cpu().numpy()
    diff = (8 * (value(h) - value(-h)) - value(2 * h) + value(-2 * h)) / (12 * h)
    assert np.all(np.abs(got - diff) <= 20 * h ** 4 * 100 / 5 + 20 * 1e-5 / h), (got, diff)
