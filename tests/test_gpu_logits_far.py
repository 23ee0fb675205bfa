"""Logits further apart than binary32's largest number: their scaled difference, and so log p, the
alternatives' and the distance from a teacher, is a number again where the scale is below one."""

import numpy as np
import pytest

import paper_1702_06943_amd as T
from logits_cases import DEV, TYPES, L, Soft, close, host, taught_tol, torch, vec, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [0.5, 0.01, 1e-30])
@pytest.mark.parametrize("n,d,kind", [(5, 9, "f32"), (5, 700, "bf16"), (300, 9001, "f32"), (2, 140001, "bf16"),
                                      (4200, 300, "f32")])
def test_far(n, d, kind, scale):
    rng = np.random.default_rng(d)
    big = torch.finfo(TYPES[kind]).max
    Z = torch.full((n, d), -big, device=DEV).to(TYPES[kind])
    Z[:, d // 2] = big
    Z[1::2, 3] = 0.0
    Z[0, 5] = -float("inf")
    at = np.r_[:min(n, 5), n - 1]
    Z64, scale = Z[at].double().cpu().numpy(), float(np.float32(scale))
    s, k = Soft(Z64, scale), 4
    ids = rng.integers(0, d, n)
    ids[:2] = [0, d // 2]
    idt = torch.from_numpy(ids).to(DEV)
    want = L.logprob(Z64, ids[at], scale, k)
    assert np.isfinite(want["logp"]).all() and want["logp"][0] < -1e8 * (scale > 1e-9)
    logp, beside = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    top, top_logp = torch.empty((n, k), dtype=torch.int64, device=DEV), torch.empty((n, k), device=DEV)
    T.toc_logprob(Z, idt, logp, top_ids=top, top_logp=top_logp, scale=scale, ws=workspace(n, d, k))
    assert np.array_equal(top[at].cpu().numpy(), want["top_ids"])
    close(top_logp[at], want["top_logp"], s.logp_tol(want["top_ids"]), "top_logp")
    dZ = torch.empty_like(Z)
    T.toc_logprob_grad(Z, dZ, idt, vec(np.ones(n)), logp=beside, scale=scale, ws=workspace(n, d))
    for got in (logp, beside):
        close(got[at], want["logp"], s.logp_tol(ids[at][:, None])[:, 0], "logp")
    # a teacher's entries at the largest logit, at the lowest and (some rows) at 0; or at the lowest alone
    for columns in ([d // 2, 0, 3], [1, 2, 2]):
        entries = np.tile(columns, (n, 1))
        t = rng.standard_normal((n, 3)).astype(np.float32)
        loss, beside = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
        T.toc_distill(Z, torch.from_numpy(entries).to(DEV), vec(t), loss, scale, ws=workspace(n, d))
        T.toc_distill_grad(Z, dZ, torch.from_numpy(entries).to(DEV), vec(t), vec(np.ones(n)), beside, scale,
                           ws=workspace(n, d))
        away = L.distill(Z64, entries[at], t[at].astype(np.float64), scale)
        tol, _ = taught_tol(s, entries[at], t[at].astype(np.float64), 1.0, None)
        for got in (loss, beside):
            got = host(got)[at]
            # half of twice the largest number, times the q of entries that sum to 1 within tol / |away|, is the
            # largest number or one step more, which is infinity
            past = np.isinf(got) & (away + tol > np.finfo(np.float32).max)
            close(np.where(past, away, got), away, tol, "loss")


@pytest.mark.parametrize("scale", [0.7, 1.0, 2.5, 1e6])
@pytest.mark.parametrize("n,d,kind", [(5, 9, "f32"), (5, 700, "bf16"), (300, 9001, "f32"), (2, 140001, "bf16")])
def test_far_entries_of_little_weight(n, d, kind, scale):
    """The share of an entry that far off is so small that its part of the distance is a number again."""
    rng = np.random.default_rng(d)
    big = torch.finfo(TYPES[kind]).max
    Z = torch.full((n, d), -big, device=DEV).to(TYPES[kind])
    Z[:, d // 2] = big
    Z64, scale = Z.double().cpu().numpy(), float(np.float32(scale))
    s = Soft(Z64, scale)
    ids = np.tile([d // 2, 0, 3], (n, 1))
    t = np.tile([0.0, -40.0, -20.0], (n, 1)) + rng.random((n, 3))
    t = t.astype(np.float32)
    loss, beside, dZ = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV), torch.empty_like(Z)
    idt, one = torch.from_numpy(ids).to(DEV), vec(np.ones(n))
    T.toc_distill(Z, idt, vec(t), loss, scale, ws=workspace(n, d))
    T.toc_distill_grad(Z, dZ, idt, vec(t), one, beside, scale, ws=workspace(n, d))
    want = L.distill(Z64, ids, t.astype(np.float64), scale)
    assert (want < 1e37).all() and (want > 1e20).all()
    tol, _ = taught_tol(s, ids, t.astype(np.float64), 1.0, None)
    for got in (loss, beside):
        close(got, want, tol, "loss")
