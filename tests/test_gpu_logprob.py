"""Log probabilities, entropy and most probable tokens on the GPU against the 64-bit oracle, and
the gradient: types, widths from one column to long rows, strides, masks that leave little or
nothing, ties, infinities, token numbers that are none, long offsets, streams and graphs."""

import numpy as np
import pytest

import paper_1702_06943_amd as T
from logits_cases import (DEV, INTS, L, TYPES, Soft, blank, close, gaps_untouched, given, grad_tol, host, logits,
                          torch, vec, workspace)

pytestmark = pytest.mark.gpu
INF = float("inf")
WIDTHS = [1, 2, 3, 4, 7, 8, 9, 63, 64, 65, 500, 511, 513, 1000, 2047, 2049, 4100, 8191, 8200, 16391, 33000]


def check(Z, Z64, ids, idt, scale, k, kind, what=""):
    """Everything toc_logprob gives, and alternatives alone, without the other outputs."""
    n, d = Z.shape
    scale = float(np.float32(scale))
    s = Soft(Z64, scale)
    want = L.logprob(Z64, ids, scale, k)
    logp, lse, h = (torch.full((n,), 7.0, device=DEV) for _ in range(3))
    top = torch.full((n, k), 7, dtype=idt.dtype, device=DEV) if k else None
    top_logp = torch.full((n, k), 7.0, device=DEV) if k else None
    T.toc_logprob(Z, idt, logp, lse, h, top, top_logp, scale, workspace(n, d, k))
    real = (ids >= 0) & (ids < d)
    columns = np.where(real, ids, 0)[:, None]
    finite(logp, want["logp"], s.logp_tol(columns)[:, 0], what + "logp")
    finite(lse, want["lse"], s.lse_tol(), what + "lse")
    close(h, want["entropy"], s.entropy_tol(), what + "entropy")
    if k:
        assert np.array_equal(top.cpu().numpy(), want["top_ids"]), what
        finite(top_logp, want["top_logp"], s.logp_tol(want["top_ids"]), what + "top_logp")
    return logp, lse, h


def finite(got, want, tol, what):
    """As close(), where infinities have to be equal."""
    got = host(got)
    ends = np.isinf(want)
    assert np.array_equal(got[ends], want[ends]), what
    close(np.where(ends, 0, got), np.where(ends, 0, want), tol, what)


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("d", WIDTHS)
def test_logprob(d, kind):
    rng = np.random.default_rng(d)
    n = 37 if d <= 2049 else 6
    for bits, gap, shift, k, scale in ((64, 0, 0, 0, 1.0), (32, 5, 1, 5, 0.37), (64, 3, 3, min(64, d + 3), 1.6)):
        Z, Z64 = logits(rng, n, d, kind, gap, shift)
        ids, idt = given(rng, n, d, bits)
        check(Z, Z64, ids, idt, scale, k, kind, f"gap {gap} k {k}: ")


@pytest.mark.parametrize("n,d", [(1, 47236), (3, 70001), (1, 262144), (2, 300007), (300, 9000), (700, 1300)])
def test_logprob_long_and_many(n, d):
    rng = np.random.default_rng(n + d)
    for kind, k in (("bf16", 20), ("f32", 64), ("f16", 1), ("bf16", 0)):
        Z, Z64 = logits(rng, n, d, kind, gap=2, shift=1)
        ids, idt = given(rng, n, d, 64)
        if n > 10:
            Z, Z64, ids, idt = Z[:20], Z64[:20], ids[:20], idt[:20]
        check(Z, Z64, ids, idt, 1.0, k, kind)


@pytest.mark.parametrize("n,d,kind,k", [(2051, 5003, "bf16", 5), (2051, 6001, "f16", 0), (2050, 2003, "f32", 32),
                                        (2050, 1501, "f16", 33), (600, 12007, "f16", 3), (400, 12007, "bf16", 64),
                                        (300, 1003, "bf16", 64), (70, 13, "f32", 64), (5003, 900, "f16", 0),
                                        (1500, 9000, "bf16", 20), (513, 17001, "bf16", 0)])
def test_lanes_by_rows(n, d, kind, k):
    """As many rows as are given, of which some are looked at."""
    rng = np.random.default_rng(n * d)
    Z = torch.randn((n, d), device=DEV, generator=torch.Generator(DEV).manual_seed(d)).mul_(3).to(TYPES[kind])
    Z[1, ::2] = -INF
    ids, idt = given(rng, n, d, 32)
    logp, lse, h = (torch.full((n,), 7.0, device=DEV) for _ in range(3))
    top = torch.full((n, k), 7, dtype=idt.dtype, device=DEV) if k else None
    top_logp = torch.full((n, k), 7.0, device=DEV) if k else None
    at = np.r_[:5, n // 2, n - 3:n]
    Z64, scale = Z[at].double().cpu().numpy(), float(np.float32(0.8))
    s, want = Soft(Z64, scale), L.logprob(Z64, ids[at], scale, k)
    real = (ids[at] >= 0) & (ids[at] < d)
    for entropy in (h, None):
        T.toc_logprob(Z, idt, logp, lse, entropy, top, top_logp, scale, workspace(n, d, k))
        finite(logp[at], want["logp"], s.logp_tol(np.where(real, ids[at], 0)[:, None])[:, 0], "logp")
        finite(lse[at], want["lse"], s.lse_tol(), "lse")
        close(h[at], want["entropy"], s.entropy_tol(), "entropy")
        if k:
            assert np.array_equal(top[at].cpu().numpy(), want["top_ids"])
            finite(top_logp[at], want["top_logp"], s.logp_tol(want["top_ids"]), "top_logp")


@pytest.mark.parametrize("low", [False, True], ids=["inf", "lowest"])
@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("d", [9, 700, 5000, 20011])
def test_masked(d, kind, low):
    """Masks that leave a share, a few, one or none of a row's columns."""
    rng = np.random.default_rng(d)
    n, bad = 9, torch.finfo(TYPES[kind]).min if low else -INF
    Z, _ = logits(rng, n, d, kind)
    keep = torch.from_numpy(rng.random((n, d)) < 0.5).to(DEV)
    keep[1:] = False
    for i, left in ((1, 5), (2, 1), (3, 2), (4, 8), (5, 1)):
        keep[i, torch.from_numpy(rng.permutation(d)[:left]).to(DEV)] = True
    keep[5] = False
    keep[5, d - 1] = True
    Z.masked_fill_(~keep, bad)                     # rows 6 to 8 are wholly masked
    ids = rng.integers(0, d, n)
    ids[8] = -1
    idt = torch.from_numpy(ids).to(DEV)
    Z64 = Z.double().cpu().numpy()
    check(Z, Z64, ids, idt, 0.8, min(d, 20), kind)
    g = rng.standard_normal((3, n))
    dZ = torch.full_like(Z, 7.0)
    T.toc_logprob_grad(Z, dZ, idt, *(vec(x) for x in g), scale=0.8, ws=workspace(n, d))
    g = g.astype(np.float32).astype(np.float64)
    scale = float(np.float32(0.8))
    want = L.logprob_grad(Z64, ids, scale, *g)
    real = ids >= 0
    target = (np.arange(d) == ids[:, None])
    close(dZ, want, grad_tol(Soft(Z64, scale), want, kind, g[0] * real, g[1], g[2], target), "dZ")
    if not low:
        assert not host(dZ)[6:].any()


@pytest.mark.parametrize("kind", sorted(TYPES))
def test_ties(kind):
    """Equal logits: all of a row, runs of columns, columns of one lane, both zeros, rising and
    falling rows; far more equal ones than alternatives."""
    d, k = 40000, 64
    j = torch.arange(d, device=DEV)
    Z = torch.stack([torch.zeros(d, device=DEV), (j % 7 == 3).float(), (j >= d - 70).float(), (j % 2048 < 8).float(),
                     (j % 8192 == 17).float() * 2, torch.where(j % 2 == 0, 0.0, -0.0), (j // 500).float(),
                     -(j // 500).float(), (j % 512 < 8).float() * 3 - (j == 512).float(),
                     torch.where(j % 1024 < 40, j % 3, -5).float()]).to(TYPES[kind])
    Z[5] = torch.where(j % 2 == 0, 0.0, -0.0).to(TYPES[kind])
    for width in (d, 9001, 2000, 500, 65):
        for bits in (32, 64):
            top = torch.empty((len(Z), k), dtype=INTS[bits], device=DEV)
            lp = torch.empty((len(Z), k), device=DEV)
            T.toc_logprob(Z[:, :width], top_ids=top, top_logp=lp, ws=workspace(len(Z), width, k))
            z = Z[:, :width].double().cpu().numpy()
            want = np.stack([L.alternatives(r, k) for r in z])
            assert np.array_equal(top.cpu().numpy(), want), width


@pytest.mark.parametrize("lanes", [16, 64, 256, 512, 1024])
@pytest.mark.parametrize("n,d", [(3, 2500), (3, 40001), (130, 400001), (3, 400001), (600, 17000)])
def test_largest_in_few_lanes(n, d, lanes):
    """The largest logits of each row, many times the alternatives, all in the columns of one lane of 16 bytes
    in so many, rising, falling and equal."""
    j = torch.arange(d, device=DEV)
    rng = np.random.default_rng(d + lanes)
    Z = torch.randn((n, d), device=DEV, generator=torch.Generator(DEV).manual_seed(d)).to(torch.bfloat16)
    at = j // 8 % lanes == 5
    for i, x in enumerate((j * (8 / d) + 10, 20 - j * (8 / d), torch.full((d,), 11.0, device=DEV))):
        Z[i::3, at] = x[at].to(torch.bfloat16)
    k = 64
    top, lp = torch.empty((n, k), dtype=torch.int32, device=DEV), torch.empty((n, k), device=DEV)
    T.toc_logprob(Z, top_ids=top, top_logp=lp, ws=workspace(n, d, k))
    for i in {0, 1, 2, n - 1, n - 2}:
        want = torch.sort(Z[i].float(), descending=True, stable=True).indices[:k]
        assert torch.equal(top[i].long(), want), i


@pytest.mark.parametrize("n,d,kind", [(1, 1 << 28, "f32"), (1, (1 << 26) + 3, "bf16"), (128, (1 << 21) + 5, "bf16")])
def test_longest_rows(n, d, kind):
    g = torch.Generator(DEV).manual_seed(n)
    Z = torch.randn((n, d), generator=g, device=DEV).to(TYPES[kind])
    Z[0, d - 1], Z[0, 12345] = 9.0, 9.0
    ids = torch.full((n,), d - 1, device=DEV)
    logp, h, lse = (torch.empty(n, device=DEV) for _ in range(3))
    top, tl = torch.empty((n, 3), dtype=torch.int64, device=DEV), torch.empty((n, 3), device=DEV)
    T.toc_logprob(Z, ids, logp, lse, h, top, tl, ws=workspace(n, d, 3))
    z = Z[0].double()
    want = torch.logsumexp(z, 0)
    lp = z - want
    # sums of positive numbers in binary32, some d / 4096 of a lane in a row: 4e-3 at the worst, 1e-4 in
    # fact (roundings of either sign)
    assert abs(float(lse[0] - want)) < 1e-4 and abs(float(logp[0] - lp[-1])) < 1e-4
    assert abs(float(h[0] + (lp.exp() * lp).sum())) < 2e-3
    assert top[0, :2].tolist() == [12345, d - 1]
    # the same numbers as a teacher's, and the gradients in place
    entries = torch.tensor([12345, 7, d - 1, -1, 7], device=DEV).expand(n, 5).contiguous()
    t = torch.tensor([1.0, 2.0, 0.5, 9.0, 0.0], device=DEV).expand(n, 5).contiguous()
    loss = torch.empty(n, device=DEV)
    dZ, c = torch.empty_like(Z), torch.ones(n, device=DEV)
    T.toc_distill_grad(Z, dZ, entries, t, c, loss, ws=workspace(n, d))
    q = torch.softmax(torch.tensor([1.0, 2.0, 0.5, 0.0], dtype=torch.float64, device=DEV), 0)
    at = torch.tensor([12345, 7, d - 1, 7], device=DEV)
    assert abs(float(loss[0] - (q * (q.log() - lp[at])).sum())) < 2e-4
    back = lp.exp().index_add_(0, at, -q)
    assert float((dZ[0].double() - back).abs().max()) < 4e-3
    T.toc_logprob_grad(Z, Z, ids, c, ws=workspace(n, d))
    back = -lp.exp()
    back[-1] += 1
    assert float((Z[0].double() - back).abs().max()) < 4e-3


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("d", [300, 3001, 30000])
def test_infinities_and_nan(d, kind):
    rng = np.random.default_rng(d)
    Z, _ = logits(rng, 6, d, kind)
    Z[0, d // 2] = INF
    Z[1, 3] = float("nan")
    Z[2, :] = float("nan")
    Z[3, 5], Z[3, d - 1] = INF, float("nan")
    Z[4, 0] = -INF
    ids = torch.tensor([1, 1, 1, -1, 0, 2], device=DEV)
    logp, lse, h = (torch.zeros(6, device=DEV) for _ in range(3))
    top, tl = torch.empty((6, 4), dtype=torch.int64, device=DEV), torch.empty((6, 4), device=DEV)
    T.toc_logprob(Z, ids, logp, lse, h, top, tl, ws=workspace(6, d, 4))
    Z64 = Z.double().cpu().numpy()
    want = L.logprob(Z64, ids.cpu().numpy(), 1.0, 4)
    assert np.array_equal(top.cpu().numpy(), want["top_ids"])
    for got, key in ((logp, "logp"), (lse, "lse"), (h, "entropy")):
        assert np.array_equal(np.isnan(host(got)), np.isnan(want[key])), key
    assert host(logp)[4] == -INF and host(logp)[3] == 0
    dZ = torch.zeros_like(Z)
    gl = torch.tensor([1.0, 0.0, 1.0, 1.0, 1.0, 1.0], device=DEV)
    T.toc_logprob_grad(Z, dZ, ids, gl, ws=workspace(6, d))
    g = host(dZ)
    assert np.isnan(g[0]).any() and np.isnan(g[2]).all()
    assert not g[1].any() and not g[3].any()                       # no coefficient: 0, whatever it holds
    again = torch.full_like(Z, 7.0)
    T.toc_logprob_grad(Z, again, ids, gl, logp=logp, ws=workspace(6, d))
    assert np.array_equal(host(again), g, equal_nan=True) and np.isnan(host(logp)[1]) and host(logp)[3] == 0
    T.toc_logprob(Z, ids, logp, ws=workspace(6, d))                # a row without a token is not read
    assert np.isnan(host(logp)[1]) and host(logp)[3] == 0
    assert abs(g[4, 0] - 1) < 1e-2 and np.isfinite(g[4:]).all()    # the masked token's own part remains


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("d", WIDTHS)
def test_grad(d, kind):
    rng = np.random.default_rng(d + 1)
    n = 37 if d <= 2049 else 6
    for bits, gap, shift, parts, scale in ((64, 0, 0, "l", 1.0), (32, 5, 1, "lse", 0.37), (64, 3, 3, "e", 1.6),
                                           (32, 0, 1, "s", 1.0)):
        Z, Z64 = logits(rng, n, d, kind, gap, shift)
        ids, idt = given(rng, n, d, bits)
        g = {p: rng.standard_normal(n).astype(np.float32) for p in parts}
        if "l" in g:
            g["l"][rng.random(n) < 0.2] = 0
        scale = float(np.float32(scale))
        dZ = blank(n, d, kind, gap, shift)
        out = [torch.zeros(n, device=DEV) for _ in range(3)]
        dev = {p: vec(x) for p, x in g.items()}
        T.toc_logprob_grad(Z, dZ, idt, dev.get("l"), dev.get("s"), dev.get("e"), *out, scale, workspace(n, d))
        assert gaps_untouched(dZ)
        want = L.logprob_grad(Z64, ids, scale, g.get("l"), g.get("s"), g.get("e"))
        real = (ids >= 0) & (ids < d)
        target = (np.arange(d) == ids[:, None])
        s = Soft(Z64, scale)
        tol = grad_tol(s, want, kind, real * g.get("l", 0.0), g.get("s", 0.0), g.get("e", 0.0), target)
        close(dZ, want, tol, f"dZ of {parts}")
        score = L.logprob(Z64, ids, scale)
        finite(out[0], score["logp"], s.logp_tol(np.where(real, ids, 0)[:, None])[:, 0], "logp")
        finite(out[1], score["lse"], s.lse_tol(), "lse")
        close(out[2], score["entropy"], s.entropy_tol(), "entropy")
        # in place, with and without the outputs: the same bits
        again = blank(n, d, kind, gap, shift)
        again.copy_(Z)
        T.toc_logprob_grad(again, again, idt, dev.get("l"), dev.get("s"), dev.get("e"), *out, scale, workspace(n, d))
        assert torch.equal(again, dZ) and gaps_untouched(again)


@pytest.mark.parametrize("n,d,kind", [(1, 47236, "bf16"), (2, 70001, "f32"), (1, 262144, "bf16"), (3, 140001, "f16"),
                                      (300, 140001, "bf16"), (1100, 8192, "f32"), (1100, 4003, "bf16"), (1000, 4003, "bf16"),
                                      (500, 9001, "f16"), (600, 9001, "bf16"), (1023, 1501, "f32"), (5003, 900, "f16")])
def test_grad_long_and_many(n, d, kind):
    rng = np.random.default_rng(n + d)
    Z = torch.randn((n, d), device=DEV, generator=torch.Generator(DEV).manual_seed(d)).mul_(3).to(TYPES[kind])
    ids, idt = given(rng, n, d, 64)
    g = rng.standard_normal((2, n)).astype(np.float32)
    dZ, logp, h = torch.empty_like(Z), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    T.toc_logprob_grad(Z, dZ, idt, vec(g[0]), None, vec(g[1]), logp, None, h, 0.9, workspace(n, d))
    if n > 10:                                     # the first and the last rows
        at = np.r_[:4, n - 4:n]
        Z, dZ, ids, g, logp, h = Z[at], dZ[at], ids[at], g[:, at], logp[at], h[at]
    Z64, scale = Z.double().cpu().numpy(), float(np.float32(0.9))
    want = L.logprob_grad(Z64, ids, scale, g[0], None, g[1])
    real = (ids >= 0) & (ids < d)
    s = Soft(Z64, scale)
    close(dZ, want, grad_tol(s, want, kind, g[0] * real, 0.0, g[1], np.arange(d) == ids[:, None]), "dZ")
    score = L.logprob(Z64, ids, scale)
    finite(logp, score["logp"], s.logp_tol(np.where(real, ids, 0)[:, None])[:, 0], "logp")
    close(h, score["entropy"], s.entropy_tol(), "entropy")


@pytest.mark.parametrize("d", [11, 3000, 50000])
def test_grad_is_the_difference(d):
    """Along a direction, central differences of toc_logprob's own outputs."""
    rng = np.random.default_rng(d)
    n, h = 4, 2.0 ** -6
    Z = logits(rng, n, d, "f32")[0]
    ids, idt = given(rng, n, d, 64)
    ids = np.abs(ids) % d
    idt = torch.from_numpy(ids).to(DEV)
    g = rng.standard_normal((3, n)).astype(np.float32)
    way = torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32)).to(DEV)
    dZ, ws = torch.empty_like(Z), workspace(n, d)
    T.toc_logprob_grad(Z, dZ, idt, *(vec(x) for x in g), ws=ws)

    def value(step):
        out = [torch.empty(n, device=DEV) for _ in range(3)]
        T.toc_logprob(Z + step * way, idt, *out, ws=ws)
        return sum(c.astype(np.float64) * host(o) for c, o in zip(g, out))

    got = (dZ.double() * way.double()).sum(1).cpu().numpy()
    diff = (8 * (value(h) - value(-h)) - value(2 * h) + value(-2 * h)) / (12 * h)
    # the formula of order h^4: fifth derivatives of log sum exp and of the entropy along `way` are
    # below 100 (|w|^5 of a few); values of size 20 and error 1e-5 over 12 h
    assert np.all(np.abs(got - diff) <= 20 * h ** 4 * 100 / 5 + 20 * 1e-5 / h), (got, diff)


def test_logits_far_apart_and_overflowing():
    """Numbers whose scaled values or differences overflow binary32, and p of 0 and 1."""
    big = 3.0e38
    Z = torch.tensor([[big, -big, 0.0, big], [-big] * 4, [0.0, 200.0, -200.0, 199.0], [1e-30, -1e-30, 0.0, 0.0]],
                     device=DEV)
    ids = torch.tensor([0, 2, 1, 0], device=DEV)
    for scale in (1.0, 5.0):
        logp, h = torch.empty(4, device=DEV), torch.empty(4, device=DEV)
        dZ = torch.empty_like(Z)
        T.toc_logprob_grad(Z, dZ, ids, torch.ones(4, device=DEV), dentropy=torch.ones(4, device=DEV), logp=logp,
                           entropy=h, scale=scale)
        l2, l4 = np.log(2), np.log(4)
        p = 1 / (1 + np.exp(-scale))
        hp = -p * np.log(p) - (1 - p) * np.log(1 - p)
        assert np.allclose(host(logp), [-l2, -l4, np.log(p), -l4], atol=1e-6)
        assert np.allclose(host(h), [l2, l4, hp, l4], atol=1e-6)
        assert np.allclose(host(dZ)[1], scale * (np.arange(4) == 2) - scale / 4, atol=2e-6)
        assert np.isfinite(host(dZ)).all()


@pytest.mark.parametrize("size", [1e3, 1e5, 3e7, 3.7e8, 4e8, 1e9, 1e12, 1e25, 3e38])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("d", [40, 5000, 140000])
def test_large_logits(d, sign, size):
    """Logits whose scaled size passes what binary32 holds to one: neighbouring numbers, equal ones and far
    ones, anywhere in a row."""
    rng = np.random.default_rng(d)
    n = 6
    top = np.float32(sign * size)
    Z = np.full((n, d), top, np.float32)
    Z -= np.abs(top) * rng.random((n, d)).astype(np.float32) * np.float32(1e-3)
    for i in range(n):
        at = rng.permutation(d)[:12]
        Z[i, at[:4]] = top
        Z[i, at[4:8]] = np.nextafter(top, np.float32(-np.inf))
        Z[i, at[8:]] = np.nextafter(Z[i, at[4:8]], np.float32(-np.inf))
        if i % 2:
            Z[i, at[:4]] = Z[i, at[9]]
    Z = np.maximum(Z, -np.finfo(np.float32).max)
    Zt, Z64 = torch.from_numpy(Z).to(DEV), Z.astype(np.float64)
    ids = np.argmax(Z, axis=1)
    ids[0] = np.argmin(Z[0])
    g = rng.standard_normal((3, n)).astype(np.float32)
    for scale in (1.0, float(np.float32(0.3))):
        s = Soft(Z64, scale)
        dZ, logp, h = torch.empty_like(Zt), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        idt = torch.from_numpy(ids).to(DEV)
        T.toc_logprob_grad(Zt, dZ, idt, *(vec(x) for x in g), logp, None, h, scale, workspace(n, d))
        want, score = L.logprob_grad(Z64, ids, scale, *g), L.logprob(Z64, ids, scale)
        close(dZ, want, grad_tol(s, want, "f32", g[0], g[1], g[2], np.arange(d) == ids[:, None]), "dZ")
        close(logp, score["logp"], s.logp_tol(ids[:, None])[:, 0], "logp")
        close(h, score["entropy"], s.entropy_tol(), "entropy")


def test_offsets_past_32_bits():
    ld, d, n = 1 << 26, 1000, 70
    buf = torch.empty(n * ld, dtype=torch.bfloat16, device=DEV)
    Z = buf.view(n, ld)[:, :d]
    Z.copy_(torch.randn((n, d), device=DEV))
    flat = Z.contiguous()
    ids = torch.arange(n, device=DEV)
    res = []
    for X in (flat, Z):
        logp, top, tl = torch.empty(n, device=DEV), torch.empty((n, 3), dtype=torch.int64, device=DEV), torch.empty((n, 3), device=DEV)
        T.toc_logprob(X, ids, logp, top_ids=top, top_logp=tl, ws=workspace(n, d, 3))
        out = torch.empty_like(flat) if X is flat else Z
        T.toc_logprob_grad(X, out, ids, torch.ones(n, device=DEV), ws=workspace(n, d))
        res.append((logp, top, tl, out))
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_more_rows_than_workgroups():
    """Four million short rows, and the last rows' outputs."""
    n, d = (1 << 22) + 77, 5
    g = torch.Generator(DEV).manual_seed(1)
    Z = torch.randn((n, d), generator=g, device=DEV)
    ids = torch.randint(0, d, (n,), generator=g, device=DEV)
    logp, top, tl = torch.empty(n, device=DEV), torch.empty((n, 2), dtype=torch.int64, device=DEV), torch.empty((n, 2), device=DEV)
    T.toc_logprob(Z, ids, logp, top_ids=top, top_logp=tl, ws=workspace(n, d, 2))
    want = torch.log_softmax(Z.double(), 1)
    assert float((logp - want.gather(1, ids[:, None])[:, 0]).abs().max()) < 2e-6
    # (a few of so many rows hold equal numbers: the lower column first)
    assert torch.equal(top, torch.sort(Z, dim=1, descending=True, stable=True).indices[:, :2])
    dZ = torch.empty_like(Z)
    T.toc_logprob_grad(Z, dZ, ids, torch.ones(n, device=DEV), ws=workspace(n, d))
    want = torch.nn.functional.one_hot(ids, d) - want.exp()
    assert float((dZ - want).abs().max()) < 2e-6


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("d", [1, 2, 7, 8, 9, 31, 127, 128, 129, 300, 572, 900, 1001, 1135, 1136, 1152])
def test_many_short_rows(d, kind):
    """So many rows that several share a wave, the last wave only partly filled; masked, padded and empty
    rows beside others."""
    rng = np.random.default_rng(d)
    n, scale = 4097 + 6, float(np.float32(0.9))
    Z, Z64 = logits(rng, n, d, kind, gap=3, shift=1, masked=0.2)
    Z[5], Z[n - 2] = -INF, -INF
    ids, idt = given(rng, n, d, 32)
    g = rng.standard_normal((3, n)).astype(np.float32)
    g[:, 7] = 0
    dZ = blank(n, d, kind, 3, 1)
    out = [torch.full((n,), 7.0, device=DEV) for _ in range(3)]
    only = torch.full((n,), 7.0, device=DEV)
    T.toc_logprob_grad(Z, dZ, idt, *(vec(x) for x in g), *out, scale)
    T.toc_logprob(Z, idt, only, scale=scale)
    assert gaps_untouched(dZ)
    at = np.r_[:40, n - 40:n]
    Z64, ids, g = Z[at].double().cpu().numpy(), ids[at], g[:, at]
    s, real = Soft(Z64, scale), (ids >= 0) & (ids < d)
    want = L.logprob_grad(Z64, ids, scale, *g)
    close(dZ[at], want, grad_tol(s, want, kind, g[0] * real, g[1], g[2], np.arange(d) == ids[:, None]), "dZ")
    score = L.logprob(Z64, ids, scale)
    for got in (out[0][at], only[at]):
        finite(got, score["logp"], s.logp_tol(np.where(real, ids, 0)[:, None])[:, 0], "logp")
    finite(out[1][at], score["lse"], s.lse_tol(), "lse")
    close(out[2][at], score["entropy"], s.entropy_tol(), "entropy")
    again = blank(n, d, kind, 3, 1)
    again.copy_(Z)
    T.toc_logprob_grad(again, again, idt, *(vec(x) for x in rng.standard_normal((3, n))), scale=scale)
    assert gaps_untouched(again)


@pytest.mark.parametrize("n,d,k", [(33, 20000, 40), (33, 1500, 40), (9, 6001, 64), (3, 140001, 20), (700, 9000, 5)])
def test_equal_calls_and_rows_alone(n, d, k):
    """Equal bits from equal calls; nothing is left in a workspace that a next call would find."""
    rng = np.random.default_rng(5)
    Z, _ = logits(rng, n, d, "bf16")
    _, idt = given(rng, n, d, 64)
    res = []
    for fill in (0, 255):
        ws = workspace(n, d, k)
        if ws is not None:
            ws.fill_(fill)
        out = [torch.full((n,), float(fill), device=DEV) for _ in range(3)]
        top, tl = torch.empty((n, k), dtype=torch.int64, device=DEV), torch.empty((n, k), device=DEV)
        T.toc_logprob(Z, idt, *out, top, tl, 1.1, ws)
        dZ = torch.empty_like(Z)
        T.toc_logprob_grad(Z, dZ, idt, out[0], out[1], out[2], scale=1.1, ws=ws)
        res.append((*out, top, tl, dZ))
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_no_rows():
    Z = torch.empty((0, 100), device=DEV)
    T.toc_logprob(Z, torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV))
    T.toc_logprob_grad(Z, Z, torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV))
