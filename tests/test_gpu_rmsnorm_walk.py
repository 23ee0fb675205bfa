"""Workgroups of the root-mean-square norm and its gradient that walk over several rows: more
rows than a launch has workgroups, in every shape that walks, rows of clearly different
magnitude so that a sum left from another row shows.  Checked on the GPU in float64 with the
oracle's mask."""

import numpy as np
import pytest

import paper_1702_06943_amd as T
from oracle import rows as R
from rows_cases import DEV, LEAST, TREE, TYPES, U, UNIT, torch

pytestmark = pytest.mark.gpu
DROP = (0.25, 0xFEEDFACE12345678, 3)
EPS = 1e-5


def inputs(n, d, kind, *scales):
    g = torch.Generator(device=DEV)
    g.manual_seed(n + d)
    by = 4.0 ** (torch.arange(n, device=DEV)[:, None] % 7 - 3)
    return [(torch.randn((n, d), generator=g, device=DEV) * by * s).to(TYPES[kind]) for s in scales]


def weights(d):
    g = torch.Generator(device=DEV)
    g.manual_seed(d)
    return 1 + 0.3 * torch.randn(d, generator=g, device=DEV)


def mask(n, d, drop):
    if not drop:
        return 1.0
    return torch.from_numpy(R.dropout(np.ones((n, d), np.float32), drop)).to(DEV)


def within(got, want, tol, what):
    off = (got.double() - want).abs() - tol
    assert not torch.isnan(off).any() and float(off.max()) <= 0, what


@pytest.mark.parametrize("drop", [None, DROP], ids=["plain", "drop"])
@pytest.mark.parametrize("eight", [False, True], ids=["same", "e4m3"])
@pytest.mark.parametrize("n,d,kind", [(2100, 8192, "bf16"), (2100, 4100, "f32"), (2060, 16384, "bf16"),
                                      (2060, 16380, "f32")])
def test_norm(n, d, kind, eight, drop):
    X, Rs = inputs(n, d, kind, 1.0, 2.0)
    w = weights(d)
    H, Y = torch.empty_like(X), torch.empty_like(X, dtype=torch.float8_e4m3fn if eight else None)
    s = torch.empty(n, device=DEV) if eight else None
    T.toc_rmsnorm(X, Y, R=Rs, H=H, w=w, eps=EPS, drop=T.Drop(*drop) if drop else None, y_scale=s)
    x = X.double() * mask(n, d, drop)
    h = Rs.double() + x
    # keep, its product and the sum; then as for few rows: the sum's tree, 1 / d, eps, the root,
    # the quotient, and what h's own errors move
    eh = 2 * U * x.abs() + 2 * U * h.abs()
    del x
    within(H, h, eh + UNIT[kind] * h.abs() + LEAST[kind], "h")
    mean = h.square().mean(1, keepdim=True) + float(np.float32(EPS))
    er = (TREE + 8) * U + (h.abs() * eh).mean(1, keepdim=True) / mean
    y = h / mean.sqrt() * w.double()
    ey = w.double().abs() * eh / mean.sqrt() + y.abs() * (er + 4 * U)
    del h, eh
    if not eight:
        within(Y, y, ey + UNIT[kind] * y.abs() + LEAST[kind], "y")
        return
    top, etop = y.abs().amax(1), ey.amax(1)
    within(s, top / 448, etop / 448 + 4 * U * top / 448, "scale")
    q, scale = Y.double(), s.double()[:, None]
    # half the distance of e4m3 neighbours at the larger of both magnitudes
    e = torch.log2(torch.maximum((y / scale).abs(), q.abs()).clamp(min=2.0 ** -6)).floor().clamp(max=8)
    within(q * scale, y, scale * 2.0 ** (e - 4) + 2 * ey + 8 * U * y.abs(), "8-bit y")


@pytest.mark.parametrize("drop", [None, DROP], ids=["plain", "drop"])
@pytest.mark.parametrize("n,d,kind", [(1300, 4096, "bf16"), (1300, 1100, "f32"), (1100, 2048, "bf16"),
                                      (700, 8192, "bf16"), (700, 4100, "f32"), (700, 16384, "bf16"),
                                      (700, 16380, "f32")])
def test_norm_grad(n, d, kind, drop):
    H, dY, dR = inputs(n, d, kind, 2.0, 1.0, 0.5)
    w = weights(d)
    dH, dX = torch.empty_like(H), torch.empty_like(H)
    dw = torch.full((d,), 9.0, device=DEV)
    ws = torch.full((T.toc_rmsnorm_grad_workspace_size(n, d),), 0xA5, dtype=torch.uint8, device=DEV)
    T.toc_rmsnorm_grad(H, dY, dH, ws, w=w, eps=EPS, dR=dR, dX=dX, dw=dw,
                       drop=T.Drop(*drop) if drop else None)
    h, dy, m = H.double(), dY.double(), mask(n, d, drop)
    r = (h.square().mean(1, keepdim=True) + float(np.float32(EPS))).rsqrt()
    g = dy * w.double()
    dh = r * g - h * r ** 3 * (g * h).mean(1, keepdim=True) + dR.double()
    terms = g.abs() * r + h.abs() * r ** 3 * (g * h).abs().mean(1, keepdim=True)
    th = 3 * (TREE + 8) * U * terms + 4 * U * dR.double().abs()
    within(dH, dh, th + UNIT[kind] * dh.abs() + LEAST[kind], "dH")
    keep = 1.0 if not drop else 65536 / (65536 - R.drop_below(drop[0]))
    dx = dh * m
    within(dX, dx, keep * th + (UNIT[kind] + 4 * U) * dx.abs() + LEAST[kind], "dX")
    parts = dy * h * r
    within(dw, parts.sum(0), (n + TREE + 16) * U * parts.abs().sum(0), "dw")
    again = torch.empty_like(dw)
    T.toc_rmsnorm_grad(H, dY, None, ws, w=w, eps=EPS, dw=again)
    assert torch.equal(again, dw)
