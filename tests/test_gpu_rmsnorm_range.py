"""The root-mean-square norm and its gradient at the ends of their range, against the 64-bit
oracle: rows whose cubed inverse root mean square is outside binary32, rows of zeros and tiny
rows under a tiny eps.  (binary16 has no such numbers.)"""

import numpy as np
import pytest

import paper_1702_06943_amd as T
from oracle import rows as R
from rows_cases import DEV, LEAST, TREE, TYPES, U, UNIT, blank, close, rows, torch, vec

pytestmark = pytest.mark.gpu
DROP = (0.25, 0x0123456789ABCDEF, 6)
KINDS = ["f32", "bf16"]


def check_grad(H, H64, dY, Y64, kind, eps, drop=None):
    """dH, dX and dw under the bounds of the gradient's other tests: r^3 carries three times r's
    error, (TREE + 8) u / 2 each, and the sum of g h its tree's."""
    n, d = H.shape
    w, w64 = vec(np.random.default_rng(d), d)
    dH, dX, dw = blank(n, d, kind), blank(n, d, kind), blank(1, d, "f32")[0]
    ws = torch.empty(max(T.toc_rmsnorm_grad_workspace_size(n, d), 16), dtype=torch.uint8, device=DEV)
    T.toc_rmsnorm_grad(H, dY, dH, ws, w=w, eps=eps, dX=dX, dw=dw, drop=T.Drop(*drop) if drop else None)
    eps = float(np.float32(eps))
    wh, wx, ww = R.rmsnorm_grad(H64, Y64, w64, eps, None, drop)
    r = 1 / np.sqrt(np.mean(H64 ** 2, axis=1, keepdims=True) + eps)
    g = Y64 * w64
    terms = np.abs(g) * r + np.abs(H64) * r ** 3 * np.mean(np.abs(g * H64), axis=1, keepdims=True)
    th = 3 * (TREE + 8) * U * terms
    close(dH, wh, th + UNIT[kind] * np.abs(wh) + LEAST[kind], "dH")
    keep = 65536 / max(65536 - R.drop_below(drop[0]), 1) if drop else 1.0
    close(dX, wx, keep * th + (UNIT[kind] + 4 * U) * np.abs(wx) + LEAST[kind], "dX")
    close(dw, ww, (n + TREE + 16) * U * np.sum(np.abs(Y64 * H64 * r), axis=0), "dw")


def along(rng, H64, size, kind):
    """dY partly along h, so that neither term of dH is small against the other."""
    Y = torch.from_numpy(rng.standard_normal(H64.shape) + 2 * H64 / size).to(TYPES[kind])
    return Y.to(DEV), Y.double().numpy()


@pytest.mark.parametrize("size", [1e10, 1e13, 1e15, 1e17])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [1, 7, 64, 300, 1000, 2049, 4099])
def test_grad_of_large_rows(d, kind, size):
    rng = np.random.default_rng(d)
    H, H64 = rows(rng, 5, d, kind, size)
    dY, Y64 = along(rng, H64, size, kind)
    for drop in (None, DROP):
        check_grad(H, H64, dY, Y64, kind, 1e-5, drop)


@pytest.mark.parametrize("eps", [1e-20, 1e-25, 1e-30])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [1, 40, 300, 4099])
def test_grad_under_a_tiny_eps(d, kind, eps):
    """Rows of zeros, as padding and dropout leave them, between tiny and ordinary rows."""
    rng = np.random.default_rng(d)
    H, H64 = rows(rng, 6, d, kind, 1.0)
    by = np.array([0.0, 1.0, 2.0 ** -40, 0.0, 2.0 ** -50, 2.0 ** 20])[:, None]
    H *= torch.from_numpy(by).to(DEV).to(H.dtype)
    dY, Y64 = rows(rng, 6, d, kind)
    check_grad(H, H64 * by, dY, Y64, kind, eps, DROP)
    # a row of zeros: dH = r g
    dH = blank(6, d, kind)
    T.toc_rmsnorm_grad(H, torch.ones_like(H), dH, None, eps=eps)
    want = float(np.float32(eps)) ** -0.5
    assert np.all(np.abs(dH[[0, 3]].double().cpu().numpy() - want) <= (4 * U + UNIT[kind]) * want)


@pytest.mark.parametrize("kind", KINDS)
def test_grad_of_dropped_rows(kind):
    """Forward with every element dropped and no residual, and back."""
    n, d, eps = 4, 136, 1e-30
    X, _ = rows(np.random.default_rng(1), n, d, kind)
    H, Y = blank(n, d, kind), blank(n, d, kind)
    T.toc_rmsnorm(X, Y, H=H, eps=eps, drop=T.Drop(1.0, 1, 2))
    assert not H.any() and not Y.any()
    dY, Y64 = rows(np.random.default_rng(2), n, d, kind)
    check_grad(H, np.zeros((n, d)), dY, Y64, kind, eps, (1.0, 1, 2))
