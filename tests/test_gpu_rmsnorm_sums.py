"""The norm's sums over long rows of numbers whose own squares are finite in binary32 while the
sum of the squares is not, against the 64-bit oracle (8-bit outputs too)."""

import numpy as np
import pytest

import paper_1702_06943_amd as T
from oracle import rows as R
from rows_cases import DEV, LEAST, TREE, TYPES, U, UNIT, blank, close, host, rows, torch, vec

pytestmark = pytest.mark.gpu
KINDS = ["f32", "bf16"]
WIDTHS = [1, 8, 60, 300, 513, 2000, 4099, 8192, 16384]


def large(rng, n, d, kind, gap=0):
    """Normal draws of standard deviation 3e18, none above 1.8e19."""
    t = np.clip(rng.standard_normal((n, d)), -5.5, 5.5) * 3e18
    X, _ = rows(rng, n, d, kind, gap=gap)
    X.copy_(torch.from_numpy(t).to(TYPES[kind]))
    return X, X.double().cpu().numpy()


@pytest.mark.parametrize("eight", [False, True], ids=["same", "e4m3"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", WIDTHS)
def test_norm(d, kind, eight):
    rng = np.random.default_rng(d)
    n = 3
    X, X64 = large(rng, n, d, kind, gap=1)
    w, w64 = vec(rng, d)
    Y = blank(n, d, torch.float8_e4m3fn if eight else kind)
    s = torch.empty(n, device=DEV) if eight else None
    T.toc_rmsnorm(X, Y, w=w, y_scale=s)
    _, y = R.rmsnorm(X64, None, w64)
    ey = np.abs(y) * (TREE + 12) * U          # the root's tree, and the products
    if not eight:
        close(Y, y, ey + UNIT[kind] * np.abs(y) + LEAST[kind], "y")
        return
    top = np.max(np.abs(y), axis=1)
    close(s, top / 448, np.max(ey, axis=1) / 448 + 4 * U * top / 448, "scale")
    q, scale = host(Y), host(s)[:, None]
    half = np.maximum(R.e4m3_half_step(y / scale), R.e4m3_half_step(q))
    close(q * scale, y, scale * half + 2 * ey + 8 * U * np.abs(y), "8-bit y")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_grad(d, kind):
    """h as above and dY of size 1 and 10, partly along h: the sum of g h, up to 1e20 d, too."""
    rng = np.random.default_rng(d)
    n = 3
    H, H64 = large(rng, n, d, kind)
    w, w64 = vec(rng, d)
    dY = torch.from_numpy(rng.standard_normal((n, d)) + 3e-18 * H64).to(TYPES[kind]).to(DEV)
    Y64 = dY.double().cpu().numpy()
    dH, dw = blank(n, d, kind), blank(1, d, "f32")[0]
    ws = torch.empty(T.toc_rmsnorm_grad_workspace_size(n, d), dtype=torch.uint8, device=DEV)
    T.toc_rmsnorm_grad(H, dY, dH, ws, w=w, dw=dw)
    wh, _, ww = R.rmsnorm_grad(H64, Y64, w64)
    r = 1 / np.sqrt(np.mean(H64 ** 2, axis=1, keepdims=True) + 1e-5)
    g = Y64 * w64
    terms = np.abs(g) * r + np.abs(H64) * r ** 3 * np.mean(np.abs(g * H64), axis=1, keepdims=True)
    close(dH, wh, 3 * (TREE + 8) * U * terms + UNIT[kind] * np.abs(wh) + LEAST[kind], "dH")
    close(dw, ww, (n + TREE + 16) * U * np.sum(np.abs(Y64 * H64 * r), axis=0), "dw")


def test_ordinary_rows_keep_their_bits():
    """Factors of 2 in all of h leave y its bits (eps far below), whatever the sums' scale is."""
    rng = np.random.default_rng(1)
    for d in (9, 300, 5000):
        X, _ = rows(rng, 4, d, "f32")
        first = None
        for e in (0, 20, -20):
            Y = blank(4, d, "f32")
            T.toc_rmsnorm((X * 2.0 ** e).contiguous(), Y, eps=1e-30)
            first = Y if first is None else first
            assert torch.equal(first, Y)
