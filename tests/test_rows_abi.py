"""Refusals of the row operators' C entry points: every argument is checked on the host
before anything is launched, so these run without a GPU (no call here reaches a launch)."""

import ctypes as C

import pytest

import paper_1702_06943_amd as T

P = 0x10000          # a pointer that no refused call follows
INF, NAN = float("inf"), float("nan")


def call(name, order, good, **changes):
    a = dict(good, **changes)
    return getattr(T.lib(), name)(*[a[k] for k in order])


EMBED = ["n", "ids", "id_bits", "n_vocab", "d", "type", "E", "lde", "scale", "drop", "out", "ldo", "s"]
EMBED_OK = dict(n=3, ids=P, id_bits=64, n_vocab=5, d=8, type=T.TOC_BF16, E=P, lde=8, scale=1.0,
                drop=None, out=P, ldo=8, s=None)
GRAD = ["n", "ids", "id_bits", "n_vocab", "d", "type", "G", "ldg", "scale", "drop", "de_type", "dE",
        "lde", "accumulate", "ws", "ws_bytes", "s"]
GRAD_OK = dict(n=3, ids=P, id_bits=32, n_vocab=5, d=8, type=T.TOC_F16, G=P, ldg=8, scale=1.0,
               drop=None, de_type=T.TOC_F32, dE=P, lde=8, accumulate=0, ws=P, ws_bytes=1 << 20, s=None)
DROP = ["n", "d", "type", "X", "ldx", "drop", "Y", "ldy", "s"]
DROP_OK = dict(n=3, d=8, type=T.TOC_F32, X=P, ldx=8, drop=None, Y=P, ldy=8, s=None)
NORM = ["n", "d", "type", "X", "ldx", "R", "ldr", "drop", "w", "eps", "H", "ldh", "y_type", "Y",
        "ldy", "y_scale", "s"]
NORM_OK = dict(n=3, d=8, type=T.TOC_BF16, X=P, ldx=8, R=P, ldr=8, drop=None, w=P, eps=1e-5, H=P,
               ldh=8, y_type=T.TOC_BF16, Y=P, ldy=8, y_scale=None, s=None)
BACK = ["n", "d", "type", "H", "ldh", "w", "eps", "dY", "lddy", "dR", "lddr", "drop", "dH", "lddh",
        "dX", "lddx", "dw", "accumulate", "ws", "ws_bytes", "s"]
BACK_OK = dict(n=3, d=8, type=T.TOC_BF16, H=P, ldh=8, w=P, eps=1e-5, dY=P, lddy=8, dR=P, lddr=8,
               drop=None, dH=P, lddh=8, dX=P, lddx=8, dw=P, accumulate=0, ws=P, ws_bytes=1 << 20, s=None)

SHARED = [("embed", "toc_embed", EMBED, EMBED_OK), ("embed_grad", "toc_embed_grad", GRAD, GRAD_OK),
          ("dropout", "toc_dropout", DROP, DROP_OK), ("norm", "toc_rmsnorm", NORM, NORM_OK),
          ("norm_grad", "toc_rmsnorm_grad", BACK, BACK_OK)]


def drop(p):
    return C.addressof(T.Drop(p, 1, 2))


@pytest.mark.parametrize("name,fn,order,good", SHARED, ids=[s[0] for s in SHARED])
def test_shared_refusals(name, fn, order, good):
    d = T.Drop(0.5, 1, 2)
    if name == "dropout":
        assert call(fn, order, good) == T.TOC_EINVAL             # drop is NULL
        good = dict(good, drop=C.addressof(d))
    assert call(fn, order, good, n=-1) == T.TOC_EINVAL
    assert call(fn, order, good, d=0) == T.TOC_EINVAL
    assert call(fn, order, good, type=7) == T.TOC_EINVAL
    assert call(fn, order, good, type=T.TOC_E4M3) == T.TOC_EINVAL
    assert call(fn, order, good, n=1 << 31) == T.TOC_EUNSUPPORTED
    wide = {k: (1 << 28) + 1 for k in order if k == "d" or k.startswith("ld")}
    assert call(fn, order, good, **wide) == T.TOC_EUNSUPPORTED
    for p in (-0.1, 1.5, NAN, INF):
        d = T.Drop(p, 1, 2)
        assert call(fn, order, good, drop=C.addressof(d)) == T.TOC_EINVAL
    size = 4 if name == "dropout" else 2
    for k in order:
        if k in ("E", "out", "G", "dE", "X", "Y", "H", "dY", "R", "dR", "dH", "dX"):
            assert call(fn, order, good, **{k: P + size // 2}) == T.TOC_EINVAL, k   # misaligned
        if k in ("E", "out", "G", "dE", "X", "Y", "dY", "ids") or (k == "H" and name == "norm_grad"):
            assert call(fn, order, good, **{k: None}) == T.TOC_EINVAL, k
        if k.startswith("ld"):
            assert call(fn, order, good, **{k: 7}) == T.TOC_EINVAL, k
    assert T.lib().toc_last_error()


@pytest.mark.parametrize("fn,order,good", [s[1:] for s in SHARED[:2]], ids=["embed", "embed_grad"])
def test_token_refusals(fn, order, good):
    assert call(fn, order, good, id_bits=16) == T.TOC_EINVAL
    assert call(fn, order, good, ids=P + 2) == T.TOC_EINVAL
    assert call(fn, order, good, n_vocab=-1) == T.TOC_EINVAL
    assert call(fn, order, good, n_vocab=1 << 31) == T.TOC_EUNSUPPORTED
    for s in (NAN, INF):
        assert call(fn, order, good, scale=s) == T.TOC_EINVAL
    d = T.Drop(0.9, 1, 2)                                         # keeps with a factor of 10
    assert call(fn, order, good, scale=1e38, drop=C.addressof(d)) == T.TOC_EINVAL
    assert call(fn, order, good, n=0, ids=None, n_vocab=0, E=None, dE=None, G=None, out=None,
                ws=None, ws_bytes=0) == 0                         # nothing to do


def test_embed_grad_refusals():
    assert call("toc_embed_grad", GRAD, GRAD_OK, de_type=T.TOC_BF16) == T.TOC_EINVAL
    assert call("toc_embed_grad", GRAD, GRAD_OK, ws=None) == T.TOC_EINVAL
    assert call("toc_embed_grad", GRAD, GRAD_OK, ws=P + 8) == T.TOC_EINVAL
    need = T.toc_embed_grad_workspace_size(3, 5, 8)
    assert call("toc_embed_grad", GRAD, GRAD_OK, ws_bytes=need - 1) == T.TOC_ESIZE
    big = (1 << 20) + 1
    assert call("toc_embed_grad", GRAD, GRAD_OK, d=big, ldg=big, lde=big) == T.TOC_EUNSUPPORTED


@pytest.mark.parametrize("fn,order,good", [s[1:] for s in SHARED[3:]], ids=["norm", "norm_grad"])
def test_norm_refusals(fn, order, good):
    for eps in (0.0, -1.0, NAN, INF):
        assert call(fn, order, good, eps=eps) == T.TOC_EINVAL
    assert call(fn, order, good, w=P + 2) == T.TOC_EINVAL
    wide = {k: 16385 for k in order if k == "d" or k.startswith("ld")}
    assert call(fn, order, good, **wide) == T.TOC_EUNSUPPORTED


def test_norm_output_refusals():
    assert call("toc_rmsnorm", NORM, NORM_OK, y_type=T.TOC_F32) == T.TOC_EINVAL
    assert call("toc_rmsnorm", NORM, NORM_OK, y_type=T.TOC_E4M3) == T.TOC_EINVAL      # no y_scale
    assert call("toc_rmsnorm", NORM, NORM_OK, y_type=T.TOC_E4M3, y_scale=P + 2) == T.TOC_EINVAL
    assert call("toc_rmsnorm", NORM, NORM_OK, n=0, X=None, R=None, H=None, Y=None) == 0
    assert call("toc_rmsnorm_grad", BACK, BACK_OK, dw=P + 2) == T.TOC_EINVAL
    assert call("toc_rmsnorm_grad", BACK, BACK_OK, ws=None) == T.TOC_EINVAL
    assert call("toc_rmsnorm_grad", BACK, BACK_OK, ws=P + 2) == T.TOC_EINVAL
    need = T.toc_rmsnorm_grad_workspace_size(3, 8)
    assert call("toc_rmsnorm_grad", BACK, BACK_OK, ws_bytes=need - 1) == T.TOC_ESIZE
    assert call("toc_rmsnorm_grad", BACK, BACK_OK, n=0, dw=None, ws=None, ws_bytes=0) == 0


def test_workspace_sizes():
    assert T.toc_embed_grad_workspace_size(0, 5, 8) == 0
    assert T.toc_rmsnorm_grad_workspace_size(0, 8) == 0
    for bad in ((-1, 5, 8), (1, -5, 8), (1, 5, 0)):
        with pytest.raises(T.TocError) as e:
            T.toc_embed_grad_workspace_size(*bad)
        assert e.value.status == T.TOC_EINVAL
    with pytest.raises(T.TocError) as e:
        T.toc_rmsnorm_grad_workspace_size(1, 16385)
    assert e.value.status == T.TOC_EUNSUPPORTED
    assert T.lib().toc_embed_grad_workspace_size(1, 1, 1, None) == T.TOC_EINVAL
    assert T.lib().toc_rmsnorm_grad_workspace_size(1, 1, None) == T.TOC_EINVAL
    # the largest call's workspace is a size, not an overflow
    assert T.toc_embed_grad_workspace_size((1 << 31) - 1, (1 << 31) - 1, 1 << 20) > 1 << 40
