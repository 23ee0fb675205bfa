"""Refusals of the C entry points on rows of logits: every argument is checked on the host before
anything is launched, so these run without a GPU (no call here reaches a launch)."""

import pytest

import paper_1702_06943_amd as T

P = 0x10000          # a pointer that no refused call follows
INF, NAN = float("inf"), float("nan")

SCORE = ["n", "d", "type", "Z", "ldz", "scale", "ids", "id_bits", "logp", "lse", "entropy", "k", "top_ids",
         "top_logp", "ws", "ws_bytes", "s"]
SCORE_GRAD = ["n", "d", "type", "Z", "ldz", "scale", "ids", "id_bits", "dlogp", "dlse", "dentropy", "logp", "lse",
              "entropy", "dZ", "lddz", "ws", "ws_bytes", "s"]
TAUGHT = ["n", "d", "type", "Z", "ldz", "scale", "k", "top_ids", "id_bits", "ldi", "top_type", "top_z", "ldt",
          "top_scale", "top_lse", "loss", "ws", "ws_bytes", "s"]
TAUGHT_GRAD = TAUGHT[:15] + ["dloss", "loss", "dZ", "lddz", "ws", "ws_bytes", "s"]
OK = dict(n=3, d=8, type=T.TOC_BF16, Z=P, ldz=8, scale=1.0, ids=P, id_bits=64, logp=P, lse=P, entropy=P, k=4,
          top_ids=P, top_logp=P, dlogp=P, dlse=P, dentropy=P, dZ=P, lddz=8, ldi=4, top_type=T.TOC_BF16, top_z=P,
          ldt=4, top_scale=1.0, top_lse=P, dloss=P, loss=P, ws=P, ws_bytes=1 << 24, s=None)
CALLS = [("toc_logprob", SCORE), ("toc_logprob_grad", SCORE_GRAD), ("toc_distill", TAUGHT),
         ("toc_distill_grad", TAUGHT_GRAD)]


def call(name, order, **changes):
    a = dict(OK, **changes)
    return getattr(T.lib(), name)(*[a[k] for k in order])


@pytest.mark.parametrize("name,order", CALLS)
def test_shared_refusals(name, order):
    def refused(status=T.TOC_EINVAL, **changes):
        assert call(name, order, **changes) == status, changes
        assert T.lib().toc_last_error()

    refused(n=-1)
    refused(d=0)
    refused(type=7)
    refused(type=T.TOC_E4M3)
    refused(n=1 << 31, status=T.TOC_EUNSUPPORTED)
    refused(d=(1 << 28) + 1, ldz=(1 << 28) + 1, lddz=(1 << 28) + 1, status=T.TOC_EUNSUPPORTED)
    for s in (0.0, -1.0, NAN, INF, 3e38):          # 3e38 log2(e) is infinite
        refused(scale=s)
    refused(id_bits=16)
    refused(Z=None)
    refused(Z=P + 1)
    refused(ldz=7)
    refused(ws=P + 8)
    for name_ in ("logp", "lse", "entropy", "dlogp", "dlse", "dentropy", "top_logp", "top_lse", "loss", "dloss"):
        if name_ in order:
            refused(**{name_: P + 2})
    if "dZ" in order:
        refused(dZ=None)
        refused(dZ=P + 1)
        refused(lddz=7)
        refused(lddz=9)                            # Z itself, with other rows
    assert call(name, order, n=0, Z=None, ids=None, logp=None, top_ids=None, top_logp=None, top_z=None, loss=None,
                dloss=None, dZ=None, dlogp=None, ws=None, ws_bytes=0) == 0        # nothing to do


def test_token_refusals():
    for name, order in CALLS[:2]:
        assert call(name, order, ids=P + 4) == T.TOC_EINVAL
        assert call(name, order, ids=None) == T.TOC_EINVAL             # logp, dlogp ask for them
    assert call(*CALLS[1], ids=None, logp=None) == T.TOC_EINVAL
    assert call(*CALLS[0], k=-1) == T.TOC_EINVAL
    assert call(*CALLS[0], k=65) == T.TOC_EUNSUPPORTED
    assert call(*CALLS[0], top_ids=None) == T.TOC_EINVAL
    assert call(*CALLS[0], top_ids=P + 4) == T.TOC_EINVAL
    assert call(*CALLS[0], top_logp=None) == T.TOC_EINVAL


def test_teacher_refusals():
    for name, order in CALLS[2:]:
        for bad in (dict(k=0), dict(k=-2), dict(top_ids=None), dict(top_ids=P + 4), dict(ldi=3), dict(ldt=3),
                    dict(top_z=None), dict(top_z=P + 1), dict(top_type=T.TOC_F16), dict(top_type=9),
                    dict(top_type=T.TOC_F32, top_z=P + 2), dict(top_scale=0.0), dict(top_scale=NAN),
                    dict(top_scale=INF)):
            assert call(name, order, **bad) == T.TOC_EINVAL, bad
        assert call(name, order, k=257, ldi=257, ldt=257) == T.TOC_EUNSUPPORTED
    assert call(*CALLS[2], loss=None) == T.TOC_EINVAL
    assert call(*CALLS[3], dloss=None) == T.TOC_EINVAL


@pytest.mark.parametrize("k", [0, 1, 20, 64])
def test_workspace_sizes(k):
    """A size covers every call of fewer rows or alternatives."""
    for d in (1, 100, 5000, 47236, 70001, 131072, 131073, 262144, 1 << 24, 1 << 28):
        last = 0
        for n in sorted({0, 1, 2, 3} | {(1 << e) + i for e in range(2, 31) for i in (-1, 0, 1)}):
            size = T.toc_logits_workspace_size(n, d, k)
            assert size >= last and size >= T.toc_logits_workspace_size(n, d, k // 2)
            assert size < 1 << 28
            last = size
    assert T.toc_logits_workspace_size(0, 100, k) == 0
    for bad, status in (((-1, 5, k), T.TOC_EINVAL), ((1, 0, k), T.TOC_EINVAL), ((1, 5, -1), T.TOC_EINVAL),
                        ((1, 5, 65), T.TOC_EUNSUPPORTED), ((1, (1 << 28) + 1, k), T.TOC_EUNSUPPORTED)):
        with pytest.raises(T.TocError) as e:
            T.toc_logits_workspace_size(*bad)
        assert e.value.status == status
    assert T.lib().toc_logits_workspace_size(1, 1, 0, None) == T.TOC_EINVAL


def test_small_workspaces():
    """One byte less than what a call asks for, at sizes that ask for some."""
    for name, order in CALLS:
        for n, d in ((1, 1 << 20), (3, 300001), (2, 1 << 26)):
            k = 4
            need = T.toc_logits_workspace_size(n, d, k if name == "toc_logprob" else 0)
            if need:
                sizes = dict(n=n, d=d, ldz=d, lddz=d, k=k)
                assert call(name, order, **sizes, ws_bytes=need - 1) == T.TOC_ESIZE
                assert call(name, order, **sizes, ws=None) == T.TOC_EINVAL
