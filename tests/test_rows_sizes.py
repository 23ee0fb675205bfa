"""Sizes that do not fit the C calls' 32- and 64-bit arguments are refused by the binding: ctypes would
cut them to their low bits, and a row of 2^32 + 8 columns would be one of 8."""

import pytest

import paper_1702_06943_amd as T

SIZES = [(T.toc_logits_workspace_size, 3), (T.toc_embed_grad_workspace_size, 3), (T.toc_rmsnorm_grad_workspace_size, 2)]


@pytest.mark.parametrize("call,args", SIZES)
def test_workspace_sizes(call, args):
    assert call(*[3] * args) >= 0
    for i in range(args):
        for size, status in (((1 << 32) + 8, T.TOC_EUNSUPPORTED), (1 << 31, T.TOC_EUNSUPPORTED),
                             ((1 << 64) + 1, T.TOC_EUNSUPPORTED), (-(1 << 32) + 5, T.TOC_EINVAL),
                             (-(1 << 64) + 5, T.TOC_EINVAL), (-1, T.TOC_EINVAL)):
            a = [3] * args
            a[i] = size
            with pytest.raises(T.TocError) as e:
                call(*a)
            assert e.value.status == status, (i, size)


@pytest.mark.gpu
def test_long_rows():
    """A row of 2^32 + 8 columns, and no rows of as many."""
    torch = pytest.importorskip("torch")
    dev = "cuda:0"
    d = (1 << 32) + 8
    for n in (0, 1):
        Z = torch.empty((n, d), dtype=torch.float16, device=dev)
        v = torch.empty(n, device=dev)
        ids = torch.zeros(n, dtype=torch.int64, device=dev)
        top = torch.zeros((n, 2), dtype=torch.int64, device=dev)
        top_z = torch.zeros((n, 2), device=dev)
        calls = [lambda: T.toc_logprob(Z, ids, v), lambda: T.toc_logprob_grad(Z, Z, ids, v),
                 lambda: T.toc_distill(Z, top, top_z, v), lambda: T.toc_distill_grad(Z, Z, top, top_z, v),
                 lambda: T.toc_embed(ids, Z, Z), lambda: T.toc_dropout(Z, Z, None), lambda: T.toc_rmsnorm(Z, Z)]
        for call in calls:
            with pytest.raises(T.TocError) as e:
                call()
            assert e.value.status == T.TOC_EUNSUPPORTED
    wide = torch.empty((0, d), dtype=torch.int64, device=dev)
    Z = torch.empty((0, 8), device=dev)
    for call in (lambda: T.toc_logprob(Z, lse=Z[:, 0], top_ids=wide, top_logp=wide.float()),
                 lambda: T.toc_distill(Z, wide, wide.float(), Z[:, 0].contiguous())):
        with pytest.raises(T.TocError) as e:
            call()
        assert e.value.status == T.TOC_EUNSUPPORTED
