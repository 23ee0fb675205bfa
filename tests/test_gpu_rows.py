"""Embedding lookup and dropout on the GPU against the 64-bit oracle: types, widths, strides,
misaligned rows, token numbers outside the table, the mask's independence of layout, in-place
calls, offsets past 32 bits, streams, graphs, and the binding's refusals."""

import numpy as np
import pytest

import paper_1702_06943_amd as T
from oracle import rows as R
from rows_cases import (DEV, LEAST, TYPES, U, UNIT, blank, close, gaps_untouched, host, rows, torch)

pytestmark = pytest.mark.gpu
DROPS = [None, (0.25, 0x123456789ABCDEF0, 0xFEDCBA9876543210)]


def tol(want, kind):
    """scale, keep and their rounding to binary32, two products; one rounding to the type."""
    return (4 * U + UNIT[kind]) * np.abs(want) + LEAST[kind]


def tokens(rng, n, V, bits):
    ids = rng.integers(0, max(V, 1), n)
    ids[rng.random(n) < 0.1] = -1
    if n > 4:
        ids[1], ids[2] = V, (1 << (bits - 1)) - 1
        ids[3], ids[4] = -(1 << (bits - 1)), max(V - 1, 0)
    return ids, torch.from_numpy(ids.astype(np.int32 if bits == 32 else np.int64)).to(DEV)


@pytest.mark.parametrize("drop", DROPS, ids=["plain", "drop"])
@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("n,d", [(1, 1), (1, 8), (1, 1000), (2, 7), (3, 9), (5, 64), (65, 63), (130, 65),
                                 (257, 300), (64, 1024), (7, 4097)])
def test_embed(n, d, kind, drop):
    rng = np.random.default_rng(n * 10007 + d)
    V, scale = 37, 1.7
    for bits, gap, shift in ((64, 0, 0), (32, 5, 1)):
        ids, idt = tokens(rng, n, V, bits)
        E, E64 = rows(rng, V, d, kind, gap=gap, shift=shift)
        out = blank(n, d, kind, gap=gap, shift=shift)
        T.toc_embed(idt, E, out, scale=scale, drop=T.Drop(*drop) if drop else None)
        want = R.embed(ids, E64, float(np.float32(scale)), drop)
        close(out, want, tol(want, kind), f"{bits}-bit ids, gap {gap}")
        assert gaps_untouched(out)


def test_embed_copies_exactly():
    rng = np.random.default_rng(3)
    for kind in TYPES:
        E, _ = rows(rng, 50, 24, kind)
        E[7, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 0.0], device=DEV)
        ids = torch.arange(49, -1, -1, device=DEV)
        out = blank(50, 24, kind)
        T.toc_embed(ids, E, out)
        assert torch.equal(torch.nan_to_num(out, nan=9.0), torch.nan_to_num(E.flip(0), nan=9.0))


def test_embed_empty():
    E = torch.ones((4, 8), device=DEV)
    T.toc_embed(torch.empty(0, dtype=torch.int64, device=DEV), E, E[:0])
    out = blank(3, 8, "f32")
    T.toc_embed(torch.arange(3, device=DEV), torch.empty((0, 8), device=DEV), out)
    assert not out.any()


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("n,d", [(1, 1), (3, 8), (9, 13), (250, 200), (33, 1023)])
def test_dropout(n, d, kind):
    rng = np.random.default_rng(n + d)
    for p in (0.0, 0.1, 0.5, 1.0, 1e-6, 0.99999):
        drop = (p, 77 + n, (1 << 63) + d)
        X, X64 = rows(rng, n, d, kind, gap=3)
        Y = blank(n, d, kind, gap=1, shift=1)
        T.toc_dropout(X, Y, T.Drop(*drop))
        want = R.dropout(X64, drop)
        close(Y, want, tol(want, kind), f"p = {p}")
        assert gaps_untouched(Y)
        inplace = X.clone()
        T.toc_dropout(inplace, inplace, T.Drop(*drop))
        assert torch.equal(inplace, Y)


def test_dropped_infinities_are_zero():
    drop = (0.5, 1, 2)
    kept = R.kept(16, 40, drop)
    for bad in (float("inf"), float("nan")):
        X = torch.full((16, 40), bad, device=DEV)
        Y = blank(16, 40, "f32")
        T.toc_dropout(X, Y, T.Drop(*drop))
        assert np.array_equal(host(Y) == 0, ~kept)
        assert not torch.isfinite(Y[torch.from_numpy(kept).to(DEV)]).any()


def test_mask_is_the_elements_own():
    """The same element is kept whatever the type, the strides, the rows around it and the
    operator that asks."""
    p = T.Drop(0.3, 99, 5)
    keep = {}
    for kind in TYPES:
        for n, d, gap in ((40, 72, 0), (40, 72, 9), (17, 72, 0), (40, 50, 0)):
            X, Y = blank(n, d, kind, gap=gap), blank(n, d, kind)
            T.toc_dropout(X, Y, p)
            keep[kind, n, d, gap] = Y != 0
    full = keep["f32", 40, 72, 0]
    for (kind, n, d, gap), k in keep.items():
        assert torch.equal(k, full[:n, :d])
    out = blank(40, 72, "f32")
    T.toc_embed(torch.zeros(40, dtype=torch.int32, device=DEV), torch.ones((1, 72), device=DEV), out,
                drop=p)
    assert torch.equal(out != 0, full)


def test_offsets_past_32_bits():
    """Table rows, and rows of strided matrices, more than 2^32 elements into their buffer."""
    V, ld, d = 70000, 65536, 16
    buf = torch.empty(V * ld, dtype=torch.bfloat16, device=DEV)
    E = buf.view(V, ld)[:, :d]
    at = torch.tensor([0, 32767, 32768, 65535, 65536, 69999], device=DEV)
    E[at] = torch.arange(6 * d, device=DEV).view(6, d).to(torch.bfloat16)
    out = blank(6, d, "bf16")
    T.toc_embed(at, E, out)
    assert torch.equal(out, torch.arange(6 * d, device=DEV).view(6, d).to(torch.bfloat16))
    drop = T.Drop(0.5, 4, 4)
    # a strided matrix of that many rows: every row's mask is its own row's
    X = torch.ones((V, d), dtype=torch.bfloat16, device=DEV)
    Y = torch.empty_like(X)
    T.toc_dropout(X, Y, drop)
    T.toc_dropout(X, E, drop)
    assert torch.equal(E, Y)


def test_another_stream_and_graph():
    rng = np.random.default_rng(8)
    E, _ = rows(rng, 100, 136, "bf16")
    ids = torch.from_numpy(rng.integers(0, 100, 300)).to(DEV)
    drop = T.Drop(0.2, 3, 3)
    want = blank(300, 136, "bf16")
    T.toc_embed(ids, E, want, 2.0, drop)
    side = torch.cuda.Stream()
    out = blank(300, 136, "bf16")
    side.wait_stream(torch.cuda.current_stream())
    T.toc_embed(ids, E, out, 2.0, drop, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            T.toc_embed(ids, E, out, 2.0, drop)
            T.toc_dropout(out, out, drop)
    T.toc_dropout(want, want, drop)
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_binding_refusals():
    E, out = torch.zeros((4, 8), device=DEV), torch.zeros((3, 8), device=DEV)
    ids = torch.zeros(3, dtype=torch.int64, device=DEV)
    bad = [
        (ids.float(), E, out), (ids[None], E, out), (ids.cpu(), E, out), (ids, E.cpu(), out),
        (ids, E, out[:2]), (ids, E, out[:, :7]), (ids, E, out.half()), (ids, E.double(), out.double()),
        (ids, E.t(), out), (ids, E[0], out), (torch.zeros(6, dtype=torch.int64, device=DEV)[::2], E, out),
        (ids, E, out[:1].expand(3, 8)),
    ]
    for a in bad:
        with pytest.raises(T.TocError) as e:
            T.toc_embed(*a)
        assert e.value.status == T.TOC_EINVAL
    for drop in (None, 0.5, T.Drop(1.5, 0, 0)):
        with pytest.raises(T.TocError) as e:
            T.toc_dropout(E, E, drop)
        assert e.value.status == T.TOC_EINVAL


def test_more_chunks_than_one_launch():
    """17 million rows of 512 bfloat16 numbers, 2^30 chunks and more: the rows of later launches
    have their own rows' masks."""
    n, d, drop = (1 << 24) + 1001, 512, (0.5, 0x1234567, 3)
    X = torch.ones((n, d), dtype=torch.bfloat16, device=DEV)
    T.toc_dropout(X, X, T.Drop(*drop))
    for row in (0, 1, (1 << 24) - 1, 1 << 24, (1 << 24) + 1, n - 1):
        q = np.arange(d // 8, dtype=np.uint64)
        fill = [np.full(d // 8, v, np.uint64) for v in (row, drop[2] & 0xFFFFFFFF, drop[2] >> 32)]
        words = R.philox4x32((q, *fill), (drop[1] & 0xFFFFFFFF, drop[1] >> 32))
        kept = np.stack([words[j // 2] >> np.uint64(16 * (j % 2)) & np.uint64(0xFFFF) for j in range(8)], 1)
        want = np.where(kept.reshape(-1) >= R.drop_below(drop[0]), 2.0, 0.0)
        assert np.array_equal(host(X[row]), want), row
