"""The embedding table's gradient on the GPU against the 64-bit oracle: types, widths, token
counts around the sort's tiles and the sums' chunks, frequent, absent and outside numbers,
accumulation, equal bits on equal calls, the adjoint of the lookup, and graphs."""

import numpy as np
import pytest

import paper_1702_06943_amd as T
from oracle import rows as R
from rows_cases import (DEV, LEAST, TYPES, U, UNIT, blank, close, gaps_untouched, rows, torch)

pytestmark = pytest.mark.gpu
DROP = (0.25, 0x0F1E2D3C4B5A6978, 41)


def run(ids, G, dE, scale=1.0, drop=None, accumulate=False, dirty=True):
    ws = torch.empty(max(T.toc_embed_grad_workspace_size(len(ids), dE.shape[0], dE.shape[1]), 16),
                     dtype=torch.uint8, device=DEV)
    if dirty:
        ws.fill_(0xA5)               # what it holds on entry does not matter
    T.toc_embed_grad(ids, G, dE, ws, scale=scale, drop=T.Drop(*drop) if drop else None,
                     accumulate=accumulate)


def on(ids, bits=64):
    return torch.from_numpy(np.asarray(ids).astype(np.int32 if bits == 32 else np.int64)).to(DEV)


def check(ids, V, d, kind, out_kind=None, scale=0.75, drop=None, bits=64, gap=0, shift=0, seed=0):
    rng = np.random.default_rng(seed)
    out_kind = out_kind or kind
    G, G64 = rows(rng, len(ids), d, kind, gap=gap, shift=shift)
    dE = blank(V, d, out_kind, gap=gap, shift=shift)
    run(on(ids, bits), G, dE, scale, drop)
    want, S, count = R.embed_grad(ids, G64, V, scale, drop)
    # at most count additions one after the other, scale and keep
    tol = (count[:, None] + 6) * U * S + UNIT[out_kind] * np.abs(want) + LEAST[out_kind]
    close(dE, want, tol, f"{len(ids)} ids of {V}, {d} columns")
    assert gaps_untouched(dE)


@pytest.mark.parametrize("drop", [None, DROP], ids=["plain", "drop"])
@pytest.mark.parametrize("kind,out_kind", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"),
                                           ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("d", [1, 7, 8, 9, 65, 300, 513, 1024])
def test_types_and_widths(d, kind, out_kind, drop):
    rng = np.random.default_rng(d)
    ids = rng.integers(-2, 50, 150)
    ids[:60] = rng.integers(0, 3, 60)
    check(ids, 48, d, kind, out_kind, drop=drop, seed=d)
    check(ids, 48, d, kind, out_kind, drop=drop, bits=32, gap=3, shift=1, seed=d)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 255, 1023, 1024, 1025, 2047, 2048, 2049,
                               4099, 20001])
def test_counts(n):
    rng = np.random.default_rng(n)
    V = 700
    ids = np.minimum(rng.zipf(1.3, n) - 1, V + 5)      # frequent numbers, some outside
    check(ids, V, 24, "f32", bits=32 if n % 2 else 64, seed=n)


@pytest.mark.parametrize("V", [1, 2, 255, 256, 511, 512, 513, 65535, 65536, 300000, 1 << 20])
def test_vocabularies(V):
    rng = np.random.default_rng(V)
    ids = np.concatenate([rng.integers(0, V, 500), [0, V - 1, V, -1, V - 1, 0]])
    check(ids, V, 8, "bf16", "f32", seed=1)


def test_runs_against_chunks():
    """Runs of one number that end on, before and after the boundaries of chunks of 16."""
    counts = [16, 16, 1, 15, 32, 17, 31, 64, 1, 1, 14, 160, 5, 11, 16]
    ids = np.repeat(np.arange(len(counts)), counts)
    for seed in range(3):
        check(np.random.default_rng(seed).permutation(ids), 40, 72, "f32", seed=seed)


@pytest.mark.parametrize("n", [1, 17, 3000, 70000])
@pytest.mark.parametrize("what", ["one", "last", "outside", "distinct"])
def test_extremes(n, what):
    V = 80000
    ids = {"one": np.zeros(n, np.int64), "last": np.full(n, V - 1), "outside": np.full(n, -7),
           "distinct": np.random.default_rng(n).permutation(V)[:n]}[what]
    rng = np.random.default_rng(n)
    G, G64 = rows(rng, n, 8, "f32")
    dE = blank(V, 8, "f32")
    run(on(ids), G, dE)
    want = np.zeros((V, 8))
    S = np.zeros((V, 8))
    if what in ("one", "last"):
        want[ids[0]], S[ids[0]] = G64.sum(0), np.abs(G64).sum(0)
    elif what == "distinct":
        want[ids], S[ids] = G64, np.abs(G64)
    close(dE, want, (n if what in ("one", "last") else 6) * U * S, what)


@pytest.mark.parametrize("kind", sorted(TYPES))
def test_accumulate_touches_only_rows_that_occur(kind):
    rng = np.random.default_rng(4)
    V, d, n = 300, 40, 900
    ids = rng.integers(0, 100, n) * 2
    ids[:400] = 4                                       # crosses chunks
    E, E64 = rows(rng, V, d, kind)
    E[1::2] = float("nan")                              # not read, not written
    before = E.clone()
    G, G64 = rows(rng, n, d, kind)
    scale = -0.01
    run(on(ids), G, E, scale, accumulate=True)
    g, S, count = R.embed_grad(ids, G64, V, float(np.float32(scale)))
    E64[1::2] = 0
    want = E64 + g
    tol = (count[:, None] + 6) * U * (S + np.abs(E64)) + UNIT[kind] * np.abs(want) + LEAST[kind]
    absent = count == 0
    assert torch.equal(torch.nan_to_num(E[torch.from_numpy(absent).to(DEV)], nan=5.0),
                       torch.nan_to_num(before[torch.from_numpy(absent).to(DEV)], nan=5.0))
    close(E[::2], want[::2], tol[::2], "accumulated rows")


def test_empty():
    dE = blank(9, 12, "bf16", gap=4)
    G = torch.empty((0, 12), dtype=torch.bfloat16, device=DEV)
    ids = torch.empty(0, dtype=torch.int32, device=DEV)
    T.toc_embed_grad(ids, G, dE, None, accumulate=True)
    assert bool((dE == 7).all())
    T.toc_embed_grad(ids, G, dE, None)
    assert not dE.any() and gaps_untouched(dE)
    T.toc_embed_grad(on([1, 2]), torch.ones((2, 12), device=DEV), torch.empty((0, 12), device=DEV),
                     torch.empty(1 << 16, dtype=torch.uint8, device=DEV))


def test_equal_calls_give_equal_bits():
    rng = np.random.default_rng(5)
    ids = on(np.minimum(rng.zipf(1.2, 30000) - 1, 999))
    G, _ = rows(rng, 30000, 120, "bf16")
    first = None
    for _ in range(4):
        dE = blank(1000, 120, "f32")
        run(ids, G, dE, drop=DROP)
        first = dE if first is None else first
        assert torch.equal(first, dE)


def test_adjoint_of_the_lookup():
    """<G, embed(E)> = <embed_grad(G), E>, and the difference quotient of <G, embed(E)> in E,
    which is linear, equals <embed_grad(G), V> for a direction V."""
    rng = np.random.default_rng(6)
    n, V, d = 2000, 300, 88
    ids = on(rng.integers(-1, V, n))
    E, E64 = rows(rng, V, d, "f32")
    W, W64 = rows(rng, V, d, "f32")
    G, G64 = rows(rng, n, d, "f32")
    drop = T.Drop(*DROP)
    dE = blank(V, d, "f32")
    run(ids, G, dE, 0.5, DROP)
    outs = []
    for table in (E, E + W / 64, E - W / 64):
        out = blank(n, d, "f32")
        T.toc_embed(ids, table.contiguous(), out, 0.5, drop)
        outs.append(out.double().cpu().numpy())
    g = dE.double().cpu().numpy()
    # 12 u per product of the left sum, (count + 6) u per entry of g with counts below 32
    bound = 50 * U * np.sum(np.abs(outs[0] * G64)) + 50 * U * np.sum(np.abs(g * E64))
    assert abs(np.sum(outs[0] * G64) - np.sum(g * E64)) <= bound
    diff = np.sum((outs[1] - outs[2]) * G64) * 32
    size = np.sum((np.abs(outs[1]) + np.abs(outs[2])) * np.abs(G64)) * 32
    assert abs(diff - np.sum(g * W64)) <= 8 * U * size + 50 * U * np.sum(np.abs(g * W64))


def test_offsets_past_32_bits():
    n, ld, d = 70000, 65536, 8
    buf = torch.empty(n * ld, dtype=torch.bfloat16, device=DEV)
    X = buf.view(n, ld)[:, :d]
    X.fill_(1.0)
    ids = torch.arange(n, device=DEV) // 7000
    dE = blank(10, d, "f32")
    run(ids, X, dE, 2.0)
    assert bool((dE == 14000.0).all())
    # the same buffer as the gradient's rows
    run(torch.arange(n - 1, -1, -1, device=DEV), torch.ones((n, d), dtype=torch.bfloat16, device=DEV), X, 3.0)
    assert bool((X == 3.0).all())


def test_graph_and_reused_workspace():
    """Replays between eager calls that leave other things in the workspace."""
    rng = np.random.default_rng(7)
    n, V, d = 5000, 2000, 64
    ids, other = on(np.minimum(rng.zipf(1.3, n) - 1, V)), on(rng.integers(0, V, n))
    G, _ = rows(rng, n, d, "f16")
    ws = torch.empty(T.toc_embed_grad_workspace_size(n, V, d), dtype=torch.uint8, device=DEV)
    want, scratch, dE = (blank(V, d, "f32") for _ in range(3))
    T.toc_embed_grad(ids, G, want, ws)
    T.toc_embed_grad(ids, G, dE, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        T.toc_embed_grad(ids, G, dE, ws)
    for _ in range(4):
        dE.fill_(3.0)
        T.toc_embed_grad(other, G, scratch, ws)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(dE, want)


def test_binding_refusals():
    ids, G, dE = on([0, 1, 2]), torch.zeros((3, 8), device=DEV), torch.zeros((4, 8), device=DEV)
    ws = torch.empty(T.toc_embed_grad_workspace_size(3, 4, 8), dtype=torch.uint8, device=DEV)
    for a in [(ids, G[:2], dE, ws), (ids, G, dE[:, :7], ws), (ids, G, dE.half(), ws), (ids, G, dE, None),
              (ids, G, dE, ws.cpu()), (ids, G, dE[0], ws), (ids.short(), G, dE, ws),
              (ids, G[:1].expand(3, 8), dE, ws)]:
        with pytest.raises(T.TocError) as e:
            T.toc_embed_grad(*a)
        assert e.value.status == T.TOC_EINVAL
    with pytest.raises(T.TocError) as e:
        T.toc_embed_grad(ids, G, dE, ws[:-16])
    assert e.value.status == T.TOC_ESIZE


def gpu_check(ids, V, G, dE, scale=1.0, accumulated=None):
    """dE against a float64 sum on the GPU (64-bit atomics: its own error is far below)."""
    ok = (ids >= 0) & (ids < V)
    at = torch.where(ok, ids, 0).long()
    terms = torch.where(ok[:, None], G.double(), 0.0) * scale
    want = torch.zeros(dE.shape, dtype=torch.float64, device=DEV).index_add_(0, at, terms)
    S = torch.zeros(dE.shape, dtype=torch.float64, device=DEV).index_add_(0, at, terms.abs())
    count = torch.zeros(V, dtype=torch.float64, device=DEV).index_add_(0, at, ok.double())
    kind = {v: k for k, v in TYPES.items()}[dE.dtype]
    tol = (count[:, None] + 6) * U * S + UNIT[kind] * want.abs() + LEAST[kind]
    assert bool(((dE.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("n,V,d,out", [
    (150001, 70000, 16, "f32"),      # more tiles than are summed without a scan
    (150001, 300000, 8, "f32"),      # three passes
    (70001, 60000, 512, "f32"),      # zeros beside both passes and the sums
    (70001, 500, 520, "bf16"),       # every row occurs, two slices, frequent numbers
    (4097, 100, 2000, "bf16"),       # the fewest tokens of the tiled sort
    (4096, 5000, 48, "f32"),         # the most of the small one
])
def test_large_calls(n, V, d, out):
    g = torch.Generator(device=DEV)
    g.manual_seed(n + V)
    law = torch.cumsum(torch.arange(1, V + 1, device=DEV, dtype=torch.float64) ** -1.1, 0)
    ids = torch.searchsorted(law, torch.rand(n, generator=g, device=DEV, dtype=torch.float64) * law[-1])
    ids = torch.where(torch.rand(n, generator=g, device=DEV) < 0.05, -1, ids)
    G = torch.randn((n, d), generator=g, device=DEV).to(torch.bfloat16)
    dE = blank(V, d, out)
    run(ids, G, dE, 0.5)
    gpu_check(ids, V, G, dE, 0.5)
    again = blank(V, d, out)
    run(ids.int(), G, again, 0.5)
    assert torch.equal(dE, again)


def test_more_rows_than_one_launch_looks_up():
    """40 million table rows: the workgroups that write zeros take several runs of rows each."""
    V, d = 40_000_000, 3
    ids = on([0, 5, V - 1, 12_345_678, 5])
    for n in (5, 5000):
        more = torch.cat([ids, torch.full((n - 5,), -1, dtype=ids.dtype, device=DEV)])
        dE = torch.full((V, d), 9.0, device=DEV)
        run(more, torch.ones((n, d), device=DEV), dE, dirty=False)
        assert float(dE.sum()) == 15.0
        assert torch.equal(dE[ids], torch.tensor([1.0, 2, 1, 1, 2], device=DEV)[:, None].expand(5, d))


def test_another_stream():
    rng = np.random.default_rng(9)
    ids, G = on(rng.integers(0, 900, 6000)), rows(rng, 6000, 72, "f32")[0]
    want, dE = blank(900, 72, "f32"), blank(900, 72, "f32")
    run(ids, G, want)
    ws = torch.empty(T.toc_embed_grad_workspace_size(6000, 900, 72), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    T.toc_embed_grad(ids, G, dE, ws, stream=side)
    side.synchronize()
    assert torch.equal(dE, want)
