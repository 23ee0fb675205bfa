"""The embedding table's gradient on each way through it, against the 64-bit oracle: up to 128
tokens in one launch and the sorts above, each with dropout, 16-bit rows, several slices of
columns, strided rows and accumulation; and numbers that begin, end and fill up at the
boundaries of the spans and workgroups of the sums."""

import numpy as np
import pytest

import paper_1702_06943_amd as T
from oracle import rows as R
from rows_cases import DEV, LEAST, U, UNIT, blank, close, gaps_untouched, rows, torch
from test_gpu_embed_grad import check, on, run

pytestmark = pytest.mark.gpu
DROP = (0.25, 0x13579BDF02468ACE, 17)
KINDS = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")]


def check_accumulate(ids, V, d, kind, drop=None, out_kind=None, gap=0, shift=0, seed=0):
    """dE = E + scale * gradient in the rows that occur; the others, NaN, are left alone."""
    rng = np.random.default_rng(seed)
    ids = np.asarray(ids)
    out_kind = out_kind or kind
    occurs = np.isin(np.arange(V), ids)
    E, E64 = rows(rng, V, d, out_kind, gap=gap, shift=shift)
    absent = torch.from_numpy(~occurs).to(DEV)
    E[absent] = float("nan")
    G, G64 = rows(rng, len(ids), d, kind, gap=gap, shift=shift)
    scale = -0.5
    run(on(ids), G, E, scale, drop, accumulate=True)
    g, S, count = R.embed_grad(ids, G64, V, scale, drop)
    want = E64 + g
    tol = (count[:, None] + 6) * U * (S + np.abs(E64)) + UNIT[out_kind] * np.abs(want) + LEAST[out_kind]
    assert torch.isnan(E[absent]).all()
    close(E[~absent], want[occurs], tol[occurs], f"{len(ids)} ids of {V}, {d} columns, accumulated")


def some_ids(n, V, seed):
    """Frequent numbers, single ones, and numbers outside the table."""
    rng = np.random.default_rng(seed)
    ids = np.minimum(rng.zipf(1.4, n) - 1, V + 3)
    ids[rng.random(n) < 0.1] = -3
    ids[0] = V - 1
    return ids


@pytest.mark.parametrize("drop", [None, DROP], ids=["plain", "drop"])
@pytest.mark.parametrize("kind,out_kind", KINDS)
@pytest.mark.parametrize("n,d", [(1, 5), (1, 1024), (2, 1100), (7, 65), (8, 513), (9, 300), (63, 24), (64, 1024),
                                 (65, 333), (100, 1), (127, 520), (128, 1024), (128, 2100), (129, 520), (129, 24)])
def test_around_one_launch(n, d, kind, out_kind, drop):
    V = 60
    ids = some_ids(n, V, n + d)
    check(ids, V, d, kind, out_kind, drop=drop, bits=32, seed=d)
    check(ids, V, d, kind, out_kind, drop=drop, gap=5, shift=1, seed=d)
    check_accumulate(ids, V, d, kind, drop, out_kind, gap=3, shift=1, seed=d)


@pytest.mark.parametrize("n", [1, 2, 60, 127, 128])
@pytest.mark.parametrize("what", ["one", "outside", "distinct", "all but one"])
def test_extremes_of_one_launch(n, what):
    V = 300
    ids = {"one": np.full(n, 7), "outside": np.full(n, V), "distinct": np.random.default_rng(n).permutation(V)[:n],
           "all but one": np.where(np.arange(n) == n // 2, 250, 3)}[what]
    check(ids, V, 520, "bf16", "f32", drop=DROP, seed=n)
    if what != "outside":
        check_accumulate(ids, V, 520, "bf16", DROP, seed=n)


@pytest.mark.parametrize("kind,out_kind", KINDS)
@pytest.mark.parametrize("n,V,d", [(130, 50, 65), (4096, 700, 24), (4097, 700, 24), (9001, 3000, 40), (5000, 300, 520)])
def test_dropout_and_accumulate_above(n, V, d, kind, out_kind):
    ids = some_ids(n, V, n)
    check(ids, V, d, kind, out_kind, drop=DROP, seed=n)
    check_accumulate(ids, V, d, kind, DROP, out_kind, seed=n)


# (type, columns, entries of a workgroup): 512 threads in groups of 8 lanes, each with a span of
# 8 entries; in groups of 64, two slices of the columns; and in groups of 32
UNITS = [("f32", 8, 512), ("bf16", 1024, 64), ("bf16", 256, 128)]


@pytest.mark.parametrize("first", [0, 1, 7])
@pytest.mark.parametrize("kind,d,unit", UNITS)
def test_runs_against_workgroups(kind, d, unit, first):
    """Runs of one number that start and end on, one before and one after the boundaries of spans
    and workgroups, and fill one and several of them; all moved on by a first number's run."""
    span = 8
    counts = [unit - 1, 1, unit, unit + 1, 2 * unit - 1, 2 * unit, 1, span - 1, 1, span, span + 1, unit - 2 * span - 1,
              3 * unit, unit - 1, 2, unit - 1, span * 3, unit - 3 * span, 1]
    if first:
        counts.insert(0, first)
    ids = np.repeat(np.arange(len(counts)), counts)
    ids = np.random.default_rng(first).permutation(np.concatenate([ids, np.full(5, -1)]))
    V = len(counts) + 2
    check(ids, V, d, kind, "f32", seed=first)
    check_accumulate(ids, V, d, kind, DROP, seed=first)


@pytest.mark.parametrize("blocks", [63, 64, 65, 66, 130])
def test_one_number_over_many_workgroups(blocks):
    kind, d, unit = UNITS[1]
    for more in (-1, 0, 1):
        ids = np.concatenate([[0], np.full(blocks * unit + more, 1), [2]])
        check(ids, 3, d, kind, "f32", seed=blocks)
