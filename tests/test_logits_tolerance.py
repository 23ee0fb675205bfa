"""What the tolerances for rows of logits count is at least what each shape of workgroup does (CPU).

A lane adds its share of a row's columns one after the other, lanes join by pairs (4 joins of 16 lanes, 6 of
64, then one for every doubling of the waves and of the parts), and each batch of chunks, each join of
waves and parts and the lanes' first common number is a move of three roundings.  logits_cases.steps()
counts 4 (d / 64 + 64) up to 6,144 columns and 4 (d / 256 + 64) from there on, as if 64 or 256 lanes had the row.
Sixteen lanes add d / 16, four times as many, but join fewer: 4 (d / 16 + 4) is below it up to 1,280
columns, and 16 lanes have rows of 1,136 at most."""

import math

import pytest

import logits_cases

# lanes, chunks of a lane in a batch, the most chunks of a row (None: any), as the kernels are launched
SCORE = [(16, 8, 142), (64, 4, 768), (256, 4, 2048), (512, 6, None), (1024, 6, None)]
GRAD = [(16, 8, 142), (64, 2, 190), (64, 8, 574), (256, 2, 766), (256, 8, 2302), (512, 6, 3582), (1024, 6, None),
        (512, 20, 10750), (1024, 12, 13310), (1024, 16, 17406)]
LONGEST = 300007          # of the tests that use these tolerances


@pytest.mark.parametrize("columns", [4, 8])
@pytest.mark.parametrize("lanes,per,most", SCORE + GRAD)
def test_steps(lanes, per, most, columns):
    for d in list(range(1, 3000)) + list(range(3000, LONGEST, 997)) + [LONGEST]:
        chunks = math.ceil(d / columns) + 1                 # a skewed row has one more
        if most is not None and chunks > most + 1:
            break
        rounds = math.ceil(chunks / lanes)
        joins = 4 if lanes == 16 else 6 + math.ceil(math.log2(max(1, lanes // 64)))
        moves = math.ceil(rounds / (per + 1)) + (1 if lanes <= 64 else 2)
        assert min(d, columns * rounds) + joins + 3 * moves <= logits_cases.steps(d), d


def test_steps_of_parts():
    """512 lanes to each of up to 64 parts, which a wave puts together."""
    for d in range(32768, LONGEST, 997):
        rounds = math.ceil((d / 4 + 1) / 512)               # (one part would have them all)
        assert 4 * rounds + 9 + 6 + 3 * (math.ceil(rounds / 7) + 3) <= logits_cases.steps(d), d
