"""How LayerNorm's backward pass cuts an example's rows, seen through its workspace: the
partial sums of a range, 2 d floats written and read, beside the operands of its rows."""
import os
import random

import pytest

from paper_2609_40335_amd import build as B
from paper_2609_40335_amd import dpghost as D


@pytest.fixture(scope="module")
def ws():
    if not os.path.exists(D.library_path()):
        B.build()
    return D.lib().dp_layernorm_backward_workspace


def test_partial_sums_stay_a_fraction_of_the_operands(ws):
    rng = random.Random(1)
    for _ in range(3000):
        b, t, d = (int(2 ** rng.uniform(0, k)) for k in (12, 16, 15))
        ranges = max(1, ws(b, t, d) // (8 * d * b))         # what is rounded up is less than a range, or counts as some
        if 8 * d * b < 4096:
            continue
        least = 16 if d <= 2048 else 8
        assert ranges <= -(-t // least), (b, t, d, ranges)
        for es in (2, 4):
            share = 16 * d * ranges / (3 * es * t * d)
            limit = (1 / 6 if d <= 2048 else 1 / 3) * 2 / es
            # an example of few rows more than a range has is cut in two of half as many
            assert share <= limit * (1 + least / t) * 1.0001 or ranges == 1, (b, t, d, es, share)
