"""The workspace of orthogonalised updates is what the header says, for callers who plan for it."""
import os
import random
import re

import pytest

from paper_2609_40335_amd import build as B
from paper_2609_40335_amd import dpghost as D

TYPES = {"DP_F32": D.DP_F32, "DP_BF16": D.DP_BF16}


@pytest.fixture(scope="module")
def ws():
    if not os.path.exists(D.library_path()):
        B.build()
    L = D.lib()

    def f(shapes, dt):
        arr = (D.dp_matrix_t * len(shapes))(*[D.dp_matrix_t(1 << 30, c, 1 << 31, c, r, c, 1.0)
                                              for r, c in shapes])
        return L.dp_orthogonalize_workspace(arr, len(shapes), dt)
    return f


def _limits():
    """(m, n, type) of the largest matrices worked without a workspace, from the header."""
    with open(os.path.join(B.ROOT, "include", "dpghost.h")) as f:
        text = " ".join(line.strip().lstrip("*").strip() for line in f)
    part = text[text.index("small enough to be worked in LDS"):]
    part = part[:part.index(")")]
    found = []
    for sizes, types in re.findall(r"((?:\d+ x \d+(?:,| or| and)? ?)+)for (both|DP_F32|DP_BF16)", part):
        for m, n in re.findall(r"(\d+) x (\d+)", sizes):
            found += [(int(m), int(n), t) for t in (TYPES if types == "both" else [types])]
    return found


def test_limits_of_the_small_form(ws):
    limits = _limits()
    assert {t for _, _, t in limits} == set(TYPES) and len(limits) >= 3, limits
    for m, n, t in limits:
        for a, b in ((m, n), (n, m)):
            assert ws([(a, b)], TYPES[t]) == 0, (a, b, t)
        assert ws([(m, n + 1)], TYPES[t]) > 0 and ws([(n + 1, m)], TYPES[t]) > 0, (m, n, t)


def _planned(m, n, dt):
    """Bytes of a matrix as the header has them."""
    up = lambda x: -(-x // 128) * 128  # noqa: E731
    s, l = up(min(m, n)), up(max(m, n))
    return 8 * s * l + (4 if dt == D.DP_BF16 and min(m, n) > 64 else 8) * s * s


def test_bytes_of_the_large_form(ws):
    rng = random.Random(5)
    side = lambda: int(2 ** rng.uniform(0, 13))  # noqa: E731
    for k in range(300):
        shapes = [(side(), side()) for _ in range(rng.choice([1, 1, 2, 5, 48]))]
        shapes += [(400, 401)]      # not a small one
        for dt in TYPES.values():
            got = ws(shapes, dt)
            most = sum(sorted((_planned(m, n, dt) for m, n in shapes), reverse=True)[:48])
            assert got <= most + 48 * 1536 + (128 << 20), (shapes, dt)
            assert got >= _planned(400, 401, dt)
    assert 68_000_000 < ws([(16, 65536)], D.DP_BF16) < 69_000_000      # two planes, 16 padded to 128
