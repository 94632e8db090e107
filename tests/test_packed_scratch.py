"""The scratch of the packed attention's backward: at most the 512 MiB that the header names, and
what its parts take. No GPU needed."""
import os
import random

import pytest

from paper_2510_00207_amd import _lib as L

MIB = 1 << 20


def ws_bytes(T, nseq, heads, kv, D, causal=True):
    return L.flowmoe_packed_attention_ws_bytes(L.make_shape(T, heads * D, 8, 1, 1, 0),
                                               L.make_packed_shape(nseq, heads, kv, D, causal))


def expected(T, nseq, heads, kv, D):
    """Sums of K and V, 32 x D floats each, of every 32-row tile and key head, a unit."""
    if T == 0 or nseq > 4096 or T <= (48 if heads // kv <= 2 else 24) * nseq:
        return 0
    rows = (T // 32 + nseq + 1) * 32 * kv
    most = -(-(256 * MIB // (8 * D)) // rows)
    units = 1 if (T + 31) // 32 * (heads // kv) <= 16 else min(most, 32)
    return units * rows * 8 * D if units > 1 else 0


@pytest.mark.parametrize("T,nseq,heads,kv,D,mb", [
    (16384, 12, 32, 8, 128, 275), (2031, 1, 16, 2, 128, 136), (32000, 1, 32, 8, 128, 525),
    (40000, 1, 32, 8, 128, 0), (300, 26, 4, 2, 64, 0),
])
def test_sizes(flowmoe_lib, T, nseq, heads, kv, D, mb):
    n = ws_bytes(T, nseq, heads, kv, D)
    assert n == expected(T, nseq, heads, kv, D) and n // 10 ** 6 == mb


def test_bound(flowmoe_lib):
    rng, most = random.Random(1), 0
    for _ in range(20000):
        kv, D = rng.choice([1, 2, 3, 4, 8, 16, 40, 64]), rng.choice([64, 128])
        heads, T = kv * rng.choice([1, 2, 3, 4, 8]), int(2 ** rng.uniform(0, 18))
        nseq = rng.choice([0, 1, rng.randint(0, max(1, T // 20))])
        n = ws_bytes(T, nseq, heads, kv, D)
        assert n == expected(T, nseq, heads, kv, D)
        most = max(most, n)
    assert 500 * MIB < most <= 512 * MIB


def test_header_names_the_bound():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    h = " ".join(open(os.path.join(root, "include", "flowmoe.h")).read().split())
    i = h.index("size_t flowmoe_packed_attention_ws_bytes")
    assert "at most 512 MiB" in h[h.rindex("/*", 0, i):i]
