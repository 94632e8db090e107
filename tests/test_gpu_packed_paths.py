"""Attention over packed sequences on every path that the sizes choose: against the fp64
definition with the tolerances of test_gpu_packed_attention.py, by the launches that a trace
names. The backward of short sequences (T <= 24 nseq, 48 nseq with groups of up to two heads) is
one launch; else there are delta's, that of dQ, dK and dV, and a join where tiles may be cut."""
import pytest
import torch

import packed_ref as R
from gpu_helpers import dev
from paper_2510_00207_amd import _lib as L
from paper_2510_00207_amd.hiprt import EventArray
from test_gpu_packed_attention import HALF, Case, within

pytestmark = pytest.mark.gpu
NAN = float("nan")
OUT = ("attn", "lse", "d_qkv", "delta")


def launches(call):
    ev = EventArray(8)
    L.flowmoe_trace_start64(ev.ev, ev.kinds, ev.pairs, (1 << 64) - 1)
    call()
    n = L.flowmoe_trace_stop()
    torch.cuda.synchronize()
    names = [L.K_NAMES[k] for k in ev.kinds[:n]]
    ev.close()
    return names


SHORT = ["attn_bwd_dkdv"]
BLOCKS = ["attn_bwd_dq", "attn_bwd_dkdv"]
JOINED = BLOCKS + ["packed_join"]


# a sequence of three tiles, empty ones, whole tiles and parts of one; T <= 24 nseq
MIXED = [70, 5, 0, 1, 33, 12, 2, 0, 32, 7]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv", [(3, 1), (6, 2), (4, 1), (8, 2), (8, 1), (16, 2), (5, 1), (2, 1), (2, 2)])
def test_short_backward_of_groups(heads, kv, causal, D):
    """A wave each for up to four of a group's heads: groups of 3 leave a wave without heads,
    of 5 and 8 give some two."""
    c = Case(MIXED, heads, kv, D, causal, 20)
    assert c.T <= 24 * len(c.lens)
    c.fwd()
    c.check_fwd()
    assert launches(c.bwd) == SHORT
    c.check_bwd()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads,kv,causal", [(6, 2, True), (8, 2, False), (2, 1, True)])
def test_short_backward_of_many_tiles(heads, kv, causal, D):
    """More than 512 tiles of the key heads: one wave a tile for a group's heads in turn."""
    lens = (MIXED * 60)[:600 // kv]
    c = Case(lens, heads, kv, D, causal, 9)
    assert (c.T // 32 + len(lens) + 1) * kv > 512 and c.T <= 24 * len(lens)
    c.fwd()
    c.check_fwd()
    assert launches(c.bwd) == SHORT
    c.check_bwd()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [[1100] + [0] * 50, [0] * 30 + [900] + [5] * 40, [300, 300] + [0] * 126])
def test_long_among_empty_and_tiny(lens, D):
    """A list of a fixed length that one or two long sequences leave nearly empty."""
    for heads, kv, causal in ((8, 2, True), (3, 1, False), (2, 2, True)):
        c = Case(lens, heads, kv, D, causal, 11)
        assert c.T <= 24 * len(lens)
        c.fwd()
        c.check_fwd()
        assert launches(c.bwd) == SHORT
        c.check_bwd()


@pytest.mark.parametrize("lens,heads,kv,D,causal", [
    ([8200], 16, 16, 128, True), ([4000] + [200] * 21, 32, 16, 128, False),
    ([4000] + [150] * 28, 32, 32, 64, True),
])
def test_join_of_two_units(lens, heads, kv, D, causal):
    """So many rows that a tile is cut in two at most."""
    c = Case(lens, heads, kv, D, causal)
    rows32 = c.T // 32 + len(lens) + 1
    assert c.n == 2 * rows32 * kv * 64 * D * 4
    c.fwd()
    c.check_fwd()
    assert launches(c.bwd) == JOINED
    c.check_bwd()
