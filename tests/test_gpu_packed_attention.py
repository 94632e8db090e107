"""Attention over packed sequences against the fp64 definition, element by element.

Tolerances. A probability is rounded to bf16 (half a step, 2^-8 relative), so attn is off by
at most 2^-8 sum P |V|, and its own rounding 2^-8 |attn|; products and sums in 32 bits and the
exponentials stay below 2^-12 of sum P |V| (scores of |q||k| <= 30 summed over 128 columns
in 32 bits are off by 128 * 2^-24 * 30 = 2.3e-4 at most, and so is a probability). lse is off
by that score error and 2^-22 of its size. Of the gradients dS is rounded, P for dV (2^-8 of
the sums of |dS| |K|, |dS| |Q|, P |dA|), the result (2^-8), and what is summed in 32 bits is
2^-10 of its terms' magnitudes: the score error of the recomputed P again, in every term, and
the sums over rows and the group's heads."""
import pytest
import torch

import packed_ref as R
from gpu_helpers import dev, need_gpu
from paper_2510_00207_amd import _lib as L

pytestmark = pytest.mark.gpu
HALF = R.HALF[torch.bfloat16]


def normal(g, *s):
    return torch.randn(*s, generator=g, device=dev()).bfloat16()


class Case:
    def __init__(self, lens, heads, kv, D, causal, tail=0, seed=0, poison=True):
        need_gpu()
        g = torch.Generator(device=dev()).manual_seed(seed)
        self.lens, self.heads, self.kv, self.D, self.causal = lens, heads, kv, D, causal
        self.live = sum(lens)
        self.T = T = self.live + tail
        self.M, self.W = heads * D, (heads + 2 * kv) * D
        self.starts = torch.tensor(R.starts_of(lens), dtype=torch.int32, device=dev())
        self.qkv, self.d_attn = normal(g, T, self.W), normal(g, T, self.M)
        if poison:  # rows of no sequence
            self.qkv[self.live:] = float("nan")
            self.d_attn[self.live:] = float("inf")
        self.shape = L.make_shape(T, self.M, 8, 1, 1, 0)
        self.packed = L.make_packed_shape(len(lens), heads, kv, D, causal)
        z = lambda *s, dtype=torch.bfloat16: torch.full(s, float("nan"), dtype=dtype, device=dev())
        f32 = torch.float32
        self.attn, self.lse = z(T, self.M), z(heads, T, dtype=f32)
        self.d_qkv, self.delta = z(T, self.W), z(heads, T, dtype=f32)
        self.n = L.flowmoe_packed_attention_ws_bytes(self.shape, self.packed)
        self.ws = torch.full((max(1, self.n),), 255, dtype=torch.uint8, device=dev())

    def fwd(self, stream=None):
        L.flowmoe_packed_attention_fwd(self.shape, self.packed, self.qkv, self.starts, self.attn,
                                       self.lse, stream=stream)

    def bwd(self, stream=None):
        L.flowmoe_packed_attention_bwd(self.shape, self.packed, self.qkv, self.starts, self.attn,
                                       self.lse, self.d_attn, self.d_qkv, self.delta, self.ws,
                                       self.n, stream=stream)

    def check_fwd(self):
        c = (self.lens, self.heads, self.kv, self.D, self.causal)
        ref, lse, mag, smax = R.attention(self.qkv, *c)
        within(self.attn, ref, (HALF + 2.0 ** -12) * mag + HALF * ref.abs())
        within(self.lse, lse, self.D * 2.0 ** -24 * smax + 2.0 ** -20 + 2.0 ** -22 * lse.abs())

    def check_bwd(self):
        c = (self.lens, self.heads, self.kv, self.D, self.causal)
        d, rnd, mag = R.attention_bwd(self.qkv, *c, self.attn, self.lse, self.d_attn)
        within(self.d_qkv, d, HALF * rnd + 2.0 ** -10 * mag + HALF * d.abs())
        assert not self.delta[:, self.live:].any()

    def check(self):
        self.fwd()
        self.check_fwd()
        self.bwd()
        self.check_bwd()


def within(got, ref, tol):
    got = got.double()
    assert torch.isfinite(got).all()
    bad = (got - ref).abs() - tol
    assert float(bad.max()) <= 0, f"{float((got - ref).abs().max()):.3e} off, {float(bad.max()):.3e} too far"


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,heads,kv,tail", [
    ([1], 1, 1, 0), ([1, 1, 1], 2, 1, 1), ([0, 5, 0, 0, 33, 0], 4, 2, 7), ([31, 32, 33], 3, 3, 0),
    ([63, 64, 65, 1], 4, 1, 130), ([127, 128, 129], 2, 2, 0), ([300], 8, 8, 0), ([700, 20], 6, 2, 90),
    ([257, 1, 1, 511, 64], 8, 2, 0), ([0, 0, 0], 2, 1, 40), ([], 2, 2, 40),
])
def test_shapes(lens, heads, kv, tail, causal, D):
    Case(lens, heads, kv, D, causal, tail).check()


@pytest.mark.parametrize("n,lens", [(100, [3, 0, 17]), (1500, [1, 2]), (5000, [1])])
def test_many_sequences(n, lens):
    """More sequences than one search of 64 finds."""
    Case((lens * n)[:n], 2, 1, 64, True, 3).check()


def test_long_sequences():
    c = Case([2500, 1700], 4, 1, 128, True)
    c.check()
    Case([3100], 2, 2, 64, False).check()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,heads,kv", [
    ([2031], 8, 1), ([1500, 3, 600], 2, 2), ([30] * 70 + [1100, 31, 700], 4, 1), ([1281], 1, 1),
])
def test_long_tiles_are_cut(lens, heads, kv, causal, D):
    """Few long tiles: cut into units, whose sums are joined; with up to 63 sequences and more."""
    c = Case(lens, heads, kv, D, causal, 9)
    assert c.n > 0
    c.check()
    want = c.d_qkv.clone()
    c.ws.fill_(255)
    c.bwd()
    assert torch.equal(c.d_qkv, want)


@pytest.mark.parametrize("n", [62, 63, 64, 65])
def test_number_of_sequences(n):
    """About where the search for a block's sequence changes, in any order of lengths."""
    g = torch.Generator().manual_seed(n)
    Case(torch.randint(0, 200, (n,), generator=g).tolist(), 4, 2, 64, True, 30).check()


@pytest.mark.parametrize("heads,kv", [(16, 2), (32, 8), (24, 8), (12, 4)])
def test_heads(heads, kv):
    """Grids with heads on XCDs of their own and without."""
    Case([200, 90], heads, kv, 64, True, 5).check()


@pytest.mark.parametrize("lens", [[40, 30, 70, 5], [20, 10, 30, 5], [130, 60, 300, 100],
                                  [900, 700, 600, 40]])
@pytest.mark.parametrize("causal", [True, False])
def test_sequences_do_not_meet(lens, causal):
    """A sequence of infinities and NaN changes no other's rows, bit for bit."""
    lo, hi = lens[0], lens[0] + lens[1]
    a = Case(lens, 4, 1, 64, causal, poison=False)
    a.fwd()
    a.bwd()
    want = [t.clone() for t in (a.attn, a.lse, a.d_qkv)]
    b = Case(lens, 4, 1, 64, causal, poison=False)
    b.qkv[lo:hi:2] = float("nan")
    b.qkv[lo + 1:hi:2] = float("inf")
    b.d_attn[lo:hi] = float("nan")
    b.fwd()
    b.bwd()
    for t, w in zip((b.attn, b.lse.T, b.d_qkv), (want[0], want[1].T, want[2])):
        assert torch.equal(t[:lo], w[:lo]) and torch.equal(t[hi:], w[hi:])


def test_rows_past_32_bit_offsets():
    """[Q | K | V] of more than 2^31 elements: the last sequences' rows."""
    n, T = 1500, 360000
    lens = [n] * (T // n - 1) + [n - 77]
    c = Case(lens, 32, 8, 128, True, 77, poison=False)
    assert c.qkv.numel() > 1 << 31
    c.fwd()
    c.bwd()
    lo, hi = c.live - lens[-1], c.live
    a = ([lens[-1]], 32, 8, 128, True)
    ref, lse, mag, smax = R.attention(c.qkv[lo:hi], *a)
    within(c.attn[lo:hi], ref, (HALF + 2.0 ** -12) * mag + HALF * ref.abs())
    within(c.lse[:, lo:hi], lse, 128 * 2.0 ** -24 * smax + 2.0 ** -20 + 2.0 ** -22 * lse.abs())
    d, rnd, mag = R.attention_bwd(c.qkv[lo:hi], *a, c.attn[lo:hi], c.lse[:, lo:hi], c.d_attn[lo:hi])
    within(c.d_qkv[lo:hi], d, HALF * rnd + 2.0 ** -10 * mag + HALF * d.abs())
    for t in (c.attn, c.d_qkv):
        assert not t[hi:].any()


def test_equal_lengths_match_the_attention():
    """Sequences of one length and heads of their own: flowmoe_attention's results."""
    c = Case([256] * 4, 4, 4, 64, True, poison=False)
    c.fwd()
    c.bwd()
    m = L.make_mha_shape(256, 4, 64, True)
    attn, lse = torch.empty_like(c.attn), torch.empty_like(c.lse)
    L.flowmoe_attention_fwd(c.shape, m, c.qkv, attn, lse)
    assert torch.equal(attn, c.attn) and torch.equal(lse, c.lse)


def test_offsets_out_of_order_stay_in_the_buffers():
    """Starts that are no list of starts: unspecified results, within the buffers."""
    c = Case([40, 30, 70, 5], 4, 2, 64, True, poison=False)
    guard = [torch.full((t.numel() + 4096,), 7.0, dtype=t.dtype, device=dev())
             for t in (c.attn, c.lse, c.d_qkv, c.delta)]
    for name, gd in zip(("attn", "lse", "d_qkv", "delta"), guard):
        t = getattr(c, name)
        setattr(c, name, gd[2048:2048 + t.numel()].view(t.shape))
    for s in ([5, -3, 1 << 30, 20, 145], [0, 145, 10, 145, 3], [145, 100, 60, 30, 0], [-1] * 5):
        c.starts = torch.tensor(s, dtype=torch.int32, device=dev())
        c.fwd()
        c.bwd()
        torch.cuda.synchronize()
        for gd in guard:
            assert (gd[:2048] == 7).all() and (gd[-2048:] == 7).all()


def test_deterministic_and_on_another_stream():
    c = Case([400, 13, 260], 8, 2, 128, True, 11)
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    want = [t.clone() for t in (c.attn, c.lse, c.d_qkv)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.fwd(s)
    c.bwd(s)
    s.synchronize()
    for t, w in zip((c.attn, c.lse, c.d_qkv), want):
        assert torch.equal(t, w)


def test_graph_follows_its_inputs():
    """A captured forward and backward, replayed with other rows and other lengths."""
    c = Case([100, 300, 57], 4, 2, 64, True, 60)
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.fwd()
        c.bwd()
    for i, lens in enumerate([[100, 300, 57], [1, 2, 500], [0, 517, 0], [100, 300, 57]]):
        other = Case(lens, 4, 2, 64, True, 517 - sum(lens), seed=i)
        for n in ("qkv", "starts", "d_attn"):
            getattr(c, n).copy_(getattr(other, n))
        c.lens, c.live = lens, sum(lens)
        graph.replay()
        torch.cuda.synchronize()
        c.check_fwd()
        c.check_bwd()
        other.fwd()
        other.bwd()
        assert torch.equal(other.attn, c.attn) and torch.equal(other.d_qkv, c.d_qkv)
