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


# (lens, heads, kv, D, causal): waves of short sequences; blocks of uncut tiles; blocks of two
# groups of waves forward, and cut tiles; one group and cut tiles
PATHS = [([20, 3, 0, 41, 9], 8, 2, 128, True), ([20, 3, 0, 41, 9], 6, 2, 64, False),
         ([100, 140], 2, 2, 64, True), ([2100], 4, 2, 128, True), ([1200, 300], 4, 1, 64, False),
         ([700, 20, 300], 4, 2, 64, True), ([700, 20, 300], 8, 2, 128, False)]


@pytest.mark.parametrize("lens,heads,kv,D,causal", PATHS)
def test_repeats_on_another_stream(lens, heads, kv, D, causal):
    """The same bits from buffers that held none of them, scratch included."""
    c = Case(lens, heads, kv, D, causal, 11)
    c.fwd()
    c.bwd()
    want = [getattr(c, n).clone() for n in OUT]
    for n in OUT:
        getattr(c, n).fill_(NAN)
    c.ws.fill_(255)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.fwd(s)
    c.bwd(s)
    s.synchronize()
    # (delta: intermediate, but every row of it is written)
    for n, w in zip(OUT, want):
        assert torch.isfinite(w).all() and torch.equal(getattr(c, n), w), n


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_gradient_of_equal_lengths(causal, D):
    """Sequences of one length and heads of their own: flowmoe_attention_bwd's gradient, each
    within its tolerance of the definition."""
    c = Case([256] * 4, 4, 4, D, causal, poison=False)
    c.fwd()
    c.bwd()
    c.check_bwd()
    d_qkv, delta = torch.full_like(c.d_qkv, NAN), torch.full_like(c.delta, NAN)
    L.flowmoe_attention_bwd(c.shape, L.make_mha_shape(256, 4, D, causal), c.qkv, c.attn, c.lse, c.d_attn,
                            d_qkv, delta)
    d, rnd, mag = R.attention_bwd(c.qkv, c.lens, 4, 4, D, causal, c.attn, c.lse, c.d_attn)
    tol = HALF * rnd + 2.0 ** -10 * mag + HALF * d.abs()
    within(d_qkv, d, tol)
    within(d_qkv, c.d_qkv.double(), 2 * tol)


@pytest.mark.parametrize("lens,heads,kv,D,causal", PATHS)
def test_starts_out_of_order_on_every_path(lens, heads, kv, D, causal):
    """Starts that are no list of starts: every buffer's surroundings stay as they are, the
    scratch's too."""
    c = Case(lens, heads, kv, D, causal, poison=False)
    T, n, guard = c.T, len(lens), {}
    for name in OUT + ("ws",):
        t = getattr(c, name)
        fill = 7 if name == "ws" else 7.0
        guard[name] = torch.full((t.numel() + 4096,), fill, dtype=t.dtype, device=dev())
        setattr(c, name, guard[name][2048:2048 + t.numel()].view(t.shape))
    up = lambda *s: (list(s) * (n + 1))[:n + 1]
    for s in (up(T, 0), up(5, -3, 1 << 30, T), up(0, T, T // 3), up(-1), up(T - 1, T // 2, 1),
              [T - i * (T // (n + 1)) for i in range(n + 1)]):
        c.starts = torch.tensor(s, dtype=torch.int32, device=dev())
        c.fwd()
        c.bwd()
        torch.cuda.synchronize()
        for name, g in guard.items():
            assert (g[:2048] == 7).all() and (g[-2048:] == 7).all(), (name, s)


def test_one_document_of_100003_tokens():
    """The last rows of the forward and of dQ, the first keys' gradients. A sum over n rows in 32 bits
    is off by n 2^-24 of its terms' magnitudes beside the other tolerances."""
    n, D, rows = 100003, 128, 96
    c = Case([n], 2, 1, D, True, 5)
    assert launches(c.fwd) == ["attn_fwd"] and launches(c.bwd) == JOINED
    x, s24, rs = c.qkv[:n].double(), n * 2.0 ** -24, D ** -0.5
    k, v = x[:, 2 * D:3 * D], x[:, 3 * D:]
    late = torch.arange(n - rows, n, device=dev())
    hidden = torch.arange(n, device=dev())[None] > late[:, None]
    dk, dv, rk, rv, mk, mv = (torch.zeros(rows, D, dtype=torch.float64, device=dev()) for _ in range(6))
    for h in range(2):
        q, o, do = (t[:, h * D:h * D + D] for t in (x, c.attn[:n].double(), c.d_attn[:n].double()))
        s = (q[late] @ k.T * rs).masked_fill(hidden, -float("inf"))
        p, lse = torch.softmax(s, 1), torch.logsumexp(s, 1)
        within(c.attn[late, h * D:h * D + D], p @ v,
               (HALF + 2.0 ** -12 + s24) * (p @ v.abs()) + HALF * (p @ v).abs())
        smax = float((q[late].abs() @ k.abs().T).max()) * rs
        within(c.lse[h, late], lse, D * 2.0 ** -24 * smax + 2.0 ** -20 + s24 + 2.0 ** -22 * lse.abs())
        delta, dmag = (do * o).sum(1), (do * o).abs().sum(1)
        p = torch.exp(s - c.lse[h, late].double()[:, None])
        ds = p * (do[late] @ v.T - delta[late, None])
        mag = p * (do[late].abs() @ v.abs().T + dmag[late, None])
        dq = ds @ k * rs
        within(c.d_qkv[late, h * D:h * D + D], dq, HALF * (ds.abs() @ k.abs() * rs) +
               (2.0 ** -10 + s24) * (mag @ k.abs() * rs) + HALF * dq.abs())
        # the first keys, seen by every query from their own on
        s = q @ k[:rows].T * rs
        s = s.masked_fill(torch.arange(rows, device=dev())[None] > torch.arange(n, device=dev())[:, None],
                          -float("inf"))
        p = torch.exp(s - c.lse[h, :n].double()[:, None])
        ds = p * (do @ v[:rows].T - delta[:, None])
        mag = p * (do.abs() @ v[:rows].abs().T + dmag[:, None])
        dk += ds.T @ q * rs
        rk += ds.abs().T @ q.abs() * rs
        mk += mag.T @ q.abs() * rs
        dv += p.T @ do
        rv += p.T @ do.abs()
        mv += p.T @ do.abs()
    for got, d, r, m in ((c.d_qkv[:rows, 2 * D:3 * D], dk, rk, mk), (c.d_qkv[:rows, 3 * D:], dv, rv, mv)):
        within(got, d, HALF * r + (2.0 ** -10 + 2 * s24) * m + HALF * d.abs())
    for t in (c.attn, c.d_qkv):
        assert not t[n:].any()


@pytest.mark.parametrize("size,path", [(100, BLOCKS), (5, SHORT)])
def test_more_sequences_than_units_are_made_for(size, path):
    """4101 sequences: a block's search takes three steps, no tile is cut."""
    lens = [size] * 4100 + [700]
    c = Case(lens, 2, 1, 64, True, 40)
    c.fwd()
    assert c.n == 0 and launches(c.bwd) == path
    for lo, hi, part in ((0, 2 * size, [size] * 2), (64 * size, 65 * size, [size]),
                         (c.live - 700 - size, c.live, [size, 700])):
        a = (part, 2, 1, 64, True)
        ref, lse, mag, smax = R.attention(c.qkv[lo:hi], *a)
        within(c.attn[lo:hi], ref, (HALF + 2.0 ** -12) * mag + HALF * ref.abs())
        within(c.lse[:, lo:hi], lse, 64 * 2.0 ** -24 * smax + 2.0 ** -20 + 2.0 ** -22 * lse.abs())
        d, rnd, mag = R.attention_bwd(c.qkv[lo:hi], *a, c.attn[lo:hi], c.lse[:, lo:hi], c.d_attn[lo:hi])
        within(c.d_qkv[lo:hi], d, HALF * rnd + 2.0 ** -10 * mag + HALF * d.abs())
    for t in (c.attn, c.d_qkv):
        assert not t[c.live:].any()
