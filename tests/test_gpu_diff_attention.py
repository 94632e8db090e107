"""Differential attention, forward and backward, against the fp64 reference, element
by element.

Tolerances count roundings, half a step of bf16 being 2^-8 of the value. Forward:
probabilities (relative to sum P_i |V|) and the output; lse and everything in fp32
stays below 2^-13 of these sums (scores are sums of at most 64 products in fp32,
|q k| summed below 64: 64 x 64 x 2^-24 = 2^-12 / sqrt(d) = 2^-15 on an exponent).
Backward, from the forward's own attn, attn2 and lse as it reads them: dS or
P_1 - lambda P_2 rounded for their product, and the output; relative to the sums of
absolute values with every difference taken as a sum."""
import numpy as np
import pytest
import torch

import oracle
from gpu_helpers import dev, host, need_gpu
from paper_2510_00207_amd import _lib as L

pytestmark = pytest.mark.gpu
H8, F = 2.0 ** -8, 2.0 ** -13


def make(nseq, seq, heads, kv, hd, seed, std=1.0):
    g = torch.Generator(device=dev()).manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=dev())
    T, M = nseq * seq, heads * hd
    qkv = (r(T, M + 2 * kv * hd) * std).bfloat16()
    return qkv, 0.2 + 0.6 * torch.rand(heads, generator=g, device=dev()), r(T, M).bfloat16()


class Call:
    """One forward and backward, outputs filled with what must be overwritten."""

    def __init__(self, nseq, seq, heads, kv, hd, causal, qkv, lam, d_attn, lens=None):
        T, M = nseq * seq, heads * hd
        d = dev()
        self.shape = L.make_shape(T, M, 8, 1, 1, 0, L.BF16)
        self.diff = L.make_diff_shape(seq, heads, kv, hd, causal)
        self.qkv, self.lam, self.d_attn = qkv, lam, d_attn
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=d)
        nan = lambda *s, dt=torch.bfloat16: torch.full(s, float("nan"), dtype=dt, device=d)
        self.attn, self.attn2, self.d_qkv = nan(T, M), nan(T, M), nan(*qkv.shape)
        self.lse, self.delta = (nan(2, heads, T, dt=torch.float32) for _ in range(2))
        self.d_lambda = torch.full((heads,), float("nan"), device=d)
        self.ws_bytes = L.flowmoe_diff_attention_ws_bytes(self.shape, self.diff)
        self.ws = torch.empty(max(1, self.ws_bytes), dtype=torch.uint8, device=d)

    def fwd(self, stream=None):
        L.flowmoe_diff_attention_fwd(self.shape, self.diff, self.qkv, self.lam, self.lens, self.attn,
                                     self.attn2, self.lse, stream=stream)

    def bwd(self, accumulate=False, stream=None):
        L.flowmoe_diff_attention_bwd(self.shape, self.diff, self.qkv, self.lam, self.lens, self.attn,
                                     self.attn2, self.lse, self.d_attn, self.d_qkv, self.delta,
                                     self.d_lambda, accumulate, self.ws, self.ws_bytes,
                                     stream=stream)

    NAMES = ("attn", "attn2", "lse", "d_qkv", "delta", "d_lambda")

    def outputs(self):
        torch.cuda.synchronize()
        return {n: getattr(self, n).clone() for n in self.NAMES}


def close(got, ref, tol, what):
    err = np.abs(host(got) - ref) - tol
    assert not np.isnan(err).any() and (err <= 0).all(), (
        what, float(np.nanmax(err)), np.unravel_index(np.nanargmax(err), err.shape))


def check(c, args):
    o = c.outputs()
    q, lam, do = host(c.qkv), host(c.lam), host(c.d_attn)
    lens = None if c.lens is None else c.lens.tolist()
    attn, attn2, lse, size = oracle.diff_attention(q, lam, *args, lens=lens)
    al = np.repeat(np.abs(lam), args[3])
    close(o["attn"], attn, (H8 + F) * (size[0] + al * size[1]) * 1.01 + 1.01 * H8 * np.abs(attn), "attn")
    close(o["attn2"], attn2, (H8 + F) * size[1] * 1.01 + 1.01 * H8 * np.abs(attn2), "attn2")
    close(o["lse"], lse, F * np.ones_like(lse), "lse")
    a, a2 = host(o["attn"]), host(o["attn2"])
    d_qkv, delta, d_lam, size = oracle.diff_attention_bwd(q, lam, a, a2, do, *args, lens=lens)
    close(o["d_qkv"], d_qkv, (H8 + F) * size * 1.01 + 1.01 * H8 * np.abs(d_qkv), "d_qkv")
    # fp32 sums of at most 128 products; over the tokens, a thread's T / 1024 and 26 more
    heads, D = args[1], args[3]
    dot = lambda x, y: np.abs(x * y).reshape(-1, heads, D).sum(2).T
    abs2 = dot(do, a2)
    big = np.stack([dot(do, a) + np.abs(lam)[:, None] * abs2, abs2])
    close(o["delta"], delta, 140 * 2.0 ** -24 * big, "delta")
    close(o["d_lambda"], d_lam, (170 + do.shape[0] / 1024) * 2.0 ** -24 * abs2.sum(1) + 1e-30, "d_lambda")


CASES = [
    # (sequences, seq_len, heads, kv_heads, head_dim, causal, lens)
    (3, 1, 2, 2, 64, True, None),
    (3, 1, 4, 1, 128, False, [1, 0, 1]),
    (2, 128, 2, 2, 64, False, None),
    (2, 200, 4, 2, 64, True, [200, 131]),
    (1, 256, 2, 2, 128, True, None),
    (2, 333, 3, 1, 128, False, [333, 64]),
    (1, 1000, 2, 1, 128, True, [999]),
    (5, 97, 3, 3, 64, False, [97, 0, 1, 96, 65]),
    (4, 300, 6, 3, 128, True, [0, 129, 300, 128]),
    (2, 520, 24, 8, 64, True, None),
    # lengths outside 0 .. seq_len are cut
    (3, 70, 2, 1, 64, True, [-5, 1000, 70]),
    # blocks of the large launches, and of the backward's units: many heads, few key heads,
    # long sequences (few steps of a unit, a short last one, units past a valid length)
    (9, 1030, 16, 4, 128, True, [1030, 1, 0, 897, 1024, 129, 1029, 500, 64]),
    (8, 1030, 16, 16, 64, False, [1030, 1000, 96, 897, 0, 31, 1029, 500]),
    (1, 2100, 8, 1, 128, True, [2090]),
    (1, 2100, 2, 1, 64, True, None),
    (2, 700, 12, 4, 64, False, [700, 450]),
    (2, 700, 12, 2, 128, False, None),
    (3, 600, 3, 3, 128, True, [600, 2, 333]),
    # dQ cut into units too, in blocks of 32 and of 64 queries, also past a valid length
    (2, 773, 2, 1, 64, False, [773, 300]),
    (1, 1500, 3, 3, 128, False, None),
    (1, 3000, 1, 1, 64, True, [1800]),
    (1, 2048, 8, 8, 128, True, [2000]),
    (1, 1100, 14, 2, 64, False, None),
    (2, 1100, 7, 7, 64, False, [40, 900]),
    (1, 2100, 12, 4, 64, True, None),
    (1, 4200, 1, 1, 128, True, [4100]),
    (1, 3500, 2, 1, 64, False, [3500]),
    # several sequences to a tile, the last tile not full, rows between that are not valid
    *[(n, s, 4, 2, d, c, [(7 * i) % (s + 2) - 1 for i in range(n)] if l else None)
      for n, s in ((1, 1), (32, 1), (70, 1), (33, 2), (21, 3), (13, 5), (4, 10), (5, 11), (3, 16), (5, 17))
      for d, c, l in ((64, True, False), (64, False, True), (128, True, True))],
    (300, 1, 40, 1, 64, False, None),
    (9, 7, 40, 1, 128, True, [7, 0, 3, 7, 7, 1, 0, 0, 5]),
    # sequences of two tiles and of one
    (90, 37, 6, 3, 128, True, None),
    (80, 64, 8, 4, 64, False, [n % 65 for n in range(80)]),
    (300, 20, 3, 3, 64, True, None),
    (200, 32, 4, 2, 128, False, [n % 33 for n in range(200)]),
    # around the tiles: one, two and three of 64 or 32 rows, a row short, whole, a row over
    *[(2, n, 1, 1, d, c, None) for n in (31, 32, 33, 63, 64, 65, 129) for d in (64, 128)
      for c in (False, True)],
    # the valid length around the tiles
    *[(1, 160, 2, 1, d, c, [n]) for n in (1, 31, 33, 64, 65, 127, 129) for d in (64, 128)
      for c in (False, True)],
]


@pytest.mark.parametrize("nseq,seq,heads,kv,hd,causal,lens", CASES)
def test_diff_attention(nseq, seq, heads, kv, hd, causal, lens):
    need_gpu()
    print(f"[diff] {nseq} x {seq}, {heads}/{kv} heads of {hd}, causal={causal}, lens={lens}",
          flush=True)
    c = Call(nseq, seq, heads, kv, hd, causal, *make(nseq, seq, heads, kv, hd, seq + hd), lens)
    c.fwd()
    c.bwd()
    check(c, (seq, heads, kv, hd, causal))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_padding_may_hold_anything(hd, causal):
    """NaN and infinities past the lengths change nothing; outputs there are zeros."""
    need_gpu()
    nseq, seq, heads, kv, lens = 4, 150, 4, 2, [150, 0, 33, 128]
    qkv, lam, d_attn = make(nseq, seq, heads, kv, hd, 5)
    a = Call(nseq, seq, heads, kv, hd, causal, qkv, lam, d_attn, lens)
    a.fwd()
    a.bwd()
    pad = torch.cat([torch.arange(seq) >= n for n in lens]).to(dev())
    q2, g2 = qkv.clone(), d_attn.clone()
    q2[pad], g2[pad] = float("nan"), float("inf")
    b = Call(nseq, seq, heads, kv, hd, causal, q2, lam, g2, lens)
    b.fwd()
    b.bwd()
    x, y = a.outputs(), b.outputs()
    for n in Call.NAMES:
        assert torch.equal(x[n], y[n]), n
    for n in ("attn", "attn2", "d_qkv"):
        assert not bool(y[n][pad].any()), n
    for n in ("lse", "delta"):
        assert not bool(y[n][:, :, pad].any()), n


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("seq", [1, 3, 10, 16])
def test_short_sequences_stay_apart(seq, hd, causal):
    """NaN and infinities of a sequence, or past its length, reach no other one."""
    need_gpu()
    nseq, heads, kv = 40, 2, 1
    lens = [seq - n % 2 for n in range(nseq)]
    qkv, lam, d_attn = make(nseq, seq, heads, kv, hd, 6)
    a = Call(nseq, seq, heads, kv, hd, causal, qkv, lam, d_attn, lens)
    a.fwd()
    a.bwd()
    bad = torch.zeros(nseq, dtype=torch.bool, device=dev())
    bad[[0, 5, 6, 38]] = True
    bad = bad.repeat_interleave(seq)
    pad = torch.cat([torch.arange(seq) >= n for n in lens]).to(dev())
    q2, g2 = qkv.clone(), d_attn.clone()
    q2[bad, ::3], g2[bad, 1::3] = float("inf"), float("nan")
    q2[pad], g2[pad] = float("nan"), float("inf")
    b = Call(nseq, seq, heads, kv, hd, causal, q2, lam, g2, lens)
    b.fwd()
    b.bwd()
    x, y = a.outputs(), b.outputs()
    for n in ("attn", "attn2", "d_qkv"):
        assert torch.equal(x[n][~bad], y[n][~bad]), n
        assert not bool(y[n][pad].any()), n
    for n in ("lse", "delta"):
        assert torch.equal(x[n][:, :, ~bad], y[n][:, :, ~bad]), n


@pytest.mark.parametrize("hd", [64, 128])
def test_large_scores(hd):
    """Scores of hundreds: one key takes the row, no exponent overflows."""
    need_gpu()
    args = (100, 2, 1, hd, True)
    c = Call(2, *args, *make(2, 100, 2, 1, hd, 9, std=8.0))
    c.fwd()
    c.bwd()
    o = c.outputs()
    q, lam = host(c.qkv), host(c.lam)
    attn, attn2, lse, size = oracle.diff_attention(q, lam, *args)
    # fp32 scores: 64 products of up to 500, 2^-24 each, on an exponent
    rel = 64 * 64 * 64 * 2.0 ** -24
    al = np.repeat(np.abs(lam), hd)
    close(o["attn"], attn, (H8 + 2 * rel) * (size[0] + al * size[1]) * 1.01 + 1.01 * H8 * np.abs(attn), "attn")
    close(o["lse"], lse, rel * np.ones_like(lse), "lse")
    assert bool(torch.isfinite(o["d_qkv"]).all()) and bool(torch.isfinite(o["d_lambda"]).all())


@pytest.mark.parametrize("nseq,seq,heads,kv,hd,causal", [
    (2, 130, 4, 1, 64, True), (1, 200, 4, 4, 128, False), (40, 32, 4, 2, 128, True),
    (9, 400, 8, 4, 128, True), (1, 700, 4, 2, 64, False), (1, 2048, 8, 2, 128, True)])
def test_lambda_of_any_sign(nseq, seq, heads, kv, hd, causal):
    """Zero, negative and large lambda, also among the heads that share a key head."""
    need_gpu()
    qkv, lam, d_attn = make(nseq, seq, heads, kv, hd, 7)
    lam[:4] = torch.tensor([0.0, -0.7, 3.0, -1e-3], device=dev())
    c = Call(nseq, seq, heads, kv, hd, causal, qkv, lam, d_attn)
    c.fwd()
    c.bwd()
    check(c, (seq, heads, kv, hd, causal))


def test_forward_alone():
    """Without attn2 and lse (no backward follows): the same attn."""
    need_gpu()
    qkv, lam, d_attn = make(2, 200, 4, 2, 64, 3)
    c = Call(2, 200, 4, 2, 64, True, qkv, lam, d_attn, [200, 77])
    c.fwd()
    o = torch.empty_like(c.attn)
    L.flowmoe_diff_attention_fwd(c.shape, c.diff, qkv, lam, c.lens, o, None, None)
    torch.cuda.synchronize()
    assert torch.equal(o, c.attn)


def test_d_lambda_accumulates_and_results_repeat():
    need_gpu()
    c = Call(2, 260, 4, 2, 128, True, *make(2, 260, 4, 2, 128, 4), [260, 100])
    c.fwd()
    c.bwd()
    first = c.outputs()
    for n in ("attn", "attn2", "lse", "d_qkv", "delta"):
        getattr(c, n).fill_(7.0)
    c.fwd()
    c.bwd(accumulate=True)
    again = c.outputs()
    for n in ("attn", "attn2", "lse", "d_qkv", "delta"):
        assert torch.equal(first[n], again[n]), n
    assert torch.equal(again["d_lambda"], first["d_lambda"] + first["d_lambda"])


def test_no_tokens():
    """No sequence of any length: nothing but dlambda's sum of nothing."""
    need_gpu()
    s = L.make_shape(0, 256, 8, 1, 1, 0, L.BF16)
    for seq, hd in ((1, 64), (4096, 64), (4096, 128)):
        m = L.make_diff_shape(seq, 256 // hd, 1, hd, True)
        assert L.flowmoe_diff_attention_ws_bytes(s, m) == 0
        L.flowmoe_diff_attention_fwd(s, m, *[None] * 6)
        dl = torch.full((256 // hd,), 3.0, device=dev())
        L.flowmoe_diff_attention_bwd(s, m, *[None] * 9, dl, True)
        assert bool((dl == 3.0).all())
        L.flowmoe_diff_attention_bwd(s, m, *[None] * 9, dl, False)
        assert not bool(dl.any())


def test_two_streams_at_once():
    need_gpu()
    cs = [Call(2, 300, 4, 2, 64, c, *make(2, 300, 4, 2, 64, 10 + c), [300, 211]) for c in (0, 1)]
    for c in cs:
        c.fwd()
        c.bwd()
    want = [c.outputs() for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    for c in cs:
        for n in Call.NAMES:
            getattr(c, n).fill_(float("nan"))
    torch.cuda.synchronize()
    for c, s in zip(cs, streams):
        c.fwd(stream=s)
    for c, s in zip(cs, streams):
        c.bwd(stream=s)
    for c, w in zip(cs, want):
        o = c.outputs()
        for n in Call.NAMES:
            assert torch.equal(o[n], w[n]), n


def test_captured_and_replayed():
    """A captured forward and backward, replayed on new inputs between eager calls."""
    need_gpu()
    args = (2, 220, 4, 2, 128, True)
    c = Call(*args, *make(2, 220, 4, 2, 128, 20), [220, 90])
    e = Call(*args, *make(2, 220, 4, 2, 128, 20), [220, 90])
    s = torch.cuda.Stream()
    c.fwd(stream=s)
    c.bwd(stream=s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.fwd()
        c.bwd()
    for k in range(3):
        qkv, lam, d_attn = make(2, 220, 4, 2, 128, 30 + k)
        lens = torch.tensor([220 - 60 * k, 17 * k], dtype=torch.int32, device=dev())
        for x in (c, e):
            x.qkv.copy_(qkv)
            x.lam.copy_(lam)
            x.d_attn.copy_(d_attn)
            x.lens.copy_(lens)
        e.fwd()
        e.bwd()
        g.replay()
        a, b = e.outputs(), c.outputs()
        for n in Call.NAMES:
            assert torch.equal(a[n], b[n]), (k, n)


def test_past_32_bit_offsets():
    """The last sequence of a batch whose qkv has more than 2^32 bytes, and more than 2^31
    elements."""
    need_gpu()
    nseq, seq, heads, kv, hd = 900, 300, 40, 20, 128
    T, M, W = nseq * seq, heads * hd, (heads + 2 * kv) * hd
    assert T * W > 1 << 31
    last, lam, d_attn = make(1, seq, heads, kv, hd, 40)
    d = dev()
    qkv = torch.zeros(T, W, dtype=torch.bfloat16, device=d)
    qkv[-seq:] = last
    do = torch.zeros(T, M, dtype=torch.bfloat16, device=d)
    do[-seq:] = d_attn
    all_ = Call(nseq, seq, heads, kv, hd, True, qkv, lam, do)
    all_.fwd()
    all_.bwd()
    torch.cuda.synchronize()
    assert not bool(all_.d_qkv[:-seq].any())
    # the last sequence's rows as a call's of their own (dlambda: the others add zeros)
    one = Call(1, seq, heads, kv, hd, True, last, lam, d_attn)
    for n in ("attn", "attn2", "d_qkv"):
        getattr(one, n).copy_(getattr(all_, n)[-seq:])
    for n in ("lse", "delta"):
        getattr(one, n).copy_(getattr(all_, n)[:, :, -seq:])
    one.d_lambda.copy_(all_.d_lambda)
    check(one, (seq, heads, kv, hd, True))
