"""The block's attention with rotary positions, differential attention and head norm
(flowmoe_diff_mha_fwd/_bwd): its steps bit for bit the single calls', its products
against fp64, element by element. A product's sum is rounded once to bf16 (2^-8 of the
value); its fp32 accumulation stays below 2^-12 of the sum of absolute products (at most
1024 of them, 2^-24 each, and as many again for the weight gradients' splits)."""
import numpy as np
import pytest
import torch

import oracle
from gpu_helpers import dev, host, need_gpu
from paper_2510_00207_amd import _lib as L

pytestmark = pytest.mark.gpu
H8, F = 2.0 ** -8, 2.0 ** -12
EPS, SCALE = 1e-5, 0.25


class Block:
    def __init__(self, nseq, seq, heads, kv, hd, causal, seed, lens=None, rot=None, layout="half"):
        T, M, W, d = nseq * seq, heads * hd, (heads + 2 * kv) * hd, dev()
        self.T, self.M, self.W, self.args = T, M, W, (seq, heads, kv, hd, causal)
        self.shape = L.make_shape(T, M, 8, 1, 1, 0, L.BF16)
        self.diff = L.make_diff_shape(seq, heads, kv, hd, causal)
        self.norm = L.make_norm_shape(heads, hd, EPS, SCALE)
        self.rope_kw = dict(heads=2 * (heads + kv), head_dim=hd // 2, rot=rot or hd // 2, layout=layout)
        self.rope = L.make_rope_shape(2 * (heads + kv), hd // 2, rot or hd // 2, seq, layout=layout)
        self.t = {}
        self.fill(seed)
        i32 = torch.int32
        self.t["lens"] = None if lens is None else torch.tensor(lens, dtype=i32, device=d)
        self.t["positions"] = (torch.arange(T, device=d) * 7 % 5000).to(i32)
        nan = lambda *s, dt=torch.bfloat16: torch.full(s, float("nan"), dtype=dt, device=d)
        f = torch.float32
        self.t.update(qkv=nan(T, W), attn=nan(T, M), attn2=nan(T, M), lse=nan(2, heads, T, dt=f),
                      normed=nan(T, M), out=nan(T, M), d_attn=nan(T, M), d_qkv=nan(T, W),
                      delta=nan(2, heads, T, dt=f), d_in=nan(T, M), dw_qkv=nan(M, W, dt=f),
                      dw_o=nan(M, M, dt=f), d_lambda=nan(heads, dt=f), dgain=nan(hd, dt=f))
        n = L.flowmoe_diff_mha_ws_bytes(self.shape, self.diff, self.norm)
        self.t["ws"] = torch.empty(max(1, n), dtype=torch.uint8, device=d)
        self.bufs = L.diff_mha_bufs(ws_bytes=n, **self.t)

    def fill(self, seed):
        g = torch.Generator(device=dev()).manual_seed(seed)
        r = lambda *s, std=1.0: (torch.randn(*s, generator=g, device=dev()) * std).bfloat16()
        T, M, W, (_, heads, _, hd, _) = self.T, self.M, self.W, self.args
        new = dict(inp=r(T, M), w_qkv=r(M, W, std=0.05), w_o=r(M, M, std=0.05), d_out=r(T, M),
                   lam=0.2 + 0.6 * torch.rand(heads, generator=g, device=dev()),
                   gain=1 + 0.2 * torch.randn(hd, generator=g, device=dev()))
        for k, v in new.items():
            if k in self.t:
                self.t[k].copy_(v)
            else:
                self.t[k] = v

    def fwd(self, rope=True, stream=None):
        L.flowmoe_diff_mha_fwd(self.shape, self.diff, self.rope if rope else None, self.norm,
                               self.bufs, stream=stream)

    def bwd(self, accumulate=False, stream=None):
        L.flowmoe_diff_mha_bwd(self.shape, self.diff, self.rope, self.norm, self.bufs, accumulate,
                               stream=stream)

    OUT = ("qkv", "attn", "attn2", "lse", "normed", "out", "d_attn", "d_qkv", "delta", "d_in", "dw_qkv",
           "dw_o", "d_lambda", "dgain")

    def outputs(self):
        torch.cuda.synchronize()
        return {n: self.t[n].clone() for n in self.OUT}


def close(got, ref, tol, what):
    err = np.abs(host(got) - ref) - tol
    assert not np.isnan(err).any() and (err <= 0).all(), (what, float(np.nanmax(err)))


@pytest.mark.parametrize("nseq,seq,heads,kv,hd,causal,lens,rot,layout", [
    (2, 100, 4, 2, 64, True, [100, 37], None, "half"),
    (3, 70, 3, 3, 128, False, None, 20, "pairs"),
    (1, 513, 8, 2, 128, True, [400], 26, "half"),
    (40, 30, 4, 4, 64, True, None, None, "pairs"),
])
def test_steps_and_products(nseq, seq, heads, kv, hd, causal, lens, rot, layout):
    need_gpu()
    b = Block(nseq, seq, heads, kv, hd, causal, 3, lens, rot, layout)
    t, T, M, W = b.t, b.T, b.M, b.W
    b.fwd(rope=False)
    raw = b.outputs()["qkv"]  # not turned
    x, wq = host(t["inp"]), host(t["w_qkv"])
    ref = x @ wq
    close(raw, ref, 1.01 * H8 * np.abs(ref) + F * (np.abs(x) @ np.abs(wq)), "qkv")
    b.fwd()
    b.bwd()
    o = b.outputs()
    # the forward's steps
    sw = L.make_shape(T, W, 8, 1, 1, 0, L.BF16)
    L.flowmoe_rope_fwd(sw, b.rope, raw, t["positions"], raw)
    assert torch.equal(raw, o["qkv"])
    z = {n: torch.empty_like(o[n]) for n in b.OUT}
    L.flowmoe_diff_attention_fwd(b.shape, b.diff, raw, t["lam"], t["lens"], z["attn"], z["attn2"], z["lse"])
    L.flowmoe_head_norm_fwd(b.shape, b.norm, z["attn"], t["gain"], z["normed"])
    for n in ("attn", "attn2", "lse", "normed"):
        assert torch.equal(z[n], o[n]), n
    n64, wo = host(o["normed"]), host(t["w_o"])
    ref = n64 @ wo
    close(o["out"], ref, 1.01 * H8 * np.abs(ref) + F * (np.abs(n64) @ np.abs(wo)), "out")
    # the backward's
    do, a, gain = host(t["d_out"]), host(o["attn"]), host(t["gain"])
    g = do @ wo.T  # rounded to bf16, then through the norm
    eps, scale = float(np.float32(EPS)), float(np.float32(SCALE))
    dx, dg = oracle.head_norm_bwd(a, g, heads, gain, eps, scale)
    v, e = np.abs(a).reshape(T, heads, hd), (H8 * np.abs(g) + F * (np.abs(do) @ np.abs(wo.T)))
    e = e.reshape(T, heads, hd) * 1.01
    r = 1 / np.sqrt((v * v).mean(2, keepdims=True) + eps)
    u = scale * np.abs(gain)
    through = lambda q: r * (u * q + v * r * r * (u * q * v).mean(2, keepdims=True))
    tol = through(e + 80 * 2.0 ** -24 * np.abs(g).reshape(T, heads, hd))
    close(o["d_attn"], dx, tol.reshape(T, M) + 1.01 * H8 * np.abs(dx), "d_attn")
    close(o["dgain"], dg, 1.1 * scale * (e * v * r).sum((0, 1)), "dgain")
    n = L.flowmoe_diff_attention_ws_bytes(b.shape, b.diff)
    L.flowmoe_diff_attention_bwd(b.shape, b.diff, raw, t["lam"], t["lens"], z["attn"], z["attn2"],
                                 z["lse"], o["d_attn"], z["d_qkv"], z["delta"], z["d_lambda"], False,
                                 torch.empty(max(1, n), dtype=torch.uint8, device=dev()), n)
    L.flowmoe_rope_bwd(sw, b.rope, z["d_qkv"], t["positions"], z["d_qkv"])
    torch.cuda.synchronize()
    for n in ("d_qkv", "delta", "d_lambda"):
        assert torch.equal(z[n], o[n]), n
    dq = host(o["d_qkv"])
    for got, A, B, half in (("d_in", dq, wq.T, H8), ("dw_o", n64.T, do, 0.0), ("dw_qkv", x.T, dq, 0.0)):
        ref = A @ B
        close(o[got], ref, 1.01 * half * np.abs(ref) + F * (np.abs(A) @ np.abs(B)), got)
    # the same again, added
    b.bwd(accumulate=True)
    o2 = b.outputs()
    for n in ("d_lambda", "dgain"):
        assert torch.equal(o2[n], o[n] + o[n]), n
    # (split sums are added to what is there one by one)
    for n, A, B in (("dw_o", n64.T, do), ("dw_qkv", x.T, dq)):
        close(o2[n], 2 * (A @ B), 2 * F * (np.abs(A) @ np.abs(B)), n)
    for n in ("d_attn", "d_qkv", "delta", "d_in"):
        assert torch.equal(o2[n], o[n]), n


def test_padded_rows_add_nothing():
    """Other finite rows past the lengths: zeros in out and d_in, the same gradients."""
    need_gpu()
    lens = [700, 0, 33]
    a, b = (Block(3, 700, 4, 2, 64, True, 31, lens) for _ in range(2))
    pad = torch.cat([torch.arange(700) >= n for n in lens]).to(dev())
    b.t["inp"][pad] *= -3
    b.t["d_out"][pad] = 100.0
    for x in (a, b):
        x.fwd()
        x.bwd()
    x, y = a.outputs(), b.outputs()
    for n in ("out", "d_in", "d_qkv", "attn"):
        assert not bool(y[n][pad].any()), n
        assert torch.equal(x[n], y[n]), n
    for n in ("dw_qkv", "dw_o", "d_lambda", "dgain"):
        assert torch.equal(x[n], y[n]), n


def test_no_tokens():
    need_gpu()
    s, d, n = (L.make_shape(0, 256, 8, 1, 1, 0, L.BF16), L.make_diff_shape(64, 4, 2, 64, True),
               L.make_norm_shape(4, 64))
    z = dict(dw_qkv=torch.ones(256, 512, device=dev()), dw_o=torch.ones(256, 256, device=dev()),
             d_lambda=torch.ones(4, device=dev()), dgain=torch.ones(64, device=dev()))
    b = L.diff_mha_bufs(**z)
    L.flowmoe_diff_mha_fwd(s, d, None, n, b)
    L.flowmoe_diff_mha_bwd(s, d, None, n, b, True)
    assert all(bool((v == 1).all()) for v in z.values())
    L.flowmoe_diff_mha_bwd(s, d, None, n, b, False)
    assert not any(bool(v.any()) for v in z.values())


def test_captured_and_replayed():
    """A captured step, replayed on new inputs between eager steps of the same block."""
    need_gpu()
    args = (2, 150, 4, 2, 64, True, 11, [150, 60])
    c, e = Block(*args), Block(*args)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.fwd()
        c.bwd()
    for k in range(3):
        for x in (c, e):
            x.fill(50 + k)
            x.t["lens"].copy_(torch.tensor([150 - 70 * k, 60 + 40 * k], dtype=torch.int32))
        e.fwd()
        e.bwd()
        g.replay()
        a, b = e.outputs(), c.outputs()
        for n in Block.OUT:
            assert torch.equal(a[n], b[n]), (k, n)


def test_gradients_against_differences():
    """Of a loss in fp64 along one direction of each learned tensor: the fp64 chain's own
    gradient by central differences, within the bf16 block's roundings. Of a sum of n terms
    with independent errors of a half step or less each of the chain's eight roundings adds
    at most 2^-8 of the root of the sum of squares; 8 x 2^-8 bounds their total where the
    terms do not cancel, so the comparison is relative to the sum of absolute terms."""
    need_gpu()
    b = Block(2, 40, 2, 1, 64, True, 21, [40, 25])
    b.fwd()
    b.bwd()
    o = b.outputs()
    h = {k: host(b.t[k]) for k in ("inp", "w_qkv", "w_o", "lam", "gain", "d_out")}
    pos = b.t["positions"].tolist()

    def loss(**kw):
        p = dict(h, **kw)
        q = oracle.rope(p["inp"] @ p["w_qkv"], pos, **b.rope_kw)
        seq, heads, kv, hd, causal = b.args
        attn = oracle.diff_attention(q, p["lam"], seq, heads, kv, hd, causal, lens=[40, 25])[0]
        return (oracle.head_norm(attn, heads, p["gain"], EPS, SCALE) @ p["w_o"] * p["d_out"]).sum()

    rng = np.random.default_rng(5)
    for name, grad in (("inp", "d_in"), ("w_qkv", "dw_qkv"), ("w_o", "dw_o"), ("lam", "d_lambda"),
                       ("gain", "dgain")):
        got = host(o[grad])
        v = rng.standard_normal(got.shape)
        num = (loss(**{name: h[name] + 1e-5 * v}) - loss(**{name: h[name] - 1e-5 * v})) / 2e-5
        assert abs((got * v).sum() - num) <= 8 * H8 * np.abs(got * v).sum(), name
