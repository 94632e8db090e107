"""The operators together, as a pre-norm block over packed documents uses them: token ids,
embedding, norm, packed attention block with rotary positions, norm of the sum, the MoE
layer; and back. Every step is compared with the fp64 definition from the tensors the
framework itself handed it, so that its tolerance is that step's own: products of K terms in
bf16 are off by K 2^-24 of the sum of their magnitudes and half a step of the result."""
import pytest
import torch

import packed_ref as R
from gpu_helpers import dev, need_gpu
from paper_2510_00207_amd import _lib as L
from paper_2510_00207_amd.layer import MoELayer

pytestmark = pytest.mark.gpu
HALF = R.HALF[torch.bfloat16]
EPS, BASE = 1e-5, 10000.0


def within(got, ref, tol):
    got = got.double()
    assert torch.isfinite(got).all()
    bad = (got - ref).abs() - tol
    assert float(bad.max()) <= 0, f"{float((got - ref).abs().max()):.3e} off, {float(bad.max()):.3e} too far"


def product(got, a, b, base=0.0, half=HALF):
    """got = base + a b"""
    a, b = a.double(), b.double()
    ref = a @ b + base
    within(got, ref, half * ref.abs() + a.shape[1] * 2.0 ** -24 * (a.abs() @ b.abs()) + 1e-30)


def turn(x, pos, heads, D, sign):
    """Rotary positions of the first heads * D columns, pairs (i, i + D / 2)."""
    th = BASE ** (-2 * torch.arange(D // 2, device=x.device, dtype=torch.float64) / D)
    ang = sign * pos.double()[:, None] * th
    c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
    y = x.double().clone()
    v = y[:, :heads * D].view(-1, heads, D)
    a, b = v[..., :D // 2].clone(), v[..., D // 2:].clone()
    v[..., :D // 2], v[..., D // 2:] = a * c - b * s, a * s + b * c
    return y


class Block:
    def __init__(self, lens, tail, heads, kv, D, rope, seed=0):
        need_gpu()
        g = torch.Generator(device=dev()).manual_seed(seed)
        self.g, self.lens, self.heads, self.kv, self.D = g, lens, heads, kv, D
        self.live, self.T = sum(lens), sum(lens) + tail
        self.M, self.W = heads * D, (heads + 2 * kv) * D
        T, M, W = self.T, self.M, self.W
        self.shape = L.make_shape(T, M, 8, 1, 1, 0)
        self.packed = L.make_packed_shape(len(lens), heads, kv, D, True)
        self.rope = L.make_rope_shape(heads + kv, D, D, 1) if rope else None
        self.starts = torch.tensor(R.starts_of(lens), dtype=torch.int32, device=dev())
        self.pos = torch.cat([torch.arange(n) for n in lens] + [torch.zeros(tail)]).int().to(dev())
        n = lambda *s, std=1.0: (torch.randn(*s, generator=g, device=dev()) * std).bfloat16()
        z = lambda *s, dtype=torch.bfloat16: torch.full(s, float("nan"), dtype=dtype, device=dev())
        f = torch.float32
        self.inp, self.d_out = n(T, M), n(T, M)
        self.w_qkv, self.w_o = n(M, W, std=M ** -0.5), n(M, M, std=M ** -0.5)
        self.t = dict(qkv=z(T, W), attn=z(T, M), lse=z(heads, T, dtype=f), out=z(T, M),
                      d_attn=z(T, M), d_qkv=z(T, W), delta=z(heads, T, dtype=f), d_in=z(T, M),
                      dw_qkv=z(M, W, dtype=f), dw_o=z(M, M, dtype=f))
        nb = L.flowmoe_packed_mha_ws_bytes(self.shape, self.packed)
        self.ws = torch.full((max(nb, 1),), 255, dtype=torch.uint8, device=dev())
        self.bufs = L.packed_mha_bufs(inp=self.inp, w_qkv=self.w_qkv, w_o=self.w_o, positions=self.pos,
                                      starts=self.starts, d_out=self.d_out, ws=self.ws, ws_bytes=nb,
                                      **self.t)

    def fwd(self, stream=None):
        L.flowmoe_packed_mha_fwd(self.shape, self.packed, self.rope, self.bufs, stream=stream)

    def bwd(self, accumulate=False, stream=None):
        L.flowmoe_packed_mha_bwd(self.shape, self.packed, self.rope, self.bufs, accumulate,
                                 stream=stream)

    def check_fwd(self):
        t, H = self.t, self.heads + self.kv
        a, b = self.inp.double(), self.w_qkv.double()
        mag = self.M * 2.0 ** -24 * (a.abs() @ b.abs())
        qkv, off = a @ b, HALF * (a @ b).abs()
        if self.rope is not None:  # rounded before and after it is turned
            two = lambda x: torch.cat([
                (x[:, :H * self.D].view(-1, H, 2, self.D // 2).sum(2, keepdim=True)
                 .expand(-1, H, 2, self.D // 2).reshape(len(x), -1)), x[:, H * self.D:]], 1)
            qkv, off, mag = turn(qkv, self.pos, H, self.D, 1), two(off), two(mag)
            off = off + HALF * (qkv.abs() + off)
        within(t["qkv"], qkv, off + 2 * mag)
        c = (self.lens, self.heads, self.kv, self.D, True)
        ref, _, m, _ = R.attention(t["qkv"], *c)
        within(t["attn"], ref, (HALF + 2.0 ** -12) * m + HALF * ref.abs())
        product(t["out"], t["attn"], self.w_o)
        assert not t["out"][self.live:].any()

    def check_bwd(self, base=0.0):
        t, H = self.t, self.heads + self.kv
        product(t["d_attn"], self.d_out, self.w_o.T)
        c = (self.lens, self.heads, self.kv, self.D, True)
        d, rnd, mag = R.attention_bwd(t["qkv"], *c, t["attn"], t["lse"], t["d_attn"])
        off = HALF * rnd + 2.0 ** -10 * mag + HALF * d.abs()
        if self.rope is not None:
            w = self.D // 2
            two = lambda x: torch.cat([
                (x[:, :H * self.D].view(-1, H, 2, w).sum(2, keepdim=True).expand(-1, H, 2, w)
                 .reshape(len(x), -1)), x[:, H * self.D:]], 1)
            d, off = turn(d, self.pos, H, self.D, -1), two(off)
            off = off + HALF * (d.abs() + off)
        within(t["d_qkv"], d, off)
        product(t["d_in"], t["d_qkv"], self.w_qkv.T)
        product(t["dw_o"], t["attn"].T, self.d_out, base, 2.0 ** -23)
        product(t["dw_qkv"], self.inp.T, t["d_qkv"], base, 2.0 ** -23)
        assert not t["d_in"][self.live:].any()


@pytest.mark.parametrize("lens,tail,heads,kv,D,rope", [
    ([5, 0, 130, 1], 9, 4, 2, 64, True), ([300, 40], 0, 2, 1, 128, True), ([64] * 5, 3, 3, 3, 64, False),
    ([1], 0, 8, 2, 64, True), ([1200], 20, 4, 1, 64, True),
])
def test_block(lens, tail, heads, kv, D, rope):
    b = Block(lens, tail, heads, kv, D, rope)
    b.fwd()
    b.check_fwd()
    b.bwd()
    b.check_bwd()
    b.t["dw_qkv"].fill_(0.25)
    b.t["dw_o"].fill_(0.25)
    b.bwd(True)
    b.check_bwd(0.25)


def test_no_tokens():
    b = Block([0, 0], 0, 2, 1, 64, True)
    b.fwd()
    b.bwd()
    assert not b.t["dw_qkv"].any() and not b.t["dw_o"].any()


def test_block_graph():
    b = Block([150, 3, 90], 13, 4, 2, 64, True)
    b.fwd()
    b.bwd()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.fwd()
        b.bwd()
    for i in range(3):
        o = Block([150, 3, 90], 13, 4, 2, 64, True, seed=i)
        for n in ("inp", "d_out", "w_qkv", "w_o"):
            getattr(b, n).copy_(getattr(o, n))
        graph.replay()
        torch.cuda.synchronize()
        o.fwd()
        o.bwd()
        for n in ("out", "d_in", "dw_qkv", "dw_o"):
            assert torch.equal(b.t[n], o.t[n]), n


def test_documents_through_a_block_and_the_experts():
    """ids -> rows -> norm -> packed attention block -> norm of the sum -> MoE layer, and back to
    the embedding's gradient."""
    lens, tail, heads, kv, D, vocab = [40, 7, 81, 100], 28, 4, 2, 64, 500
    b = Block(lens, tail, heads, kv, D, True)
    T, M, g, d = b.T, b.M, b.g, dev()
    ids = torch.randint(0, vocab, (T,), generator=g, device=d, dtype=torch.int32)
    ids[b.live:] = -1
    table = torch.randn(vocab, M, generator=g, device=d).bfloat16()
    gains = [1 + 0.1 * torch.randn(M, generator=g, device=d) for _ in range(2)]
    bias = [0.1 * torch.randn(M, generator=g, device=d) for _ in range(2)]
    emb = L.make_embed_shape(vocab, 0.5)
    buf = lambda *s, dtype=torch.bfloat16: torch.full(s, float("nan"), dtype=dtype, device=d)
    x0, n1, h, dx0 = buf(T, M), b.inp, buf(T, M), buf(T, M)
    moe = MoELayer(T_total=T, M=M, H=64, E=4, k=2, f=2.0)
    for w in (moe.w_gate, moe.w1, moe.w2):
        w.copy_(torch.randn(w.shape, generator=g, device=d) * 0.05)
    n2 = moe.x
    L.flowmoe_embed_fwd(b.shape, emb, ids, table, x0)
    L.flowmoe_layer_norm_fwd(b.shape, EPS, x0, None, gains[0], bias[0], None, n1)
    b.fwd()
    L.flowmoe_layer_norm_fwd(b.shape, EPS, b.t["out"], x0, gains[1], bias[1], h, n2)
    moe.forward()
    # y = h + experts(norm(h)); its gradient dy
    dy = torch.randn(T, M, generator=g, device=d).bfloat16()
    moe.dy.copy_(dy)
    moe.backward()
    ws_n = L.flowmoe_layer_norm_ws_bytes(b.shape)
    ws = torch.empty(max(1, ws_n), dtype=torch.uint8, device=d)
    dg, db = [buf(M, dtype=torch.float32) for _ in range(2)], [buf(M, dtype=torch.float32) for _ in range(2)]
    dh = b.d_out
    L.flowmoe_layer_norm_bwd(b.shape, EPS, h, gains[1], moe.dx, dy, dh, dg[1], db[1], False, ws, ws_n)
    b.bwd()
    L.flowmoe_layer_norm_bwd(b.shape, EPS, x0, gains[0], b.t["d_in"], dh, dx0, dg[0], db[0], False, ws, ws_n)
    ne = L.flowmoe_embed_ws_bytes(b.shape, emb)
    dtable = buf(vocab, M, dtype=torch.float32)
    L.flowmoe_embed_bwd(b.shape, emb, ids, dx0, dtable, False,
                        torch.empty(ne, dtype=torch.uint8, device=d), ne)
    # each step from what it was given
    assert torch.equal(x0, (table.float()[ids.long().clamp(min=0)] * 0.5 * (ids >= 0)[:, None]).bfloat16())
    E24 = 2.0 ** -24
    off = lambda n, r, x, gn: ((M + 20) * E24 * (n.abs() + r * x.abs().mean(1, keepdim=True)) * gn.abs() +
                               4 * E24 * (x.abs() * r * gn.abs() + 2))
    y, x, n, r = R.layer_norm(x0, None, gains[0], bias[0], EPS)
    within(n1, y, HALF * y.abs() + off(n, r, x, gains[0].double()))
    b.check_fwd()
    y, x, n, r = R.layer_norm(b.t["out"], x0, gains[1], bias[1], EPS)
    within(n2, y, HALF * y.abs() + off(n, r, x, gains[1].double()))
    within(h, x, 2 * HALF * x.abs())
    b.check_bwd()
    for i, (xi, dyi, ds, got) in enumerate([(x0, b.t["d_in"], dh, dx0), (h, moe.dx, dy, dh)]):
        dx, rg, rb, mg, mb, mag = R.layer_norm_bwd(xi, gains[i], dyi, ds, EPS)
        _, x, n, r = R.layer_norm(xi, None, None, None, EPS)
        noff = (M + 20) * E24 * (1 + r * x.abs().mean(1, keepdim=True))
        within(got, dx, HALF * dx.abs() + (4 * noff + 8 * E24) * mag)
        within(dg[i], rg, (T + 20) * E24 * mg + (noff * (1 + n.abs()) * dyi.double().abs()).sum(0))
        within(db[i], rb, (T + 20) * E24 * mb)
    ref, mag = R.embed_bwd(ids, dx0, vocab, 0.5)
    within(dtable, ref, (T + 2) * E24 * mag)
