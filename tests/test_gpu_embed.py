"""Embedding lookup and its gradient against the fp64 definition.

Tolerances: a looked-up row is one product in 32 bits and the output's rounding; of an f32
table the product's rounding alone. A row of the gradient of n tokens is a sum of n terms
in 32 bits (n 2^-24 of the sum of their magnitudes) and a product."""
import pytest
import torch

import packed_ref as R
from gpu_helpers import dev, need_gpu
from paper_2510_00207_amd import _lib as L

pytestmark = pytest.mark.gpu
E24 = 2.0 ** -24
TD = {"bf16": torch.bfloat16, "f32": torch.float32}


class Case:
    def __init__(self, T, M, vocab, dtype="bf16", scale=1.7, seed=0, ids=None):
        need_gpu()
        g = torch.Generator(device=dev()).manual_seed(seed)
        td = TD[dtype]
        self.T, self.M, self.vocab, self.scale, self.td = T, M, vocab, scale, td
        if ids is None:  # among them some of no row
            ids = torch.randint(-2, vocab + 2, (T,), generator=g, device=dev())
        self.ids = ids.to(device=dev(), dtype=torch.int32)
        self.table = torch.randn(vocab, M, generator=g, device=dev()).to(td)
        self.dy = torch.randn(T, M, generator=g, device=dev()).to(td)
        self.y = torch.full((T, M), float("nan"), dtype=td, device=dev())
        self.dtable = torch.full((vocab, M), float("nan"), device=dev())
        self.shape = L.make_shape(T, M, 8, 1, 1, 0, L.F32 if dtype == "f32" else L.BF16)
        self.embed = L.make_embed_shape(vocab, scale)
        self.n = L.flowmoe_embed_ws_bytes(self.shape, self.embed)
        self.ws = torch.full((max(1, self.n),), 255, dtype=torch.uint8, device=dev())

    def fwd(self, **kw):
        L.flowmoe_embed_fwd(self.shape, self.embed, self.ids, self.table, self.y, **kw)

    def bwd(self, accumulate=False, **kw):
        L.flowmoe_embed_bwd(self.shape, self.embed, self.ids, self.dy, self.dtable, accumulate,
                            self.ws, self.n, **kw)

    def check_fwd(self):
        ref = R.embed(self.ids, self.table, self.embed.scale)
        half = R.HALF[self.td] + (E24 if self.td == torch.bfloat16 else 0)
        within(self.y, ref, half * ref.abs())

    def check_bwd(self, base=None):
        ref, mag = R.embed_bwd(self.ids, self.dy, self.vocab, self.embed.scale)
        on = (self.ids >= 0) & (self.ids < self.vocab)
        n = torch.bincount(self.ids[on].long(), minlength=self.vocab)[:, None]
        if base is not None:
            ref, mag = ref + base.double(), mag + base.double().abs()
            assert torch.equal(self.dtable[n[:, 0] == 0], base[n[:, 0] == 0])
        within(self.dtable, ref, (n + 2) * E24 * mag)


def within(got, ref, tol):
    got = got.double()
    assert torch.isfinite(got).all()
    bad = (got - ref).abs() - tol
    assert bad.numel() == 0 or float(bad.max()) <= 0, (
        f"{float((got - ref).abs().max()):.3e} off, {float(bad.max()):.3e} too far")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,M,vocab", [
    (1, 8, 1), (1, 1024, 3), (2, 64, 7), (63, 72, 50), (64, 512, 5), (65, 520, 300), (200, 1032, 1),
    (255, 40, 2), (256, 40, 2), (257, 2056, 11), (1000, 264, 5003), (1023, 8, 70000), (4096, 128, 3),
    (4097, 128, 30), (5000, 96, 257), (10000, 64, 65536), (9999, 16, 65535),
])
def test_shapes(T, M, vocab, dtype):
    c = Case(T, M, vocab, dtype)
    c.fwd()
    c.check_fwd()
    c.bwd()
    c.check_bwd()
    base = torch.randn(vocab, M, device=dev())
    c.dtable.copy_(base)
    c.bwd(True)
    c.check_bwd(base)


@pytest.mark.parametrize("T", [128, 300, 4096, 20000])
def test_one_id(T):
    """Every token the same row, whole chunks of it and a rest; then all of no row."""
    for M, ids in [(64, torch.full((T,), 3)), (520, torch.full((T,), 0)),
                   (64, torch.full((T,), -1)), (64, torch.full((T,), 1 << 30))]:
        c = Case(T, M, 9, ids=ids)
        c.fwd()
        c.check_fwd()
        c.bwd()
        c.check_bwd()
        base = torch.randn(9, M, device=dev())
        c.dtable.copy_(base)
        c.bwd(True)
        c.check_bwd(base)


def test_runs_at_the_windows_edges():
    """Runs of one id that end at, before and behind the multiples of 64."""
    runs = [64, 64, 63, 1, 65, 127, 128, 129, 192, 2, 320, 7, 1, 1, 56, 64]
    ids = torch.cat([torch.full((n,), 2 * i) for i, n in enumerate(runs)])
    c = Case(len(ids), 72, 40, ids=ids[torch.randperm(len(ids), generator=torch.Generator().manual_seed(3))])
    c.bwd()
    c.check_bwd()
    base = torch.randn(40, 72, device=dev())
    c.dtable.copy_(base)
    c.bwd(True)
    c.check_bwd(base)


def test_many_tokens():
    """More items than 256 blocks of 1024 sort, four passes of digits."""
    g = torch.Generator(device=dev()).manual_seed(9)
    T, vocab = 300007, (1 << 24) + 5
    ids = torch.exp(torch.rand(T, generator=g, device=dev(), dtype=torch.float64) * 16.6).long()
    c = Case(T, 8, vocab, "f32", ids=ids)
    c.fwd()
    c.check_fwd()
    c.bwd()
    c.check_bwd()


def test_no_tokens():
    c = Case(0, 64, 30)
    c.fwd()
    c.bwd()
    assert float(c.dtable.abs().max()) == 0
    c.dtable.fill_(2.0)
    c.bwd(True)
    assert (c.dtable == 2).all()


def test_rows_of_no_id_may_hold_anything():
    c = Case(500, 64, 20)
    c.dy[(c.ids < 0) | (c.ids >= 20)] = float("nan")
    c.bwd()
    assert torch.isfinite(c.dtable).all()


def test_table_past_32_bit_offsets():
    need_gpu()
    V, M = 140000, 16384  # 2^31 elements and more
    table = torch.zeros(V, M, dtype=torch.bfloat16, device=dev())
    rows = torch.tensor([0, V - 1, 131072, 70000])
    for r in rows.tolist():
        table[r] = float(r % 251 + 1)
    y = torch.empty(4, M, dtype=torch.bfloat16, device=dev())
    s = L.make_shape(4, M, 8, 1, 1, 0)
    L.flowmoe_embed_fwd(s, L.make_embed_shape(V), rows.int().to(dev()), table, y)
    want = (rows % 251 + 1).to(dev()).bfloat16()[:, None].expand(-1, M)
    assert torch.equal(y, want)
    del table
    d = torch.full((V, M), 1.0, device=dev())
    e = L.make_embed_shape(V)
    n = L.flowmoe_embed_ws_bytes(s, e)
    L.flowmoe_embed_bwd(s, e, rows.int().to(dev()), y, d, True, torch.empty(n, dtype=torch.uint8, device=dev()), n)
    for r in range(4):
        assert (d[rows[r]] == 1 + want[r].float()).all()
    d[rows] = 1.0
    assert float(d.min()) == 1 and float(d.max()) == 1


def test_deterministic_graph_and_stream():
    c = Case(5000, 256, 3000)
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.fwd()
        c.bwd()
    for i in range(3):
        o = Case(5000, 256, 3000, seed=i)
        for n in ("ids", "table", "dy"):
            getattr(c, n).copy_(getattr(o, n))
        graph.replay()
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        o.fwd(stream=s)
        o.bwd(stream=s)
        s.synchronize()
        assert torch.equal(c.y, o.y) and torch.equal(c.dtable, o.dtable)
        c.check_bwd()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,M,vocab", [
    (8, 1032, 1), (9, 512, 1), (33, 4104, 2), (512, 520, 3), (512, 4104, 40000), (513, 1032, 2),
    (1024, 8, 1), (1024, 2056, 600), (1025, 2056, 600),
])
def test_few_tokens(T, M, vocab, dtype):
    """Either side of the sizes at which a wave, a block or a launch has enough tokens, with runs of
    a few, of dozens and of all tokens, and one id before and behind them all."""
    g = torch.Generator().manual_seed(T)
    ids = torch.randint(0, vocab, (T,), generator=g)
    ids[torch.rand(T, generator=g) < 0.1] = vocab // 2
    ids[torch.rand(T, generator=g) < 0.1] = -1
    ids[0] = ids[-1] = vocab - 1
    c = Case(T, M, vocab, dtype, ids=ids)
    c.bwd()
    c.check_bwd()
    first = c.dtable.clone()
    c.dtable.fill_(float("nan"))
    c.bwd()
    assert torch.equal(first, c.dtable)
    base = torch.randn(vocab, M, device=dev())
    c.dtable.copy_(base)
    c.bwd(True)
    c.check_bwd(base)


def test_many_rows_of_no_id_may_hold_anything():
    c = Case(5000, 64, 20)
    c.dy[(c.ids < 0) | (c.ids >= 20)] = float("nan")
    c.bwd()
    assert torch.isfinite(c.dtable).all()


def test_few_tokens_graph_and_stream():
    """As test_deterministic_graph_and_stream; such calls take no workspace."""
    c = Case(700, 264, 900)
    assert c.n == 0
    c.bwd()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.flowmoe_embed_bwd(c.shape, c.embed, c.ids, c.dy, c.dtable, False, None, 0)
    for i in range(3):
        o = Case(700, 264, 900, seed=i)
        c.ids.copy_(o.ids)
        c.dy.copy_(o.dy)
        graph.replay()
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        o.bwd(stream=s)
        s.synchronize()
        assert torch.equal(c.dtable, o.dtable)
        c.check_bwd()


@pytest.mark.parametrize("T,M,vocab", [
    (1025, 520, 3), (2047, 8, 200), (2049, 8, 255), (3000, 72, 70000), (8191, 8, 40), (8192, 512, 300),
    (8193, 512, 300), (8193, 504, 70000), (8192, 8, 1 << 17),
])
def test_ranked_and_sorted(T, M, vocab):
    """Either side of the sizes at which ids are ranked or sorted and rows are wide or narrow."""
    c = Case(T, M, vocab, "f32" if T % 2 else "bf16")
    c.bwd()
    c.check_bwd()
    first = c.dtable.clone()
    c.dtable.fill_(float("nan"))
    c.bwd()
    assert torch.equal(first, c.dtable)
    base = torch.randn(vocab, M, device=dev())
    c.dtable.copy_(base)
    c.bwd(True)
    c.check_bwd(base)
