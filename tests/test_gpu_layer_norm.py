"""Layer norm against the fp64 definition, element by element.

Tolerances: with N = M + 20 32-bit operations in a row's longest sum at most (they are sums
of sums, so far fewer count), mean, variance and row sums are off by N 2^-24 of their terms'
magnitudes; an output is, besides its own rounding (half a step of its type), off by a few
2^-24 of n gain and bias and by the relative error of r. dgain and dbias sum over T rows: (T +
20) 2^-24 of the sum of magnitudes, and n's own error in each term."""
import pytest
import torch

import packed_ref as R
from gpu_helpers import dev, need_gpu
from paper_2510_00207_amd import _lib as L

pytestmark = pytest.mark.gpu
E24 = 2.0 ** -24
EPS = 1e-5
TD = {"bf16": torch.bfloat16, "f32": torch.float32}


class Case:
    def __init__(self, T, M, dtype="bf16", res=True, affine=True, seed=0, mean=0.3, std=2.0):
        need_gpu()
        g = torch.Generator(device=dev()).manual_seed(seed)
        self.T, self.M, self.td = T, M, TD[dtype]
        r = lambda *s: torch.randn(*s, generator=g, device=dev())
        self.x = (r(T, M) * std + mean).to(self.td)
        self.res = r(T, M).to(self.td) if res else None
        self.gain = 1 + 0.1 * r(M) if affine else None
        self.bias = 0.1 * r(M) if affine else None
        self.dy, self.d_sum = r(T, M).to(self.td), r(T, M).to(self.td) if res else None
        nan = lambda *s, dtype=self.td: torch.full(s, float("nan"), dtype=dtype, device=dev())
        self.sum, self.y, self.dx = nan(T, M) if res else None, nan(T, M), nan(T, M)
        self.dgain, self.dbias = (nan(M, dtype=torch.float32) for _ in range(2))
        self.shape = L.make_shape(T, M, 8, 1, 1, 0, L.F32 if dtype == "f32" else L.BF16)
        self.n = L.flowmoe_layer_norm_ws_bytes(self.shape)
        self.ws = torch.full((max(1, self.n),), 255, dtype=torch.uint8, device=dev())

    def fwd(self, **kw):
        L.flowmoe_layer_norm_fwd(self.shape, EPS, self.x, self.res, self.gain, self.bias, self.sum,
                                 self.y, **kw)

    def bwd(self, accumulate=False, **kw):
        L.flowmoe_layer_norm_bwd(self.shape, EPS, self.x, self.gain, self.dy, self.d_sum, self.dx,
                                 self.dgain, self.dbias, accumulate, self.ws, self.n, **kw)

    def check_fwd(self):
        y, h, n, r = R.layer_norm(self.x, self.res, self.gain, self.bias, EPS)
        g = 1 if self.gain is None else self.gain.double().abs()
        # r and the mean's share of n: N 2^-24 of the row's mean magnitude
        off = (self.M + 20) * E24 * (n.abs() + r * h.abs().mean(1, keepdim=True)) * g
        off = off + 4 * E24 * (y.abs() + h.abs() * r * g + 1)
        within(self.y, y, R.HALF[self.td] * y.abs() + off)
        if self.sum is not None:
            within(self.sum, h, 2 * R.HALF[self.td] * h.abs() + 1e-30)

    def check_bwd(self, base=0.0):
        dx, dg, db, mg, mb, mag = R.layer_norm_bwd(self.x, self.gain, self.dy, self.d_sum, EPS)
        _, h, n, r = R.layer_norm(self.x, None, None, None, EPS)
        noff = (self.M + 20) * E24 * (1 + r * h.abs().mean(1, keepdim=True))
        within(self.dx, dx, R.HALF[self.td] * dx.abs() + (4 * noff + 8 * E24) * mag)
        within(self.dgain, dg + base, (self.T + 20) * E24 * mg + (noff * (1 + n.abs()) * self.dy.double().abs()).sum(0) +
               4 * E24 * abs(base))
        within(self.dbias, db + base, (self.T + 20) * E24 * mb + 4 * E24 * abs(base))


def within(got, ref, tol):
    got = got.double()
    assert torch.isfinite(got).all()
    bad = (got - ref).abs() - tol
    assert float(bad.max()) <= 0, f"{float((got - ref).abs().max()):.3e} off, {float(bad.max()):.3e} too far"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,M,res,affine", [
    (1, 8, True, True), (1, 16384, True, True), (3, 24, False, True), (5, 504, True, False),
    (7, 512, False, False), (9, 520, True, True), (33, 1024, True, True), (2, 1032, False, True),
    (64, 2040, True, True), (10, 2056, True, True), (17, 4096, True, True), (5, 4104, True, False),
    (3, 8200, True, True), (1000, 64, True, True), (2500, 96, False, True), (600, 4096, True, True),
])
def test_shapes(T, M, res, affine, dtype):
    c = Case(T, M, dtype, res, affine)
    c.fwd()
    c.check_fwd()
    c.bwd()
    c.check_bwd()


def test_more_rows_than_blocks():
    c = Case(9001, 264)
    c.fwd()
    c.check_fwd()
    c.bwd()
    c.check_bwd()


def test_rows_past_32_bit_offsets():
    """More than 2^31 elements: the last rows, and the sums over all."""
    T, M = 530000, 4096
    c = Case(8, M, res=False)
    x = c.x.repeat(T // 8, 1)
    dy = c.dy.repeat(T // 8, 1)
    s = L.make_shape(T, M, 8, 1, 1, 0)
    y = torch.zeros_like(x)
    L.flowmoe_layer_norm_fwd(s, EPS, x, None, c.gain, c.bias, None, y)
    c.fwd()
    assert torch.equal(y[-8:], c.y) and torch.equal(y[T // 2:T // 2 + 8], c.y)
    n = L.flowmoe_layer_norm_ws_bytes(s)
    ws = torch.empty(n, dtype=torch.uint8, device=dev())
    L.flowmoe_layer_norm_bwd(s, EPS, x, c.gain, dy, None, y, c.dgain, c.dbias, False, ws, n)
    got, db = c.dgain.clone(), c.dbias.clone()
    c.bwd()
    assert torch.equal(y[-8:], c.dx) and torch.equal(y[T // 2:T // 2 + 8], c.dx)
    # T / 8 times the eight rows' sums: T 2^-24 of the magnitudes
    _, dg, dbr, mg, mb, _ = R.layer_norm_bwd(c.x, c.gain, c.dy, None, EPS)
    within(got, dg * (T // 8), (T + 20) * E24 * mg * (T // 8) + 1e-3 * mg)
    within(db, dbr * (T // 8), (T + 20) * E24 * mb * (T // 8))


def test_trace_of_kinds_past_31():
    from paper_2510_00207_amd.hiprt import EventArray
    c = Case(3000, 512)
    ev = EventArray(8)
    L.flowmoe_trace_start64(ev.ev, ev.kinds, ev.pairs, L.kind_mask(["layer_norm", "layer_norm_bwd"]))
    c.fwd()
    c.bwd()
    n = L.flowmoe_trace_stop()
    assert [L.K_NAMES[k] for k in ev.kinds[:n]] == ["layer_norm", "layer_norm_bwd", "layer_norm_bwd"]
    assert all(ev.elapsed_ms(i) > 0 for i in range(n))
    ev.close()


def test_unaligned_parameters():
    """Gains, biases and their gradients at 4 bytes past a 16-byte boundary."""
    for T, M in ((3, 40), (2000, 1032), (5, 8200)):
        c = Case(T, M)
        c.fwd()
        c.bwd()
        want = [t.clone() for t in (c.y, c.dx, c.dgain, c.dbias)]
        off = lambda t: torch.cat([t.new_zeros(1), t])[1:]
        c.gain, c.bias, c.dgain, c.dbias = (off(t) for t in (c.gain, c.bias, c.dgain, c.dbias))
        assert c.gain.data_ptr() % 16 == 4 and c.dgain.data_ptr() % 16 == 4
        c.fwd()
        c.bwd()
        assert all(torch.equal(t, w) for t, w in zip((c.y, c.dx, c.dgain, c.dbias), want))


def test_large_mean():
    """Deviations far below the mean: the squares are of deviations, not of the values."""
    c = Case(40, 1000, "f32", mean=1000.0, std=1.0)
    c.fwd()
    c.check_fwd()
    c.bwd()
    c.check_bwd()


def test_constant_rows():
    c = Case(4, 256, "f32", res=False)
    c.x[:] = 3.0
    c.fwd()
    assert torch.equal(c.y, c.bias.expand(4, -1))
    c.bwd()
    assert torch.isfinite(c.dx).all() and float(c.dgain.abs().max()) == 0


@pytest.mark.parametrize("T,M", [(3, 40), (2000, 1024)])
def test_accumulate(T, M):
    c = Case(T, M)
    c.dgain.fill_(0.5)
    c.dbias.fill_(0.5)
    c.bwd(True)
    c.check_bwd(0.5)


def test_no_rows():
    c = Case(0, 64)
    c.fwd()
    c.bwd()
    assert float(c.dgain.abs().max()) == 0 and float(c.dbias.abs().max()) == 0
    c.dgain.fill_(2.0)
    c.bwd(True)
    assert (c.dgain == 2).all()


@pytest.mark.parametrize("T", [4, 3000])
def test_in_place_and_without_parameter_gradients(T):
    c = Case(T, 1000)
    c.fwd()
    c.bwd()
    want, ws, wy = c.dx.clone(), c.sum.clone(), c.y.clone()
    x, res, dy, d_sum = (t.clone() for t in (c.x, c.res, c.dy, c.d_sum))
    L.flowmoe_layer_norm_fwd(c.shape, EPS, x, res, c.gain, c.bias, x, res)
    assert torch.equal(x, ws) and torch.equal(res, wy)
    L.flowmoe_layer_norm_bwd(c.shape, EPS, c.x, c.gain, dy, c.d_sum, dy, None, None, False)
    assert torch.equal(dy, want)
    L.flowmoe_layer_norm_bwd(c.shape, EPS, c.x, c.gain, c.dy, d_sum, d_sum, None, None, False)
    assert torch.equal(d_sum, want)
    x = c.x.clone()
    L.flowmoe_layer_norm_bwd(c.shape, EPS, x, c.gain, c.dy, c.d_sum, x, None, None, False)
    assert torch.equal(x, want)
    g1, b1 = c.dgain.clone(), c.dbias.clone()
    L.flowmoe_layer_norm_bwd(c.shape, EPS, c.x, c.gain, c.dy, c.d_sum, c.dx, c.dgain, None, False,
                             c.ws, c.n)
    c.dgain.copy_(g1)
    L.flowmoe_layer_norm_bwd(c.shape, EPS, c.x, c.gain, c.dy, c.d_sum, c.dx, None, c.dbias, False,
                             c.ws, c.n)
    assert torch.equal(c.dgain, g1) and torch.equal(c.dbias, b1)


def test_gradient_against_differences():
    """f32: the loss sum(w y) along a direction; a central difference of step e is off by O(e^2)
    and by the outputs' roundings, 2^-24 sum |w y| / e."""
    c = Case(6, 200, "f32", res=False)
    c.bwd()
    g = torch.Generator(device=dev()).manual_seed(5)
    v = torch.randn(6, 200, generator=g, device=dev())
    x, e, f = c.x.clone(), 2.0 ** -7, []
    for s in (1, -1):
        c.x = x + s * e * v
        c.fwd()
        f.append((c.y.double() * c.dy.double()).sum())
    mag = float((c.y * c.dy).abs().sum())
    want = float((c.dx.double() * v.double()).sum())
    assert abs(float(f[0] - f[1]) / (2 * e) - want) <= 4 * E24 * mag / e + 8 * e * e * float(c.dx.abs().sum())


def test_graph_and_stream():
    c = Case(3000, 512)
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.fwd()
        c.bwd()
    for i in range(3):
        o = Case(3000, 512, seed=i + 1)
        for n in ("x", "res", "dy", "d_sum"):
            getattr(c, n).copy_(getattr(o, n))
        c.gain, c.bias = c.gain.copy_(o.gain), c.bias.copy_(o.bias)
        graph.replay()
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        o.fwd(stream=s)
        o.bwd(stream=s)
        s.synchronize()
        for n in ("y", "sum", "dx", "dgain", "dbias"):
            assert torch.equal(getattr(c, n), getattr(o, n)), n
        c.check_fwd()
        c.check_bwd()
