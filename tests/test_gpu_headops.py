"""Rotary positions and head norm against the fp64 reference, element by element.

Tolerances count roundings. Rotary positions: cosine and sine are within 8 half
steps of fp32 (the angle's fraction of a turn rounded to fp32, 2 pi 2^-25, and the
functions' own), two products and a sum make 3 more: 12 x 2^-24 (|u| + |v|) mscale,
plus half a step of the output's type. Head norm: a sum of at most 512 squares over a
lane's 8 and six exchanges, a reciprocal root and three products: 32 x 2^-24."""
import numpy as np
import pytest
import torch

import oracle
from gpu_helpers import dev, host, need_gpu
from paper_2510_00207_amd import _lib as L

pytestmark = pytest.mark.gpu
TD = {"bf16": torch.bfloat16, "f32": torch.float32}
DT = {"bf16": L.BF16, "f32": L.F32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a step, relative
U = 2.0 ** -24


def normal(seed, *shape, dtype="bf16"):
    g = torch.Generator(device=dev()).manual_seed(seed)
    return torch.randn(*shape, generator=g, device=dev()).to(TD[dtype])


def close(got, ref, tol, what):
    err = np.abs(host(got) - ref) - tol
    assert not np.isnan(err).any() and (err <= 0).all(), (
        what, float(err.max()), np.unravel_index(err.argmax(), err.shape))


BANDS = dict(scaling="bands", factor=8.0, orig_len=256.0, low=1.0, high=32.0, mscale=1.2)
ROPE_CASES = [
    # (T, M, heads, head_dim, rot, layout, dtype, scaling, positions)
    (1, 64, 1, 64, 64, "half", "bf16", {}, None),
    (7, 2048, 32, 64, 64, "half", "bf16", BANDS, "far"),
    (130, 1544, 12, 128, 64, "pairs", "f32", dict(scaling="linear", factor=4.0), "row"),
    (65, 520, 4, 128, 128, "half", "bf16", dict(scaling="base", factor=8.0), "far"),
    (33, 96, 1, 96, 48, "half", "f32", {}, "far"),
    (5, 80, 1, 80, 40, "pairs", "bf16", {}, "row"),
    (9, 512, 1, 512, 512, "pairs", "bf16", {}, "row"),
    (9, 1024, 2, 512, 512, "half", "f32", BANDS, "far"),
    # turned columns that no vector holds whole
    (19, 200, 3, 64, 2, "half", "bf16", {}, "far"),
    (19, 200, 3, 64, 50, "half", "f32", {}, "far"),
    (19, 200, 3, 64, 30, "pairs", "bf16", {}, "row"),
    (4, 24, 3, 8, 6, "pairs", "f32", {}, "row"),
    (257, 8, 1, 8, 8, "pairs", "bf16", {}, "far"),
    (300, 5128, 65, 72, 16, "half", "bf16", {}, "row"),
    # heads that do not divide a block's threads, more heads than it holds
    (1030, 2400, 30, 80, 80, "half", "bf16", {}, "row"),
    (1100, 480, 6, 80, 42, "half", "f32", BANDS, "far"),
    (70, 2640, 11, 240, 240, "half", "bf16", {}, "row"),
    (2, 512, 1, 512, 510, "half", "bf16", {}, "row"),
]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("T,M,heads,hd,rot,layout,dtype,scaling,positions", ROPE_CASES)
def test_rope(T, M, heads, hd, rot, layout, dtype, scaling, positions, back):
    need_gpu()
    seq = 50
    print(f"[rope] T={T} M={M} heads={heads} hd={hd} rot={rot} {layout} {dtype}", flush=True)
    x = normal(T + M, T, M, dtype=dtype)
    rng = np.random.default_rng(T)
    p = None
    if positions == "far":
        p = rng.integers(-2 ** 31, 2 ** 31 - 1, T)
        p[:4] = [0, -1, 2 ** 31 - 1, -2 ** 31][:T]
    elif positions == "row":
        p = rng.integers(0, 5000, T)
    pos = None if p is None else torch.from_numpy(p.astype(np.int32)).to(dev())
    s = L.make_shape(T, M, 8, 1, 1, 0, DT[dtype])
    r = L.make_rope_shape(heads, hd, rot, seq, layout=layout, **scaling)
    call = L.flowmoe_rope_bwd if back else L.flowmoe_rope_fwd
    y = torch.full_like(x, 7.0)
    call(s, r, x, pos, y)
    z = x.clone()  # in place
    call(s, r, z, pos, z)
    torch.cuda.synchronize()
    xh = host(x)
    at = np.arange(T) % seq if p is None else p
    ref = oracle.rope(xh, at, heads, hd, rot, layout, back=back, **scaling)
    # |u| + |v| of each column's pair
    size = np.zeros_like(xh)
    i = np.arange(rot // 2)
    a, b = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    for h in range(heads):
        size[:, h * hd + a] = size[:, h * hd + b] = np.abs(xh[:, h * hd + a]) + np.abs(xh[:, h * hd + b])
    # (angles in double, here and there: up to 16 roundings of 2^-53 of a position's radians)
    ang = 16 * 2.0 ** -53 * np.abs(np.asarray(at, np.float64))[:, None]
    tol = (12 * U + ang) * scaling.get("mscale", 1.0) * size
    tol += 1.01 * HALF[dtype] * np.abs(ref) * (size > 0)
    n = heads * hd
    close(y[:, :n], ref[:, :n], tol[:, :n], "y")
    assert bool((y[:, n:] == 7.0).all()), "columns past the heads were written"
    assert torch.equal(z[:, :n], y[:, :n]) and torch.equal(z[:, n:], x[:, n:])


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("T,heads,hd,rot", [
    (9, 3, 128, 64), (33, 4, 64, 50), (1100, 2, 64, 2), (5, 2, 8, 6), (70, 11, 240, 238)])
def test_rope_copies_the_other_columns(T, heads, hd, rot, layout, dtype, back):
    """Columns past rot_dim bit for bit, infinities, NaN and -0 among them, which reach no
    turned column either; out of place and in place."""
    need_gpu()
    M = heads * hd + 8
    x = normal(T + rot, T, M, dtype=dtype)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    # inf, -inf, quiet and signalling NaN, -0, 0, the smallest denormal, 1.5
    odd = [0x7F80, 0xFF80, 0x7FC1, 0x7F81, 0x8000, 0, 1, 0x3FC0]
    if dtype == "f32":
        odd = [v << 16 if v != 1 else 1 for v in odd]
    np_bits = np.array(odd, np.uint16 if dtype == "bf16" else np.uint32)
    odd = torch.from_numpy(np_bits.view(np.int16 if dtype == "bf16" else np.int32)).to(dev())
    col = torch.arange(M, device=dev())
    other = (col < heads * hd) & (col % hd >= rot)
    i = torch.arange(T, device=dev())[:, None] * 3 + col[None, :]
    z = x.clone()
    z.view(bits)[:, other] = odd[i % 8][:, other]
    s = L.make_shape(T, M, 8, 1, 1, 0, DT[dtype])
    r = L.make_rope_shape(heads, hd, rot, 50, layout=layout, mscale=1.25)
    call = L.flowmoe_rope_bwd if back else L.flowmoe_rope_fwd
    want, got = x.clone(), torch.full_like(z, 7.0)
    call(s, r, x, None, want)
    call(s, r, z, None, got)
    kept = z.clone()
    call(s, r, z, None, z)  # in place
    torch.cuda.synchronize()
    turned = (col < heads * hd) & ~other
    for y in (got, z):
        assert torch.equal(y.view(bits)[:, other], kept.view(bits)[:, other])
        assert torch.equal(y[:, turned], want[:, turned])


def test_rope_forward_then_backward_is_the_identity():
    need_gpu()
    x = normal(3, 300, 512, dtype="f32")
    s = L.make_shape(300, 512, 8, 1, 1, 0, L.F32)
    for layout in ("half", "pairs"):
        r = L.make_rope_shape(4, 128, 128, 100, layout=layout)
        y, z = torch.empty_like(x), torch.empty_like(x)
        L.flowmoe_rope_fwd(s, r, x, None, y)
        L.flowmoe_rope_bwd(s, r, y, None, z)
        torch.cuda.synchronize()
        # two turns, each within 12 half steps of the pair's |u| + |v| <= 2 max |x|
        assert float((z - x).abs().max()) <= 2 * 13 * U * 2 * 1.5 * float(x.abs().max())


def test_rope_past_32_bit_offsets():
    """The last rows of a tensor of more than 2^32 bytes."""
    need_gpu()
    T, M = (1 << 18) + 3, 8320
    assert T * M * 2 > 1 << 32
    x = torch.zeros(T, M, dtype=torch.bfloat16, device=dev())
    x[-5:] = normal(5, 5, M)
    s = L.make_shape(T, M, 8, 1, 1, 0, L.BF16)
    r = L.make_rope_shape(65, 128, 128, T)
    L.flowmoe_rope_fwd(s, r, x.data_ptr(), None, x)
    s5 = L.make_shape(5, M, 8, 1, 1, 0, L.BF16)
    y = normal(5, 5, M)
    pos = torch.arange(T - 5, T, dtype=torch.int32, device=dev())
    L.flowmoe_rope_fwd(s5, r, y, pos, y)
    torch.cuda.synchronize()
    assert torch.equal(x[-5:], y) and not bool(x[:-5].any())


NORM_CASES = [
    # (T, heads, head_dim, dtype)
    (1, 1, 8, "bf16"), (1, 1, 512, "f32"), (3, 5, 24, "f32"), (257, 8, 64, "f32"),
    (100, 3, 200, "bf16"), (333, 4, 128, "bf16"), (77, 2, 256, "bf16"), (64, 1, 96, "f32"),
    (4000, 16, 128, "bf16"), (2500, 33, 32, "f32"), (10, 2, 504, "bf16"),
]


@pytest.mark.parametrize("gained", [True, False])
@pytest.mark.parametrize("T,heads,hd,dtype", NORM_CASES)
def test_head_norm(T, heads, hd, dtype, gained):
    need_gpu()
    print(f"[norm] T={T} heads={heads} hd={hd} {dtype}", flush=True)
    M, eps, scale = heads * hd, 1e-3, 0.3
    x, dy = normal(T, T, M, dtype=dtype), normal(T + 1, T, M, dtype=dtype)
    x[T // 2] *= 1e-3  # a row that eps governs
    if T > 2:
        x[0] = 0.0
    gain = 1 + 0.5 * normal(7, hd, dtype="f32") if gained else None
    s = L.make_shape(T, M, 8, 1, 1, 0, DT[dtype])
    n = L.make_norm_shape(heads, hd, eps, scale)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dgain = torch.full((hd,), 3.0, device=dev())
    need = L.flowmoe_head_norm_ws_bytes(s, n)
    ws = torch.empty(max(1, need), dtype=torch.uint8, device=dev())
    L.flowmoe_head_norm_fwd(s, n, x, gain, y)
    L.flowmoe_head_norm_bwd(s, n, x, gain, dy, dx, dgain, False, ws, need)
    dg2, dx2, y2 = dgain.clone(), dy.clone(), x.clone()
    L.flowmoe_head_norm_bwd(s, n, x, gain, dx2, dx2, dg2, True, ws, need)  # dx over dy, added
    L.flowmoe_head_norm_fwd(s, n, y2, gain, y2)  # in place
    dx3 = torch.empty_like(x)
    L.flowmoe_head_norm_bwd(s, n, x, gain, dy, dx3, None, False)  # without dgain, no scratch
    torch.cuda.synchronize()
    xh, dyh, gh = host(x), host(dy), None if gain is None else host(gain)
    eps, scale = float(np.float32(eps)), float(np.float32(scale))
    ref = oracle.head_norm(xh, heads, gh, eps, scale)
    close(y, ref, (1.01 * HALF[dtype] + 32 * U) * np.abs(ref), "y")
    rdx, rdg = oracle.head_norm_bwd(xh, dyh, heads, gh, eps, scale)
    v, d = np.abs(xh).reshape(T, heads, hd), np.abs(dyh).reshape(T, heads, hd)
    r = 1 / np.sqrt((v * v).mean(2, keepdims=True) + eps)
    u = scale * d * (1 if gh is None else np.abs(gh))
    size = (r * (u + v * r * r * (u * v).mean(2, keepdims=True))).reshape(T, M)
    close(dx, rdx, 1.01 * HALF[dtype] * np.abs(rdx) + 80 * U * size, "dx")
    # a sum over a thread's rows, the block's groups and the blocks, at most T heads + 200 long
    path = 64 + min(T * heads, 400)
    close(dgain, rdg, path * U * scale * (d * v * r).sum((0, 1)), "dgain")
    assert torch.equal(dx2, dx) and torch.equal(y2, y) and torch.equal(dx3, dx)
    assert torch.equal(dg2, dgain + dgain)


def test_head_norm_of_no_tokens():
    need_gpu()
    s, n = L.make_shape(0, 64, 8, 1, 1, 0, L.F32), L.make_norm_shape(1, 64)
    L.flowmoe_head_norm_fwd(s, n, None, None, None)
    dg = torch.full((64,), 3.0, device=dev())
    L.flowmoe_head_norm_bwd(s, n, None, None, None, None, dg, True)
    assert bool((dg == 3.0).all())
    L.flowmoe_head_norm_bwd(s, n, None, None, None, None, dg, False)
    assert not bool(dg.any())
