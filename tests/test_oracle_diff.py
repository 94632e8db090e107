"""The fp64 references of rotary positions, head norm and differential attention
against their definitions: gradients against central differences, rotations against
complex numbers, the attention against a softmax written for one row."""
import math

import numpy as np
import pytest

from oracle import diff_ref as R


def numgrad(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("scaling", [
    dict(), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
    dict(scaling="bands", factor=8.0, orig_len=64.0, low=1.0, high=8.0)])
def test_rope_is_a_turn_of_pairs(layout, scaling):
    rng = np.random.default_rng(1)
    heads, hd, rot = 2, 12, 8
    x = rng.standard_normal((5, 30))
    pos = np.array([0, 1, 7, -3, 100000])
    th = R.rope_angles(rot, **scaling)
    y = R.rope(x, pos, heads, hd, rot, layout, mscale=1.25, **scaling)
    for h in range(heads):
        for i in range(rot // 2):
            a, b = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
            z = (x[:, h * hd + a] + 1j * x[:, h * hd + b]) * 1.25 * np.exp(1j * pos * th[i])
            np.testing.assert_allclose(y[:, h * hd + a] + 1j * y[:, h * hd + b], z, atol=1e-12)
    kept = np.r_[8:12, 20:30]
    assert np.array_equal(y[:, kept], x[:, kept])
    w = rng.standard_normal(x.shape)
    g = R.rope(w, pos, heads, hd, rot, layout, back=True, mscale=1.25, **scaling)
    f = lambda t: (R.rope(t, pos, heads, hd, rot, layout, mscale=1.25, **scaling) * w).sum()
    np.testing.assert_allclose(g, numgrad(f, x), atol=1e-7)


def test_rope_scalings():
    th = R.rope_angles(16)
    np.testing.assert_allclose(th, [10000.0 ** (-i / 8) for i in range(8)], rtol=1e-14)
    np.testing.assert_allclose(R.rope_angles(16, scaling="linear", factor=4), th / 4)
    b = R.rope_angles(16, scaling="base", factor=4)
    assert b[0] == 1.0 and math.isclose(b[-1], th[-1] / 4)  # fastest as it was, slowest slowed
    g = R.rope_angles(16, scaling="bands", factor=4, orig_len=1000, low=1, high=32)
    turns = 1000 * th / (2 * np.pi)
    assert (turns > 32).any() and (turns < 1).any()
    np.testing.assert_allclose(g[turns >= 32], th[turns >= 32])
    np.testing.assert_allclose(g[turns <= 1], th[turns <= 1] / 4)


@pytest.mark.parametrize("gain", [False, True])
def test_head_norm_gradients(gain):
    rng = np.random.default_rng(2)
    x, w = rng.standard_normal((3, 16)), rng.standard_normal((3, 16))
    x[1, 8:] = 0.0
    g = 1 + rng.standard_normal(8) if gain else None
    kw = dict(eps=1e-2, scale=0.7)
    y = R.head_norm(x, 2, g, **kw)
    row = x[2, 8:]
    np.testing.assert_allclose(y[2, 8:], 0.7 * (1 if g is None else g) * row /
                               math.sqrt(row @ row / 8 + 1e-2))
    dx, dg = R.head_norm_bwd(x, w, 2, g, **kw)
    np.testing.assert_allclose(dx, numgrad(lambda t: (R.head_norm(t, 2, g, **kw) * w).sum(), x),
                               atol=1e-7)
    g0 = np.ones(8) if g is None else g
    np.testing.assert_allclose(dg, numgrad(lambda t: (R.head_norm(x, 2, t, **kw) * w).sum(), g0),
                               atol=1e-7)


CASE = dict(seq_len=5, heads=4, kv_heads=2, head_dim=4)


def _inputs(seed, T=10):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((T, 16 + 2 * 8)), rng.uniform(-0.3, 0.9, 4),
            rng.standard_normal((T, 16)))


def test_diff_attention_of_one_row():
    qkv, lam, _ = _inputs(3)
    attn, attn2, lse, _ = R.diff_attention(qkv, lam, causal=True, lens=[5, 3], **CASE)
    # token 2 of sequence 1 (valid: 3 tokens), head 3 (key head 1)
    t, keys = 7, [5, 6, 7]
    w = []
    for i in (0, 1):
        s = [qkv[t, 12 + 2 * i:14 + 2 * i] @ qkv[j, 20 + 2 * i:22 + 2 * i] / math.sqrt(2) for j in keys]
        e = [math.exp(v) for v in s]
        assert math.isclose(lse[i, 3, t], math.log(sum(e)))
        w.append([v / sum(e) for v in e])
    o = [sum(wj * qkv[j, 28:32] for wj, j in zip(wi, keys)) for wi in w]
    np.testing.assert_allclose(attn2[t, 12:], o[1])
    np.testing.assert_allclose(attn[t, 12:], o[0] - lam[3] * o[1])
    assert not attn[8:].any() and not lse[:, :, 8:].any()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens", [None, [5, 3], [0, 1]])
def test_diff_attention_gradients(causal, lens):
    qkv, lam, w = _inputs(4)
    kw = dict(causal=causal, lens=lens, **CASE)
    attn, attn2, _, _ = R.diff_attention(qkv, lam, **kw)
    d_qkv, delta, d_lam, _ = R.diff_attention_bwd(qkv, lam, attn, attn2, w, **kw)
    f = lambda q, l: (R.diff_attention(q, l, **kw)[0] * w).sum()
    np.testing.assert_allclose(d_qkv, numgrad(lambda t: f(t, lam), qkv), atol=1e-7)
    np.testing.assert_allclose(d_lam, numgrad(lambda t: f(qkv, t), lam), atol=1e-7)
    np.testing.assert_allclose(d_lam, -delta[1].sum(1), atol=1e-12)
