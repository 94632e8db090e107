"""The references' gradients against central differences of their forwards, in fp64 on the
CPU. A central difference of step e is off by O(e^2) and by rounding of about 1e-16 / e: 1e-6
relative at e = 1e-5 is far above both."""
import pytest
import torch

import packed_ref as R


def directional(f, x, v, e=1e-5):
    return float((f(x + e * v) - f(x - e * v)) / (2 * e))


@pytest.mark.parametrize("heads,kv,causal", [(2, 2, True), (4, 2, True), (3, 1, False)])
def test_attention_gradient(heads, kv, causal):
    g = torch.Generator().manual_seed(heads)
    D, lens, T = 8, [5, 0, 1, 7], 15
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    qkv, w = r(T, (heads + 2 * kv) * D), r(T, heads * D)
    attn, lse, _, _ = R.attention(qkv, lens, heads, kv, D, causal)
    d, _, _ = R.attention_bwd(qkv, lens, heads, kv, D, causal, attn, lse, w)
    loss = lambda x: (R.attention(x, lens, heads, kv, D, causal)[0] * w).sum()
    for _ in range(3):
        v = r(*qkv.shape)
        assert directional(loss, qkv, v) == pytest.approx(float((d * v).sum()), rel=1e-6, abs=1e-7)
    assert d[13:].abs().max() == 0


def test_layer_norm_gradient():
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    x, gain, bias, w, ds = r(6, 24) * 2 + 0.5, r(24), r(24), r(6, 24), r(6, 24)
    dx, dg, db, *_ = R.layer_norm_bwd(x, gain, w, ds, 1e-5)
    y = lambda a, b, c: (R.layer_norm(a, None, b, c, 1e-5)[0] * w).sum()
    for f, at, d in [(lambda t: y(t, gain, bias) + (t * ds).sum(), x, dx),
                     (lambda t: y(x, t, bias), gain, dg), (lambda t: y(x, gain, t), bias, db)]:
        v = r(*at.shape)
        assert directional(f, at, v) == pytest.approx(float((d * v).sum()), rel=1e-6, abs=1e-7)


def test_embed_gradient():
    g = torch.Generator().manual_seed(2)
    ids = torch.tensor([3, 0, 3, -1, 9, 10, 3])
    table, w = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((10, 8), (7, 8)))
    d, _ = R.embed_bwd(ids, w, 10, 0.7)
    v = torch.randn(10, 8, generator=g, dtype=torch.float64)
    f = lambda t: (R.embed(ids, t, 0.7) * w).sum()
    assert directional(f, table, v) == pytest.approx(float((d * v).sum()), rel=1e-6, abs=1e-7)
