"""fp64 references of the packed attention, the layer norm and the embedding, from their
definitions, with what their tolerances need: the sums of magnitudes that a rounding of a
factor scales with."""
import math

import torch

# a rounding to nearest is off by at most half a step, relative to the value
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def starts_of(lens):
    s = [0]
    for n in lens:
        s.append(s[-1] + n)
    return s


def attention(qkv, lens, heads, kv, D, causal):
    """(attn, lse, sum of P |V|, largest sum of |q| |k| / sqrt(D)) of the rows, zeros in those
    of no sequence."""
    T = qkv.shape[0]
    x = qkv.double()
    z = lambda *s: torch.zeros(*s, dtype=torch.float64, device=qkv.device)
    attn, mag, lse, smax = z(T, heads * D), z(T, heads * D), z(heads, T), 0.0
    for a, b in zip(starts_of(lens), starts_of(lens)[1:]):
        if a == b:
            continue
        for h in range(heads):
            q, k, v = (x[a:b, c * D:c * D + D] for c in columns(h, heads, kv))
            s = scores(q, k, causal)
            lse[h, a:b] = torch.logsumexp(s, 1)
            p = torch.softmax(s, 1)
            attn[a:b, h * D:h * D + D] = p @ v
            mag[a:b, h * D:h * D + D] = p @ v.abs()
            smax = max(smax, float((q.abs() @ k.abs().T).max()) / math.sqrt(D))
    return attn, lse, mag, smax


def columns(h, heads, kv):
    g = h // (heads // kv)
    return h, heads + g, heads + kv + g


def scores(q, k, causal):
    s = q @ k.T / math.sqrt(q.shape[1])
    if causal:
        s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1), -math.inf)
    return s


def attention_bwd(qkv, lens, heads, kv, D, causal, attn, lse, d_attn):
    """(d_qkv; the same sums of the magnitudes of what is rounded; and of what is summed in
    32 bits), from the forward's attn and lse as given."""
    x, o, do_ = qkv.double(), attn.double(), d_attn.double()
    d, rnd, mag = (torch.zeros_like(x) for _ in range(3))
    rs = 1 / math.sqrt(D)
    for a, b in zip(starts_of(lens), starts_of(lens)[1:]):
        if a == b:
            continue
        for h in range(heads):
            cq, ck, cv = (slice(c * D, c * D + D) for c in columns(h, heads, kv))
            q, k, v = x[a:b, cq], x[a:b, ck], x[a:b, cv]
            do = do_[a:b, h * D:h * D + D]
            oh = o[a:b, h * D:h * D + D]
            p = torch.exp(scores(q, k, causal) - lse[h, a:b].double()[:, None])
            ds = p * (do @ v.T - (do * oh).sum(1, keepdim=True))
            dm = p * (do.abs() @ v.abs().T + (do * oh).abs().sum(1, keepdim=True))
            d[a:b, cq] += ds @ k * rs
            d[a:b, ck] += ds.T @ q * rs
            d[a:b, cv] += p.T @ do
            rnd[a:b, cq] += ds.abs() @ k.abs() * rs
            rnd[a:b, ck] += ds.abs().T @ q.abs() * rs
            rnd[a:b, cv] += p.T @ do.abs()
            mag[a:b, cq] += dm @ k.abs() * rs
            mag[a:b, ck] += dm.T @ q.abs() * rs
            mag[a:b, cv] += p.T @ do.abs()
    return d, rnd, mag


def layer_norm(x, res, gain, bias, eps):
    """(y, h, n, r)"""
    h = x.double() + (0 if res is None else res.double())
    mu = h.mean(1, keepdim=True)
    r = 1 / torch.sqrt(((h - mu) ** 2).mean(1, keepdim=True) + eps)
    n = (h - mu) * r
    y = n if gain is None else n * gain.double()
    return y if bias is None else y + bias.double(), h, n, r


def layer_norm_bwd(x, gain, dy, d_sum, eps):
    """(dx, dgain, dbias, sum of |dy n|, sum of |dy|, magnitude of dx's terms)"""
    _, _, n, r = layer_norm(x, None, None, None, eps)
    dy = dy.double()
    u = dy if gain is None else dy * gain.double()
    dx = r * (u - u.mean(1, keepdim=True) - n * (u * n).mean(1, keepdim=True))
    mag = r * (u.abs() + u.abs().mean(1, keepdim=True) + n.abs() * (u * n).abs().mean(1, keepdim=True))
    if d_sum is not None:
        dx = dx + d_sum.double()
        mag = mag + d_sum.double().abs()
    return dx, (dy * n).sum(0), dy.sum(0), (dy * n).abs().sum(0), dy.abs().sum(0), mag


def embed(ids, table, scale):
    there = (ids >= 0) & (ids < table.shape[0])
    y = table.double()[ids.long().clamp(0, table.shape[0] - 1)] * scale
    return y * there[:, None]


def embed_bwd(ids, dy, vocab, scale):
    """(dtable, sum of |scale dy|)"""
    there = (ids >= 0) & (ids < vocab)
    d = torch.zeros(vocab, dy.shape[1], dtype=torch.float64, device=dy.device)
    m = torch.zeros_like(d)
    i = ids.long()[there]
    d.index_add_(0, i, dy.double()[there])
    m.index_add_(0, i, dy.double()[there].abs())
    return d * scale, m * abs(scale)
