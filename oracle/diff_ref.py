"""fp64 reference of the differential attention block's operators (test
infrastructure only): rotary positions (arXiv 2104.09864; the bands scaling of
arXiv 2309.00071, Sec. 3.2), differential attention (arXiv 2410.05258, Sec.
2.1) and the RMS norm of each head, forward and backward.

Every function is the definition written out with numpy, per sequence and head;
nothing is blocked, fused or reordered. Gradients are the chain rule.
"""
from __future__ import annotations

import numpy as np


# ---- rotary positions ---------------------------------------------------------
def rope_angles(rot, base=10000.0, scaling="none", factor=1.0, orig_len=0.0, low=1.0, high=32.0):
    """theta_i, the angle per token of each of the rot / 2 pairs."""
    i = np.arange(rot // 2, dtype=np.float64)
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2.0))
    theta = base ** (-2.0 * i / rot)
    if scaling == "linear":
        theta = theta / factor
    elif scaling == "bands":
        g = np.clip((orig_len * theta / (2 * np.pi) - low) / (high - low), 0.0, 1.0)
        theta = theta * (g + (1.0 - g) / factor)
    return theta


def rope(x, pos, heads, head_dim, rot, layout="half", back=False, mscale=1.0, **scaling):
    """x (T x M) with its first heads * head_dim columns turned at positions pos (T);
    back: the gradient's turn. Other columns are returned as they are."""
    phi = np.asarray(pos, np.float64)[:, None] * rope_angles(rot, **scaling)
    c, s = mscale * np.cos(phi), mscale * np.sin(phi) * (-1.0 if back else 1.0)
    y = np.array(x, np.float64)
    for h in range(heads):
        i = np.arange(rot // 2)
        a, b = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
        a, b = a + h * head_dim, b + h * head_dim
        y[:, a], y[:, b] = x[:, a] * c - x[:, b] * s, x[:, a] * s + x[:, b] * c
    return y


# ---- head norm ----------------------------------------------------------------
def head_norm(x, heads, gain=None, eps=1e-5, scale=1.0):
    """scale * gain * x / sqrt(mean(x^2) + eps) of each head's columns."""
    v = x.reshape(x.shape[0], heads, -1)
    g = np.ones(v.shape[2]) if gain is None else gain
    return (scale * g * v / np.sqrt((v * v).mean(2, keepdims=True) + eps)).reshape(x.shape)


def head_norm_bwd(x, dy, heads, gain=None, eps=1e-5, scale=1.0):
    """(dx, dgain)."""
    v, d = x.reshape(x.shape[0], heads, -1), dy.reshape(x.shape[0], heads, -1)
    g = np.ones(v.shape[2]) if gain is None else gain
    rms = np.sqrt((v * v).mean(2, keepdims=True) + eps)
    n = v / rms
    u = scale * g * d
    dx = (u - n * (u * n).mean(2, keepdims=True)) / rms
    return dx.reshape(x.shape), scale * (d * n).sum((0, 1))


# ---- differential attention -----------------------------------------------------
def _lens(T, seq_len, lens):
    n = T // seq_len
    return [seq_len] * n if lens is None else [min(max(int(v), 0), seq_len) for v in lens]


def diff_parts(qkv, seq_len, heads, kv_heads, head_dim, causal, lens=None):
    """For every sequence and head: (rows, h, its query columns, its key columns, its value
    columns, [P_1, P_2], [lse_1, lse_2]) over the sequence's valid tokens (at least one)."""
    D, d, M = head_dim, head_dim // 2, heads * head_dim
    for b, n in enumerate(_lens(qkv.shape[0], seq_len, lens)):
        if n == 0:
            continue
        rows = slice(b * seq_len, b * seq_len + n)
        for h in range(heads):
            g = h // (heads // kv_heads)
            cq, ck, cv = h * D, M + g * D, M + (kv_heads + g) * D
            p, lse = [], []
            for i in (0, 1):
                s = qkv[rows, cq + i * d:cq + (i + 1) * d] @ \
                    qkv[rows, ck + i * d:ck + (i + 1) * d].T / np.sqrt(d)
                if causal:
                    s = np.where(np.tril(np.ones((n, n), bool)), s, -np.inf)
                m = s.max(1, keepdims=True)
                e = np.exp(s - m)
                z = e.sum(1, keepdims=True)
                p.append(e / z)
                lse.append((m + np.log(z))[:, 0])
            yield rows, h, cq, ck, cv, p, lse


def diff_attention(qkv, lam, seq_len, heads, kv_heads, head_dim, causal, lens=None):
    """attn (T x M), attn2 = P_2 V (T x M), lse (2 x heads x T), and `size` (2 x T x M), the
    sums P_i |V| that the rounding of probabilities is relative to."""
    T, D = qkv.shape[0], head_dim
    attn, attn2 = np.zeros((T, heads * D)), np.zeros((T, heads * D))
    size = np.zeros((2, T, heads * D))
    lse = np.zeros((2, heads, T))
    for rows, h, cq, ck, cv, p, l in diff_parts(qkv, seq_len, heads, kv_heads, D, causal, lens):
        v, col = qkv[rows, cv:cv + D], slice(h * D, (h + 1) * D)
        attn2[rows, col] = p[1] @ v
        attn[rows, col] = p[0] @ v - lam[h] * attn2[rows, col]
        size[0, rows, col], size[1, rows, col] = p[0] @ np.abs(v), p[1] @ np.abs(v)
        lse[:, h, rows] = l
    return attn, attn2, lse, size


def diff_attention_bwd(qkv, lam, attn, attn2, d_attn, seq_len, heads, kv_heads, head_dim, causal,
                       lens=None):
    """Gradients from the forward's attn and attn2: d_qkv (T x W), delta (2 x heads x T),
    d_lambda (heads), and `size` (T x W), sums of absolute values behind each element of
    d_qkv, every difference taken as a sum (what the rounding of its parts is relative to)."""
    D, d = head_dim, head_dim // 2
    d_qkv, size = np.zeros(qkv.shape), np.zeros(qkv.shape)
    delta, d_lam = np.zeros((2, heads, qkv.shape[0])), np.zeros(heads)
    for rows, h, cq, ck, cv, p, _ in diff_parts(qkv, seq_len, heads, kv_heads, D, causal, lens):
        col = slice(h * D, (h + 1) * D)
        do, v = d_attn[rows, col], qkv[rows, cv:cv + D]
        d2 = (do * attn2[rows, col]).sum(1)
        d1 = (do * attn[rows, col]).sum(1) + lam[h] * d2
        delta[0, h, rows], delta[1, h, rows] = d1, d2
        d_lam[h] -= d2.sum()
        dp = do @ v.T
        d_qkv[rows, cv:cv + D] += (p[0] - lam[h] * p[1]).T @ do
        size[rows, cv:cv + D] += (p[0] + abs(lam[h]) * p[1]).T @ np.abs(do)
        for i, w, dl in ((0, p[0], d1), (1, -lam[h] * p[1], d2)):
            q, k = (slice(c0 + i * d, c0 + (i + 1) * d) for c0 in (cq, ck))
            ds, sz = w * (dp - dl[:, None]), np.abs(w) * (np.abs(dp) + np.abs(dl)[:, None])
            d_qkv[rows, q] = ds @ qkv[rows, k] / np.sqrt(d)
            d_qkv[rows, k] += ds.T @ qkv[rows, q] / np.sqrt(d)
            size[rows, q] = sz @ np.abs(qkv[rows, k]) / np.sqrt(d)
            size[rows, k] += sz.T @ np.abs(qkv[rows, q]) / np.sqrt(d)
    return d_qkv, delta, d_lam, size
