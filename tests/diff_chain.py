"""The gradients of the differential attention block as one chain in fp64, from its inputs
alone, and how far the roundings of a bf16 block may move them (imported by
tests/test_diff_chain.py and tests/test_gpu_diff_chain.py).

Every tensor that the block keeps or multiplies in bf16 passes through `rnd`, so that an
error can be put there and followed to the gradients. Half a step of bf16 is 2^-8 of the
value. `bounds` puts an error of that size and of either sign into every element of one
such tensor at a time and takes the root mean square (over a few draws of the signs) of
how far each gradient moves in the 2-norm; a block's own error at that place is no larger
in any element and of independent signs. The sum over all places (as if all of them moved
a gradient the same way), twice (a scalar's error is one draw, not a norm), bounds the
block's. fp32 sums (2^-13 and less) lie far below."""
import numpy as np

import oracle
from oracle.diff_ref import diff_parts

H8 = 2.0 ** -8
GRADS = ("d_in", "dw_qkv", "dw_o", "d_lambda", "dgain")
PLACES = ("qkv", "turned", "p1", "p2", "attn", "attn2", "normed", "g", "d_attn", "p12", "ds1", "ds2",
          "d_qkv", "d_turned", "d_in")


def keep(name, x):
    return x


def forward(p, args, rope, pos, lens, norm, rnd=keep):
    """(qkv as turned, attn, attn2, normed); rope: keywords of oracle.rope, or None."""
    seq, heads, kv, D, causal = args
    q = rnd("qkv", p["inp"] @ p["w_qkv"])
    if rope is not None:
        n = rope["heads"] * rope["head_dim"]
        q = np.concatenate([rnd("turned", oracle.rope(q, pos, **rope)[:, :n]), q[:, n:]], 1)
    attn, attn2 = np.zeros((q.shape[0], heads * D)), np.zeros((q.shape[0], heads * D))
    for rows, h, cq, ck, cv, pr, _ in diff_parts(q, *args, lens=lens):
        v, col = q[rows, cv:cv + D], slice(h * D, (h + 1) * D)
        o1, o2 = rnd("p1", pr[0]) @ v, rnd("p2", pr[1]) @ v
        attn2[rows, col] = o2
        attn[rows, col] = o1 - p["lam"][h] * o2
    attn, attn2 = rnd("attn", attn), rnd("attn2", attn2)
    return q, attn, attn2, rnd("normed", oracle.head_norm(attn, heads, p["gain"], *norm))


def gradients(p, args, rope, pos, lens, norm, rnd=keep):
    """The gradients GRADS of sum(out * d_out)."""
    seq, heads, kv, D, causal = args
    d, lam = D // 2, p["lam"]
    q, attn, attn2, normed = forward(p, args, rope, pos, lens, norm, rnd)
    g = rnd("g", p["d_out"] @ p["w_o"].T)
    da, dgain = oracle.head_norm_bwd(attn, g, heads, p["gain"], *norm)
    da = rnd("d_attn", da)
    dq, d_lam = np.zeros(q.shape), np.zeros(heads)
    for rows, h, cq, ck, cv, pr, _ in diff_parts(q, *args, lens=lens):
        col = slice(h * D, (h + 1) * D)
        do, v = da[rows, col], q[rows, cv:cv + D]
        d2 = (do * attn2[rows, col]).sum(1, keepdims=True)
        d1 = (do * attn[rows, col]).sum(1, keepdims=True) + lam[h] * d2
        d_lam[h] -= d2.sum()
        dp = do @ v.T
        dq[rows, cv:cv + D] += rnd("p12", pr[0] - lam[h] * pr[1]).T @ do
        for i, ds in ((0, pr[0] * (dp - d1)), (1, pr[1] * (dp - d2))):
            ds = rnd(f"ds{i + 1}", ds) * (1.0 if i == 0 else -lam[h]) / np.sqrt(d)
            qi, ki = slice(cq + i * d, cq + (i + 1) * d), slice(ck + i * d, ck + (i + 1) * d)
            dq[rows, qi] = ds @ q[rows, ki]
            dq[rows, ki] += ds.T @ q[rows, qi]
    dq = rnd("d_qkv", dq)
    if rope is not None:
        n = rope["heads"] * rope["head_dim"]
        dq = np.concatenate([rnd("d_turned", oracle.rope(dq, pos, back=True, **rope)[:, :n]), dq[:, n:]], 1)
    return {"d_in": rnd("d_in", dq @ p["w_qkv"].T), "dw_qkv": p["inp"].T @ dq,
            "dw_o": normed.T @ p["d_out"], "d_lambda": d_lam, "dgain": dgain}


def loss(p, args, rope, pos, lens, norm):
    return (forward(p, args, rope, pos, lens, norm)[3] @ p["w_o"] * p["d_out"]).sum()


def bounds(p, *rest, draws=4, seed=0):
    """(gradients, the 2-norm that each one's error may have)."""
    ref = gradients(p, *rest)
    rng = np.random.default_rng(seed)
    total = {n: 0.0 for n in GRADS}
    for place in PLACES:
        sq = {n: 0.0 for n in GRADS}
        for _ in range(draws):
            off = lambda name, x: x * (1 + H8 * rng.choice((-1.0, 1.0), x.shape)) if name == place else x
            moved = gradients(p, *rest, rnd=off)
            for n in GRADS:
                sq[n] += ((moved[n] - ref[n]) ** 2).sum() / draws
        for n in GRADS:
            total[n] += 2.0 * np.sqrt(sq[n])
    return ref, total


def within(got, ref, bound):
    """Whether a gradient lies within its bound of the reference."""
    got = np.asarray(got, np.float64)
    return bool(np.isfinite(got).all()) and np.linalg.norm(got - ref) <= bound


# (sequences, seq_len, heads, kv_heads, head_dim, causal, lens, rot_dim or None: not turned,
# layout, with a gain)
CASES = [
    (2, 40, 4, 2, 64, True, [40, 25], 32, "half", True),
    (3, 33, 3, 1, 128, False, None, None, "half", True),
    (2, 70, 3, 3, 64, True, [70, 1], 20, "pairs", False),
    (12, 10, 4, 1, 64, False, [n % 11 for n in range(12)], None, "half", False),
]
