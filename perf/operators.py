"""The operators of a differential attention block, as cases to time and compare.

A program that trains such a block turns the queries and keys by their positions
(rotary positions), takes the difference of two softmax maps per head
(differential attention) and normalises every head's output before the output
projection (head norm); its backward pass runs the three in reverse. The cases
are single calls of these, in each direction, over the sizes of moe_inputs'
configurations (widths 64 to 4096, sequences of 64, 512 and 4096 tokens, heads
of 64 and 128, up to 16384 tokens) and over ragged ones: padded batches,
sequences of any length, keys and values shared by groups of heads, rotations
of a part of the head.

With ``own`` false ``run`` computes the operators from elementary torch
operations in 32 bits (angles in 64); with ``own`` true it calls the framework.
``exact`` computes them in 64 bits, a sequence at a time.

Inputs: activations and gradients N(0, 1); lambda uniform in [0.2, 0.8] (its
initial values over a network's depth); gains 1 + N(0, 0.1^2).
"""
import math

import torch

own = False

TD = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS, SCALE = 1e-5, 0.2  # of the head norm: 1 - lambda_init of a deep layer


# ---- the cases ---------------------------------------------------------------------
def _rope(dir, T, heads, hd, rot, layout, scaling="none", dtype="bf16", pad=0, pos="row", seq=4096):
    return dict(kind="rope_" + dir, T=T, heads=heads, hd=hd, rot=rot, layout=layout,
                scaling=scaling, dtype=dtype, ld=heads * hd + pad, pos=pos, seq=seq)


def _diff(dir, nseq, seq, heads, kv, hd, causal, pad=0):
    """pad > 0: sequence i has seq - (i * pad) % (seq + 1) valid tokens."""
    return dict(kind="diff_" + dir, nseq=nseq, seq=seq, heads=heads, kv=kv, hd=hd, causal=causal,
                pad=pad)


def _norm(dir, T, heads, hd, dtype="bf16"):
    return dict(kind="norm_" + dir, T=T, heads=heads, hd=hd, dtype=dtype)


def listed():
    return [
        # one token of each of 64 sequences at far, unrelated positions of a stretched context
        dict(name="rope_tokens", **_rope("fwd", 64, 32, 64, 64, "half", "bands", pos="far")),
        # an fp32 layer that turns half of each head, adjacent pairs, inside wider rows
        dict(name="rope_bwd_part_f32",
             **_rope("bwd", 4100, 12, 128, 64, "pairs", "linear", "f32", pad=520, seq=1025)),
        # queries and keys of the largest configuration, inside the rows of [Q | K | V]
        dict(name="rope_large", **_rope("fwd", 16384, 64, 128, 128, "half", "base", pad=4096)),
        # a few short sentences, the shortest of them empty
        dict(name="diff_fwd_short", **_diff("fwd", 4, 77, 4, 4, 64, False, 26)),
        # an ordinary padded batch of a bidirectional model
        dict(name="diff_fwd_padded", **_diff("fwd", 16, 500, 16, 8, 64, False, 23)),
        # the largest: long causal sequences
        dict(name="diff_fwd_long", **_diff("fwd", 4, 4096, 32, 32, 128, True)),
        # the gradients of a few short causal sentences
        dict(name="diff_bwd_short", **_diff("bwd", 4, 77, 4, 2, 64, True, 13)),
        # four query heads to a key head, an odd length, a padded batch
        dict(name="diff_bwd_shared", **_diff("bwd", 2, 2031, 16, 4, 128, True, 600)),
        # the largest backward
        dict(name="diff_bwd_long", **_diff("bwd", 4, 4096, 32, 32, 128, True)),
        # the heads of a small fp32 layer
        dict(name="norm_fwd_f32", **_norm("fwd", 257, 8, 64, "f32")),
        # the heads of the largest configuration, each direction
        dict(name="norm_fwd_large", **_norm("fwd", 16384, 32, 128)),
        dict(name="norm_bwd_large", **_norm("bwd", 16384, 32, 128)),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["rope_fwd", "rope_bwd", "diff_fwd", "diff_fwd", "diff_bwd", "diff_bwd",
                       "norm_fwd", "norm_bwd"])
    op, dir = kind.split("_")
    while True:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if op == "rope":
            hd = rng.choice([32, 64, 64, 80, 128, 128, 256])
            rot = rng.choice([hd, hd, hd // 2, 2 * rng.randint(2, hd // 2)])
            c = _rope(dir, int(_log(rng, 1, 20000)), int(_log(rng, 1, 65)), hd, rot,
                      rng.choice(["half", "pairs"]), rng.choice(["none", "linear", "base", "bands"]),
                      dtype, rng.choice([0, 0, 8 * rng.randint(1, 300)]),
                      rng.choice(["row", "row", "far"]), int(_log(rng, 1, 8192)))
            most = 5.4e8
        elif op == "norm":
            c = _norm(dir, int(_log(rng, 1, 20000)), int(_log(rng, 1, 65)),
                      rng.choice([32, 64, 64, 96, 128, 128, 200, 256]), dtype)
            most = 4.2e8
        else:
            hd, seq, kv = rng.choice([64, 128]), int(_log(rng, 1, 6000)), rng.choice([1, 2, 3, 4, 8, 16])
            c = _diff(dir, max(1, int(_log(rng, 1, 16384)) // seq), seq, kv * rng.choice([1, 1, 2, 4]),
                      kv, hd, rng.random() < 0.6, rng.choice([0, 0, rng.randint(1, seq)]))
            most = 1e9
        w = work(c)
        # no dearer than the largest listed case of its kind
        if w["bytes"] <= most and w["flops"] <= {"fwd": 8e11, "bwd": 1.3e12}[dir] and (
                op != "diff" or 4 * c["nseq"] * c["heads"] * c["seq"] ** 2 <= 9e9):
            return c


def _lens(c):
    return [c["seq"] - (i * c["pad"]) % (c["seq"] + 1) for i in range(c["nseq"])]


def work(c):
    op, dir = c["kind"].split("_")
    if op == "diff":
        n, D = _lens(c), c["hd"]
        pairs = c["heads"] * sum(v * (v + 1) // 2 if c["causal"] else v * v for v in n)
        T, live, M = c["nseq"] * c["seq"], sum(n), c["heads"] * D
        qkv, stat = M + 2 * c["kv"] * D, 2 * c["heads"]
        if dir == "fwd":
            # scores of both maps, values of both; [Q | K | V] in, two outputs and lse out
            return {"flops": 6 * D * pairs, "bytes": 2 * live * qkv + T * (4 * M + 4 * stat)}
        # scores, dP, dV, dQ and dK; [Q | K | V], two outputs, their gradient and lse in
        return {"flops": 10 * D * pairs,
                "bytes": live * (2 * qkv + 6 * M + 4 * stat) + T * (2 * qkv + 4 * stat)}
    es = 4 if c["dtype"] == "f32" else 2
    n = c["T"] * c["heads"] * c["hd"]
    if op == "rope":
        return {"flops": 3 * c["T"] * c["heads"] * c["rot"],
                "bytes": 2 * n * es + (4 * c["T"] if c["pos"] == "far" else 0)}
    return {"flops": (4 if dir == "fwd" else 10) * n, "bytes": (2 if dir == "fwd" else 3) * n * es}


# ---- inputs ------------------------------------------------------------------------
def _normal(g, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def prepare(case, seed):
    c, g = dict(case), torch.Generator(device="cuda").manual_seed(int(seed) + 1)
    s = dict(case=c)
    op, dir = c["kind"].split("_")
    if op == "rope":
        # (rows of ld columns, of which the operator fills the first heads * hd)
        s["x"] = _normal(g, c["T"], c["ld"], dtype=TD[c["dtype"]])
        s["y"] = torch.zeros_like(s["x"])
        s["pos"] = None if c["pos"] == "row" else torch.randint(
            0, 1 << 17, (c["T"],), generator=g, device="cuda", dtype=torch.int32)
    elif op == "norm":
        td, M = TD[c["dtype"]], c["heads"] * c["hd"]
        s["x"] = _normal(g, c["T"], M, dtype=td)
        s["gain"] = 1 + 0.1 * torch.randn(c["hd"], generator=g, device="cuda")
        s["y"] = torch.zeros_like(s["x"])
        if dir == "bwd":
            s["dy"] = _normal(g, c["T"], M, dtype=td)
            s["dgain"] = torch.zeros(c["hd"], device="cuda")
    else:
        T, M = c["nseq"] * c["seq"], c["heads"] * c["hd"]
        s["qkv"] = _normal(g, T, M + 2 * c["kv"] * c["hd"])
        s["lam"] = 0.2 + 0.6 * torch.rand(c["heads"], generator=g, device="cuda")
        s["lens"] = torch.tensor(_lens(c), dtype=torch.int32, device="cuda") if c["pad"] else None
        if dir == "fwd":
            s["attn"] = torch.zeros(T, M, dtype=torch.bfloat16, device="cuda")
            s["attn2"] = torch.zeros_like(s["attn"])
            s["lse"] = torch.zeros(2, c["heads"], T, device="cuda")
        else:
            # what the forward kept
            f = _diff_fwd(s)
            s.update(attn=f["attn"], attn2=f["attn2"], lse=f["lse"])
            s["d_attn"] = _normal(g, T, M)
            s["d_qkv"] = torch.zeros_like(s["qkv"])
            s["delta"] = torch.zeros(2, c["heads"], T, device="cuda")
            s["d_lam"] = torch.zeros(c["heads"], device="cuda")
    return s


# ---- the plain forms ---------------------------------------------------------------
FACTOR, ORIG, LOW, HIGH, BASE = 8.0, 4096, 1.0, 32.0, 10000.0


def _mscale(c):
    return 0.1 * math.log(FACTOR) + 1.0 if c["scaling"] == "bands" else 1.0


def _rope_plain(s, sign):
    c = s["case"]
    T, H, hd, rot = c["T"], c["heads"], c["hd"], c["rot"]
    i = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    base = BASE * FACTOR ** (rot / (rot - 2)) if c["scaling"] == "base" else BASE
    th = base ** (-2 * i / rot)
    if c["scaling"] == "linear":
        th = th / FACTOR
    if c["scaling"] == "bands":
        keep = ((ORIG * th / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        th = th * (keep + (1 - keep) / FACTOR)
    pos = torch.arange(T, device="cuda") % c["seq"] if s["pos"] is None else s["pos"]
    ang = (pos.double()[:, None] * th)[:, None]  # T x 1 x rot / 2
    cs, sn = (torch.cos(ang) * _mscale(c)).float(), (torch.sin(ang) * (sign * _mscale(c))).float()
    x = s["x"][:, :H * hd].reshape(T, H, hd).float()
    if c["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        r = torch.cat([a * cs - b * sn, a * sn + b * cs], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        r = torch.stack([a * cs - b * sn, a * sn + b * cs], -1).reshape(T, H, rot)
    y = s["y"]
    y[:, :H * hd] = torch.cat([r, x[..., rot:]], -1).reshape(T, H * hd).to(y.dtype)
    return y


def _norm_plain(s, bwd):
    c = s["case"]
    x = s["x"].float().view(-1, c["heads"], c["hd"])
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    if not bwd:
        return (x * r * (SCALE * s["gain"])).view(c["T"], -1).to(s["x"].dtype)
    dy = s["dy"].float().view_as(x)
    u = dy * (SCALE * s["gain"])
    dx = r * (u - x * (r * r * (u * x).mean(-1, keepdim=True)))
    return {"dx": dx.view(c["T"], -1).to(s["x"].dtype),
            "dgain": SCALE * (dy * x * r).sum(0).sum(0)}


def _parts(s):
    """Q, K (nseq x heads x 2 x seq x d) and V (nseq x heads x seq x D) in 32 bits, the
    shared ones repeated, and the pairs that are not seen (nseq x 1 x seq x seq)."""
    c = s["case"]
    B, N, H, G, D = c["nseq"], c["seq"], c["heads"], c["kv"], c["hd"]
    x = s["qkv"].float().view(B, N, H + 2 * G, D)
    n = torch.arange(N, device="cuda")
    lens = torch.full((B,), N, device="cuda") if s["lens"] is None else s["lens"]
    pad = n >= lens[:, None]
    # (values of padded rows are whatever the batch holds)
    x = x.masked_fill(pad[..., None, None], 0.0)
    two = lambda t: t.reshape(B, N, H, 2, D // 2).permute(0, 2, 3, 1, 4).contiguous()
    k, v = (x[:, :, H + i * G:H + (i + 1) * G].repeat_interleave(H // G, 2) for i in (0, 1))
    out = pad[:, None, :, None] | pad[:, None, None, :]
    if c["causal"]:
        out = out | (n[None, :] > n[:, None])
    return two(x[:, :, :H]), two(k), v.transpose(1, 2).contiguous(), out


def _rows(s, t):
    """nseq x heads x seq x D as T x M."""
    c = s["case"]
    return t.transpose(1, 2).reshape(c["nseq"] * c["seq"], -1)


def _stat(s, t):
    """nseq x heads x 2 x seq as 2 x heads x T."""
    return t.permute(2, 1, 0, 3).reshape(2, s["case"]["heads"], -1).contiguous()


def _diff_fwd(s):
    c = s["case"]
    q, k, v, out = _parts(s)
    sc = (q @ k.transpose(-1, -2).contiguous()).mul_((c["hd"] // 2) ** -0.5)
    sc.masked_fill_(out[:, :, None], -math.inf)
    m = sc.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = sc.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    l = torch.where(l == 0, torch.ones_like(l), l)
    lse = (m + torch.log(l))[..., 0]
    p.div_(l)
    o1, o2 = p[:, :, 0] @ v, p[:, :, 1] @ v
    return {"attn": _rows(s, o1 - s["lam"][:, None, None] * o2).bfloat16(),
            "attn2": _rows(s, o2).bfloat16(), "lse": _stat(s, lse)}


def _diff_bwd(s):
    c = s["case"]
    B, N, H, G, D = c["nseq"], c["seq"], c["heads"], c["kv"], c["hd"]
    q, k, v, out = _parts(s)
    rs = (D // 2) ** -0.5
    lse = s["lse"].view(2, H, B, N).permute(2, 1, 0, 3)
    sc = (q @ k.transpose(-1, -2).contiguous()).mul_(rs).masked_fill_(out[:, :, None], -math.inf)
    p = sc.sub_(lse[..., None]).exp_()
    heads = lambda t: t.float().view(B, N, H, D).transpose(1, 2).contiguous()
    do, lam = heads(s["d_attn"]), s["lam"][:, None, None]
    seen = ~out.all(-1, keepdim=True)
    do = torch.where(seen, do, torch.zeros_like(do))
    d2 = (do * heads(s["attn2"])).sum(-1, keepdim=True)
    d1 = (do * heads(s["attn"])).sum(-1, keepdim=True) + lam * d2
    dp = do @ v.transpose(-1, -2).contiguous()
    dv = (p[:, :, 0] - lam * p[:, :, 1]).transpose(-1, -2).contiguous() @ do
    p[:, :, 0].mul_(dp - d1).mul_(rs)
    p[:, :, 1].mul_(dp.sub_(d2)).mul_(-rs * lam)
    dq, dk = p @ k, p.transpose(-1, -2).contiguous() @ q
    cols = lambda t: t.permute(0, 3, 1, 2, 4).reshape(B * N, H, D)
    share = lambda t: t.view(B * N, G, H // G, D).sum(2)
    return {"d_qkv": torch.cat([cols(dq), share(cols(dk)), share(_rows(s, dv).view(B * N, H, D))],
                               1).reshape(B * N, -1).bfloat16(),
            "d_lambda": -d2.sum((0, 2, 3))}


# ---- the framework's calls -----------------------------------------------------------
def _plan(s):
    """Shapes and scratch that a program makes once."""
    from paper_2510_00207_amd import _lib as L
    c = s["case"]
    op = c["kind"].split("_")[0]
    dt = L.F32 if c.get("dtype") == "f32" else L.BF16
    if op == "rope":
        shape = L.make_shape(c["T"], c["ld"], 8, 1, 1, 0, dtype=dt)
        kw = dict(none={}, linear=dict(factor=FACTOR), base=dict(factor=FACTOR),
                  bands=dict(factor=FACTOR, orig_len=ORIG, low=LOW, high=HIGH))[c["scaling"]]
        return L, shape, L.make_rope_shape(c["heads"], c["hd"], c["rot"], c["seq"],
                                           layout=c["layout"], base=BASE, scaling=c["scaling"],
                                           mscale=_mscale(c), **kw)
    T = c["nseq"] * c["seq"] if op == "diff" else c["T"]
    shape = L.make_shape(T, c["heads"] * c["hd"], 8, 1, 1, 0, dtype=dt)
    if op == "norm":
        sub = L.make_norm_shape(c["heads"], c["hd"], eps=EPS, scale=SCALE)
        n = L.flowmoe_head_norm_ws_bytes(shape, sub)
    else:
        sub = L.make_diff_shape(c["seq"], c["heads"], c["kv"], c["hd"], c["causal"])
        n = L.flowmoe_diff_attention_ws_bytes(shape, sub)
    s["ws"], s["ws_bytes"] = torch.empty(max(1, n), dtype=torch.uint8, device="cuda"), n
    return L, shape, sub


def _own(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    L, shape, sub = s["plan"]
    kind = s["case"]["kind"]
    if kind == "rope_fwd":
        L.flowmoe_rope_fwd(shape, sub, s["x"], s["pos"], s["y"])
        return s["y"]
    if kind == "rope_bwd":
        L.flowmoe_rope_bwd(shape, sub, s["x"], s["pos"], s["y"])
        return s["y"]
    if kind == "norm_fwd":
        L.flowmoe_head_norm_fwd(shape, sub, s["x"], s["gain"], s["y"])
        return s["y"]
    if kind == "norm_bwd":
        L.flowmoe_head_norm_bwd(shape, sub, s["x"], s["gain"], s["dy"], s["y"], s["dgain"], False,
                                s["ws"], s["ws_bytes"])
        return {"dx": s["y"], "dgain": s["dgain"]}
    if kind == "diff_fwd":
        L.flowmoe_diff_attention_fwd(shape, sub, s["qkv"], s["lam"], s["lens"], s["attn"],
                                     s["attn2"], s["lse"])
        return {n: s[n] for n in ("attn", "attn2", "lse")}
    L.flowmoe_diff_attention_bwd(shape, sub, s["qkv"], s["lam"], s["lens"], s["attn"], s["attn2"],
                                 s["lse"], s["d_attn"], s["d_qkv"], s["delta"], s["d_lam"], False,
                                 s["ws"], s["ws_bytes"])
    return {"d_qkv": s["d_qkv"], "d_lambda": s["d_lam"]}


def run(s):
    if own:
        return _own(s)
    kind = s["case"]["kind"]
    if kind.startswith("rope"):
        return _rope_plain(s, 1 if kind == "rope_fwd" else -1)
    if kind.startswith("norm"):
        return _norm_plain(s, kind == "norm_bwd")
    return _diff_fwd(s) if kind == "diff_fwd" else _diff_bwd(s)


# ---- from the definitions, in 64 bits --------------------------------------------------
def _exact_rope(c, s, back):
    T, H, hd, rot = c["T"], c["heads"], c["hd"], c["rot"]
    freq = []
    for j in range(rot // 2):
        b = BASE * (FACTOR ** (rot / (rot - 2.0)) if c["scaling"] == "base" else 1.0)
        f = math.exp(-2.0 * j / rot * math.log(b))
        if c["scaling"] == "linear":
            f /= FACTOR
        elif c["scaling"] == "bands":
            turns = ORIG * f / (2 * math.pi)
            w = min(1.0, max(0.0, (turns - LOW) / (HIGH - LOW)))
            f = w * f + (1 - w) * f / FACTOR
        freq.append(f)
    freq = torch.tensor(freq, dtype=torch.float64, device="cuda")
    pos = (torch.arange(T, device="cuda") % c["seq"] if s["pos"] is None else s["pos"]).double()
    # the pair as a complex number, times m e^(+- i phi)
    turn = torch.polar(torch.full((T, rot // 2), _mscale(c), dtype=torch.float64, device="cuda"),
                       (-1.0 if back else 1.0) * pos[:, None] * freq[None, :])
    y = s["y"].double()
    v = y[:, :H * hd].unflatten(1, (H, hd))
    x = s["x"].double()[:, :H * hd].unflatten(1, (H, hd))
    i = torch.arange(rot // 2, device="cuda")
    ia, ib = (i, i + rot // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
    z = torch.complex(x[..., ia], x[..., ib]) * turn[:, None]
    v.copy_(x)
    v[..., ia], v[..., ib] = z.real, z.imag
    return y


def _exact_norm(c, s, back):
    x, g = s["x"].double().unflatten(1, (c["heads"], c["hd"])), SCALE * s["gain"].double()
    rms = torch.sqrt(x.pow(2).sum(-1, keepdim=True) / c["hd"] + EPS)
    if not back:
        return (x / rms * g).flatten(1)
    dy = s["dy"].double().view_as(x)
    n = x / rms
    u = dy * g
    return {"dx": ((u - n * (u * n).sum(-1, keepdim=True) / c["hd"]) / rms).flatten(1),
            "dgain": SCALE * (dy * n).sum((0, 1))}


def _exact_diff(c, s, back):
    N, H, G, D = c["seq"], c["heads"], c["kv"], c["hd"]
    d, T = D // 2, c["nseq"] * N
    z = lambda *sh: torch.zeros(*sh, dtype=torch.float64, device="cuda")
    lam = s["lam"].double()
    attn, attn2, lse = z(T, H * D), z(T, H * D), z(2, H, T)
    dqkv, dlam = z(T, (H + 2 * G) * D), z(H)
    for b, n in enumerate(_lens(c)):
        rows = slice(b * N, b * N + n)
        x = s["qkv"][rows].double()
        for h in range(H):
            g = h // (H // G)
            cq, ck, cv = h * D, (H + g) * D, (H + G + g) * D
            v = x[:, cv:cv + D]
            col = slice(h * D, h * D + D)
            a = []
            for i in (0, 1):
                t = x[:, cq + i * d:cq + i * d + d] @ x[:, ck + i * d:ck + i * d + d].T / math.sqrt(d)
                if c["causal"]:
                    t = t.masked_fill(torch.ones_like(t, dtype=torch.bool).triu(1), -math.inf)
                if not back:
                    lse[i, h, rows] = torch.logsumexp(t, 1) if n else lse[i, h, rows]
                    a.append(torch.softmax(t, 1))
                else:
                    a.append(torch.exp(t - s["lse"][i, h, rows].double()[:, None]))
            if not back:
                o2 = a[1] @ v
                attn2[rows, col] = o2
                attn[rows, col] = a[0] @ v - lam[h] * o2
                continue
            do = s["d_attn"][rows, col].double()
            e2 = (do * s["attn2"][rows, col].double()).sum(1, keepdim=True)
            e1 = (do * s["attn"][rows, col].double()).sum(1, keepdim=True) + lam[h] * e2
            dlam[h] -= e2.sum()
            dp = do @ v.T
            dqkv[rows, cv:cv + D] += (a[0] - lam[h] * a[1]).T @ do
            for i, ds in ((0, a[0] * (dp - e1)), (1, -lam[h] * a[1] * (dp - e2))):
                q0, k0 = cq + i * d, ck + i * d
                dqkv[rows, q0:q0 + d] = ds @ x[:, k0:k0 + d] / math.sqrt(d)
                dqkv[rows, k0:k0 + d] += ds.T @ x[:, q0:q0 + d] / math.sqrt(d)
    if back:
        return {"d_qkv": dqkv, "d_lambda": dlam}
    return {"attn": attn, "attn2": attn2, "lse": lse}


def exact(case, seed):
    op, dir = case["kind"].split("_")
    if op == "diff" and case["nseq"] * case["heads"] > 20000:
        return None  # (a few launches for each head of each sequence)
    s = prepare(case, seed)
    fn = {"rope": _exact_rope, "norm": _exact_norm, "diff": _exact_diff}[op]
    return fn(dict(case), s, dir == "bwd")
