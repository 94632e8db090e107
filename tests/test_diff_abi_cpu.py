"""Refusals of the differential attention block's calls, before anything is enqueued
(no GPU needed; the fake addresses are never dereferenced)."""
import pytest

from paper_2510_00207_amd import _lib as L

FAKE = 0x10000
BIG = 1 << 40  # a workspace of any size


def refused(status, text, call):
    with pytest.raises(L.FlowMoEError) as ei:
        call()
    assert ei.value.status == status and text in str(ei.value), str(ei.value)


def calls(s, sub):
    """Every entry point that takes the sub-shape's type, with valid pointers."""
    return {
        L.RopeShape: [lambda: L.flowmoe_rope_fwd(s, sub, FAKE, None, FAKE, stream=0),
                      lambda: L.flowmoe_rope_bwd(s, sub, FAKE, FAKE, FAKE, stream=0)],
        L.NormShape: [lambda: L.flowmoe_head_norm_fwd(s, sub, FAKE, None, FAKE, stream=0),
                      lambda: L.flowmoe_head_norm_bwd(s, sub, FAKE, None, FAKE, FAKE, FAKE, 0, FAKE,
                                                      BIG, stream=0)],
        L.DiffShape: [lambda: L.flowmoe_diff_attention_fwd(s, sub, FAKE, FAKE, None, FAKE, FAKE, FAKE,
                                                           stream=0),
                      lambda: L.flowmoe_diff_attention_bwd(s, sub, *[FAKE] * 10, 0, FAKE, BIG,
                                                           stream=0)],
    }[type(sub)]


def shape(T=64, M=256, dtype=L.BF16):
    return L.make_shape(T, M, 8, 1, 1, 0, dtype)


def rope(**kw):
    a = dict(heads=2, head_dim=64, rot_dim=64, seq_len=16)
    a.update(kw)
    return L.make_rope_shape(**a)


@pytest.mark.parametrize("sub", [rope(), L.make_norm_shape(4, 64),
                                 L.make_diff_shape(16, 4, 2, 64, True)])
def test_shapes_refused(flowmoe_lib, sub):
    for s, status, text in [(shape(T=-1), L.ERR_INVALID, "T = -1"),
                            (shape(M=0), L.ERR_INVALID, "M = 0"),
                            (shape(M=252), L.ERR_INVALID, "multiple of 8"),
                            (shape(dtype=5), L.ERR_INVALID, "dtype 5"),
                            (shape(T=1 << 30, M=1 << 20), L.ERR_UNSUPPORTED, "too large")]:
        for call in calls(s, sub):
            refused(status, text, call)


BANDS = dict(scaling="bands", factor=4.0, orig_len=100.0)


@pytest.mark.parametrize("kw,status,text", [
    (dict(heads=0), L.ERR_INVALID, "heads"), (dict(heads=5), L.ERR_INVALID, "heads * head_dim"),
    (dict(heads=1 << 30), L.ERR_INVALID, "heads * head_dim"),
    (dict(head_dim=60), L.ERR_INVALID, "head_dim"), (dict(head_dim=0), L.ERR_INVALID, "head_dim"),
    (dict(head_dim=520, rot_dim=8), L.ERR_UNSUPPORTED, "head_dim"),
    (dict(rot_dim=0), L.ERR_INVALID, "rot_dim"), (dict(rot_dim=33), L.ERR_INVALID, "rot_dim"),
    (dict(rot_dim=66), L.ERR_INVALID, "rot_dim"), (dict(layout=2), L.ERR_INVALID, "layout"),
    (dict(scaling=4), L.ERR_INVALID, "scaling"), (dict(scaling=-1), L.ERR_INVALID, "scaling"),
    (dict(seq_len=0), L.ERR_INVALID, "seq_len"), (dict(base=1.0), L.ERR_INVALID, "base"),
    (dict(base=float("nan")), L.ERR_INVALID, "base"), (dict(base=float("inf")), L.ERR_INVALID, "base"),
    (dict(mscale=float("inf")), L.ERR_INVALID, "mscale"),
    (dict(scaling="linear", factor=0.5), L.ERR_INVALID, "factor"),
    (dict(scaling="base", factor=float("nan")), L.ERR_INVALID, "factor"),
    (dict(scaling="base", factor=2.0, rot_dim=2), L.ERR_INVALID, "rot_dim > 2"),
    (dict(scaling="base", factor=1e300, base=1e300), L.ERR_INVALID, "too large"),
    (dict(BANDS, orig_len=0.0), L.ERR_INVALID, "orig_len"),
    (dict(BANDS, low=32.0), L.ERR_INVALID, "low"),
    (dict(BANDS, high=float("nan")), L.ERR_INVALID, "low"),
])
def test_rope_refusals(flowmoe_lib, kw, status, text):
    for call in calls(shape(), rope(**kw)):
        refused(status, text, call)


@pytest.mark.parametrize("mscale", [1e39, -1e39, 1e300, float("nan"), 1e-40, -1e-46, 5e-324])
def test_rope_mscale_as_the_kernel_holds_it_refused(flowmoe_lib, mscale):
    """Values that a float would hold as infinite, denormal or zero."""
    for call in calls(shape(), rope(mscale=mscale)):
        refused(L.ERR_INVALID, "mscale", call)


@pytest.mark.parametrize("sub,status,text", [
    (L.make_norm_shape(3, 64), L.ERR_INVALID, "heads * head_dim"),
    (L.make_norm_shape(0, 64), L.ERR_INVALID, "heads * head_dim"),
    (L.make_norm_shape(64, 4), L.ERR_INVALID, "head_dim"),
    (L.make_norm_shape(4, 64, eps=0.0), L.ERR_INVALID, "eps"),
    (L.make_norm_shape(4, 64, eps=1e-40), L.ERR_INVALID, "eps"),
    (L.make_norm_shape(4, 64, eps=float("nan")), L.ERR_INVALID, "eps"),
    (L.make_norm_shape(4, 64, scale=float("inf")), L.ERR_INVALID, "scale"),
    (L.make_diff_shape(16, 4, 2, 32, True), L.ERR_UNSUPPORTED, "head_dim"),
    (L.make_diff_shape(16, 2, 2, 64, True), L.ERR_INVALID, "heads * head_dim"),
    (L.make_diff_shape(16, 4, 3, 64, True), L.ERR_INVALID, "kv_heads"),
    (L.make_diff_shape(16, 4, 0, 64, True), L.ERR_INVALID, "kv_heads"),
    (L.make_diff_shape(16, 4, 8, 64, True), L.ERR_INVALID, "kv_heads"),
    (L.make_diff_shape(0, 4, 2, 64, True), L.ERR_INVALID, "seq_len"),
    (L.make_diff_shape(24, 4, 2, 64, True), L.ERR_INVALID, "whole number of sequences"),
    (L.DiffShape(16, 4, 2, 64, 2), L.ERR_INVALID, "causal"),
])
def test_norm_and_diff_refusals(flowmoe_lib, sub, status, text):
    for call in calls(shape(), sub):
        refused(status, text, call)


def test_sizes_refused(flowmoe_lib):
    refused(L.ERR_UNSUPPORTED, "head_dim", lambda: L.flowmoe_head_norm_fwd(
        shape(M=520), L.make_norm_shape(1, 520), FAKE, None, FAKE, stream=0))
    d = L.make_diff_shape(16, 4, 2, 64, True)
    refused(L.ERR_UNSUPPORTED, "BF16", lambda: L.flowmoe_diff_attention_fwd(
        shape(dtype=L.F32), d, FAKE, FAKE, None, FAKE, None, None, stream=0))
    wide = L.make_diff_shape(16, 1 << 16, 1, 64, True)
    refused(L.ERR_UNSUPPORTED, "too large", lambda: L.flowmoe_diff_attention_fwd(
        shape(T=16, M=1 << 22), wide, FAKE, FAKE, None, FAKE, None, None, stream=0))
    # 2^23 tiles of 512 threads are more than a grid holds
    many = L.make_diff_shape(1, 1, 1, 64, True)
    refused(L.ERR_UNSUPPORTED, "too many", lambda: L.flowmoe_diff_attention_fwd(
        shape(T=1 << 23, M=64), many, FAKE, FAKE, None, FAKE, None, None, stream=0))
    refused(L.ERR_UNSUPPORTED, "too large", lambda: L.flowmoe_rope_fwd(
        shape(T=1, M=1 << 27), rope(), FAKE, None, FAKE, stream=0))


def test_null_and_misaligned_refused(flowmoe_lib):
    s, r, n, d = shape(), rope(), L.make_norm_shape(4, 64), L.make_diff_shape(16, 4, 2, 64, True)
    inv = L.ERR_INVALID

    def each(fn, args, checks):
        for i, (name, null_ok, align) in enumerate(checks):
            if not null_ok:
                refused(inv, f"{name} is null", lambda: fn(*args[:i], None, *args[i + 1:]))
            refused(inv, f"{name} is not {align}-byte aligned",
                    lambda: fn(*args[:i], FAKE + align // 2, *args[i + 1:]))

    each(lambda *a: L.flowmoe_rope_fwd(s, r, *a, stream=0), [FAKE] * 3,
         [("x", 0, 16), ("positions", 1, 4), ("y", 0, 16)])
    each(lambda *a: L.flowmoe_rope_bwd(s, r, *a, stream=0), [FAKE] * 3,
         [("dy", 0, 16), ("positions", 1, 4), ("dx", 0, 16)])
    each(lambda *a: L.flowmoe_head_norm_fwd(s, n, *a, stream=0), [FAKE] * 3,
         [("x", 0, 16), ("gain", 1, 4), ("y", 0, 16)])
    each(lambda *a: L.flowmoe_head_norm_bwd(s, n, *a, 0, FAKE, BIG, stream=0), [FAKE] * 5,
         [("x", 0, 16), ("gain", 1, 4), ("dy", 0, 16), ("dx", 0, 16), ("dgain", 1, 4)][:4])
    each(lambda *a: L.flowmoe_diff_attention_fwd(s, d, *a, stream=0), [FAKE] * 6,
         [("qkv", 0, 16), ("lambda", 0, 4), ("lens", 1, 4), ("attn", 0, 16), ("attn2", 1, 16),
          ("lse", 1, 4)])
    each(lambda *a: L.flowmoe_diff_attention_bwd(s, d, *a, 0, FAKE, BIG, stream=0), [FAKE] * 10,
         [("qkv", 0, 16), ("lambda", 0, 4), ("lens", 1, 4), ("attn", 0, 16), ("attn2", 0, 16),
          ("lse", 0, 4), ("d_attn", 0, 16), ("d_qkv", 0, 16), ("delta", 0, 4), ("d_lambda", 0, 4)])
    refused(inv, "dgain is not 4-byte aligned", lambda: L.flowmoe_head_norm_bwd(
        s, n, FAKE, None, FAKE, FAKE, FAKE + 2, 0, FAKE, BIG, stream=0))


def test_workspaces_checked(flowmoe_lib):
    s, n = shape(T=1024), L.make_norm_shape(4, 64)
    need = L.flowmoe_head_norm_ws_bytes(s, n)
    assert need >= 64 * 4
    for ws, have in ((FAKE, need - 1), (None, need)):
        refused(L.ERR_WORKSPACE, "flowmoe_head_norm_bwd", lambda: L.flowmoe_head_norm_bwd(
            s, n, FAKE, None, FAKE, FAKE, FAKE, 0, ws, have, stream=0))
    assert L.flowmoe_head_norm_ws_bytes(shape(M=0), n) == 0
    assert L.flowmoe_diff_attention_ws_bytes(s, L.make_diff_shape(16, 4, 3, 64, True)) == 0


def test_no_tokens(flowmoe_lib):
    """Nothing to do and no tensor needed, but for the backward's sums."""
    s, d = shape(T=0), L.make_diff_shape(16, 4, 2, 64, True)
    L.flowmoe_rope_fwd(s, rope(), None, None, None, stream=0)
    L.flowmoe_rope_bwd(s, rope(), None, None, None, stream=0)
    L.flowmoe_head_norm_fwd(s, L.make_norm_shape(4, 64), None, None, None, stream=0)
    L.flowmoe_head_norm_bwd(s, L.make_norm_shape(4, 64), *[None] * 5, 0, stream=0)
    L.flowmoe_diff_attention_fwd(s, d, *[None] * 6, stream=0)
    refused(L.ERR_INVALID, "d_lambda is null", lambda: L.flowmoe_diff_attention_bwd(
        s, d, *[None] * 10, 0, stream=0))


def mha_bufs(**kw):
    b = {n: FAKE for n in L._DIFF_MHA_FIELDS}
    b.update(ws_bytes=BIG, **kw)
    return L.diff_mha_bufs(**b)


def test_diff_mha_refusals(flowmoe_lib):
    s, d, n = shape(), L.make_diff_shape(16, 4, 2, 64, True), L.make_norm_shape(4, 64)
    r = L.make_rope_shape(12, 32, 32, 16)
    both = lambda *a: [lambda: L.flowmoe_diff_mha_fwd(*a, stream=0),
                       lambda: L.flowmoe_diff_mha_bwd(*a, 0, stream=0)]
    for rr, text in ((L.make_rope_shape(8, 32, 32, 16), "Q's and K's"),
                     (L.make_rope_shape(6, 64, 32, 16), "Q's and K's"),
                     (L.make_rope_shape(12, 32, 32, 64), "seq_len"),
                     (L.make_rope_shape(12, 32, 34, 16), "rot_dim")):
        for call in both(s, d, rr, n, mha_bufs()):
            refused(L.ERR_INVALID, text, call)
    for nn, text in ((L.make_norm_shape(2, 128), "norm's heads"), (L.make_norm_shape(4, 64, eps=-1.0), "eps")):
        for call in both(s, d, r, nn, mha_bufs()):
            refused(L.ERR_INVALID, text, call)
    for call in both(shape(dtype=L.F32), d, r, n, mha_bufs()):
        refused(L.ERR_UNSUPPORTED, "BF16", call)
    nullable = ("gain", "positions", "lens", "dgain", "ws")
    fwd = ("in", "w_qkv", "w_o", "lambda", "qkv", "attn", "attn2", "lse", "normed", "out")
    names = [x for x in L._DIFF_MHA_FIELDS if x not in nullable]
    for x in names:
        calls_ = both(s, d, r, n, mha_bufs(**{x: None}))
        if x in fwd:
            refused(L.ERR_INVALID, f"bufs->{x} is null", calls_[0])
        if x != "out":
            refused(L.ERR_INVALID, f"bufs->{x} is null", calls_[1])
    for x in ("gain", "positions", "lens"):
        for call in both(s, d, r, n, mha_bufs(**{x: FAKE + 2})):
            refused(L.ERR_INVALID, f"bufs->{x} is not 4-byte aligned", call)
    s = shape(T=1024)
    need = L.flowmoe_diff_mha_ws_bytes(s, d, n)
    assert need >= 64 * 4 and need >= max(L.flowmoe_diff_attention_ws_bytes(s, d), L.flowmoe_head_norm_ws_bytes(s, n))
    b = mha_bufs()
    b.ws_bytes = need - 1
    refused(L.ERR_WORKSPACE, "flowmoe_diff_mha_bwd", lambda: L.flowmoe_diff_mha_bwd(s, d, r, n, b, 0,
                                                                                    stream=0))
    with pytest.raises(KeyError):
        L.diff_mha_bufs(w1=None)
    # no tokens: the forward has nothing to do, the backward's sums stay to be written
    L.flowmoe_diff_mha_fwd(shape(T=0), d, r, n, L.diff_mha_bufs(), stream=0)
    refused(L.ERR_INVALID, "dw_qkv is null", lambda: L.flowmoe_diff_mha_bwd(
        shape(T=0), d, r, n, L.diff_mha_bufs(), 0, stream=0))


def test_more_tokens_than_a_grid_holds_refused(flowmoe_lib):
    """Four tokens to a block of 256 threads: from 2^26 of them on HIP would cut a grid off."""
    with pytest.raises(L.FlowMoEError) as ei:
        L.flowmoe_rope_fwd(shape(T=1 << 26, M=2048), L.make_rope_shape(32, 64, 64, 16), FAKE, None, FAKE,
                           stream=0)
    assert ei.value.status == L.ERR_HIP and "invalid configuration" in str(ei.value)


def test_block_of_more_tokens_than_positions_reach_refused(flowmoe_lib):
    """Where the positions' grid would be cut off the block enqueues nothing, its first
    products neither."""
    T = 1 << 26
    s, d, n = shape(T=T, M=256), L.make_diff_shape(4096, 2, 2, 128, True), L.make_norm_shape(2, 128)
    r = L.make_rope_shape(8, 64, 64, 4096)
    for call in (lambda: L.flowmoe_diff_mha_fwd(s, d, r, n, mha_bufs(), stream=0),
                 lambda: L.flowmoe_diff_mha_bwd(s, d, r, n, mha_bufs(), 0, stream=0)):
        refused(L.ERR_HIP, "invalid configuration", call)
