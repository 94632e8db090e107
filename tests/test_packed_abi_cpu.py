"""Refusals of the packed attention's, the layer norm's and the embedding's calls, before
anything is enqueued (no GPU needed; the fake addresses are never dereferenced)."""
import ctypes
import os
import re

import pytest

from paper_2510_00207_amd import _lib as L

FAKE = 0x10000
BIG = 1 << 40  # a workspace of any size


def refused(status, text, call):
    with pytest.raises(L.FlowMoEError) as ei:
        call()
    assert ei.value.status == status and text in str(ei.value), str(ei.value)


def shape(T=64, M=256, dtype=L.BF16):
    return L.make_shape(T, M, 8, 1, 1, 0, dtype)


PACKED, EMBED = L.make_packed_shape(3, 4, 2, 64, True), L.make_embed_shape(100)
MHA = [n for n in L._PACKED_MHA_FIELDS if n != "ws"]


def mha_bufs(**kw):
    a = {n: FAKE for n in MHA}
    a.update(ws=FAKE, ws_bytes=BIG)
    a["inp"] = a.pop("in")
    a.update(kw)
    return L.packed_mha_bufs(**a)


def calls(s, sub):
    """Every entry point of a kind, with valid pointers."""
    if isinstance(sub, L.PackedShape):
        return [lambda: L.flowmoe_packed_attention_fwd(s, sub, FAKE, FAKE, FAKE, FAKE, stream=0),
                lambda: L.flowmoe_packed_attention_bwd(s, sub, *[FAKE] * 7, FAKE, BIG, stream=0),
                lambda: L.flowmoe_packed_mha_fwd(s, sub, None, mha_bufs(), stream=0),
                lambda: L.flowmoe_packed_mha_bwd(s, sub, None, mha_bufs(), 0, stream=0)]
    if isinstance(sub, L.EmbedShape):
        return [lambda: L.flowmoe_embed_fwd(s, sub, FAKE, FAKE, FAKE, stream=0),
                lambda: L.flowmoe_embed_bwd(s, sub, FAKE, FAKE, FAKE, 0, FAKE, BIG, stream=0)]
    return [lambda: L.flowmoe_layer_norm_fwd(s, sub, FAKE, None, None, None, None, FAKE, stream=0),
            lambda: L.flowmoe_layer_norm_bwd(s, sub, FAKE, None, FAKE, None, FAKE, FAKE, FAKE, 0,
                                             FAKE, BIG, stream=0)]


@pytest.mark.parametrize("sub", [PACKED, EMBED, 1e-5])
def test_shapes_refused(flowmoe_lib, sub):
    for s, status, text in [(shape(T=-1), L.ERR_INVALID, "T = -1"),
                            (shape(M=0), L.ERR_INVALID, "M = 0"),
                            (shape(M=252), L.ERR_INVALID, "multiple of 8"),
                            (shape(dtype=5), L.ERR_INVALID, "dtype 5"),
                            (shape(T=1 << 30, M=1 << 20), L.ERR_UNSUPPORTED, "too large")]:
        for call in calls(s, sub):
            refused(status, text, call)


@pytest.mark.parametrize("sub,status,text", [
    (L.make_packed_shape(3, 4, 2, 32, True), L.ERR_UNSUPPORTED, "head_dim"),
    (L.make_packed_shape(3, 2, 2, 64, True), L.ERR_INVALID, "heads * head_dim"),
    (L.make_packed_shape(3, 0, 1, 64, True), L.ERR_INVALID, "heads * head_dim"),
    (L.make_packed_shape(3, 4, 3, 64, True), L.ERR_INVALID, "kv_heads"),
    (L.make_packed_shape(3, 4, 0, 64, True), L.ERR_INVALID, "kv_heads"),
    (L.make_packed_shape(3, 4, 8, 64, True), L.ERR_INVALID, "kv_heads"),
    (L.make_packed_shape(-1, 4, 2, 64, True), L.ERR_INVALID, "nseq"),
    (L.make_packed_shape(1 << 30, 4, 2, 64, True), L.ERR_UNSUPPORTED, "too many attention tiles"),
    (L.PackedShape(3, 4, 2, 64, 2), L.ERR_INVALID, "causal"),
    (L.make_embed_shape(0), L.ERR_INVALID, "vocab"), (L.make_embed_shape(-5), L.ERR_INVALID, "vocab"),
    (L.make_embed_shape(1 << 30), L.ERR_UNSUPPORTED, "too large"),
    (L.make_embed_shape(9, float("inf")), L.ERR_INVALID, "scale"),
    (L.make_embed_shape(9, float("nan")), L.ERR_INVALID, "scale"),
    (0.0, L.ERR_INVALID, "eps"), (-1e-5, L.ERR_INVALID, "eps"), (1e-40, L.ERR_INVALID, "eps"),
    (float("nan"), L.ERR_INVALID, "eps"), (float("inf"), L.ERR_INVALID, "eps"),
])
def test_refusals(flowmoe_lib, sub, status, text):
    s = shape(T=1 << 20, M=4096) if isinstance(sub, L.EmbedShape) and sub.vocab == 1 << 30 else shape()
    for call in calls(s, sub):
        refused(status, text, call)


def test_types_and_widths(flowmoe_lib):
    for call in calls(shape(dtype=L.F32), PACKED):
        refused(L.ERR_UNSUPPORTED, "BF16", call)
    for call in calls(shape(T=4, M=1 << 22), L.make_packed_shape(1, 1 << 16, 1, 64, True)):
        refused(L.ERR_UNSUPPORTED, "too large", call)
    for call in calls(shape(M=16392), 1e-5):
        refused(L.ERR_UNSUPPORTED, "16384", call)


def test_pointers(flowmoe_lib):
    s, n = shape(), 0
    args = ["qkv", "starts", "attn", "lse"]
    for i, name in enumerate(args):
        a = [FAKE] * 4
        a[i] = None
        refused(L.ERR_INVALID, name, lambda: L.flowmoe_packed_attention_fwd(s, PACKED, *a, stream=0))
        a[i] = FAKE + 2
        refused(L.ERR_INVALID, name, lambda: L.flowmoe_packed_attention_fwd(s, PACKED, *a, stream=0))
    args = ["qkv", "starts", "attn", "lse", "d_attn", "d_qkv", "delta"]
    for i, name in enumerate(args):
        a = [FAKE] * 7
        a[i] = None
        refused(L.ERR_INVALID, name,
                lambda: L.flowmoe_packed_attention_bwd(s, PACKED, *a, FAKE, BIG, stream=0))
    bwd = {"d_out", "d_attn", "d_qkv", "delta", "d_in", "dw_qkv", "dw_o"}
    rope = L.make_rope_shape(6, 64, 64, 1)
    for name in MHA:
        b = mha_bufs(**{"inp" if name == "in" else name: FAKE + 2})
        what = f"bufs->{name}"
        refused(L.ERR_INVALID, what, lambda: L.flowmoe_packed_mha_bwd(s, PACKED, rope, b, 0, stream=0)
                if name in bwd else L.flowmoe_packed_mha_fwd(s, PACKED, rope, b, stream=0))
    for rp, text in [(L.make_rope_shape(6, 32, 32, 1), "are not Q's and K's"),
                     (L.make_rope_shape(4, 64, 64, 1), "are not Q's and K's"),
                     (L.make_rope_shape(6, 64, 65, 1), "rot_dim")]:
        refused(L.ERR_INVALID, text, lambda: L.flowmoe_packed_mha_fwd(s, PACKED, rp, mha_bufs(), stream=0))
    refused(L.ERR_INVALID, "positions",
            lambda: L.flowmoe_packed_mha_fwd(s, PACKED, rope, mha_bufs(positions=None), stream=0))
    for i, name in enumerate(["x", "res", "gain", "bias", "sum", "y"]):
        a = [FAKE] * 4 + [2 * FAKE, FAKE]
        a[i] = FAKE + 2
        refused(L.ERR_INVALID, name, lambda: L.flowmoe_layer_norm_fwd(s, 1e-5, *a, stream=0))
    refused(L.ERR_INVALID, "one buffer", lambda: L.flowmoe_layer_norm_fwd(
        s, 1e-5, FAKE, FAKE, None, None, FAKE, FAKE, stream=0))
    for i, name in enumerate(["x", "gain", "dy", "d_sum", "dx", "dgain", "dbias"]):
        a = [FAKE] * 7
        a[i] = FAKE + 2
        refused(L.ERR_INVALID, name,
                lambda: L.flowmoe_layer_norm_bwd(s, 1e-5, *a, 0, FAKE, BIG, stream=0))
    for i, name in enumerate(["ids", "table", "y"]):
        a = [FAKE] * 3
        a[i] = None
        refused(L.ERR_INVALID, name, lambda: L.flowmoe_embed_fwd(s, EMBED, *a, stream=0))
    for i, name in enumerate(["ids", "dy", "dtable"]):
        a = [FAKE] * 3
        a[i] = FAKE + 2
        refused(L.ERR_INVALID, name,
                lambda: L.flowmoe_embed_bwd(s, EMBED, *a, 0, FAKE, BIG, stream=0))


def test_workspaces(flowmoe_lib):
    s = shape(T=4096)
    for n, call in [
        (L.flowmoe_layer_norm_ws_bytes(s), lambda ws, n: L.flowmoe_layer_norm_bwd(
            s, 1e-5, FAKE, None, FAKE, None, FAKE, FAKE, FAKE, 0, ws, n, stream=0)),
        (L.flowmoe_embed_ws_bytes(s, EMBED), lambda ws, n: L.flowmoe_embed_bwd(
            s, EMBED, FAKE, FAKE, FAKE, 0, ws, n, stream=0))]:
        assert n > 0
        refused(L.ERR_WORKSPACE, str(n), lambda: call(FAKE, n - 1))
        refused(L.ERR_WORKSPACE, "null", lambda: call(None, n))
        refused(L.ERR_INVALID, "ws", lambda: call(FAKE + 8, n))
    bad = shape(M=100)
    assert L.flowmoe_layer_norm_ws_bytes(bad) == 0
    assert L.flowmoe_embed_ws_bytes(bad, EMBED) == 0
    assert L.flowmoe_packed_attention_ws_bytes(bad, PACKED) == 0
    assert L.flowmoe_packed_mha_ws_bytes(bad, PACKED) == 0


def test_nothing_to_do(flowmoe_lib):
    """Calls without tokens take null pointers and enqueue nothing."""
    s = shape(T=0)
    L.flowmoe_packed_attention_fwd(s, PACKED, None, None, None, None, stream=0)
    L.flowmoe_packed_attention_bwd(s, PACKED, *[None] * 7, stream=0)
    L.flowmoe_packed_mha_fwd(s, PACKED, None, L.packed_mha_bufs(), stream=0)
    L.flowmoe_layer_norm_fwd(s, 1e-5, *[None] * 6, stream=0)
    L.flowmoe_layer_norm_bwd(s, 1e-5, *[None] * 7, 0, stream=0)
    L.flowmoe_embed_fwd(s, EMBED, None, None, None, stream=0)
    L.flowmoe_embed_bwd(s, EMBED, None, None, FAKE, 1, stream=0)


def test_binding_matches_header(flowmoe_lib):
    """The structs' fields and the trace kinds, in the header's order."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    h = open(os.path.join(root, "include", "flowmoe.h")).read()
    h = re.sub(r"/\*.*?\*/", "", h, flags=re.S)

    def fields(name):
        body = h[:h.index("} " + name)]
        body = body[body.rindex("{") + 1:]
        return re.findall(r"(\w+)\s*[;,]", body)

    assert fields("flowmoe_packed_mha_bufs_t") == [n for n, _ in L.PackedMhaBufs._fields_]
    assert fields("flowmoe_packed_shape_t") == [n for n, _ in L.PackedShape._fields_]
    assert fields("flowmoe_embed_shape_t") == [n for n, _ in L.EmbedShape._fields_]
    kinds = dict((int(v), n.lower()) for n, v in re.findall(r"FLOWMOE_K_(\w+) = (\d+)", h))
    assert [kinds[i] for i in range(32, len(L.K_NAMES))] == L.K_NAMES[32:]
    assert max(kinds) + 1 == len(L.K_NAMES) <= 64


def test_trace_mask_of_64_bits(flowmoe_lib):
    refused(L.ERR_INVALID, "pairs", lambda: L.flowmoe_trace_start64(None, None, -1, 1 << 33))
    L.flowmoe_trace_start64(None, None, 0, (1 << 64) - 1)
    assert L.flowmoe_trace_stop() == 0
    assert L.kind_mask(["layer_norm", "embed"]) == (1 << 32) | (1 << 34)
    with pytest.raises(ValueError, match="trace_start64"):  # (ctypes would cut it to 32 bits)
        L.flowmoe_trace_start(None, None, 0, L.kind_mask(["layer_norm"]))
    assert ctypes.sizeof(L.PackedMhaBufs) == 8 * (len(L._PACKED_MHA_FIELDS) + 1)
