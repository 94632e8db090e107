"""Masks of flowmoe_trace_start: what programs passed while there were 32 kinds is taken, and a
kind past 31 beside one of the first 32 is traced, not cut off. No GPU needed but for the last
test."""
import ctypes

import pytest

from paper_2510_00207_amd import _lib as L

ALL = (1 << 64) - 1


@pytest.fixture
def entries(flowmoe_lib, monkeypatch):
    """The entry points that the binding calls, with the mask each of them gets."""
    got = []

    class Lib:
        def flowmoe_trace_start(self, events, kinds, pairs, mask):
            got.append((32, ctypes.c_uint32(mask).value))
            return 0

        def flowmoe_trace_start64(self, events, kinds, pairs, mask):
            got.append((64, ctypes.c_uint64(mask).value))
            return 0

    monkeypatch.setattr(L, "load", lambda: Lib())
    return got


FIRST, PAST = L.kind_mask(L.K_NAMES[:32]), L.kind_mask(L.K_NAMES[32:])


@pytest.mark.parametrize("mask,want", [
    (0, (32, 0)), (1, (32, 1)), (FIRST, (32, FIRST)), (0xFFFFFFFF, (32, 0xFFFFFFFF)),
    # every kind, by name and as a number
    (L.kind_mask(L.K_NAMES), (64, FIRST | PAST)), (-1, (64, ALL)), (ALL, (64, ALL)),
    # all but one of the first 32, of those past them
    (~L.kind_mask(["gate"]), (64, ALL - 1)),
    (L.kind_mask(n for n in L.K_NAMES if n != "embed"), (64, (FIRST | PAST) - L.kind_mask(["embed"]))),
    (L.kind_mask(["rope", "layer_norm"]), (64, L.kind_mask(["rope", "layer_norm"]))),
])
def test_masks_taken(entries, mask, want):
    L.flowmoe_trace_start(None, None, 0, mask)
    assert entries == [want]


@pytest.mark.parametrize("mask", [PAST, L.kind_mask(["packed_join"]), 1 << 63])
def test_kinds_past_31_alone_are_refused(entries, mask):
    with pytest.raises(ValueError, match="trace_start64"):
        L.flowmoe_trace_start(None, None, 0, mask)
    assert entries == []


@pytest.mark.gpu
@pytest.mark.parametrize("mask", [L.kind_mask(L.K_NAMES), -1, L.kind_mask(["rope", "layer_norm"])])
def test_kinds_recorded(mask):
    import torch

    from gpu_helpers import dev, need_gpu
    from paper_2510_00207_amd.hiprt import EventArray
    need_gpu()
    T, M = 70, 256
    x = torch.randn(T, M, device=dev()).bfloat16()
    y, s = torch.empty_like(x), L.make_shape(T, M, 8, 1, 1, 0)
    ev = EventArray(8)
    L.flowmoe_trace_start(ev.ev, ev.kinds, ev.pairs, mask)
    L.flowmoe_rope_fwd(s, L.make_rope_shape(4, 64, 64, T), x, None, y)
    L.flowmoe_layer_norm_fwd(s, 1e-5, x, None, None, None, None, y)
    torch.cuda.synchronize()
    n = L.flowmoe_trace_stop()
    assert [L.K_NAMES[k] for k in ev.kinds[:n]] == ["rope", "layer_norm"]
    ev.close()
