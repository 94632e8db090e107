"""Every gradient of the differential attention block (flowmoe_diff_mha_fwd/_bwd) against
the fp64 chain from the same inputs, in the 2-norm, within the bounds of diff_chain.py;
with and without positions and a gain."""
import pytest
import torch

import diff_chain as C
from gpu_helpers import host, need_gpu
from paper_2510_00207_amd import _lib as L
from test_gpu_diff_mha import EPS, SCALE, Block

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", C.CASES)
def test_gradients_against_the_chain(case):
    need_gpu()
    nseq, seq, heads, kv, hd, causal, lens, rot, layout, gained = case
    b = Block(nseq, seq, heads, kv, hd, causal, 61, lens, rot, layout)
    if rot is None:
        b.rope = None
    if not gained:
        b.t["gain"] = None
    b.bufs = L.diff_mha_bufs(ws_bytes=b.bufs.ws_bytes, **b.t)
    b.fwd()
    b.bwd()
    o = b.outputs()
    p = {k: host(b.t[k]) for k in ("inp", "w_qkv", "w_o", "lam", "d_out")}
    p["gain"] = host(b.t["gain"] if gained else torch.ones(hd))
    ref, bound = C.bounds(p, b.args, b.rope_kw if rot else None, b.t["positions"].tolist(), lens,
                          (EPS, SCALE))
    for n in C.GRADS:
        assert C.within(host(o[n]), ref[n], bound[n]), n
    # without dgain: the others as they were
    b.t["dgain"] = None
    b.bufs = L.diff_mha_bufs(ws_bytes=b.bufs.ws_bytes, **b.t)
    b.bwd()
    torch.cuda.synchronize()
    for n in C.GRADS[:4]:
        assert torch.equal(b.t[n], o[n]), n
