"""The fp64 chain of the differential attention block's gradients: against central
differences; and that its bounds pass a block that rounds and reject wrong ones."""
import numpy as np
import pytest

import diff_chain as C

NORM = (1e-5, 0.25)


def setup(case, seed=3):
    nseq, seq, heads, kv, hd, causal, lens, rot, layout, gained = case
    T, M, W = nseq * seq, heads * hd, (heads + 2 * kv) * hd
    rng = np.random.default_rng(seed)
    r = lambda *s, std=1.0: to_bf16(std * rng.standard_normal(s))
    p = dict(inp=r(T, M), w_qkv=r(M, W, std=0.05), w_o=r(M, M, std=0.05), d_out=r(T, M),
             lam=rng.uniform(0.2, 0.8, heads),
             gain=1 + 0.2 * rng.standard_normal(hd) if gained else np.ones(hd))
    rope = None if rot is None else dict(heads=2 * (heads + kv), head_dim=hd // 2, rot=rot, layout=layout)
    return p, (seq, heads, kv, hd, causal), rope, np.arange(T) * 7 % 5000, lens, NORM


def to_bf16(x):
    """Rounded to nearest, ties to even."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    b = (b + 0x7FFF + (b >> 16 & 1)) & 0xFFFF0000
    return b.astype(np.uint32).view(np.float32).astype(np.float64)


@pytest.mark.parametrize("case", C.CASES)
def test_chain_against_differences(case):
    """Along each gradient itself, where the terms add up."""
    s = setup(case)
    p, rest = s[0], s[1:]
    ref = C.gradients(*s)
    for name, grad in (("inp", "d_in"), ("w_qkv", "dw_qkv"), ("w_o", "dw_o"), ("lam", "d_lambda"),
                       ("gain", "dgain")):
        v = ref[grad] / np.linalg.norm(ref[grad])
        at = lambda h: C.loss(dict(p, **{name: p[name] + h * v}), *rest)
        num = (8 * (at(1e-3) - at(-1e-3)) - (at(2e-3) - at(-2e-3))) / 12e-3
        assert abs(num - np.linalg.norm(ref[grad])) <= 1e-6 * abs(num), name


@pytest.mark.parametrize("case", C.CASES)
def test_bounds_pass_roundings_and_reject_mistakes(case):
    s = setup(case)
    p, args, rope, pos, lens, norm = s
    ref, bound = C.bounds(*s)
    rounded = C.gradients(*s, rnd=lambda name, x: to_bf16(x))
    for n in C.GRADS:
        print(n, np.linalg.norm(ref[n]), bound[n] / np.linalg.norm(ref[n]),
              np.linalg.norm(rounded[n] - ref[n]) / bound[n])
        assert C.within(rounded[n], ref[n], bound[n]), n
        for what, wrong in (("negated", -ref[n]), ("half", ref[n] / 2), ("larger", 1.5 * ref[n]),
                            ("reversed", ref[n][::-1]), ("shifted", np.roll(ref[n], 1, -1)),
                            ("nothing", 0 * ref[n])):
            assert not C.within(wrong, ref[n], bound[n]), (n, what)

    def rejected(wrong, grads):
        for n in grads:
            assert not C.within(wrong[n], ref[n], bound[n]), n

    chain = lambda **kw: C.gradients(dict(p, **kw.pop("p", {})), *[
        kw.get(k, v) for k, v in zip(("args", "rope", "pos", "lens", "norm"), s[1:])])
    rejected(chain(args=args[:4] + (not args[4],)), ("d_in", "dw_qkv", "dw_o"))
    rejected(chain(p=dict(lam=-p["lam"])), C.GRADS)
    rejected(chain(norm=(norm[0], 1.0)), C.GRADS)
    if rope is None:
        turned = dict(heads=2 * (args[1] + args[2]), head_dim=args[3] // 2, rot=args[3] // 2)
        rejected(chain(rope=turned), ("d_in", "dw_qkv"))
    else:
        rejected(chain(rope=None), ("d_in", "dw_qkv"))
        rejected(chain(pos=pos[::-1]), ("d_in", "dw_qkv"))
    if lens is not None:
        rejected(chain(lens=None), C.GRADS)
    # the second map's part of dQ and dK, and the norm's projection, left out
    rejected(C.gradients(*s, rnd=lambda name, x: 0 * x if name == "ds2" else x), ("d_in", "dw_qkv"))
    rejected(C.gradients(*s, rnd=lambda name, x: 0 * x if name == "p2" else x), C.GRADS)
