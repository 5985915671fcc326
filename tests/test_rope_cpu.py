"""Rotary positions without a GPU: the tables of the scalings, the oracle's own properties, the host's refusals."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2608_20427_b200 as bf1
from oracle import cache_oracle as C
from paper_2608_20427_b200 import binding

CFGS = [dict(dim=128), dict(dim=16, base=500.0), dict(dim=64, scaling="linear", factor=4.0), dict(dim=96, scaling="ntk", factor=8.0),
        dict(dim=128, base=1e6, scaling="yarn", factor=16.0, original_len=4096),
        dict(dim=32, scaling="yarn", factor=2.0, original_len=100, beta_fast=4.0, beta_slow=1.0)]


@pytest.mark.parametrize("kw", CFGS, ids=lambda k: "-".join(str(v) for v in k.values()))
def test_tables(kw):
    want, magnitude = C.rope_turns(**kw)
    rope = bf1.plan_rope(bf1.RopeCfg(**kw), "cpu")
    assert rope.dim == kw["dim"] and rope.turns.dtype.itemsize == 8
    assert np.allclose(rope.turns.numpy(), want, rtol=1e-14, atol=0) and abs(rope.magnitude - magnitude) < 1e-14
    assert bf1.plan_rope(bf1.RopeCfg(magnitude=0.5, **kw), "cpu").magnitude == 0.5


def test_the_oracle_depends_on_distances_only():
    """<R(p) x, R(s) y> is a function of p - s: what the operator is for."""
    rng = np.random.default_rng(1)
    turns, _ = C.rope_turns(32)
    for layout in ("half", "interleaved"):
        x, y = rng.standard_normal((2, 1, 1, 64))
        dot = [float((C.rotate(x, [p], turns, 1.0, layout)[0, 0] * C.rotate(y, [p + 5], turns, 1.0, layout)[0, 0]).sum()) for p in (0, 3, 1000)]
        assert max(dot) - min(dot) < 1e-11
        # position 0 is the identity, the transpose turns back
        assert np.array_equal(C.rotate(x, [0], turns, 1.0, layout), x)
        assert np.allclose(C.rotate(C.rotate(x, [77], turns, 1.0, layout), [77], turns, 1.0, layout, back=True), x, atol=1e-14)


def test_refusals():
    lib = bf1.load()
    for kw, code in ((dict(dim=24), -2), (dict(dim=0), -2), (dict(dim=64, base=1.0), -1), (dict(dim=64, base=math.nan), -1),
                     (dict(dim=64, scaling="linear", factor=0.5), -1), (dict(dim=64, scaling="yarn", factor=2.0), -1),
                     (dict(dim=64, scaling="yarn", factor=2.0, original_len=10, beta_fast=1.0, beta_slow=1.0), -1)):
        with pytest.raises(bf1.Bf1Error) as e:
            bf1.plan_rope(bf1.RopeCfg(**kw), "cpu")
        assert e.value.code == code
    with pytest.raises(ValueError):
        bf1.plan_rope(bf1.RopeCfg(64, scaling="stretched"), "cpu")
    with pytest.raises(ValueError):
        bf1.plan_rope(bf1.RopeCfg(64, layout="thirds"), "cpu")
    with pytest.raises(ValueError):
        bf1.Rope.from_turns([0.1] * 12, "half", 1.0, "cpu")

    fake = ctypes.c_void_p(0x1000)
    rows = lambda p=0x1000, row=128, head=64: ctypes.byref(binding._RowsC(p, row, head))  # noqa: E731
    rope = lambda dim=64, layout=0, turns=0x1000: ctypes.byref(binding._RopeC(dim, layout, 1.0, turns))  # noqa: E731

    def call(q=None, k=None, pos=fake, tokens=4, hq=2, hkv=1, d=64, r=None, oq=None, ok=None):
        rcs = [f(q or rows(), k or rows(), pos, tokens, hq, hkv, d, r or rope(), oq or rows(0x2000), ok or rows(0x3000), None)
               for f in (lib.bf1_rope_fwd, lib.bf1_rope_bwd)]
        assert rcs[0] == rcs[1]
        return rcs[0]

    assert call(tokens=0) == 0                                   # nothing to do, nothing launched
    assert call(tokens=-1) == -1 and call(hq=0) == -1 and call(hkv=-1) == -1
    assert call(d=96) == -2 and call(hq=65535, hkv=1) == -2
    assert call(pos=None) == -1
    assert call(q=rows(None)) == -1 and call(oq=rows(None)) == -1 and call(k=rows(None)) == -1 and call(ok=rows(None)) == -1
    assert call(q=rows(0x1008)) == -1 and b"aligned" in lib.bf1_last_error()
    assert call(q=rows(row=12)) == -1 and call(k=rows(head=65)) == -1
    assert call(r=rope(dim=128)) == -2 and call(r=rope(dim=24)) == -2 and call(r=rope(layout=2)) == -1 and call(r=rope(turns=None)) == -1
    assert call(q=rows(0x2000, row=256)) == -1 and b"in place" in lib.bf1_last_error()


def test_outputs_without_their_inputs_are_refused():
    """Before anything else is looked at, the device included."""
    q = torch.zeros((2, 1, 64), dtype=torch.bfloat16)
    pos = torch.zeros(2, dtype=torch.int32)
    rope = bf1.plan_rope(bf1.RopeCfg(64), "cpu")
    for call in (bf1.rope_fwd, bf1.rope_bwd):
        with pytest.raises(AssertionError, match="out_k is given without k"):
            call(q, None, pos, rope, out_k=torch.zeros_like(q))
    pages = torch.zeros((1, 64, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(AssertionError, match="out_q is given without q"):
        bf1.cache_write(q, q, pages, pages, bf1.CachePlan.empty(1, 2, "cpu"), rope=rope, out_q=torch.zeros_like(q))
