"""One-token decode over 8-bit pages without a GPU: the oracle against library attention, the host's refusals."""
import ctypes
import math

import numpy as np
import torch

import paper_2608_20427_b200 as bf1
from oracle import cache_oracle as C
from paper_2608_20427_b200 import binding


def test_the_oracle_is_attention_over_the_listed_keys():
    rng = np.random.default_rng(2)
    hq, hkv, d, pages = 4, 2, 64, 6
    codes = [C.to_e4m3(rng.standard_normal((pages, 64, hkv, d)) * 50) for _ in range(2)]
    scales = [2.0 ** rng.integers(-8, -5, (pages, hkv)) for _ in range(2)]
    q = rng.standard_normal((3, hq, d))
    lists, lens = [[4, 0, 2], [5], []], [150, 64, 0]
    o, lse = C.decode(q, *codes, *scales, lists, lens)
    assert np.isnan(o[2]).all() and np.isnan(lse[:, 2]).all()
    for s in range(2):
        k, v = (torch.tensor((c[lists[s]] * w[lists[s]][:, None, :, None]).reshape(-1, hkv, d)[:lens[s]]).transpose(0, 1) for c, w in zip(codes, scales))
        want = torch.nn.functional.scaled_dot_product_attention(torch.tensor(q[s])[:, None], k, v, enable_gqa=True)[:, 0]
        assert np.allclose(o[s], want.numpy(), rtol=1e-12, atol=1e-12)
        x = torch.einsum("hd,hnd->hn", torch.tensor(q[s]), k.repeat_interleave(2, 0)) / math.sqrt(d)
        assert np.allclose(lse[:, s], torch.logsumexp(x, 1).numpy(), rtol=1e-13)


def test_refusals():
    lib = bf1.load()
    f = ctypes.c_void_p(0x1000)
    plan = lambda deg=11, count=0x1000, page=0x1000, block=0x1000, status=0x1000: ctypes.byref(binding._DecodePlanC(deg, count, page, block, status))  # noqa: E731

    def call(q=f, kp=f, vp=f, ks=f, vs=f, pages=1, lens=f, batch=1, hq=2, hkv=1, d=64, p=None, ws=f, o=f, lse=f):
        return lib.bf1_decode_fwd_fp8(q, kp, vp, ks, vs, pages, lens, batch, hq, hkv, d, 0.0, p or plan(), ws, o, lse, None)

    assert call(batch=0) == 0
    for name in ("q", "kp", "vp", "ks", "vs", "lens", "ws", "o", "lse"):
        assert call(**{name: None}) == -1, name
    for kw in (dict(count=None), dict(page=None), dict(block=None), dict(status=None)):
        assert call(p=plan(**kw)) == -1
    assert call(batch=-1) == -1 and call(pages=0) == -1 and call(hq=0) == -1 and call(hkv=0) == -1 and call(hq=3, hkv=2) == -1
    assert call(hq=8) == -2 and call(hq=3) == -2 and call(d=96) == -2
    for name in ("q", "kp", "vp", "o", "ws"):
        assert call(**{name: ctypes.c_void_p(0x1008)}) == -1 and b"aligned" in lib.bf1_last_error()
    assert call(p=plan(0)) == -2 and call(batch=65536) == -2 and call(pages=1 << 25) == -2 and call(hq=65536, hkv=65536) == -2
    assert call(p=plan(1 << 22), batch=1024) == -2
    assert call(batch=0, p=plan(100000)) == 0                      # lists may be of any length
    for args in ((-1, 2, 1, 1, 64), (1, 3, 2, 1, 64), (1, 2, 1, 0, 64), (1, 2, 1, 1, 0), (1, 0, 1, 1, 64)):
        assert lib.bf1_decode_fp8_workspace_bytes(*args) == -1
    assert 16 <= lib.bf1_decode_fp8_workspace_bytes(1024, 32, 8, 10 ** 6, 128) < 8 << 20


def test_refusals_of_packed_rows():
    lib = bf1.load()
    f = ctypes.c_void_p(0x1000)
    plan = ctypes.byref(binding._DecodePlanC(11, 0x1000, 0x1000, 0x1000, 0x1000))

    def call(q=f, rows=4, cu=f, batch=2, hq=2, hkv=1, d=64, o=f, lse=f):
        return lib.bf1_decode_fwd_fp8_packed(q, rows, cu, f, f, f, f, 1, f, batch, hq, hkv, d, 0.0, plan, f, o, lse, None)

    assert call(batch=0) == 0 and call(rows=0) == 0                 # nothing to do, nothing launched
    assert call(cu=None) == -1 and call(q=None) == -1 and call(o=None) == -1 and call(lse=None) == -1
    assert call(rows=-1) == -1 and call(batch=-1) == -1 and call(hq=3, hkv=2) == -1
    assert call(hq=8) == -2 and call(d=96) == -2 and call(batch=65536) == -2
