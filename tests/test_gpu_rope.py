"""Rotary positions on the GPU against 64 bits: layouts, parts of a head, scalings, strides, padding, far positions, gradients."""
import numpy as np
import pytest
import torch

import paper_2608_20427_b200 as bf1
from oracle import cache_oracle as C

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def inputs(tokens, hq, hkv, d, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((tokens, hq, d), generator=g).to(torch.bfloat16).to(DEV), torch.randn((tokens, hkv, d), generator=g).to(torch.bfloat16).to(DEV))


def check(got, x, positions, cfg, back=False):
    """The result's rounding to bf16, and in 32 bits: the angle to 2^-22 of a radian (half a step of a number up to 1 in turns of
    a half, times pi), sine and cosine to 2^-22, two products and a sum of 2^-24 each: below 2^-20 (|x| + |y|) magnitude."""
    turns, magnitude = C.rope_turns(cfg.dim, cfg.base, cfg.scaling, cfg.factor, cfg.original_len, cfg.beta_fast, cfg.beta_slow)
    x = x.double().cpu().numpy()
    want = C.rotate(x, positions, turns, magnitude, cfg.layout, back)
    got = got.double().cpu().numpy()
    live = np.asarray(positions) >= 0
    pair = np.abs(x)
    r = cfg.dim
    if cfg.layout == "half":
        pair[..., :r] = np.tile(pair[..., :r // 2] + pair[..., r // 2:r], 2)
    else:
        pair[..., :r] = np.repeat(pair[..., 0:r:2] + pair[..., 1:r:2], 2, axis=-1)
    limit = np.abs(want) * 2.0 ** -8 + pair * magnitude * 2.0 ** -20
    assert (np.abs(got - want)[live] <= limit[live]).all()
    assert np.array_equal(got[live][..., r:], x[live][..., r:])        # carried over
    return live


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("tokens,hq,hkv,d,dim", [(1, 1, 1, 64, 64), (1, 16, 8, 128, 128), (3, 5, 0, 64, 16), (17, 4, 4, 128, 96), (33, 2, 1, 64, 32),
                                                 (301, 8, 2, 128, 64), (5, 40, 3, 128, 16), (130, 7, 1, 64, 48)])
def test_forward_and_gradient(layout, tokens, hq, hkv, d, dim):
    q, k = inputs(tokens, hq, max(hkv, 1), d, tokens + d)
    cfg = bf1.RopeCfg(dim, layout=layout)
    rope = bf1.plan_rope(cfg, DEV)
    pos = [(7 * t * t + 11) % 5000 for t in range(tokens)]
    p = torch.tensor(pos, dtype=torch.int32, device=DEV)
    for back, call in ((False, bf1.rope_fwd), (True, bf1.rope_bwd)):
        oq, ok = call(q, k if hkv else None, p, rope)
        check(oq, q, pos, cfg, back)
        if hkv:
            check(ok, k, pos, cfg, back)
        else:
            assert ok is None


@pytest.mark.parametrize("kw", [dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=4.0, base=1e6),
                                dict(scaling="yarn", factor=8.0, original_len=512)], ids=lambda k: k["scaling"])
def test_scaled(kw):
    q, k = inputs(40, 4, 2, 128, 5)
    cfg = bf1.RopeCfg(128, **kw)
    pos = [0, 1, 2, 511, 512, 513, 4095, 4096] * 5
    oq, ok = bf1.rope_fwd(q, k, torch.tensor(pos, dtype=torch.int32, device=DEV), bf1.plan_rope(cfg, DEV))
    check(oq, q, pos, cfg)
    check(ok, k, pos, cfg)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_positions_keep_their_angle(layout):
    """2^31 - 1 with a first frequency of one radian: 32-bit angles would be off by a hundred radians."""
    pos = [2 ** 31 - 1, 2 ** 30 + 1, 16777217, 16777219, 1000003, 999999]
    q, k = inputs(len(pos), 2, 1, 64, 6)
    cfg = bf1.RopeCfg(64, layout=layout)
    oq, ok = bf1.rope_fwd(q, k, torch.tensor(pos, dtype=torch.int32, device=DEV), bf1.plan_rope(cfg, DEV))
    turns, _ = C.rope_turns(64)
    got, x = oq.double().cpu().numpy(), q.double().cpu().numpy()
    # the oracle's own product position * turns is off by 2^-53 * 2^31 / 2 pi turns here: 2^-22 of a radian more
    want = C.rotate(x, pos, turns, 1.0, layout)
    size = np.abs(x)
    pair = np.tile(size[..., :32] + size[..., 32:], 2) if layout == "half" else np.repeat(size[..., 0::2] + size[..., 1::2], 2, axis=-1)
    assert (np.abs(got - want) <= np.abs(want) * 2.0 ** -8 + pair * 2.0 ** -19).all()


def test_strided_parts_of_a_projection_and_head_major_rows():
    tokens, hq, hkv, d = 37, 4, 2, 64
    row = torch.randn((tokens, (hq + 2 * hkv) * d), device=DEV).to(torch.bfloat16)
    q, k = row[:, :hq * d].view(tokens, hq, d), row[:, hq * d:(hq + hkv) * d].view(tokens, hkv, d)
    pos = torch.arange(tokens, dtype=torch.int32, device=DEV)
    rope = bf1.plan_rope(bf1.RopeCfg(64), DEV)
    want = bf1.rope_fwd(q.contiguous(), k.contiguous(), pos, rope)
    got = bf1.rope_fwd(q, k, pos, rope)
    assert all(x.is_contiguous() and torch.equal(x, y) for x, y in zip(got, want))
    # head by head, into head by head
    qh, kh = q.transpose(0, 1).contiguous().transpose(0, 1), k.transpose(0, 1).contiguous().transpose(0, 1)
    oh = [torch.empty_like(x) for x in (qh, kh)]
    assert not oh[0].is_contiguous()
    bf1.rope_fwd(qh, kh, pos, rope, out_q=oh[0], out_k=oh[1])
    assert all(torch.equal(x, y) for x, y in zip(oh, want))
    # in place, in the projection's output; the values beside them stay
    v = row[:, (hq + hkv) * d:].clone()
    oq, ok = bf1.rope_fwd(q, k, pos, rope, out_q=q, out_k=k)
    assert oq.data_ptr() == q.data_ptr() and torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(row[:, (hq + hkv) * d:], v)


def test_padding_rows_stay_and_empty_calls_do_nothing():
    q, k = inputs(9, 2, 1, 64, 8)
    pos = [3, -1, 5, -7, 0, 1, 2, 3, -1]
    cfg = bf1.RopeCfg(32)
    out = [torch.full_like(x, float("nan")) for x in (q, k)]
    bf1.rope_fwd(q, k, torch.tensor(pos, dtype=torch.int32, device=DEV), bf1.plan_rope(cfg, DEV), out_q=out[0], out_k=out[1])
    for got, x in zip(out, (q, k)):
        live = check(got, x, pos, cfg)
        assert torch.isnan(got[torch.tensor(~live, device=DEV)].float()).all()
    oq, ok = bf1.rope_fwd(q[:0], k[:0], torch.zeros(0, dtype=torch.int32, device=DEV), bf1.plan_rope(cfg, DEV))
    assert oq.shape == (0, 2, 64) and ok.shape == (0, 1, 64)


def test_rows_beyond_32_bits():
    tokens, h, d = (1 << 31) // (64 * 128) + 5, 64, 128
    q = torch.zeros((tokens, h, d), dtype=torch.bfloat16, device=DEV)
    q[-5:] = inputs(5, h, 1, d, 13)[0]
    pos = torch.full((tokens,), -1, dtype=torch.int32, device=DEV)
    pos[-5:] = torch.arange(5, dtype=torch.int32, device=DEV) + 99
    rope = bf1.plan_rope(bf1.RopeCfg(d), DEV)
    want = bf1.rope_fwd(q[-5:], None, pos[-5:], rope)[0]
    assert torch.equal(bf1.rope_fwd(q, None, pos, rope, out_q=q)[0][-5:], want)


def test_gradient_against_differences():
    """d/dx <g, R x> along a direction, from the forward alone: the forward is linear, so a step of any size gives the slope up to
    rounding.  x, y of bf16 values: <g, R x> rounds each product's factor by 2^-8 at most."""
    d, tokens = 64, 5
    q, _ = inputs(tokens, 3, 1, d, 9)
    g, _ = inputs(tokens, 3, 1, d, 10)
    pos = torch.tensor([0, 1, 100, 4097, 77], dtype=torch.int32, device=DEV)
    for layout in ("half", "interleaved"):
        rope = bf1.plan_rope(bf1.RopeCfg(d, layout=layout), DEV)
        y = bf1.rope_fwd(q, None, pos, rope)[0].double()
        dx = bf1.rope_bwd(g, None, pos, rope)[0].double()
        left, right = (g.double() * y).sum((1, 2)), (dx * q.double()).sum((1, 2))
        limit = 2.0 ** -8 * ((g.double() * y).abs() + (dx * q.double()).abs()).sum((1, 2)) * 1.01
        assert ((left - right).abs() <= limit).all()


def test_other_stream_and_graph():
    q, k = inputs(50, 4, 2, 128, 11)
    pos = torch.arange(50, dtype=torch.int32, device=DEV)
    rope = bf1.plan_rope(bf1.RopeCfg(128), DEV)
    want = bf1.rope_fwd(q, k, pos, rope)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = bf1.rope_fwd(q, k, pos, rope, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    out = [torch.zeros_like(x) for x in (q, k)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bf1.rope_fwd(q, k, pos, rope, out_q=out[0], out_k=out[1])
    q.mul_(2)
    graph.replay()
    again = bf1.rope_fwd(q, k, pos, rope)
    assert all(torch.equal(x, y) for x, y in zip(out, again)) and not torch.equal(out[0], want[0])


def test_refusals_of_the_binding():
    q, k = inputs(4, 2, 1, 64, 12)
    pos = torch.zeros(4, dtype=torch.int32, device=DEV)
    rope = bf1.plan_rope(bf1.RopeCfg(64), DEV)
    for bad in (lambda: bf1.rope_fwd(q.float(), k, pos, rope), lambda: bf1.rope_fwd(q, k[:3], pos, rope), lambda: bf1.rope_fwd(q, k, pos[:3], rope),
                lambda: bf1.rope_fwd(q, k, pos.long(), rope), lambda: bf1.rope_fwd(q, k, pos.cpu(), rope), lambda: bf1.rope_fwd(q, k.cpu(), pos, rope),
                lambda: bf1.rope_fwd(q, k, pos, rope, out_q=torch.empty_like(k)), lambda: bf1.rope_fwd(q, None, pos, rope, out_q=q[:1].expand(4, 2, 64)), lambda: bf1.rope_fwd(q.transpose(1, 2), None, pos, rope),
                lambda: bf1.rope_fwd(q, k, pos, bf1.plan_rope(bf1.RopeCfg(64), "cpu"))):   # (a table on the host is not read)
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(bf1.Bf1Error):
        bf1.rope_fwd(q, k, pos, bf1.plan_rope(bf1.RopeCfg(128), DEV))
