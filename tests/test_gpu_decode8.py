"""One-token decode over 8-bit pages against 64 bits: tails, empty sequences, long and short lists, cut ones, what lies behind the
newest token, scales and queries of all sizes, and a serving loop that fills the cache it reads."""
import math

import numpy as np
import pytest
import torch

import paper_2608_20427_b200 as bf1
from oracle import cache_oracle as C

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
E4M3 = torch.float8_e4m3fn
DENSE = dict(block=64, local_blocks=1 << 20, global_first=0, dyadic=0)


def logical(n, dense):
    j = (n - 1) // 64
    if n == 0:
        return []
    if dense:
        return list(range(j + 1))
    return sorted({j, 0} | {j - w for w in (1, 2) if w <= j} | {j - (1 << k) for k in range(20) if j >= 1 << k})


class Cache:
    """Pages of random numbers; `lens` tokens per sequence, pages in random order."""

    def __init__(self, lens, hkv, d, dense, seed, room=5, exponents=(-9, -5)):
        g = torch.Generator().manual_seed(seed)
        self.lens = lens
        self.lists = [logical(n, dense) for n in lens]
        held = [(n + 63) // 64 for n in lens]
        need = sum(len(x) for x in self.lists)
        perm = [int(x) for x in torch.randperm(need + room, generator=g)]
        table = torch.full((len(lens), max(max(held), 1)), -1, dtype=torch.int32)
        for s, x in enumerate(self.lists):
            for b in x:
                table[s, b] = perm.pop()
        self.lists = [[int(table[s, b]) for b in x] for s, x in enumerate(self.lists)]
        shape = (need + room, 64, hkv, d)
        self.kp, self.vp = ((torch.randn(shape, generator=g) * 60).clamp(-448, 448).to(E4M3) for _ in range(2))
        self.ks, self.vs = (2.0 ** torch.randint(*exponents, shape[:1] + (hkv,), generator=g).float() for _ in range(2))
        self.table = table
        self.cfg = bf1.RouteCfg(**DENSE) if dense else bf1.RouteCfg()

    def garbage_behind(self):
        """NaN wherever nothing has been written."""
        used = {p for x in self.lists for p in x}
        for t in (self.kp, self.vp):
            u = t.view(torch.uint8)
            for p in range(u.shape[0]):
                if p not in used:
                    u[p] = 0x7f
            for x, n in zip(self.lists, self.lens):
                if n % 64:
                    u[x[-1], n % 64:] = 0xff
        for t in (self.ks, self.vs):
            for p in range(t.shape[0]):
                if p not in used:
                    t[p] = float("nan")


def run(c, q, scale=None, plan=None, times=2):
    lens = torch.tensor(c.lens, dtype=torch.int32, device=DEV)
    plan = plan or bf1.plan_decode(lens, c.table.to(DEV), c.cfg)
    batch, hq, d = q.shape
    ws = bf1.decode_fp8_workspace(batch, hq, c.kp.shape[2], plan.max_degree, d, DEV)
    ws.fill_(0xff)                                                 # NaN, whatever it is read as
    out = torch.full((batch, hq, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    lse = torch.full((hq, batch), float("nan"), device=DEV)
    args = [t.to(DEV) for t in (q, c.kp, c.vp, c.ks, c.vs)]
    first = None
    for _ in range(times):
        bf1.decode_fwd_fp8(*args, lens, plan, ws, scale=scale, out=out, lse=lse)
        torch.cuda.synchronize()
        first = first or (out.clone(), lse.clone())
    assert torch.equal(first[0].view(torch.int16), out.view(torch.int16)) and torch.equal(first[1].view(torch.int32), lse.view(torch.int32))
    return out, lse, plan


def check(c, q, out, lse, scale=None):
    """What may be off: the result's rounding, 2^-8 of it; the weights' rounding to f16, 2^-11 of each (below 2^-14 of the largest 2^-25 in all);
    a score, by the sum of its d products in 32 bits (d 2^-24 of their absolute sum), and by its product with two scales and its difference to the
    maximum (2^-21 of the largest score); an exponential, 2^-22.  The weights' errors count on the mean of |v|."""
    q64, kp, vp, ks, vs = (t.double().cpu().numpy() for t in (q, c.kp, c.vp, c.ks, c.vs))
    batch, hq, d = q.shape
    group = hq // kp.shape[2]
    want, want_lse = C.decode(q64, kp, vp, ks, vs, c.lists, c.lens, scale)
    by = scale or 1 / math.sqrt(d)
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for s, (x, n) in enumerate(zip(c.lists, c.lens)):
        if n == 0:
            assert np.isnan(got[s]).all() and np.isnan(got_lse[:, s]).all()        # not written
            continue
        keys = (len(x) - 1) * 64 + (n - 1) % 64 + 1
        for h in range(hq):
            j = h // group
            k = np.abs(kp[x, :, j] * ks[x, j][:, None, None]).reshape(-1, d)[:keys]
            v = np.abs(vp[x, :, j] * vs[x, j][:, None, None]).reshape(-1, d)[:keys]
            score = by * ((kp[x, :, j] * ks[x, j][:, None, None]).reshape(-1, d)[:keys] @ q64[s, h])
            sums = by * (k @ np.abs(q64[s, h])).max()
            off = d * 2.0 ** -24 * sums + 2.0 ** -21 * (np.abs(score).max() + 1)
            w = np.exp(score - want_lse[h, s])
            mean, rest = w @ v, 2.0 ** -25 * v.sum(0) * w.max()
            limit = 2.0 ** -8 * np.abs(want[s, h]) + (2.0 ** -11 + 2 * off) * 1.01 * mean + rest
            assert (np.abs(got[s, h] - want[s, h]) <= limit).all(), (s, h, np.abs(got[s, h] - want[s, h]).max(), limit.min())
            assert abs(got_lse[h, s] - want_lse[h, s]) <= off + 2.0 ** -21 * (1 + abs(want_lse[h, s])), (s, h)


def queries(batch, hq, d, seed, size=1.0):
    return (torch.randn((batch, hq, d), generator=torch.Generator().manual_seed(seed)) * size).to(torch.bfloat16)


@pytest.mark.parametrize("dense", [False, True], ids=["route", "dense"])
@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (4, 2, 128), (8, 2, 64), (16, 8, 128), (8, 2, 128), (1, 1, 128), (6, 3, 64)])
def test_tails_and_empty_sequences(hq, hkv, d, dense):
    lens = [1, 64, 65, 0, 257, 1000, 0, 4097, 63, 128]
    c = Cache(lens, hkv, d, dense, seed=hq + d)
    q = queries(len(lens), hq, d, 1)
    out, lse, plan = run(c, q)
    assert plan.status.item() == 0
    check(c, q, out, lse)
    c.garbage_behind()
    again, lse2, _ = run(c, q)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse.view(torch.int32), lse2.view(torch.int32))


@pytest.mark.parametrize("lens,hq,hkv,d,dense", [([1], 2, 1, 64, False), ([130], 1, 1, 64, True), ([32768], 16, 8, 128, False), ([20011], 8, 2, 64, True),
                                                 ([40000, 3], 4, 1, 128, True), ([9000] * 3 + [1, 0, 70], 16, 4, 128, True), ([0, 0], 2, 1, 64, False),
                                                 ([64 * 40, 0, 0, 64 * 40 + 1], 2, 2, 128, True)])
def test_long_and_short_lists(lens, hq, hkv, d, dense):
    """Lists that many cuts go through, runs without a page, single pages."""
    c = Cache(lens, hkv, d, dense, seed=len(lens))
    q = queries(len(lens), hq, d, 2)
    out, lse, _ = run(c, q)
    check(c, q, out, lse)


@pytest.mark.parametrize("batch,hq,hkv", [(300, 2, 1), (1024, 2, 1), (1025, 4, 1), (1500, 2, 2)])
def test_batches(batch, hq, hkv):
    """Up to 1024 lists are cut into equal runs, more are walked whole."""
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in rng.integers(0, 500, batch)]
    c = Cache(lens, hkv, 64, False, seed=3)
    q = queries(batch, hq, 64, 3)
    out, lse, _ = run(c, q)
    check(c, q, out, lse)


@pytest.mark.parametrize("batch,hq,hkv,d,most", [(90, 4, 2, 64, 2500), (41, 16, 4, 128, 1900), (150, 1, 1, 128, 1700), (1024, 2, 1, 64, 1800), (3, 2, 1, 64, 30000), (1100, 2, 1, 64, 6000), (9, 16, 4, 64, 29000),
                                                     (5, 4, 1, 128, 27000)])
def test_runs_through_lists_of_all_lengths(batch, hq, hkv, d, most):
    """Long lists that fill the GPU: equal runs of the row of all pages, empty lists among them, lists cut once, often and not at all."""
    rng = np.random.default_rng(batch)
    lens = [int(most ** rng.random()) if rng.random() < 0.9 else 0 for _ in range(batch)]
    lens[batch // 2], lens[0], lens[-1] = most, 0, 65
    c = Cache(lens, hkv, d, True, seed=batch)
    c.garbage_behind()
    q = queries(batch, hq, d, 14)
    out, lse, plan = run(c, q)
    assert plan.status.item() == 0
    check(c, q, out, lse)


@pytest.mark.parametrize("hkv,group,lens", [(64, 1, [5000, 64, 0, 1700]), (700, 2, [100, 65]), (700, 1, [1800, 3]), (36, 4, [130, 7])])
def test_many_heads(hkv, group, lens):
    """More KV heads than a run to each, lists for every SM from few sequences."""
    c = Cache(lens, hkv, 64, True, seed=hkv)
    q = queries(len(lens), hkv * group, 64, 15)
    out, lse, _ = run(c, q)
    check(c, q, out, lse)


def test_scales_of_all_sizes_and_a_given_softmax_scale():
    """A page's weights are rounded against the softmax's maximum alone: a page of tiny values beside huge ones loses nothing of its own."""
    c = Cache([1000, 64, 130], 2, 64, True, seed=4, exponents=(-9, -8))
    c.vs *= 2.0 ** torch.randint(-60, 60, c.vs.shape, generator=torch.Generator().manual_seed(5)).float()
    c.ks *= 1.37                                                    # no power of two
    q = queries(3, 4, 64, 4)
    out, lse, _ = run(c, q, scale=0.03)
    check(c, q, out, lse, scale=0.03)


@pytest.mark.parametrize("size", [1e-30, 1e-3, 300.0, 1e30])
def test_queries_of_all_sizes(size):
    c = Cache([300, 65], 1, 128, True, seed=6)
    q = queries(2, 2, 128, 6, size)
    c.ks = (c.ks.double() / size).float()
    out, lse, _ = run(c, q)
    check(c, q, out, lse)
    assert torch.isfinite(out).all()


def test_what_is_not_finite_stays_in_its_list():
    """NaN in a key or a value, an infinity in a query: NaN in that sequence's and head's result, others as they were."""
    c = Cache([200, 70, 300], 2, 64, True, seed=7)
    q = queries(3, 4, 64, 7)
    base, base_lse, _ = run(c, q)
    c.kp.view(torch.uint8)[c.lists[0][1], 5, 0, 9] = 0x7f            # a key of sequence 0, KV head 0
    c.vp.view(torch.uint8)[c.lists[2][0], 63, 1, 3] = 0xff           # a value of sequence 2, KV head 1
    q[1, 3, 0] = float("inf")
    out, lse, _ = run(c, q)
    bad = torch.zeros((3, 4, 64), dtype=torch.bool)
    bad[0, :2] = True
    bad[2, 2:, 3] = True
    bad[1, 3] = True
    assert torch.isnan(out[bad.to(DEV)]).all() and torch.equal(out[~bad.to(DEV)], base[~bad.to(DEV)])
    gone = torch.zeros((4, 3), dtype=torch.bool)
    gone[:2, 0] = gone[3, 1] = True
    assert torch.isnan(lse[gone.to(DEV)]).all() and torch.equal(lse[~gone.to(DEV)], base_lse[~gone.to(DEV)])


def test_equal_scores_give_the_mean():
    """Queries of zero: every key counts alike; the LSE is the log of their number."""
    c = Cache([1000, 1, 64], 1, 64, True, seed=8)
    out, lse, _ = run(c, torch.zeros((3, 2, 64), dtype=torch.bfloat16))
    check(c, torch.zeros((3, 2, 64)), out, lse)
    assert np.allclose(lse[0].cpu(), np.log([1000, 1, 64]), atol=1e-5)


def test_another_64_tokens_and_bad_pages_are_reported():
    c = Cache([100, 200], 1, 64, False, seed=9)
    q = queries(2, 2, 64, 9)
    lens = torch.tensor([100, 200], dtype=torch.int32, device=DEV)
    plan = bf1.plan_decode(lens, c.table.to(DEV), c.cfg)
    c.lens = [128, 200]                                             # still the plan's blocks
    out, lse, _ = run(c, q, plan=plan)
    assert plan.status.item() == 0
    check(c, q, out, lse)
    c.lens = [129, 200]
    out, lse, _ = run(c, q, plan=plan)
    assert plan.status.item() == 8 and torch.isnan(out[0]).all() and torch.isfinite(out[1]).all()
    plan = bf1.plan_decode(lens, c.table.to(DEV), c.cfg)
    plan.page[0, 0] = c.kp.shape[0]
    plan.page[0, 1] = -1
    c.lens = [100, 200]
    out, lse, _ = run(c, q, plan=plan)                              # page 0 is read in their place
    assert plan.status.item() == 8 and torch.isfinite(out[1]).all()


def test_pages_beyond_32_bits():
    hkv, d = 8, 128
    pages = (1 << 31) // (64 * hkv * d) + 30
    c = Cache([500, 64], hkv, d, True, seed=10)
    n = c.kp.shape[0]
    big = [torch.zeros((pages, 64, hkv, d), dtype=torch.uint8, device=DEV) for _ in range(2)]
    ks, vs = (torch.ones((pages, hkv), device=DEV) for _ in range(2))
    for b, t in zip(big, (c.kp, c.vp)):
        b[-n:] = t.view(torch.uint8).to(DEV)
    ks[-n:], vs[-n:] = c.ks.to(DEV), c.vs.to(DEV)
    q = queries(2, 16, d, 10)
    out, lse, _ = run(c, q)
    table = torch.where(c.table >= 0, c.table + pages - n, c.table).to(DEV)
    lens = torch.tensor(c.lens, dtype=torch.int32, device=DEV)
    plan = bf1.plan_decode(lens, table, c.cfg)
    ws = bf1.decode_fp8_workspace(2, 16, hkv, plan.max_degree, d, DEV)
    far, far_lse = bf1.decode_fwd_fp8(q.to(DEV), big[0].view(E4M3), big[1].view(E4M3), ks, vs, lens, plan, ws)
    assert torch.equal(far, out) and torch.equal(far_lse, lse)


def test_graph_and_another_stream():
    c = Cache([3000, 64, 777], 2, 128, True, seed=11)
    q = queries(3, 4, 128, 11)
    want, want_lse, plan = run(c, q)
    lens = torch.tensor(c.lens, dtype=torch.int32, device=DEV)
    args = [t.to(DEV) for t in (q, c.kp, c.vp, c.ks, c.vs)] + [lens, plan]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = bf1.decode_fwd_fp8(*args, bf1.decode_fp8_workspace(3, 4, 2, plan.max_degree, 128, DEV), stream=side)
    side.synchronize()
    assert torch.equal(got[0], want) and torch.equal(got[1], want_lse)
    ws = bf1.decode_fp8_workspace(3, 4, 2, plan.max_degree, 128, DEV)
    out, lse = torch.zeros_like(want), torch.zeros_like(want_lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bf1.decode_fwd_fp8(*args, ws, out=out, lse=lse)
    for _ in range(3):
        out.zero_()
        graph.replay()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_refusals_of_the_binding():
    c = Cache([100], 1, 64, False, seed=12)
    q, kp, vp, ks, vs = (t.to(DEV) for t in (queries(1, 2, 64, 12), c.kp, c.vp, c.ks, c.vs))
    lens = torch.tensor([100], dtype=torch.int32, device=DEV)
    plan = bf1.plan_decode(lens, c.table.to(DEV), c.cfg)
    ws = bf1.decode_fp8_workspace(1, 2, 1, plan.max_degree, 64, DEV)
    f = bf1.decode_fwd_fp8
    for bad in (lambda: f(q.float(), kp, vp, ks, vs, lens, plan, ws), lambda: f(q, kp.view(torch.uint8), vp, ks, vs, lens, plan, ws),
                lambda: f(q, kp, vp[:1], ks, vs, lens, plan, ws), lambda: f(q, kp, vp, ks[:1], vs, lens, plan, ws),
                lambda: f(q, kp, vp, ks, vs.double(), lens, plan, ws), lambda: f(q, kp, vp, ks, vs, lens.long(), plan, ws),
                lambda: f(q, kp, vp, ks, vs, lens, plan, ws[:100]), lambda: f(q, kp.cpu(), vp, ks, vs, lens, plan, ws),
                lambda: f(q, kp, vp, ks, vs, torch.cat((lens, lens)), plan, ws), lambda: f(q, kp, vp, ks, vs, lens, bf1.DecodePlan.empty(1, 4, "cpu"), ws),
                lambda: f(q, kp, vp, ks, vs, lens, bf1.DecodePlan.empty(2, 4, DEV), ws), lambda: f(q, kp, vp, ks, vs, lens, plan, ws.cpu()),
                lambda: f(q, kp, vp, ks, vs, lens, plan, ws, out=torch.zeros_like(q).float()), lambda: f(q, kp, vp, ks, vs, lens, plan, ws, lse=torch.zeros((1, 2), device=DEV))):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(bf1.Bf1Error):
        f(torch.cat([q] * 4, 1), kp, vp, ks, vs, lens, plan, bf1.decode_fp8_workspace(1, 8, 1, plan.max_degree, 64, DEV))
    o, lse = f(q[:0], kp, vp, ks, vs, lens[:0], bf1.DecodePlan.empty(0, 4, DEV), ws)
    assert o.shape == (0, 2, 64) and lse.shape == (2, 0)


@pytest.mark.parametrize("dense", [False, True], ids=["route", "dense"])
def test_a_serving_loop(dense):
    """Prompts, then tokens: plan_cache, rope and write, plan_decode, decode, lengths on the device all the while, one captured step;
    every step against attention in 64 bits over the keys and values as they went in (which the cache holds to 2^-4 of each)."""
    hq, hkv, d, pages, batch = 4, 2, 64, 40, 3
    g = torch.Generator().manual_seed(13)
    cfg = bf1.RopeCfg(32)
    rope = bf1.plan_rope(cfg, DEV)
    route = bf1.RouteCfg(**DENSE) if dense else bf1.RouteCfg()
    kp, vp = (torch.full((pages, 64, hkv, d), 0x7f, dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2))
    ks, vs = (torch.full((pages, hkv), float("nan"), device=DEV) for _ in range(2))
    lens = torch.zeros(batch, dtype=torch.int32, device=DEV)
    table = torch.full((batch, 10), -1, dtype=torch.int32, device=DEV)
    stack, count = torch.arange(pages, dtype=torch.int32, device=DEV), torch.tensor([pages], dtype=torch.int32, device=DEV)
    new = torch.tensor([130, 0, 62], dtype=torch.int32, device=DEV)
    seen = [[], [], []]

    def draw(n):
        q = torch.randn((n, hq, d), generator=g).to(torch.bfloat16).to(DEV)
        return q, *(torch.randn((n, hkv, d), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))

    def keep(k, v, plan):
        cu = plan.cu_tokens.tolist()
        turned = bf1.rope_fwd(k, None, plan.positions, rope)[0].double().cpu().numpy()
        for s in range(batch):
            for t in range(cu[s], cu[s + 1]):
                seen[s].append((turned[t], v[t].double().cpu().numpy()))

    # the prompts
    _, k, v = draw(200)
    plan = bf1.plan_cache(lens, new, table, pages, 200, stack, count, seqlens_out=lens, free_count_out=count)
    bf1.cache_write(bf1.rope_fwd(k, None, plan.positions, rope)[0], v, kp, vp, plan, ks, vs)
    keep(k, v, plan)
    # the step, captured: its inputs are refilled in place
    step = bf1.CachePlan.empty(batch, batch, DEV)
    q, k, v = draw(batch)
    pages_plan = bf1.plan_decode(lens, table, route)
    ws = bf1.decode_fp8_workspace(batch, hq, hkv, pages_plan.max_degree, d, DEV)
    turned, out = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.zeros((hq, batch), device=DEV)
    new.zero_()

    def body():
        bf1.plan_cache(lens, new, table, pages, batch, stack, count, plan=step, seqlens_out=lens, free_count_out=count)
        bf1.cache_write(k, v, kp, vp, step, ks, vs, rope=rope, q=q, out_q=turned)
        bf1.plan_decode(lens, table, route, plan=pages_plan)
        bf1.decode_fwd_fp8(turned, kp, vp, ks, vs, lens, pages_plan, ws, out=out, lse=lse)

    body()                                                          # adds nothing
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        body()
    new.fill_(1)
    for i in range(70):
        for t, x in zip((q, k, v), draw(batch)):
            t.copy_(x)
        graph.replay()
        keep(k, v, step)
        assert step.status.item() == 0 and pages_plan.status.item() == 0 and lens.tolist() == [len(x) for x in seen]
        if i % 10 not in (0, 3):
            continue
        for s in range(batch):
            n = len(seen[s])
            rows = [r for b in logical(n, dense) for r in range(64 * b, min(64 * b + 64, n))]
            kk, vv = np.stack([seen[s][r][0] for r in rows]), np.stack([seen[s][r][1] for r in rows])
            qq = turned[s].double().cpu().numpy()
            for h in range(hq):
                key = kk[:, h // 2]
                x = key @ qq[h] / math.sqrt(d)
                # a number of the cache is off by 2^-4 of itself, or by 2^-10 of a scale that is below max / 224, twice that where the scale
                # has grown; the keys seen here have been rounded to bf16 besides
                off = (np.abs(key) * (2.0 ** -4 + 2.0 ** -7) + np.abs(key).max() / 224 * 2.0 ** -9) @ np.abs(qq[h]) / math.sqrt(d)
                w = np.exp(x - x.max())
                val = vv[:, h // 2]
                o = (w @ val) / w.sum()
                e = np.expm1(2 * off.max())
                limit = e * (w @ np.abs(val - o)) / w.sum() * 1.1 + (w @ np.abs(val)) / w.sum() * 2.0 ** -4 * (1 + e) + np.abs(val).max() / 224 * 2.0 ** -9 + 2.0 ** -7 * np.abs(o)
                assert (np.abs(out[s, h].double().cpu().numpy() - o) <= limit).all()
                assert abs(lse[h, s].item() - (x.max() + math.log(w.sum()))) <= off.max() + 1e-3
    # one sequence leaves: its pages come back and its row of the results stays as it is
    before = count.item()
    was = out[0].clone()
    held = (lens[0].item() + 63) // 64
    new.copy_(torch.tensor([-1, 1, 1], dtype=torch.int32))
    graph.replay()
    assert lens[0].item() == 0 and count.item() >= before + held - 2 and torch.equal(out[0], was) and pages_plan.count[0].item() == 0


def check_beside(c, q, out, lse):
    """As `check`, with what is small held to its own size: a weight's rounding to f16 is 2^-11 of it, but for those below 2^-29 of the
    largest among the sixteen keys of a page that a warp takes together, which are off by half of 2^-39 of that one."""
    q64, kp, vp, ks, vs = (t.double().cpu().numpy() for t in (q, c.kp, c.vp, c.ks, c.vs))
    batch, hq, d = q.shape
    want, want_lse = C.decode(q64, kp, vp, ks, vs, c.lists, c.lens)
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for s, (x, n) in enumerate(zip(c.lists, c.lens)):
        keys = (len(x) - 1) * 64 + (n - 1) % 64 + 1
        for h in range(hq):
            j = h // (hq // kp.shape[2])
            k = (kp[x, :, j] * ks[x, j][:, None, None]).reshape(-1, d)[:keys]
            v = np.abs(vp[x, :, j] * vs[x, j][:, None, None]).reshape(-1, d)[:keys]
            score = k @ q64[s, h] / math.sqrt(d)
            off = d * 2.0 ** -24 * (np.abs(k) @ np.abs(q64[s, h])).max() / math.sqrt(d) + 2.0 ** -21 * (np.abs(score).max() + 1)
            w = np.exp(score - want_lse[h, s])
            limit = 2.0 ** -8 * np.abs(want[s, h]) + (2.0 ** -11 + 2 * off) * 1.01 * (w @ v)
            for i in range(0, keys, 16):
                limit = limit + 2.0 ** -40 * w[i:i + 16].max() * v[i:i + 16].sum(0)
            assert (np.abs(got[s, h] - want[s, h]) <= limit).all(), (s, h, (np.abs(got[s, h] - want[s, h]) / limit).max())
            assert abs(got_lse[h, s] - want_lse[h, s]) <= off + 2.0 ** -21 * (1 + abs(want_lse[h, s])), (s, h)


@pytest.mark.parametrize("lens,hq,hkv,d,dense", [([30000], 2, 1, 128, True), ([1536, 700, 65, 40], 16, 8, 128, True), ([32768], 4, 1, 64, False), ([500] * 160, 1, 1, 64, True),
                                                 ([22000, 100, 3000], 8, 2, 64, True)], ids=["runs", "parts", "route", "whole", "runs-64"])
@pytest.mark.parametrize("nats", [12.0, 17.0, 18.5, 20.0, 30.0])
def test_a_sink_takes_nothing_from_the_others(nats, lens, hq, hkv, d, dense):
    """One key far above all others and with a value of zero: the result is the others', with their digits, however small their weights."""
    c = Cache(lens, hkv, d, dense, seed=16)
    c.kp = (c.kp.float() / 16).to(E4M3)
    c.ks.fill_(2.0 ** -5)
    q = torch.ones((len(lens), hq, d), dtype=torch.bfloat16) * (torch.randint(0, 2, (len(lens), hq, d), generator=torch.Generator().manual_seed(17)) * 2 - 1)
    q[:, :] = q[:, :1]                                              # one sign pattern for the heads, so that one key is everyone's sink
    for s, x in enumerate(c.lists):
        at = (7 * s) % min(lens[s], 64)                             # in the first page of the list
        c.kp[x[0], at] = (q[s, 0].float() * (nats / math.sqrt(d)) * 32).to(E4M3)
        c.vp[x[0], at] = 0
    out, lse, _ = run(c, q)
    check_beside(c, q, out, lse)


@pytest.mark.parametrize("lens,hq,hkv,d", [([256] * 3, 2, 1, 128), ([256] * 160, 2, 1, 128), ([25600], 2, 1, 128), ([25600], 2, 1, 64)], ids=["parts", "whole", "runs", "runs-64"])
def test_pages_of_small_weights_and_large_values(lens, hq, hkv, d):
    """Every other page has scores 18 nats below its neighbours' and values 2^40 times theirs: it is what the result is made of."""
    for odd in (0, 1):
        c = Cache(lens, hkv, d, True, seed=18)
        c.kp = (c.kp.float() / 16).to(E4M3)
        c.ks.fill_(2.0 ** -5)
        q = torch.ones((len(lens), hq, d), dtype=torch.bfloat16)
        c.vs.fill_(2.0 ** -7)
        for x in c.lists:
            for b, p in enumerate(x):
                if b % 2 == odd:
                    c.kp[p] = (c.kp[p].float() + 18.0 / math.sqrt(d) * 32).to(E4M3)
                    c.vs[p] = 2.0 ** -47
        out, lse, _ = run(c, q)
        check_beside(c, q, out, lse)


# ---- a step's packed rows ------------------------------------------------------------------------------------------------------------
def packed(counts, spare=0):
    cu = np.concatenate([[0], np.cumsum(counts)])
    return torch.tensor(cu, dtype=torch.int32, device=DEV), int(cu[-1]) + spare


@pytest.mark.parametrize("lens,counts,hq,hkv,d,dense", [([70, 300, 0, 64, 1, 129], [1, 0, 0, 3, 1, 129], 4, 2, 64, False), ([20000, 65, 9000, 3], [0, 1, 1, 2], 16, 8, 128, True),
                                                        ([26000, 500, 27000, 1], [1, 0, 1, 1], 2, 1, 64, True), ([300] * 200, [1, 0, 2, 1] * 50, 2, 1, 128, False),
                                                        ([100, 200], [0, 0], 2, 2, 64, False), ([2000] * 90, [0, 1, 1] * 30, 8, 2, 64, True)],
                         ids=["parts", "runs", "runs-64", "whole", "none", "runs-many"])
def test_packed_rows(lens, counts, hq, hkv, d, dense):
    """Every sequence with tokens in the step is decoded from the row of its newest one, the others are passed over."""
    c = Cache(lens, hkv, d, dense, seed=19)
    cu, rows = packed(counts, spare=2)
    q = queries(rows, hq, d, 20).to(DEV)
    lens_d = torch.tensor(lens, dtype=torch.int32, device=DEV)
    plan = bf1.plan_decode(lens_d, c.table.to(DEV), c.cfg)
    ws = bf1.decode_fp8_workspace(len(lens), hq, hkv, plan.max_degree, d, DEV)
    ws.fill_(0xff)
    out, lse = torch.full_like(q, float("nan")), torch.full((hq, rows), float("nan"), device=DEV)
    args = [t.to(DEV) for t in (c.kp, c.vp, c.ks, c.vs)]
    got = bf1.decode_fwd_fp8(q, *args, lens_d, plan, ws, out=out, lse=lse, cu_tokens=cu)
    assert got[0] is out and got[1] is lse and plan.status.item() == 0
    live = [s for s, n in enumerate(counts) if n > 0 and lens[s] > 0]
    at = [int(cu[s + 1]) - 1 for s in live]
    c.lens = [n if s in live else 0 for s, n in enumerate(lens)]
    mine = torch.zeros((len(lens), hq, d), dtype=torch.bfloat16)
    mine[live] = q[at].cpu()
    spread, spread_lse = (torch.full(s, float("nan"), dtype=t) for s, t in ((mine.shape, torch.bfloat16), ((hq, len(lens)), torch.float32)))
    spread[live], spread_lse[:, live] = out[at].cpu(), lse[:, at].cpu()
    c.lists = [x if n else [] for x, n in zip(c.lists, c.lens)]
    check(c, mine, spread, spread_lse)
    others = [r for r in range(rows) if r not in at]
    assert torch.isnan(out[others]).all() and torch.isnan(lse[:, others]).all()
    own = bf1.decode_fwd_fp8(q, *args, lens_d, plan, ws, cu_tokens=cu)                 # with results of its own
    assert torch.equal(own[0][at], out[at]) and torch.equal(own[1][:, at], lse[:, at])


def test_packed_rows_outside_the_arrays_are_refused():
    c = Cache([100, 200, 300], 1, 64, False, seed=21)
    lens = torch.tensor(c.lens, dtype=torch.int32, device=DEV)
    args = [t.to(DEV) for t in (c.kp, c.vp, c.ks, c.vs)]
    q = queries(3, 2, 64, 22).to(DEV)
    ws = bf1.decode_fp8_workspace(3, 2, 1, 17, 64, DEV)
    plan = bf1.plan_decode(lens, c.table.to(DEV), c.cfg)
    want = bf1.decode_fwd_fp8(q, *args, lens, plan, ws)[0]
    for offsets, good in (([0, 1, 4, 3], [0]), ([-1, 1, 2, 3], [1, 2]), ([0, 1, 2, 2 ** 31 - 1], [0, 1]), ([-5, -2, -1, 0], [])):
        plan = bf1.plan_decode(lens, c.table.to(DEV), c.cfg)
        out = torch.full_like(q, float("nan"))
        bf1.decode_fwd_fp8(q, *args, lens, plan, ws, out=out, cu_tokens=torch.tensor(offsets, dtype=torch.int32, device=DEV))
        assert plan.status.item() == 8 and torch.equal(out[good], want[good])
        assert torch.isnan(out[[s for s in range(3) if s not in good]]).all()


def test_refusals_of_packed_rows():
    c = Cache([100], 1, 64, False, seed=12)
    q, kp, vp, ks, vs = (t.to(DEV) for t in (queries(3, 2, 64, 12), c.kp, c.vp, c.ks, c.vs))
    lens = torch.tensor([100], dtype=torch.int32, device=DEV)
    plan = bf1.plan_decode(lens, c.table.to(DEV), c.cfg)
    ws = bf1.decode_fp8_workspace(1, 2, 1, plan.max_degree, 64, DEV)
    cu = torch.tensor([0, 3], dtype=torch.int32, device=DEV)
    f = lambda q=q, lens=lens, **kw: bf1.decode_fwd_fp8(q, kp, vp, ks, vs, lens, plan, ws, **kw)  # noqa: E731
    for bad in (lambda: f(), lambda: f(cu_tokens=cu[:1]), lambda: f(cu_tokens=cu.long()), lambda: f(cu_tokens=cu.cpu()), lambda: f(cu_tokens=cu[None]),
                lambda: f(lens=torch.cat((lens, lens)), cu_tokens=cu), lambda: f(cu_tokens=cu, out=torch.zeros_like(q[:1])), lambda: f(cu_tokens=cu, lse=torch.zeros((2, 1), device=DEV))):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(TypeError):
        f(cu_tokens=[0, 3])
    o, lse = f(q=q[:0], cu_tokens=torch.zeros(2, dtype=torch.int32, device=DEV))
    assert o.shape == (0, 2, 64) and lse.shape == (2, 0)


@pytest.mark.parametrize("dense", [False, True], ids=["route", "dense"])
def test_a_serving_step_with_idle_and_released_sequences(dense):
    """The step of a serving loop, captured: sequences wait, end and begin again, each is decoded with its own query.  Against 64 bits over
    the numbers that the cache holds, rows of nobody left as they were."""
    hq, hkv, d, pages, batch = 4, 2, 64, 60, 5
    g = torch.Generator().manual_seed(23)
    rng = np.random.default_rng(23)
    rope = bf1.plan_rope(bf1.RopeCfg(64), DEV)
    route = bf1.RouteCfg(**DENSE) if dense else bf1.RouteCfg()
    kp, vp = (torch.full((pages, 64, hkv, d), 0x7f, dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2))
    ks, vs = (torch.full((pages, hkv), float("nan"), device=DEV) for _ in range(2))
    lens = torch.zeros(batch, dtype=torch.int32, device=DEV)
    new = torch.zeros(batch, dtype=torch.int32, device=DEV)
    table = torch.full((batch, 10), -1, dtype=torch.int32, device=DEV)
    stack, count = torch.arange(pages, dtype=torch.int32, device=DEV), torch.tensor([pages], dtype=torch.int32, device=DEV)
    rows = 90
    step = bf1.CachePlan.empty(batch, rows, DEV)
    lists = bf1.plan_decode(lens, table, route)
    ws = bf1.decode_fp8_workspace(batch, hq, hkv, lists.max_degree, d, DEV)
    q, k, v = (torch.zeros((rows, h, d), dtype=torch.bfloat16, device=DEV) for h in (hq, hkv, hkv))
    turned, out, lse = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((hq, rows), device=DEV)

    def body():
        bf1.plan_cache(lens, new, table, pages, rows, stack, count, plan=step, seqlens_out=lens, free_count_out=count)
        bf1.plan_decode(lens, table, route, plan=lists)
        bf1.cache_write(k, v, kp, vp, step, ks, vs, rope=rope, q=q, out_q=turned)
        bf1.decode_fwd_fp8(turned, kp, vp, ks, vs, lens, lists, ws, out=out, lse=lse, cu_tokens=step.cu_tokens)

    body()                                                          # adds nothing
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        body()
    held = [0] * batch
    for i in range(40):
        counts = [int(rng.choice([1, 1, 0, -1 if n else 0, 40])) if i else 60 - 20 * s * (s < 3) for s, n in enumerate(held)]
        while sum(max(n, 0) for n in counts) > rows:
            counts[counts.index(max(counts))] = 1
        new.copy_(torch.tensor(counts, dtype=torch.int32))
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g).to(torch.bfloat16))
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        graph.replay()
        held = [0 if n < 0 else old + n for n, old in zip(counts, held)]
        assert step.status.item() == 0 and lists.status.item() == 0 and lens.tolist() == held
        cu = step.cu_tokens.tolist()
        live = [s for s, n in enumerate(counts) if n > 0]
        at = [cu[s + 1] - 1 for s in live]
        c = Cache.__new__(Cache)
        c.kp, c.vp, c.ks, c.vs = (t.cpu() for t in (kp, vp, ks, vs))
        c.lens = [held[s] for s in live]
        c.lists = [[int(table[s, b]) for b in logical(held[s], dense)] for s in live]
        check(c, turned[at].cpu(), out[at], lse[:, at])
        others = [r for r in range(rows) if r not in at]
        assert torch.isnan(out[others]).all() and torch.isnan(lse[:, others]).all()


@pytest.mark.parametrize("lens,hq,hkv,d", [([300] * 3, 4, 2, 64), ([256] * 160, 2, 1, 128), ([26000, 70], 2, 1, 128), ([100], 2, 2, 64)], ids=["parts", "whole", "runs", "one"])
def test_nothing_is_done_behind_a_wait_that_ran_out(lens, hq, hkv, d):
    """The bit that a launch leaves behind when it has given up a wait: later ones on its status word write nothing, until a plan clears it."""
    c = Cache(lens, hkv, d, True, seed=24)
    q = queries(len(lens), hq, d, 24)
    lens_d = torch.tensor(lens, dtype=torch.int32, device=DEV)
    plan = bf1.plan_decode(lens_d, c.table.to(DEV), c.cfg)
    plan.status.fill_(4)
    out, lse, _ = run(c, q, plan=plan)
    assert torch.isnan(out).all() and torch.isnan(lse).all() and plan.status.item() == 4
    bf1.plan_decode(lens_d, c.table.to(DEV), c.cfg, plan=plan)
    out, lse, _ = run(c, q, plan=plan)
    assert plan.status.item() == 0
    check(c, q, out, lse)


def test_the_most_lists_that_are_cut():
    """1024 lists of up to 29 pages are dealt in runs, 1025 walked whole: the workspace, which runs alone write to, says so.  The same data on both sides."""
    rng = np.random.default_rng(25)
    lens = [int(x) for x in rng.integers(0, 1850, 1025)]
    lens[3] = 1850
    c = Cache(lens, 1, 64, True, seed=25)
    q = queries(1025, 2, 64, 25)
    args = [t.to(DEV) for t in (c.kp, c.vp, c.ks, c.vs)]
    results = []
    for batch in (1024, 1025):
        lens_d = torch.tensor(lens[:batch], dtype=torch.int32, device=DEV)
        plan = bf1.plan_decode(lens_d, c.table[:batch].contiguous().to(DEV), c.cfg)
        ws = torch.full_like(bf1.decode_fp8_workspace(1024, 2, 1, plan.max_degree, 64, DEV), 0x5a)
        out, lse = torch.full((batch, 2, 64), float("nan"), dtype=torch.bfloat16, device=DEV), torch.full((2, batch), float("nan"), device=DEV)
        bf1.decode_fwd_fp8(q[:batch].to(DEV), *args, lens_d, plan, ws, out=out, lse=lse)
        assert plan.status.item() == 0 and ws.ne(0x5a).any().item() == (batch == 1024)
        results.append((out, lse))
    check(c, q, *results[1])
    c.lens, c.lists = lens[:1024], c.lists[:1024]
    check(c, q[:1024], *results[0])
