"""Filling the paged cache on the GPU: the tables of a step (whole numbers, equal to the oracle's) and the write against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2608_20427_b200 as bf1
from oracle import cache_oracle as C

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
E4M3 = torch.float8_e4m3fn


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def tables(lens, pages, width, rng):
    """A page table for the cached tokens and a stack of what is left of `pages`."""
    perm = [int(x) for x in rng.permutation(pages)]
    table = [[-1] * width for _ in lens]
    for s, n in enumerate(lens):
        for b in range((n + 63) // 64):
            table[s][b] = perm.pop()
    return table, perm


def stack_of(free, pages):
    t = torch.full((pages,), -9, dtype=torch.int32, device=DEV)
    t[:len(free)] = ints(free) if free else t[:0]
    return t


def check_step(plan, lens, new, table_in, table, stack, free, pages, tokens):
    want = C.plan_cache(lens, new, table_in, pages, tokens, free)
    lens_w, table_w, free_w, cu, pos, slots, units = want
    assert plan.status.item() == 0
    assert plan.seqlens.tolist() == lens_w and plan.cu_tokens.tolist() == cu and table.tolist() == table_w
    pad = [-1] * (tokens - len(pos))
    assert plan.positions.tolist() == pos + pad and plan.slots.tolist() == slots + pad
    assert plan.num_units.item() == len(units)
    assert plan.units.tolist() == units + [[-1] * 4] * (plan.units.shape[0] - len(units))
    if free is not None:
        assert plan.free_count.item() == len(free_w) and stack[:len(free_w)].tolist() == free_w
    return want


STEPS = {
    "one-token": ([0], [1], 1),
    "one-token-later": ([127], [1], 1),
    "page-is-full": ([128], [1], 5),
    "prompt-and-tokens": ([0, 5, 64, 63, 0, 130], [200, 1, 1, 2, 0, 64], 300),
    "released": ([100, 0, 64, 65, 1], [-1, 128, -1, 1, -1], 129),
    "nothing-new": ([3, 0, 70], [0, 0, 0], 4),
    "no-tokens-at-all": ([3, 70], [-1, 0], 0),
}


@pytest.mark.parametrize("name", STEPS)
def test_a_step(name):
    lens, new, tokens = STEPS[name]
    rng = np.random.default_rng(len(name))
    pages, width = 30, 6
    table_in, free = tables(lens, pages, width, rng)
    table, stack = ints(table_in), stack_of(free, pages)
    plan = bf1.plan_cache(ints(lens), ints(new), table, pages, tokens, stack, ints([len(free)]))
    check_step(plan, lens, new, table_in, table, stack, free, pages, tokens)
    # the same pages without a stack: the table is complete
    full = ints(C.plan_cache(lens, new, table_in, pages, tokens, free)[1])
    again = bf1.plan_cache(ints(lens), ints(new), full, pages, tokens)
    assert torch.equal(again.slots, plan.slots) and torch.equal(again.units, plan.units) and torch.equal(again.seqlens, plan.seqlens)


@pytest.mark.parametrize("batch,tokens", [(1, 40000), (700, 3000), (1023, 5000), (1024, 5000), (1025, 5000), (5000, 30000), (40000, 90000)])
def test_random_steps(batch, tokens):
    """One cluster of one or eight CTAs, one chunk of sequences or many."""
    rng = np.random.default_rng(batch)
    width = 700 if batch == 1 else 9
    lens = [int(x) for x in rng.integers(0, 300, batch)]
    new = [int(x) for x in rng.choice([0, 1, 1, 1, -1, 2, 9], batch)]
    if batch == 1:
        new = [39000]
    for s in range(0, batch, 97):
        if batch > 1 and sum(max(x, 0) for x in new) < tokens - 250:
            new[s] = int(rng.integers(60, 240))
    held = sum((n + 63) // 64 for n in lens)
    grow = sum((n + max(a, 0) + 63) // 64 - (n + 63) // 64 for n, a in zip(lens, new))
    pages = held + grow + 3
    table_in, free = tables(lens, pages, width, rng)
    table, stack = ints(table_in), stack_of(free, pages)
    plan = bf1.plan_cache(ints(lens), ints(new), table, pages, tokens, stack, ints([len(free)]))
    check_step(plan, lens, new, table_in, table, stack, free, pages, tokens)


def test_many_steps_in_place_and_in_a_graph():
    """Lengths and stack updated in place by one captured step that is replayed with other new lengths."""
    rng = np.random.default_rng(8)
    batch, pages, width, tokens = 40, 200, 10, 700
    lens, free = [0] * batch, [int(x) for x in rng.permutation(pages)]
    table_h = [[-1] * width for _ in range(batch)]
    dl, dn, table, stack, count = ints(lens), ints([0] * batch), ints(table_h), stack_of(free, pages), ints([pages])
    plan = bf1.CachePlan.empty(batch, tokens, DEV)

    def step():
        bf1.plan_cache(dl, dn, table, pages, tokens, stack, count, plan=plan, seqlens_out=dl, free_count_out=count)

    step()                                                       # adds nothing
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    done = refused = 0
    for i in range(60):
        new = [int(x) for x in rng.choice([0, 1, 1, 1, 1, -1, 64, 120] if i % 3 == 0 else [1, 1, 1, 0], batch)]
        dn.copy_(ints(new))
        before = (dl.tolist(), table.tolist(), count.item(), stack[:count.item()].tolist())
        graph.replay()
        try:
            lens, table_h, free, cu, pos, slots, units = C.plan_cache(lens, new, table_h, pages, tokens, free)
        except C.Refused:
            refused += 1
            assert plan.status.item() != 0 and plan.num_units.item() == 0 and plan.cu_tokens.tolist() == [0] * (batch + 1)
            assert (dl.tolist(), table.tolist(), count.item(), stack[:count.item()].tolist()) == before
            continue
        done += 1
        assert plan.status.item() == 0 and dl.tolist() == lens and table.tolist() == table_h
        assert count.item() == len(free) and stack[:len(free)].tolist() == free
        assert plan.slots[:len(slots)].tolist() == slots and plan.units[:len(units)].tolist() == units
    assert done > 20 and refused > 2


@pytest.mark.parametrize("lens,new,tokens,free,bits", [
    ([5, -1], [1, 1], 9, 5, 1), ([5, 0], [1, -2], 9, 5, 1), ([5, 256], [1, 1], 9, 5, 1), ([0, 2 ** 31 - 1], [1, 1], 9, 5, 1),
    ([5, 0], [2 ** 31 - 1, 1], 9, 5, 1), ([5, 0], [5, 5], 9, 5, 2), ([0, 0], [65, 65], 200, 3, 2), ([0, 0], [64, 64], 200, -1, 2),
    ([64, 0], [-1, 64], 200, 10, 2)])
def test_refused_steps_change_nothing(lens, new, tokens, free, bits):
    pages, width = 10, 4
    table_in = [[7, 8, 9, 6], [1, 2, 3, 4]]
    table, stack = ints(table_in), stack_of([5, 0, 3, 2, 1, 9, 8, 7, 6, 4], pages)
    was = stack.clone()
    plan = bf1.CachePlan.empty(2, tokens, DEV)
    for t in (plan.seqlens, plan.positions, plan.slots, plan.units, plan.num_units, plan.cu_tokens):
        t.fill_(77)
    bf1.plan_cache(ints(lens), ints(new), table, pages, tokens, stack, ints([free]), plan=plan)
    assert plan.status.item() == bits
    assert plan.seqlens.tolist() == lens and plan.free_count.item() == free and table.tolist() == table_in and torch.equal(stack, was)
    assert plan.cu_tokens.tolist() == [0, 0, 0] and plan.num_units.item() == 0
    assert all((t == -1).all().item() for t in (plan.positions, plan.slots, plan.units))
    with pytest.raises(bf1.Bf1Error):
        plan.check_status()


def test_bad_pages_are_reported_and_not_written():
    table, pages = ints([[99, -3], [0, 1]]), 4
    plan = bf1.plan_cache(ints([10, 60]), ints([60, 10]), table, pages, 70)
    assert plan.status.item() == 8
    assert plan.slots.tolist() == [-1] * 60 + [60, 61, 62, 63] + list(range(64, 70))
    assert plan.units.tolist() == [[0, 54, -1, 10], [54, 6, -1, 0], [60, 4, 0, 60], [64, 6, 1, 0], [-1] * 4]
    k = torch.ones((70, 1, 64), dtype=torch.bfloat16, device=DEV)
    kp, vp = (torch.zeros((pages, 64, 1, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    bf1.cache_write(k, k, kp, vp, plan)
    assert plan.status.item() == 8 and kp[0, 60:].eq(1).all() and kp[1, :6].eq(1).all() and kp.sum().item() == 10 * 64


# ---- the write --------------------------------------------------------------------------------------------------------------------------
def cache(pages, hkv, d, fp8, g):
    """Pages full of something, with scales that are powers of two."""
    if fp8:
        kp, vp = ((torch.randn((pages, 64, hkv, d), generator=g) * 40).clamp(-448, 448).to(E4M3).to(DEV) for _ in range(2))
        ks, vs = (2.0 ** torch.randint(-9, -5, (pages, hkv), generator=g).float().to(DEV) for _ in range(2))
        return kp, vp, ks, vs
    kp, vp = (torch.randn((pages, 64, hkv, d), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    return kp, vp, None, None


def check_write(got, before, x, plan, scales=None, scales_before=None, exact_input=True):
    """Pages in 8 bits hold whole numbers of steps: equal to the oracle's where the input is exact.  Where the input has been rotated in
    32 bits (off by 2^-20 of the pair, see the rotation's own tests) a value may lie across a tie: one step, 2^-3 of the value, or the
    smallest step, 2^-9."""
    want = before.double().cpu().numpy()
    ws = None if scales is None else scales_before.double().cpu().numpy()
    units = [u for u in plan.units.tolist() if u[1] > 0]
    C.write_pages(want, ws, x, units)
    got = got.double().cpu().numpy()
    if scales is not None:
        assert np.array_equal(scales.double().cpu().numpy(), ws)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    if exact_input:
        assert same.all()
    elif scales is not None:
        assert (same | (np.abs(got - want) <= np.maximum(np.abs(want) * 2.0 ** -3, 2.0 ** -9))).all() and same.mean() > 0.999
    else:
        rows = np.zeros(want.shape[:2], bool)
        for first, count, page, row in units:
            rows[page, row:row + count] = True
        assert same[~rows].all()
        assert (np.abs(got - want) <= np.abs(want) * 2.0 ** -8 + 2.0 ** -17).all()


WRITES = [([0], [1]), ([63], [1]), ([64], [1]), ([10, 0, 127, 64, 31], [1, 1, 1, 0, 1]), ([0, 61, 64, 5], [64, 6, 129, 200]), ([3, 3], [2, 5]), ([1], [63]),
          ([0] * 40, [1] * 40), ([61] + [9] * 39, [55] + [0] * 20 + [1] * 19)]


@pytest.mark.parametrize("fp8", [True, False], ids=["e4m3", "bf16"])
@pytest.mark.parametrize("hkv,d", [(1, 64), (3, 128), (8, 64)])
@pytest.mark.parametrize("lens,new", WRITES, ids=lambda v: "-".join(str(x) for x in v[:5]))
def test_write(lens, new, hkv, d, fp8):
    g = torch.Generator().manual_seed(sum(lens) + hkv + d)
    rng = np.random.default_rng(5)
    tokens, pages = sum(new) + 3, 60 + len(lens)
    table_in, free = tables(lens, pages, 8, rng)
    plan = bf1.plan_cache(ints(lens), ints(new), ints(table_in), pages, tokens, stack_of(free, pages), ints([len(free)]))
    # sizes all over the place, so that scales of partial pages have to grow, or stay
    size = 10.0 ** torch.empty((tokens, hkv, 1)).uniform_(-2, 1, generator=g)
    k, v = ((torch.randn((tokens, hkv, d), generator=g) * size).to(torch.bfloat16) for _ in range(2))
    k[sum(new):] = float("nan")                                   # rows behind the last token are not read
    v[sum(new):] = float("nan")
    kp, vp, ks, vs = cache(pages, hkv, d, fp8, g)
    was = [None if t is None else t.clone() for t in (kp, vp, ks, vs)]
    assert bf1.cache_write(k.to(DEV), v.to(DEV), kp, vp, plan, ks, vs) is None
    assert plan.status.item() == 0
    check_write(kp, was[0], k.double().numpy(), plan, ks, was[2])
    check_write(vp, was[1], v.double().numpy(), plan, vs, was[3])
    now = [None if t is None else t.clone() for t in (kp, vp, ks, vs)]
    bf1.cache_write(k.to(DEV), v.to(DEV), kp, vp, plan, ks, vs)   # the same once more changes nothing
    assert all(x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(now, (kp, vp, ks, vs)))


def test_a_refused_step_writes_nothing():
    """Its plan has no units and no positions: pages, scales and rotated queries stay as they are."""
    g = torch.Generator().manual_seed(3)
    rope = bf1.plan_rope(bf1.RopeCfg(64), DEV)
    for tokens in (3, 40):                                          # both kernels
        kp, vp, ks, vs = cache(4, 2, 64, True, g)
        was = [t.clone() for t in (kp, vp, ks, vs)]
        plan = bf1.plan_cache(ints([0, 0, 0]), ints([1, 1, 1000]), ints([[0], [1], [2]]), 4, tokens)
        assert plan.status.item() & 1
        k = torch.ones((tokens, 2, 64), dtype=torch.bfloat16, device=DEV)
        out = torch.full_like(k, 5.0)
        bf1.cache_write(k, k, kp, vp, plan, ks, vs, rope=rope, q=k, out_q=out)
        assert out.eq(5).all() and all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(was, (kp, vp, ks, vs)))


def test_scales_grow_token_by_token_as_for_the_whole_page():
    """64 single tokens, each larger than those before it: the scale is at every step the whole page's."""
    hkv, d = 2, 64
    g = torch.Generator().manual_seed(7)
    x = (torch.randn((64, hkv, d), generator=g) * 1.5 ** torch.arange(64.0)[:, None, None] * 1e-3).to(torch.bfloat16)
    kp, vp = (torch.zeros((1, 64, hkv, d), device=DEV).to(E4M3) for _ in range(2))
    ks, vs = (torch.full((1, hkv), 2.0 ** 90, device=DEV) for _ in range(2))      # left over from another sequence
    for n in range(64):
        plan = bf1.plan_cache(ints([n]), ints([1]), ints([[0]]), 1, 1)
        bf1.cache_write(x[n:n + 1].to(DEV), x[n:n + 1].neg().to(DEV), kp, vp, plan, ks, vs)
        want = [C.page_scale(x[:n + 1, h].double().numpy()) for h in range(hkv)]
        assert ks[0].tolist() == want and vs[0].tolist() == want
    whole = bf1.plan_cache(ints([0]), ints([64]), ints([[0]]), 1, 64)
    kw, vw = torch.zeros_like(kp), torch.zeros_like(vp)
    bf1.cache_write(x.to(DEV), x.neg().to(DEV), kw, vw, whole, ks.clone(), vs.clone())
    # only values below 2^-6 of the scale have been rounded on the way: each move rounds by half of 2^-9 at most, and halves what was off
    off = (kp.double() - kw.double()).abs()
    assert (off[kw.double().abs() >= 2.0 ** -6] <= 2.0 ** -9).all() and off.max().item() <= 2.0 ** -9
    assert torch.equal(vp.double(), -kp.double())


@pytest.mark.parametrize("many", [False, True], ids=["token", "page"])
def test_values_that_are_not_finite_and_zeros(many):
    """Infinities and NaN are stored as NaN and do not count for the scale; a page of zeros has the smallest scale."""
    n = 64 if many else 1
    x = torch.zeros((n, 3, 64), dtype=torch.bfloat16)
    x[0, 0, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 3.0])
    x[0, 1, 5] = 3.3895313892515355e38                              # the largest there is
    plan = bf1.plan_cache(ints([0]), ints([n]), ints([[0]]), 1, n)
    kp, vp = (torch.zeros((1, 64, 3, 64), device=DEV).to(E4M3) for _ in range(2))
    ks, vs = (torch.ones((1, 3), device=DEV) for _ in range(2))
    bf1.cache_write(x.to(DEV), x.to(DEV), kp, vp, plan, ks, vs)
    assert ks[0].tolist() == [2.0 ** -7, 2.0 ** 120, 2.0 ** -64] and torch.equal(ks, vs)
    got = kp[0, 0].float().cpu()
    assert torch.isnan(got[0, :3]).all() and got[0, 3] == 384.0 and got[1, 5] == 256.0 and got[2].eq(0).all()
    assert torch.isfinite(kp[0].float()).sum().item() == 64 * 3 * 64 - 3


@pytest.mark.parametrize("fp8", [True, False], ids=["e4m3", "bf16"])
@pytest.mark.parametrize("layout,dim,d,hq,hkv", [("half", 128, 128, 16, 8), ("half", 48, 64, 3, 1), ("interleaved", 64, 64, 8, 2), ("interleaved", 32, 128, 5, 5)])
@pytest.mark.parametrize("lens,new", [([5, 1000, 63], [1, 1, 1]), ([100, 0], [90, 70]), ([50] + [7] * 29, [36] + [0] * 8 + [1] * 21), ([3, 62], [1, 2])],
                         ids=["tokens", "prompts", "prompt-among-tokens", "few"])
def test_write_with_a_rope(lens, new, layout, dim, d, hq, hkv, fp8):
    g = torch.Generator().manual_seed(dim + hq)
    tokens, pages = sum(new) + 2, 40
    pages += len(lens)
    table_in, free = tables(lens, pages, 18, np.random.default_rng(6))
    plan = bf1.plan_cache(ints(lens), ints(new), ints(table_in), pages, tokens, stack_of(free, pages), ints([len(free)]))
    k, v = (torch.randn((tokens, hkv, d), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    q = torch.randn((tokens, hq, d), generator=g).to(torch.bfloat16).to(DEV)
    cfg = bf1.RopeCfg(dim, layout=layout)
    rope = bf1.plan_rope(cfg, DEV)
    kp, vp, ks, vs = cache(pages, hkv, d, fp8, g)
    was = [None if t is None else t.clone() for t in (kp, vp, ks, vs)]
    out = torch.full_like(q, 7.0)
    assert bf1.cache_write(k, v, kp, vp, plan, ks, vs, rope=rope, q=q, out_q=out) is out
    turns, _ = C.rope_turns(dim)
    pos = plan.positions.tolist()
    x = C.rotate(k.double().cpu().numpy(), pos, turns, 1.0, layout)
    x = np.nan_to_num(x, nan=0.0)
    check_write(kp, was[0], x, plan, ks, was[2], exact_input=False)
    check_write(vp, was[1], v.double().cpu().numpy(), plan, vs, was[3])
    want, want_k = bf1.rope_fwd(q, k, plan.positions, rope)
    n = sum(new)
    assert torch.equal(out[:n], want[:n]) and out[n:].eq(7).all()
    if not fp8:                                                      # bit for bit what the rotation and a plain write give
        kp2, vp2 = was[0].clone(), was[1].clone()
        bf1.cache_write(want_k, v, kp2, vp2, plan)
        assert torch.equal(kp, kp2) and torch.equal(vp, vp2)
    assert bf1.cache_write(k, v, kp, vp, plan, ks, vs, rope=rope) is None      # keys alone
    made = bf1.cache_write(k, v, kp, vp, plan, ks, vs, rope=rope, q=q)
    assert torch.equal(made[:n], want[:n])


def test_strided_rows_far_pages_and_another_stream():
    """K and V as parts of a projection's output, pages beyond 2^31 elements of the cache, a stream of its own."""
    hkv, d = 8, 128
    pages = (1 << 31) // (64 * hkv * d) + 40
    g = torch.Generator().manual_seed(12)
    row = torch.randn((66, 4 * hkv * d), generator=g).to(torch.bfloat16).to(DEV)
    k, v = row[:, hkv * d:2 * hkv * d].view(66, hkv, d), row[:, 3 * hkv * d:].view(66, hkv, d)
    kp, vp = (torch.zeros((pages, 64, hkv, d), dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2))
    ks, vs = (torch.ones((pages, hkv), device=DEV) for _ in range(2))
    plan = bf1.plan_cache(ints([0]), ints([66]), ints([[pages - 1, pages - 3]]), pages, 66)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    bf1.cache_write(k, v, kp, vp, plan, ks, vs, stream=side)
    side.synchronize()
    for pg, x, sc in ((kp, k, ks), (vp, v, vs)):
        x = x.double().cpu().numpy()
        want, ws = np.zeros((2, 64, hkv, d)), np.ones((2, hkv))
        C.write_pages(want, ws, x, [[0, 64, 0, 0], [64, 2, 1, 0]])
        assert np.array_equal(pg[[pages - 1, pages - 3]].double().cpu().numpy(), want) and np.array_equal(sc[[pages - 1, pages - 3]].double().cpu().numpy(), ws)
        assert sc.ne(1).sum().item() == 2 * hkv and not pg.view(torch.uint8)[:pages - 3].any().item()


def test_refusals_of_the_binding():
    k = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device=DEV)
    plan = bf1.plan_cache(ints([0]), ints([4]), ints([[0]]), 2, 4)
    kp, vp = (torch.zeros((2, 64, 2, 64), dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2))
    ks, vs = (torch.ones((2, 2), device=DEV) for _ in range(2))
    for bad in (lambda: bf1.cache_write(k, k, kp, vp, plan), lambda: bf1.cache_write(k, k, kp, vp, plan, ks), lambda: bf1.cache_write(k, k[:3], kp, vp, plan, ks, vs),
                lambda: bf1.cache_write(k, k, kp[:, :32], vp, plan, ks, vs), lambda: bf1.cache_write(k, k, kp[:, :, :1], vp, plan, ks, vs),
                lambda: bf1.cache_write(k, k, kp, vp[:1], plan, ks, vs), lambda: bf1.cache_write(k, k, kp, vp, plan, ks[:1], vs),
                lambda: bf1.cache_write(k, k, kp, vp, plan, ks.double(), vs), lambda: bf1.cache_write(k.cpu(), k, kp, vp, plan, ks, vs),
                lambda: bf1.cache_write(k, k, kp.cpu(), vp, plan, ks, vs), lambda: bf1.cache_write(k, k, kp, vp, bf1.CachePlan.empty(1, 4, "cpu"), ks, vs),
                lambda: bf1.cache_write(k, k, kp, vp, plan, ks, vs, rope=bf1.plan_rope(bf1.RopeCfg(64), "cpu")),
                lambda: bf1.cache_write(k, k, kp, vp, plan, ks, vs, rope=bf1.plan_rope(bf1.RopeCfg(64), DEV), q=k[:3]),
                lambda: bf1.plan_cache(ints([0]), ints([4, 1]), ints([[0]]), 2, 4), lambda: bf1.plan_cache(ints([0]), ints([4]), ints([[0], [1]]), 2, 4),
                lambda: bf1.plan_cache(ints([0]), ints([4]).long(), ints([[0]]), 2, 4), lambda: bf1.plan_cache(ints([0]), ints([4]).cpu(), ints([[0]]), 2, 4),
                lambda: bf1.plan_cache(ints([0]), ints([4]), ints([[0]]), 2, 4, ints([1]), ints([1])), lambda: bf1.plan_cache(ints([0]), ints([4]), ints([[0]]), 2, 4, ints([1, 0])),
                lambda: bf1.plan_cache(ints([0]), ints([4]), ints([[0]]), 2, 4, plan=bf1.CachePlan.empty(1, 4, "cpu")),
                lambda: bf1.plan_cache(ints([0]), ints([4]), ints([[0]]), 0, 4)):
        with pytest.raises(AssertionError):
            bad()
    for bad in (lambda: bf1.cache_write(k, k, kp, vp, bf1.CachePlan.empty(1, 5, DEV), ks, vs), lambda: bf1.cache_write(k, k, kp, vp, plan, ks, vs, q=k),
                lambda: bf1.cache_write(k, k, kp, vp, plan, ks, vs, rope=bf1.plan_rope(bf1.RopeCfg(128), DEV))):
        with pytest.raises(bf1.Bf1Error):
            bad()
