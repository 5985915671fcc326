"""Filling the paged cache without a GPU: the oracle's numbers in 8 bits, the tables' invariants, the host's refusals."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2608_20427_b200 as bf1
from oracle import cache_oracle as C
from paper_2608_20427_b200 import binding


def test_numbers_in_8_bits_are_those_of_the_type():
    """All 256 codes come back as they are; what lies between goes to the nearer, ties to the even one (torch's conversion)."""
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    fine = codes[np.isfinite(codes)]
    assert np.array_equal(C.to_e4m3(fine), fine) and fine.max() == C.E4M3_MAX
    rng = np.random.default_rng(3)
    x = np.concatenate([rng.standard_normal(4000) * s for s in (1e-3, 0.02, 1.0, 100.0)] + [(fine[:-1] + fine[1:]) / 2]).clip(-448, 448)
    x = x.astype(np.float32).astype(np.float64)
    assert np.array_equal(C.to_e4m3(x), torch.tensor(x, dtype=torch.float32).to(torch.float8_e4m3fn).double().numpy())
    assert np.isnan(C.to_e4m3([np.inf, -np.inf, np.nan])).all()


def test_scale_of_a_page():
    assert C.page_scale(np.array([0.0])) == 2.0 ** -64 and C.page_scale(np.array([np.nan, np.inf])) == 2.0 ** -64
    for top, e in ((448.0, 0), (448.0001, 1), (447.0, 0), (224.0, -1), (224.001, 0), (3.5, -7), (3.53, -6), (1e-30, -64), (2.0 ** 127 * 1.9, 120)):
        assert C.page_scale(np.array([0.0, -top, np.inf])) == 2.0 ** e, top


def test_steps_of_the_tables_keep_every_page_once():
    rng = np.random.default_rng(4)
    pages, width, batch = 60, 12, 9
    lens, table, free = [0] * batch, [[-1] * width for _ in range(batch)], [int(x) for x in rng.permutation(pages)]
    for step in range(200):
        new = [int(rng.choice([0, 1, 1, 1, 30, 130, -1])) for _ in range(batch)]
        try:
            lens, table, free, cu, pos, slots, units = C.plan_cache(lens, new, table, pages, 1000, free)
        except C.Refused:
            continue
        held = [p for n, row in zip(lens, table) for p in row[:(n + 63) // 64]]
        assert sorted(held + free) == list(range(pages))
        assert len(set(slots)) == len(slots) and sum(u[1] for u in units) == len(slots) == cu[-1]
        assert len(units) <= bf1.load().bf1_cache_plan_units(batch, len(slots))
    assert lens != [0] * batch


def test_the_bound_on_units_is_reached():
    lib = bf1.load()
    for lens, new in (([63], [66]), ([63] * 3, [2, 2, 2]), ([0], [64]), ([1], [1])):
        table = [list(range(10 * s, 10 * s + 9)) for s in range(len(lens))]
        units = C.plan_cache(lens, new, table, 100, sum(new))[6]
        assert len(units) <= lib.bf1_cache_plan_units(len(lens), sum(new))
    assert lib.bf1_cache_plan_units(3, 6) == 6 and lib.bf1_cache_plan_units(1, 66) == 3
    assert lib.bf1_cache_plan_units(0, 0) == 1 and lib.bf1_cache_plan_units(-1, 5) == -1 and lib.bf1_cache_plan_units(5, -1) == -1


def plan_c(batch=2, tokens=8, cap=8, **kw):
    fields = dict(seqlens=0x1000, free_count=0x1000, cu_tokens=0x1000, positions=0x1000, slots=0x1000, units=0x1000, num_units=0x1000, starts=0x1000,
                  status=0x1000)
    fields.update(kw)
    return ctypes.byref(binding._CachePlanC(batch, tokens, cap, *fields.values()))


def test_refusals_of_the_tables():
    lib = bf1.load()
    f = 0x1000

    def call(lens=f, new=f, table=f, width=4, pages=10, free=f, count=f, plan=None):
        return lib.bf1_plan_cache(lens, new, table, width, pages, free, count, plan or plan_c(), None)

    assert lib.bf1_plan_cache(f, f, f, 4, 10, f, f, None, None) == -1
    assert call(lens=None) == -1 and call(new=None) == -1 and call(table=None) == -1
    assert call(free=None) == -1 and call(count=None) == -1
    assert call(width=0) == -2 and call(pages=0) == -2 and call(width=(1 << 24) + 1) == -2 and call(pages=1 << 25) == -2
    for name in ("seqlens", "free_count", "cu_tokens", "positions", "slots", "units", "num_units", "starts", "status"):
        assert call(plan=plan_c(**{name: None})) == -1, name
    assert call(plan=ctypes.byref(binding._CachePlanC(2, 8, 8, *[0x1000] * 5, 0x1008, *[0x1000] * 3))) == -1
    assert call(plan=plan_c(starts=0x1004)) == -1 and b"aligned" in lib.bf1_last_error()
    assert call(plan=plan_c(batch=-1)) == -1 and call(plan=plan_c(batch=65536)) == -1 and call(plan=plan_c(tokens=-1)) == -1
    assert call(plan=plan_c(tokens=(1 << 30) + 1)) == -1
    short = binding._CachePlanC(2, 8, 3, *[0x1000] * 9)
    assert lib.bf1_plan_cache(f, f, f, 4, 10, f, f, ctypes.byref(short), None) == -3


def test_refusals_of_the_write():
    lib = bf1.load()
    f = ctypes.c_void_p(0x1000)
    rows = lambda p=0x1000, row=128, head=64: ctypes.byref(binding._RowsC(p, row, head))  # noqa: E731
    rope = lambda dim=64: ctypes.byref(binding._RopeC(dim, 0, 1.0, 0x1000))  # noqa: E731

    def call(k=None, v=None, q=None, tokens=8, hq=0, hkv=1, d=64, plan=None, r=None, pages=10, kp=f, vp=f, ks=f, vs=f, oq=None):
        return lib.bf1_cache_write(k or rows(), v or rows(), q, tokens, hq, hkv, d, plan or plan_c(), r, pages, kp, vp, ks, vs, oq, None)

    assert lib.bf1_cache_write(rows(), rows(), None, 8, 0, 1, 64, None, None, 10, f, f, f, f, None, None) == -1
    assert call(tokens=7) == -1 and b"plan is for" in lib.bf1_last_error()
    assert call(tokens=-1) == -1 and call(hkv=0) == -1 and call(hq=-1) == -1 and call(pages=0) == -1
    assert call(d=96) == -2 and call(hkv=65536) == -2
    assert call(kp=None) == -1 and call(vp=None) == -1 and call(kp=ctypes.c_void_p(0x1008)) == -1
    assert call(ks=None) == -1 and call(vs=None) == -1
    assert call(k=rows(None)) == -1 and call(v=rows(0x1002)) == -1 and call(k=rows(row=4)) == -1
    assert call(hq=2, q=rows(), oq=rows()) == -1 and b"rope" in lib.bf1_last_error()      # queries without a rope
    assert call(hq=2, q=rows(), oq=rows(None), r=rope()) == -1 and call(hq=2, q=rows(None), oq=rows(), r=rope()) == -1
    assert call(hq=2, q=rows(), oq=rows(row=256), r=rope()) == -1 and b"in place" in lib.bf1_last_error()
    assert call(r=rope(128)) == -2
    short = binding._CachePlanC(2, 8, 3, *[0x1000] * 9)
    assert call(plan=ctypes.byref(short)) == -3
    assert call(tokens=0, plan=plan_c(tokens=0)) == 0 and call(plan=plan_c(batch=0)) == 0   # nothing to do, nothing launched


def test_plans_of_the_binding():
    p = bf1.CachePlan.empty(3, 100, "cpu")
    assert p.units.shape == (7, 4) and p.c.capacity_units == 7 and p.c.capacity_tokens == 100 and p.c.batch == 3
    with pytest.raises(ValueError):
        bf1.CachePlan.empty(-1, 5, "cpu")
    with pytest.raises(ValueError):
        bf1.plan_cache(torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros((3, 4), dtype=torch.int32), 10, 99, plan=p)
