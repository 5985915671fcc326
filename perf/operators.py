"""The operators around the paged cache: what is measured of them, in which cases, and what a pass cannot do without.

  rope    rotary positions on the queries and keys of a packed batch (`rope_fwd`), and in training on their gradients (`rope_bwd`)
  tables  a serving step's page table, positions, slots and write units, built from the requests' lengths (`plan_cache`)
  write   a step's keys and values put into the pages (`cache_write`): in 8 bits with a scale for each page and KV head, or in
          bf16; for single tokens the rotation of queries and keys is part of the call
  decode  one token per sequence over a cache in 8 bits (`decode_fwd_fp8`), along the BF1 route or over every page

Where `own` is false `run` computes the same in elementary torch operations.
"""
import math

import torch

own = False

PAGE = 64
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -64


# ---- cases ------------------------------------------------------------------------------------------------------------------

def _text(values):
    return " ".join(str(int(v)) for v in values)


def _numbers(text):
    return [int(x) for x in text.split()]


def _rope(name, lens, hq, hkv, d, rot, layout, scaling="none", grad=False, fused=False):
    """`lens` tokens per sequence, positions from 0 in each; `fused`: q and k are parts of one projection's output."""
    case = {"op": "rope", "lens": _text(lens), "hq": hq, "hkv": hkv, "d": d, "rot": rot, "layout": layout, "scaling": scaling,
            "grad": grad, "fused": fused, "first": 0}
    return dict(case, name=name) if name else case


def _tables(name, old, new, spare, max_pages):
    """`old` cached tokens and `new` tokens of every sequence (-1: it is released); `spare` rows behind the last token."""
    case = {"op": "tables", "old": _text(old), "new": _text(new), "spare": spare, "max_pages": max_pages}
    return dict(case, name=name) if name else case


def _write(name, old, new, hq, hkv, d, fp8=True, rot=0, layout="half"):
    """`rot` dimensions are rotated in the call (0: none; then there are no queries either)."""
    case = {"op": "write", "old": _text(old), "new": _text(new), "hq": hq, "hkv": hkv, "d": d, "fp8": fp8, "rot": rot, "layout": layout}
    return dict(case, name=name) if name else case


def _decode(name, lens, hq, hkv, d, dense=False):
    case = {"op": "decode", "lens": _text(lens), "hq": hq, "hkv": hkv, "d": d, "dense": dense}
    return dict(case, name=name) if name else case


_SERVING = [65536 - 1777 * i - 13 * (i % 5) for i in range(32)]


def listed():
    return [
        # one decode step of eight users over a bf16 cache: the smallest call, launches and host work
        dict(_rope("rope_step_8", [1] * 8, 16, 8, 128, 128, "half"), first=20011),
        # a training step's layer on packed documents: queries and keys in the output of one projection, their gradients back into one
        _rope("rope_train_4k", [130, 2048, 777, 65, 1, 1075], 16, 8, 128, 128, "interleaved", grad=True, fused=True),
        # a long prompt, positions stretched beyond the length the model was trained at
        _rope("rope_32k", [32768], 16, 8, 128, 128, "half", scaling="yarn"),
        # a decode step of a serving batch: every sequence grows by a token, some by a page
        _tables("tables_step_32", _SERVING, [1] * 32, 0, 1025),
        # a step that takes in long and short prompts beside decoding sequences and lets finished ones go
        _tables("tables_mixed_512", [(977 * i) % 4000 for i in range(512)],
                [-1 if i % 16 == 3 else 1 if i % 4 else 1 + (2749 * i) % 2048 for i in range(512)], 100, 128),
        # the next token of eight users
        _write("write_step_8", [32767, 999, 20010, 64, 32000, 4096, 9998, 16383], [1] * 8, 16, 8, 128, rot=128),
        # the next token of a large serving batch
        _write("write_step_256", [(977 * i) % 30000 for i in range(256)], [1] * 256, 16, 8, 128, rot=128),
        # a prompt's keys and values, rotated already for its attention, some of it behind what is cached
        _write("write_prompts_32k", [0, 1000, 65, 0], [16384, 3001, 1038, 12345], 16, 8, 128),
        # one user's next token, along the route
        _decode("decode_1", [32768], 16, 8, 128),
        # a serving batch along the route
        _decode("decode_32", _SERVING, 16, 8, 128),
        # a layer that stays dense, one user with a long context
        _decode("decode_dense_100k", [100003], 16, 8, 128, dense=True),
        # a layer that stays dense, users with contexts of all lengths
        _decode("decode_dense_24", [32768 - 1361 * i - 7 * (i % 3) for i in range(24)], 16, 8, 128, dense=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _split(rng, total, parts):
    parts = min(parts, total)
    cuts = sorted(rng.sample(range(1, total), parts - 1)) if parts > 1 else []
    return [b - a for a, b in zip([0] + cuts, cuts + [total])]


def draw(rng):
    op = rng.choice(["rope", "tables", "write", "write", "decode", "decode", "decode"])
    hkv = rng.choice([1, 2, 4, 8])
    hq, d = hkv * rng.choice([1, 2, 2, 4]), rng.choice([64, 128, 128])
    layout = rng.choice(["half", "half", "interleaved"])
    rot = rng.choice([d, d, d // 2, d // 4])
    if op == "rope":
        total = _log_int(rng, 1, 32768 if hq <= 16 else 16384)
        case = _rope(None, _split(rng, total, rng.choice([1, 1, 3, 9])), hq, hkv, d, rot, layout,
                     rng.choice(["none", "linear", "ntk", "yarn"]), rng.random() < 0.4, rng.random() < 0.5)
        return dict(case, first=rng.choice([0, 0, _log_int(rng, 1, 1000000)]))
    if op == "tables":
        batch = _log_int(rng, 1, 1000)
        old = [rng.choice([0, _log_int(rng, 1, 8000)]) for _ in range(batch)]
        long = rng.random()
        new = [-1 if rng.random() < 0.05 else 0 if rng.random() < 0.05 else _log_int(rng, 1, 1000) if rng.random() < long else 1 for _ in range(batch)]
        new[0] = max(new[0], 1)
        return _tables(None, old, new, rng.choice([0, 0, rng.randrange(1, 200)]), 150)
    if op == "write":
        if rng.random() < 0.5:
            batch = _log_int(rng, 1, 400)
            return _write(None, [rng.choice([0, _log_int(rng, 1, 60000), _log_int(rng, 1, 60000)]) for _ in range(batch)], [1] * batch,
                          hq, hkv, d, rng.random() < 0.75, rot, layout)
        new = _split(rng, _log_int(rng, 10, 24000), rng.choice([1, 2, 5, 17]))
        return _write(None, [rng.choice([0, rng.randrange(5000)]) for _ in new], new, hq, hkv, d, rng.random() < 0.75,
                      rng.choice([0, 0, rot]), layout)
    dense = rng.random() < 0.4
    batch = _log_int(rng, 1, 20 if dense else 200)
    most = min(131072, 390000 * 1024 // (hkv * d * batch)) if dense else 65536   # (dense: about what the largest listed case reads)
    lens = [_log_int(rng, 1, most) for _ in range(batch)]
    return _decode(None, lens, hq, hkv, d, dense)


# ---- what a program has in hand ------------------------------------------------------------------------------------------------

def _rope_cfg(case):
    more = {"none": {}, "linear": {"factor": 4.0}, "ntk": {"factor": 4.0},
            "yarn": {"factor": 8.0, "original_len": 4096}}[case.get("scaling", "none")]
    return dict({"dim": case["rot"], "base": 1000000.0, "layout": case["layout"], "scaling": case.get("scaling", "none")}, **more)


def _frequencies(cfg):
    """Radians per position of every pair, and the factor on the rotated values."""
    r, base, s = cfg["dim"], cfg["base"], cfg.get("factor", 1.0)
    if cfg["scaling"] == "ntk":
        base = base * s ** (r / (r - 2))
    f = base ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)
    if cfg["scaling"] == "linear":
        f = f / s
    magnitude = 1.0
    if cfg["scaling"] == "yarn":
        rounds = cfg["original_len"] * f / (2 * math.pi)
        keep = ((rounds - 1.0) / (32.0 - 1.0)).clamp(0, 1)
        f = keep * f + (1 - keep) * f / s
        magnitude = 0.1 * math.log(s) + 1.0
    return f, magnitude


def _lists(case):
    """Logical pages that the newest token of every sequence reads, ascending."""
    out = []
    for n in _numbers(case["lens"]):
        j = (n - 1) // PAGE
        if case["dense"]:
            out.append(list(range(j + 1)))
        else:
            out.append(sorted({j, 0} | {j - w for w in (1, 2) if w <= j} | {j - (1 << k) for k in range(j.bit_length()) if j >= 1 << k}))
    return out


def _randn(shape, gen, dev, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=dev).normal_(generator=gen)


def _prepare_rope(case, gen, dev):
    lens, hq, hkv, d = _numbers(case["lens"]), case["hq"], case["hkv"], case["d"]
    total = sum(lens)
    state = {"positions": torch.cat([torch.arange(n, dtype=torch.int32) for n in lens]).to(dev) + case["first"]}

    def pair():
        if case["fused"]:   # [q | k | v] of a token in one row
            row = _randn((total, (hq + 2 * hkv) * d), gen, dev)
            return row[:, :hq * d].view(total, hq, d), row[:, hq * d:(hq + hkv) * d].view(total, hkv, d)
        return _randn((total, hq, d), gen, dev), _randn((total, hkv, d), gen, dev)

    state["q"], state["k"] = pair()
    if case["grad"]:
        state["d_q"], state["d_k"] = _randn((total, hq, d), gen, dev), _randn((total, hkv, d), gen, dev)
        row = torch.zeros((total, (hq + 2 * hkv) * d), dtype=torch.bfloat16, device=dev) if case["fused"] else None
        state["into_q"] = row[:, :hq * d].view(total, hq, d) if case["fused"] else torch.empty_like(state["d_q"])
        state["into_k"] = row[:, hq * d:(hq + hkv) * d].view(total, hkv, d) if case["fused"] else torch.empty_like(state["d_k"])
    return state


def _prepare_tables(case, gen, dev):
    old, new = _numbers(case["old"]), _numbers(case["new"])
    batch, max_pages = len(old), case["max_pages"]
    held = [(n + PAGE - 1) // PAGE for n in old]
    needed = sum((o + max(n, 0) + PAGE - 1) // PAGE - h for o, n, h in zip(old, new, held))
    pool = sum(held) + needed + 50
    where = torch.randperm(pool, generator=gen, device=dev).to(torch.int32)
    count = torch.tensor(held, device=dev)
    at = torch.arange(max_pages, device=dev)
    start = torch.cumsum(count, 0) - count
    index = (start[:, None] + at).clamp(max=pool - 1)
    table = torch.where(at < count[:, None], where[index], torch.full((), -1, dtype=torch.int32, device=dev))
    free = torch.full((pool,), -1, dtype=torch.int32, device=dev)
    free[:pool - sum(held)] = where[sum(held):]
    return {"lens": torch.tensor(old, dtype=torch.int32, device=dev), "new": torch.tensor(new, dtype=torch.int32, device=dev),
            "table": table.contiguous(), "free": free, "free_count": torch.tensor([pool - sum(held)], dtype=torch.int32, device=dev),
            "num_pages": pool, "tokens": sum(max(n, 0) for n in new) + case["spare"]}


def _e4m3(shape, gen, dev):
    """Values as a cache holds them: normal ones under a scale that leaves the largest within range."""
    out = torch.empty(shape, dtype=E4M3, device=dev)
    step = max(1, (1 << 27) // max(1, out[0].numel()))
    for i in range(0, shape[0], step):
        out[i:i + step] = (torch.empty((min(step, shape[0] - i),) + tuple(shape[1:]), device=dev).normal_(generator=gen) * 64).clamp(-E4M3_MAX, E4M3_MAX).to(E4M3)
    return out


def _scales(shape, gen, dev):
    return 2.0 ** torch.randint(-8, -5, shape, generator=gen, device=dev).float()


def _prepare_write(case, gen, dev):
    old, new, hq, hkv, d = _numbers(case["old"]), _numbers(case["new"]), case["hq"], case["hkv"], case["d"]
    total = sum(new)
    units = sum((o + n - 1) // PAGE - o // PAGE + 1 for o, n in zip(old, new))
    state = {"lens": torch.tensor(old, dtype=torch.int32, device=dev), "new": torch.tensor(new, dtype=torch.int32, device=dev), "tokens": total}
    # the pages that the step writes stand anywhere among others; those before them are not touched and share one
    state["num_pages"] = units + 37
    where = torch.randperm(state["num_pages"], generator=gen, device=dev).to(torch.int32).cpu()
    table = torch.full((len(old), max((o + n + PAGE - 1) // PAGE for o, n in zip(old, new))), int(where[-1]), dtype=torch.int32)
    at = 0
    for s, (o, n) in enumerate(zip(old, new)):
        first, last = o // PAGE, (o + n - 1) // PAGE
        table[s, first:last + 1] = where[at:at + last + 1 - first]
        at += last + 1 - first
    state["table"] = table.to(dev)
    state["map"] = _maps(state["lens"], state["new"], state["table"], total)
    state["k"], state["v"] = _randn((total, hkv, d), gen, dev), _randn((total, hkv, d), gen, dev)
    if case["rot"]:
        state["q"] = _randn((total, hq, d), gen, dev)
        state["out_q"] = torch.zeros_like(state["q"])
    shape = (state["num_pages"], PAGE, hkv, d)
    if case["fp8"]:
        state["k_pages"], state["v_pages"] = _e4m3(shape, gen, dev), _e4m3(shape, gen, dev)
        state["k_scales"], state["v_scales"] = _scales(shape[:1] + (hkv,), gen, dev), _scales(shape[:1] + (hkv,), gen, dev)
    else:
        state["k_pages"], state["v_pages"] = _randn(shape, gen, dev), _randn(shape, gen, dev)
    return state


def _prepare_decode(case, gen, dev):
    lens, hq, hkv, d = _numbers(case["lens"]), case["hq"], case["hkv"], case["d"]
    lists = _lists(case)
    held = [(n + PAGE - 1) // PAGE for n in lens]
    pool = sum(len(x) for x in lists) + 11   # the pages that nobody's newest token reads need no room here
    where = torch.randperm(pool, generator=gen, device=dev).to(torch.int32).cpu()
    degree = max(len(x) for x in lists)
    pages = torch.full((len(lens), degree), -1, dtype=torch.int32)
    table = torch.full((len(lens), max(held)), -1, dtype=torch.int32)
    at = 0
    for s, x in enumerate(lists):
        pages[s, :len(x)] = where[at:at + len(x)]
        table[s, torch.tensor(x)] = where[at:at + len(x)]
        at += len(x)
    state = {"lens": torch.tensor(lens, dtype=torch.int32, device=dev), "table": table.to(dev), "pages": pages.to(dev),
             "keys": torch.tensor([(len(x) - 1) * PAGE + n - (n - 1) // PAGE * PAGE for x, n in zip(lists, lens)], device=dev)}
    shape = (pool, PAGE, hkv, d)
    state["k_pages"], state["v_pages"] = _e4m3(shape, gen, dev), _e4m3(shape, gen, dev)
    state["k_scales"], state["v_scales"] = _scales(shape[:1] + (hkv,), gen, dev), _scales(shape[:1] + (hkv,), gen, dev)
    state["q"] = _randn((len(lens), hq, d), gen, dev)
    state["out"] = torch.zeros_like(state["q"])
    state["lse"] = torch.zeros((hq, len(lens)), dtype=torch.float32, device=dev)
    return state


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    state = {"rope": _prepare_rope, "tables": _prepare_tables, "write": _prepare_write, "decode": _prepare_decode}[case["op"]](case, gen, dev)
    state["case"] = case
    if case.get("rot"):
        cfg = _rope_cfg(case)
        f, state["magnitude"] = _frequencies(cfg)
        state["frequencies"] = f.to(dev)
    if own:   # the handles that a program makes once
        import paper_2608_20427_b200 as bf1
        state["lib"] = bf1
        if case.get("rot"):
            state["rope"] = bf1.plan_rope(bf1.RopeCfg(**cfg), dev)
        if case["op"] == "tables":
            state["plan"] = bf1.CachePlan.empty(len(_numbers(case["old"])), state["tokens"], dev)
        if case["op"] == "write":
            state["plan"] = bf1.plan_cache(state["lens"], state["new"], state["table"], state["num_pages"], state["tokens"])
        if case["op"] == "decode":
            cfg = bf1.RouteCfg(64, 1 << 20, 0, 0) if case["dense"] else bf1.RouteCfg()
            state["plan"] = bf1.plan_decode(state["lens"], state["table"], cfg)
            state["work"] = bf1.decode_fp8_workspace(len(_numbers(case["lens"])), case["hq"], case["hkv"], state["plan"].max_degree, case["d"], dev)
    return state


# ---- the plain forms -------------------------------------------------------------------------------------------------------------

def _rotate(x, positions, f, magnitude, layout, sign=1.0):
    """Rotary positions in 32 bits, the angles in 64; x [T, H, d] -> float32."""
    angle = positions.double()[:, None] * f
    cos, sin = (angle.cos() * magnitude).float()[:, None], (angle.sin() * (sign * magnitude)).float()[:, None]
    r = 2 * f.numel()
    x = x.float()
    if layout == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    return torch.cat((turned, x[..., r:]), -1)


def _maps(lens, new, table, tokens):
    """(offsets, positions, slots, units, their number) of a step's tokens, pages as the table has them."""
    old, new = lens.long(), new.long().clamp(min=0)
    batch, dev = old.numel(), old.device
    none = torch.full((), -1, dtype=torch.int64, device=dev)
    end = torch.cumsum(new, 0)
    t = torch.arange(tokens, device=dev)
    s = torch.searchsorted(end, t, right=True)
    real, s = s < batch, s.clamp(max=batch - 1)
    pos = torch.where(real, old[s] + t - (end[s] - new[s]), none)
    slots = torch.where(real, table[s, pos.clamp(min=0) // PAGE].long() * PAGE + pos % PAGE, none)
    count = torch.where(new > 0, (old + new - 1) // PAGE - old // PAGE + 1, torch.zeros_like(new))
    last = torch.cumsum(count, 0)
    u = torch.arange(max(1, min(tokens, tokens // PAGE + 2 * batch)), device=dev)
    s = torch.searchsorted(last, u, right=True)
    real, s = s < batch, s.clamp(max=batch - 1)
    page = old[s] // PAGE + u - (last[s] - count[s])
    first = torch.maximum(old[s], page * PAGE)
    stop = torch.minimum(old[s] + new[s], page * PAGE + PAGE)
    units = torch.stack((end[s] - new[s] + first - old[s], stop - first, table[s, page.clamp(min=0, max=table.shape[1] - 1)].long(), first % PAGE), 1)
    units = torch.where(real[:, None], units, none)
    offsets = torch.cat((torch.zeros_like(end[:1]), end))
    return {k: v.int() for k, v in (("offsets", offsets), ("positions", pos), ("slots", slots), ("units", units), ("num_units", last[-1:]))}


def _run_tables(state):
    lens, new, table, free, count = state["lens"], state["new"], state["table"], state["free"], state["free_count"]
    held = (lens + PAGE - 1) // PAGE
    gone = new < 0
    after = torch.where(gone, torch.zeros_like(lens), lens + new)
    at = torch.arange(table.shape[1], device=lens.device)
    # released pages onto the stack, in order of sequences and pages
    back = torch.where(gone, held, torch.zeros_like(held))
    to = count + (torch.cumsum(back, 0) - back)[:, None] + at
    room = torch.cat((free, free[:1]))
    room.scatter_(0, torch.where(at < back[:, None], to, torch.full_like(to, free.numel())).flatten(), table.flatten())
    free.copy_(room[:-1])
    count = count + back.sum()
    # new pages from its top
    want = torch.where(gone, torch.zeros_like(held), (after + PAGE - 1) // PAGE - held)
    first = torch.cumsum(want, 0) - want
    index = count - 1 - (first[:, None] + at - held[:, None])
    fresh = (at >= held[:, None]) & (at < (held + want)[:, None])
    table.copy_(torch.where(fresh, free[index.clamp(min=0, max=free.numel() - 1).long()], table))
    m = _maps(lens, new, table, state["tokens"])
    return table, free, after, (count - want.sum()).int(), m["offsets"], m["positions"], m["slots"], m["units"], m["num_units"]


def _quantize(pages, scales, x, units):
    """Rows x [T, H, d] (float32) into the pages of the units, in 8 bits; the rows already there are kept under the new scale."""
    first, count, page, row0 = units.long().unbind(1)
    row = torch.arange(PAGE, device=x.device)
    rel = row - row0[:, None]
    fresh = (rel >= 0) & (rel < count[:, None])
    rows = x[(first[:, None] + rel).clamp(min=0, max=x.shape[0] - 1)]
    top = torch.where(fresh[:, :, None, None], rows.abs(), torch.zeros_like(rows)).amax((1, 3))
    mantissa, exponent = torch.frexp(top / E4M3_MAX)
    exponent = torch.where(mantissa == 0.5, exponent - 1, exponent)
    scale = torch.ldexp(torch.ones_like(top), exponent).clamp(min=SCALE_MIN)
    before = scales[page]
    scale = torch.where(row0[:, None] > 0, torch.maximum(scale, before), scale)
    there = pages[page]
    kept = (there.float() * (before / scale)[:, None, :, None]).to(E4M3).view(torch.uint8)
    put = (rows / scale[:, None, :, None]).to(E4M3).view(torch.uint8)
    out = torch.where(fresh[:, :, None, None], put, torch.where((row < row0[:, None])[:, :, None, None], kept, there.view(torch.uint8)))
    pages.view(torch.uint8)[page] = out
    scales[page] = scale


def _run_write(state):
    case, m = state["case"], state["map"]
    k, v = state["k"].float(), state["v"].float()
    if case["rot"]:
        k = _rotate(state["k"], m["positions"], state["frequencies"], state["magnitude"], case["layout"])
        state["out_q"].copy_(_rotate(state["q"], m["positions"], state["frequencies"], state["magnitude"], case["layout"]))
    if case["fp8"]:
        units = m["units"][:state["num_pages"] - 37]
        _quantize(state["k_pages"], state["k_scales"], k, units)
        _quantize(state["v_pages"], state["v_scales"], v, units)
    else:
        slots = m["slots"].long()
        state["k_pages"].flatten(0, 1)[slots] = k.to(torch.bfloat16)
        state["v_pages"].flatten(0, 1)[slots] = v.to(torch.bfloat16)


def _run_decode(state):
    q, pages = state["q"], state["pages"]
    batch, hq, d = q.shape
    hkv = state["k_pages"].shape[2]
    which = pages.clamp(min=0).long()
    k = (state["k_pages"][which].float() * state["k_scales"][which][:, :, None, :, None]).flatten(1, 2)   # [batch, keys, hkv, d]
    v = (state["v_pages"][which].float() * state["v_scales"][which][:, :, None, :, None]).flatten(1, 2)
    scores = torch.einsum("bhgd,bnhd->bhgn", q.float().view(batch, hkv, hq // hkv, d), k) / math.sqrt(d)
    dead = torch.arange(k.shape[1], device=q.device) >= state["keys"][:, None]
    scores = scores.masked_fill(dead[:, None, None], float("-inf"))
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    state["out"].copy_((torch.einsum("bhgn,bnhd->bhgd", p, v) / total).reshape(batch, hq, d))
    state["lse"].copy_((top + torch.log(total)).reshape(batch, hq).t())


def run(state):
    case = state["case"]
    if case["op"] == "rope":
        if own:
            lib, rope, pos = state["lib"], state["rope"], state["positions"]
            out = lib.rope_fwd(state["q"], state["k"], pos, rope)
            if case["grad"]:
                out += lib.rope_bwd(state["d_q"], state["d_k"], pos, rope, out_q=state["into_q"], out_k=state["into_k"])
            return out
        how = (state["positions"], state["frequencies"], state["magnitude"], case["layout"])
        out = tuple(_rotate(x, *how).to(torch.bfloat16) for x in (state["q"], state["k"]))
        if case["grad"]:
            state["into_q"].copy_(_rotate(state["d_q"], *how, sign=-1.0))
            state["into_k"].copy_(_rotate(state["d_k"], *how, sign=-1.0))
            out += (state["into_q"], state["into_k"])
        return out
    if case["op"] == "tables":
        if own:
            p = state["lib"].plan_cache(state["lens"], state["new"], state["table"], state["num_pages"], state["tokens"],
                                        free_pages=state["free"], free_count=state["free_count"], plan=state["plan"])
            return state["table"], state["free"], p.seqlens, p.free_count, p.cu_tokens, p.positions, p.slots, p.units, p.num_units
        return _run_tables(state)
    if case["op"] == "write":
        if own:
            state["lib"].cache_write(state["k"], state["v"], state["k_pages"], state["v_pages"], state["plan"], k_scales=state.get("k_scales"),
                                     v_scales=state.get("v_scales"), rope=state.get("rope"), q=state.get("q"), out_q=state.get("out_q"))
        else:
            _run_write(state)
        return [state[x] for x in ("k_pages", "v_pages", "k_scales", "v_scales", "out_q") if x in state]
    if own:
        return state["lib"].decode_fwd_fp8(state["q"], state["k_pages"], state["v_pages"], state["k_scales"], state["v_scales"], state["lens"],
                                           state["plan"], state["work"], out=state["out"], lse=state["lse"])
    _run_decode(state)
    return state["out"], state["lse"]


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------------

def work(case):
    if case["op"] == "tables":
        old, new = _numbers(case["old"]), _numbers(case["new"])
        tokens = sum(max(n, 0) for n in new)
        units = sum((o + n - 1) // PAGE - o // PAGE + 1 for o, n in zip(old, new) if n > 0)
        fresh = sum((o + n + PAGE - 1) // PAGE - (o + PAGE - 1) // PAGE for o, n in zip(old, new) if n > 0)
        back = sum((o + PAGE - 1) // PAGE for o, n in zip(old, new) if n < 0)
        return {"bytes": 16 * len(old) + 8 * (tokens + case["spare"]) + 20 * units + 8 * (fresh + back), "flops": 0}
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] == "rope":
        values = sum(_numbers(case["lens"])) * (hq + hkv) * (2 if case["grad"] else 1)
        return {"bytes": 4 * values * d + 4 * sum(_numbers(case["lens"])), "flops": 3 * values * case["rot"]}
    if case["op"] == "write":
        old, new = _numbers(case["old"]), _numbers(case["new"])
        tokens = sum(new)
        units = sum((o + n - 1) // PAGE - o // PAGE + 1 for o, n in zip(old, new))
        moved = tokens * hkv * 2 * d * (3 if case["fp8"] else 4) + units * (16 + (8 * hkv if case["fp8"] else 0))
        turned = tokens * (hq + hkv) * case["rot"]
        if case["rot"]:
            moved += tokens * hq * 4 * d
        return {"bytes": moved, "flops": 3 * turned + 4 * tokens * hkv * d}
    keys = pages = 0
    for n, x in zip(_numbers(case["lens"]), _lists(case)):
        keys += (len(x) - 1) * PAGE + n - (n - 1) // PAGE * PAGE
        pages += len(x)
    return {"bytes": 2 * keys * hkv * d + pages * (4 + 8 * hkv) + len(_numbers(case["lens"])) * hq * (4 * d + 4), "flops": 4 * d * keys * hq}


# ---- in 64 bits --------------------------------------------------------------------------------------------------------------------

def _exact_rotation(x, positions, case, sign=1.0):
    """Every pair as a complex number times magnitude * exp(i sign angle)."""
    cfg = _rope_cfg(case)
    r, s = cfg["dim"], cfg.get("factor", 1.0)
    f = []
    for i in range(r // 2):
        if cfg["scaling"] == "ntk":
            w = math.exp(-2 * i / r * (math.log(cfg["base"]) + r / (r - 2) * math.log(s)))
        else:
            w = math.exp(-2 * i / r * math.log(cfg["base"]))
        if cfg["scaling"] == "linear":
            w /= s
        if cfg["scaling"] == "yarn":
            g = min(1.0, max(0.0, (cfg["original_len"] * w / (2 * math.pi) - 1.0) / 31.0))
            w = g * w + (1 - g) * w / s
        f.append(w)
    size = 0.1 * math.log(s) + 1.0 if cfg["scaling"] == "yarn" else 1.0
    angle = torch.outer(positions.double(), torch.tensor(f, dtype=torch.float64, device=x.device)) * sign
    by = torch.polar(torch.full_like(angle, size), angle)[:, None]
    y = x.double().clone()
    even, odd = (slice(0, r // 2), slice(r // 2, r)) if cfg["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    z = torch.complex(y[..., even], y[..., odd]) * by
    y[..., even], y[..., odd] = z.real, z.imag
    return y


def _exact_pages(pages, scales, x, units):
    held, scale = pages.double(), scales.double().clone()
    for first, count, page, row in units.tolist():
        if count < 0:
            continue
        rows = x[first:first + count]
        need = torch.exp2(torch.ceil(torch.log2(rows.abs().amax((0, 2)) / E4M3_MAX) - 1e-12)).clamp(min=SCALE_MIN)
        if row:
            need = torch.maximum(need, scale[page])
            held[page, :row] = (held[page, :row] * (scale[page] / need)[None, :, None]).to(E4M3).double()
        held[page, row:row + count] = (rows / need[None, :, None]).to(E4M3).double()
        scale[page] = need
    return held, scale


def exact(case, seed):
    if case["op"] == "tables":
        return None
    state = prepare(case, seed)
    if case["op"] == "rope":
        out = [_exact_rotation(state[x], state["positions"], case) for x in ("q", "k")]
        return out + ([_exact_rotation(state[x], state["positions"], case, -1.0) for x in ("d_q", "d_k")] if case["grad"] else [])
    if case["op"] == "write":
        m = state["map"]
        k, v = state["k"].double(), state["v"].double()
        if case["rot"]:
            k = _exact_rotation(state["k"], m["positions"], case)
        if case["fp8"]:
            (k_pages, k_scales), (v_pages, v_scales) = (_exact_pages(state[n + "_pages"], state[n + "_scales"], x, m["units"]) for n, x in (("k", k), ("v", v)))
            out = [k_pages, v_pages, k_scales, v_scales]
        else:
            out = []
            for n, x in (("k", k), ("v", v)):
                pages = state[n + "_pages"].double()
                for first, count, page, row in m["units"].tolist():
                    if count > 0:
                        pages[page, row:row + count] = x[first:first + count]
                out.append(pages)
        return out + ([_exact_rotation(state["q"], m["positions"], case)] if case["rot"] else [])
    q, hkv, d = state["q"].double(), case["hkv"], case["d"]
    o, lse = torch.zeros_like(q), torch.zeros_like(state["lse"], dtype=torch.float64)
    group = case["hq"] // hkv
    for s, n in enumerate(state["keys"].tolist()):
        which = state["pages"][s, :(n + PAGE - 1) // PAGE].long()
        for h in range(hkv):
            k = (state["k_pages"][which, :, h].double() * state["k_scales"][which, h].double()[:, None, None]).reshape(-1, d)[:n]
            v = (state["v_pages"][which, :, h].double() * state["v_scales"][which, h].double()[:, None, None]).reshape(-1, d)[:n]
            x = k @ q[s, h * group:(h + 1) * group].t() / math.sqrt(d)
            lse[h * group:(h + 1) * group, s] = torch.logsumexp(x, 0)
            o[s, h * group:(h + 1) * group] = torch.softmax(x, 0).t() @ v
    return o, lse
