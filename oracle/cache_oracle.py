"""Plain 64-bit implementations of the operators around the paged cache: rotary positions, the step's tables, the cache write and
one-token attention over pages in 8 bits.  Written from the definitions in include/bf1.h, in numpy and Python loops, and used
by the tests only."""
import math

import numpy as np

PAGE = 64
E4M3_MAX = 448.0
MIN_SCALE = 2.0 ** -64


# ---- rotary positions ---------------------------------------------------------------------------------------------------------
def rope_turns(dim, base=10000.0, scaling="none", factor=1.0, original_len=0.0, beta_fast=32.0, beta_slow=1.0):
    """(turns per position of every pair, magnitude)."""
    if scaling == "ntk":
        base *= factor ** (dim / (dim - 2))
    out = []
    for i in range(dim // 2):
        t = base ** (-2 * i / dim) / (2 * math.pi)
        if scaling == "linear":
            t /= factor
        elif scaling == "yarn":
            n = original_len * t
            if n <= beta_slow:
                t /= factor
            elif n < beta_fast:
                w = (n - beta_slow) / (beta_fast - beta_slow)
                t = w * t + (1 - w) * t / factor
        out.append(t)
    return np.array(out), 0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0


def rotation(position, turns, magnitude, d, layout):
    """The d x d matrix that a head's column vector is multiplied with."""
    r = 2 * len(turns)
    m = np.eye(d)
    for i, t in enumerate(turns):
        x, y = (i, i + r // 2) if layout == "half" else (2 * i, 2 * i + 1)
        a = 2 * math.pi * math.fmod(position * t, 1.0)
        m[x, x] = m[y, y] = magnitude * math.cos(a)
        m[x, y], m[y, x] = -magnitude * math.sin(a), magnitude * math.sin(a)
    return m


def rotate(x, positions, turns, magnitude, layout, back=False):
    """x [T, H, d] -> float64; tokens of negative position come out as NaN (they are not written)."""
    x = np.asarray(x, dtype=np.float64)
    out = np.full(x.shape, np.nan)
    for t, p in enumerate(positions):
        if p >= 0:
            m = rotation(int(p), turns, magnitude, x.shape[2], layout)
            out[t] = x[t] @ (m if back else m.T)
    return out


# ---- numbers in 8 bits: four exponent bits, three of fraction -------------------------------------------------------------------
def to_e4m3(x):
    """Nearest value, ties to even; what is not finite becomes NaN.  |x| <= 448 is the caller's business."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(all="ignore"):
        exponent = np.maximum(np.floor(np.log2(np.where(x == 0, 1.0, np.abs(x)))), -6.0)
        exponent = np.where(np.abs(x) < 2.0 ** exponent, np.maximum(exponent - 1, -6), exponent)   # (log2 may be a step off)
        exponent = np.where(np.abs(x) >= 2.0 ** (exponent + 1), exponent + 1, exponent)
        step = 2.0 ** (exponent - 3)
        return np.where(np.isfinite(x), np.rint(x / step) * step, np.nan)


def page_scale(rows):
    """The smallest power of two, 2^-64 at least, under which the finite values of `rows` are within +-448."""
    top = float(np.max(np.abs(rows), initial=0.0, where=np.isfinite(rows)))
    e = -64
    while top > E4M3_MAX * 2.0 ** e:
        e += 1
    return 2.0 ** e


def write_pages(pages, scales, x, units):
    """Rows x [T, H, d] (float64) put into `pages` [P, 64, H, d] (values as stored, float64), in place; scales [P, H] or None (not
    in 8 bits: the rows are stored as they are)."""
    for first, count, page, row in units:
        for h in range(x.shape[1]):
            rows = x[first:first + count, h]
            if scales is None:
                pages[page, row:row + count, h] = rows
                continue
            scale = page_scale(rows)
            if row > 0:
                scale = max(scale, scales[page, h])
                if scale != scales[page, h]:
                    pages[page, :row, h] = to_e4m3(pages[page, :row, h] * (scales[page, h] / scale))
            scales[page, h] = scale
            pages[page, row:row + count, h] = to_e4m3(rows / scale)


# ---- the tables of a step ---------------------------------------------------------------------------------------------------------
class Refused(Exception):
    pass


def plan_cache(lens, new, table, num_pages, tokens, free=None):
    """One step: (lens, table, free list, offsets, positions, slots, units) after it, as plain lists.  `free` None: the pages are
    in the table already.  Raises Refused where nothing is done."""
    lens, table = list(lens), [list(r) for r in table]
    width = len(table[0]) if table else 0
    pages_of = lambda n: (n + PAGE - 1) // PAGE  # noqa: E731
    for n, a in zip(lens, new):
        if n < 0 or a < -1 or pages_of(n + max(a, 0)) > width:
            raise Refused("lengths")
    if sum(max(a, 0) for a in new) > tokens:
        raise Refused("tokens")
    stack = None if free is None else list(free)
    if stack is not None:
        for s, a in enumerate(new):
            if a < 0:
                stack += table[s][:pages_of(lens[s])]
        if len(stack) > num_pages:
            raise Refused("more free pages than there are")
        if sum(pages_of(n + a) - pages_of(n) for n, a in zip(lens, new) if a > 0) > len(stack):
            raise Refused("pages")
    offsets, positions, slots, units = [0], [], [], []
    for s, a in enumerate(new):
        n = lens[s]
        for i in range(max(a, 0)):
            p = n + i
            if p % PAGE == 0 and stack is not None:
                table[s][p // PAGE] = stack.pop()
            page = table[s][p // PAGE]
            good = 0 <= page < num_pages
            if i == 0 or p % PAGE == 0:
                units.append([len(positions), 0, page if good else -1, p % PAGE])
            units[-1][1] += 1
            positions.append(p)
            slots.append(page * PAGE + p % PAGE if good else -1)
        lens[s] = 0 if a < 0 else n + a
        offsets.append(len(positions))
    return lens, table, stack, offsets, positions, slots, units


# ---- one token per sequence over its pages ------------------------------------------------------------------------------------------
def decode(q, k_pages, v_pages, k_scales, v_scales, lists, lens, scale=None):
    """q [B, hq, d]; pages [P, 64, hkv, d] (values as stored); lists: physical pages of every sequence, the last one holding token
    lens - 1.  (o [B, hq, d], lse [hq, B]) in float64, NaN for empty sequences."""
    q = np.asarray(q, dtype=np.float64)
    batch, hq, d = q.shape
    group = hq // k_pages.shape[2]
    scale = 1 / math.sqrt(d) if scale is None else scale
    o, lse = np.full(q.shape, np.nan), np.full((hq, batch), np.nan)
    for s, (pages, n) in enumerate(zip(lists, lens)):
        if n == 0:
            continue
        keys = (len(pages) - 1) * PAGE + (n - 1) % PAGE + 1
        pages = list(pages)
        for h in range(hq):
            j = h // group
            k = (k_pages[pages, :, j] * k_scales[pages, j][:, None, None]).reshape(-1, d)[:keys]
            v = (v_pages[pages, :, j] * v_scales[pages, j][:, None, None]).reshape(-1, d)[:keys]
            x = scale * (k @ q[s, h])
            top = x.max()
            w = np.exp(x - top)
            o[s, h] = (w @ v) / w.sum()
            lse[h, s] = top + math.log(w.sum())
    return o, lse
