"""Thin Python binding of the BF1 C-ABI library (argument marshalling only).

Every step of the operator runs in the library's CUDA kernels.  PyTorch is used for device
memory, streams and nothing else.  There is no CPU or PyTorch fallback: if the shared
library cannot be built or loaded, importing callers get an exception.

The calls that launch kernels go through the extension module `_host` (csrc/bf1_host.cpp), which takes the
tensors apart and calls the C ABI; what only computes sizes on the host uses ctypes.
"""
from __future__ import annotations

import ctypes
import importlib.util
import math
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

from . import build as _build

BF1_OK = 0
DEV_BAD_SEQLENS, DEV_CAPACITY, DEV_WAIT_TIMEOUT, DEV_BAD_ROUTE = 1, 2, 4, 8

EXPORTS = ("bf1_route_capacity", "bf1_plan_route", "bf1_attn_fwd", "bf1_dense_causal_fwd",
           "bf1_attn_fwd_noalloc", "bf1_plan_decode", "bf1_decode_workspace_bytes", "bf1_decode_fwd",
           "bf1_attn_bwd", "bf1_attn_bwd_workspace_bytes", "bf1_shard_needed_blocks", "bf1_plan_route_shard",
           "bf1_shard_needed_blocks_strided", "bf1_plan_route_shard_strided",
           "bf1_rope_turns", "bf1_rope_fwd", "bf1_rope_bwd",
           "bf1_decode_fp8_workspace_bytes", "bf1_decode_fwd_fp8", "bf1_decode_fwd_fp8_packed", "bf1_cache_plan_units", "bf1_plan_cache", "bf1_cache_write",
           "bf1_last_error", "bf1_version")


class RouteCfg(ctypes.Structure):
    """Mirror of bf1_route_cfg.  Defaults: the paper's reported configuration (Section 3.1)."""
    _fields_ = [("block", ctypes.c_int32), ("local_blocks", ctypes.c_int32),
                ("global_first", ctypes.c_int32), ("dyadic", ctypes.c_int32)]

    def __init__(self, block: int = 64, local_blocks: int = 2, global_first: int = 1, dyadic: int = 1):
        super().__init__(block, local_blocks, global_first, dyadic)


class _RouteC(ctypes.Structure):
    """Mirror of bf1_route."""
    _fields_ = [("capacity_qblocks", ctypes.c_int32), ("max_degree", ctypes.c_int32),
                ("qb_seq", ctypes.c_void_p), ("qb_block", ctypes.c_void_p),
                ("kv_count", ctypes.c_void_p), ("kv_idx", ctypes.c_void_p),
                ("pair_count", ctypes.c_void_p), ("order", ctypes.c_void_p),
                ("total_pairs", ctypes.c_void_p), ("num_qblocks", ctypes.c_void_p),
                ("status", ctypes.c_void_p), ("sched", ctypes.c_void_p)]


class _DecodePlanC(ctypes.Structure):
    """Mirror of bf1_decode_plan."""
    _fields_ = [("max_degree", ctypes.c_int32), ("count", ctypes.c_void_p), ("page", ctypes.c_void_p),
                ("block", ctypes.c_void_p), ("status", ctypes.c_void_p)]


class _RopeCfgC(ctypes.Structure):
    """Mirror of bf1_rope_cfg."""
    _fields_ = [("dim", ctypes.c_int32), ("scaling", ctypes.c_int32), ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("original_len", ctypes.c_double), ("beta_fast", ctypes.c_double), ("beta_slow", ctypes.c_double)]


class _RopeC(ctypes.Structure):
    """Mirror of bf1_rope."""
    _fields_ = [("dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("magnitude", ctypes.c_float), ("turns", ctypes.c_void_p)]


class _RowsC(ctypes.Structure):
    """Mirror of bf1_rows."""
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class _CachePlanC(ctypes.Structure):
    """Mirror of bf1_cache_plan."""
    _fields_ = [("batch", ctypes.c_int32), ("capacity_tokens", ctypes.c_int32), ("capacity_units", ctypes.c_int32),
                ("seqlens", ctypes.c_void_p), ("free_count", ctypes.c_void_p), ("cu_tokens", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("slots", ctypes.c_void_p), ("units", ctypes.c_void_p), ("num_units", ctypes.c_void_p), ("starts", ctypes.c_void_p),
                ("status", ctypes.c_void_p)]


class Bf1Error(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("bf1 error %d: %s" % (code, msg))
        self.code = code


_lib = None


def load():
    """Load (building first if needed) libbf1.so and declare its signatures."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.build()
    L = ctypes.CDLL(path)
    i32, i64, vp, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float
    L.bf1_route_capacity.restype = ctypes.c_int
    L.bf1_route_capacity.argtypes = [i32, i64, i32, ctypes.POINTER(RouteCfg), ctypes.POINTER(i32), ctypes.POINTER(i32)]
    L.bf1_plan_route.restype = ctypes.c_int
    L.bf1_plan_route.argtypes = [vp, i32, i64, i32, ctypes.POINTER(RouteCfg), ctypes.POINTER(_RouteC), vp]
    L.bf1_attn_fwd.restype = ctypes.c_int
    L.bf1_attn_fwd.argtypes = [vp, vp, vp, vp, i32, i64, i32, i32, i32, i32, f32, ctypes.POINTER(_RouteC), vp, vp, vp]
    L.bf1_dense_causal_fwd.restype = ctypes.c_int
    L.bf1_dense_causal_fwd.argtypes = [vp, vp, vp, vp, i32, i64, i32, i32, i32, i32, f32, vp, vp, vp, vp]
    L.bf1_attn_fwd_noalloc.restype = ctypes.c_int
    L.bf1_attn_fwd_noalloc.argtypes = [vp, vp, vp, vp, i32, i64, i32, i32, i32, i32, f32, ctypes.POINTER(RouteCfg),
                                       vp, vp, vp, vp]
    L.bf1_plan_decode.restype = ctypes.c_int
    L.bf1_plan_decode.argtypes = [vp, vp, i32, i32, ctypes.POINTER(RouteCfg), ctypes.POINTER(_DecodePlanC), vp]
    L.bf1_decode_workspace_bytes.restype = i64
    L.bf1_decode_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
    L.bf1_decode_fwd.restype = ctypes.c_int
    L.bf1_decode_fwd.argtypes = [vp, vp, vp, i32, vp, i32, i32, i32, i32, f32, ctypes.POINTER(_DecodePlanC), vp, vp,
                                 vp, vp]
    L.bf1_attn_bwd_workspace_bytes.restype = i64
    L.bf1_attn_bwd_workspace_bytes.argtypes = [ctypes.POINTER(_RouteC), i64, i32, i32, i32]
    L.bf1_attn_bwd.restype = ctypes.c_int
    L.bf1_attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i64, i32, i32, i32, i32, f32, ctypes.POINTER(_RouteC),
                               vp, vp, vp, vp, vp]
    L.bf1_shard_needed_blocks.restype = ctypes.c_int
    L.bf1_shard_needed_blocks.argtypes = [i64, ctypes.POINTER(RouteCfg), i32, i32, ctypes.POINTER(i32), i32, ctypes.POINTER(i32)]
    L.bf1_plan_route_shard.restype = ctypes.c_int
    L.bf1_plan_route_shard.argtypes = [i64, i32, i32, ctypes.POINTER(RouteCfg), vp, i32, ctypes.POINTER(_RouteC), vp, vp]
    L.bf1_shard_needed_blocks_strided.restype = ctypes.c_int
    L.bf1_shard_needed_blocks_strided.argtypes = [i64, ctypes.POINTER(RouteCfg), i32, i32, i32, ctypes.POINTER(i32), i32,
                                                  ctypes.POINTER(i32)]
    L.bf1_plan_route_shard_strided.restype = ctypes.c_int
    L.bf1_plan_route_shard_strided.argtypes = [i64, i32, i32, i32, ctypes.POINTER(RouteCfg), vp, i32, ctypes.POINTER(_RouteC),
                                               vp, vp]
    rows, ropep = ctypes.POINTER(_RowsC), ctypes.POINTER(_RopeC)
    L.bf1_rope_turns.restype = ctypes.c_int
    L.bf1_rope_turns.argtypes = [ctypes.POINTER(_RopeCfgC), ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    for name in ("bf1_rope_fwd", "bf1_rope_bwd"):
        getattr(L, name).restype = ctypes.c_int
        getattr(L, name).argtypes = [rows, rows, vp, i32, i32, i32, i32, ropep, rows, rows, vp]
    cache = ctypes.POINTER(_CachePlanC)
    L.bf1_cache_plan_units.restype = i32
    L.bf1_cache_plan_units.argtypes = [i32, i32]
    L.bf1_plan_cache.restype = ctypes.c_int
    L.bf1_plan_cache.argtypes = [vp, vp, vp, i32, i32, vp, vp, cache, vp]
    L.bf1_cache_write.restype = ctypes.c_int
    L.bf1_cache_write.argtypes = [rows, rows, rows, i32, i32, i32, i32, cache, ropep, i32, vp, vp, vp, vp, rows, vp]
    L.bf1_decode_fp8_workspace_bytes.restype = i64
    L.bf1_decode_fp8_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
    L.bf1_decode_fwd_fp8.restype = ctypes.c_int
    L.bf1_decode_fwd_fp8.argtypes = [vp, vp, vp, vp, vp, i32, vp, i32, i32, i32, i32, f32, ctypes.POINTER(_DecodePlanC), vp, vp, vp, vp]
    L.bf1_decode_fwd_fp8_packed.restype = ctypes.c_int
    L.bf1_decode_fwd_fp8_packed.argtypes = [vp, i32, vp, vp, vp, vp, vp, i32, vp, i32, i32, i32, i32, f32, ctypes.POINTER(_DecodePlanC), vp, vp, vp, vp]
    L.bf1_last_error.restype = ctypes.c_char_p
    L.bf1_last_error.argtypes = []
    L.bf1_version.restype = ctypes.c_int
    _lib = L
    return L


_host_module = None


def _host():
    """The extension module of the call path (built first if needed)."""
    global _host_module
    if _host_module is None:
        load()
        name = __package__ + "._host"
        spec = importlib.util.spec_from_file_location(name, _build.build_host())
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.set_error(Bf1Error)
        _host_module = module
    return _host_module


def _check(rc: int):
    if rc != BF1_OK:
        raise Bf1Error(rc, load().bf1_last_error().decode())


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> Optional[int]:
    """None stands for the current stream of the current device."""
    return None if stream is None else int(stream.cuda_stream)


def _raw_stream(stream: Optional[torch.cuda.Stream]) -> int:
    return int((stream if stream is not None else torch.cuda.current_stream()).cuda_stream)


def route_capacity(batch: int, total_tokens: int, max_seqlen: int, cfg: Optional[RouteCfg] = None):
    """(capacity_qblocks, max_degree) for a batch; host only."""
    cfg = cfg or RouteCfg()
    cap, deg = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(load().bf1_route_capacity(batch, total_tokens, max_seqlen, ctypes.byref(cfg),
                                     ctypes.byref(cap), ctypes.byref(deg)))
    return cap.value, deg.value


@dataclass
class Route:
    """Device arrays of a planned route plus the C struct that points at them."""
    cfg: RouteCfg
    capacity_qblocks: int
    max_degree: int
    qb_seq: torch.Tensor
    qb_block: torch.Tensor
    kv_count: torch.Tensor
    kv_idx: torch.Tensor
    pair_count: torch.Tensor
    order: torch.Tensor
    total_pairs: torch.Tensor
    num_qblocks: torch.Tensor
    status: torch.Tensor
    sched: torch.Tensor
    c: _RouteC = None

    @staticmethod
    def empty(capacity_qblocks: int, max_degree: int, device, cfg: Optional[RouteCfg] = None) -> "Route":
        i32 = dict(dtype=torch.int32, device=device)
        r = Route(cfg=cfg or RouteCfg(), capacity_qblocks=capacity_qblocks, max_degree=max_degree,
                  qb_seq=torch.empty(capacity_qblocks, **i32), qb_block=torch.empty(capacity_qblocks, **i32),
                  kv_count=torch.empty(capacity_qblocks, **i32),
                  kv_idx=torch.empty((capacity_qblocks, max_degree), **i32),
                  pair_count=torch.empty(capacity_qblocks, **i32), order=torch.empty(capacity_qblocks, **i32),
                  total_pairs=torch.zeros(1, dtype=torch.int64, device=device),
                  num_qblocks=torch.zeros(1, **i32), status=torch.zeros(1, **i32),
                  sched=torch.zeros(2, **i32))
        r.c = _RouteC(capacity_qblocks, max_degree, r.qb_seq.data_ptr(), r.qb_block.data_ptr(),
                      r.kv_count.data_ptr(), r.kv_idx.data_ptr(), r.pair_count.data_ptr(), r.order.data_ptr(),
                      r.total_pairs.data_ptr(), r.num_qblocks.data_ptr(), r.status.data_ptr(),
                      r.sched.data_ptr())
        return r

    @staticmethod
    def from_host(qb_seq, qb_block, kv_count, kv_idx, pair_count, order, total_pairs: int, device,
                  cfg: Optional[RouteCfg] = None) -> "Route":
        """Upload a route the caller built on the host (any ascending lists whose last entry is the
        query block itself; kv_idx [slots, max_degree] padded with -1).  Marshalling only.  The forward takes the
        slots in any order; the backward wants the blocks of a sequence in consecutive slots (see bf1_attn_bwd)."""
        kv_idx = torch.as_tensor(kv_idx, dtype=torch.int32)
        slots, max_degree = kv_idx.shape
        r = Route.empty(max(slots, 1), max_degree, device, cfg)
        for name, src in (("qb_seq", qb_seq), ("qb_block", qb_block), ("kv_count", kv_count),
                          ("pair_count", pair_count), ("order", order)):
            getattr(r, name)[:slots].copy_(torch.as_tensor(src, dtype=torch.int32))
        r.kv_idx[:slots].copy_(kv_idx)
        r.total_pairs.fill_(int(total_pairs))
        r.num_qblocks.fill_(slots)
        return r

    def check_status(self):
        """Synchronising read of the device status word; raises if any BF1_DEV_* bit is set."""
        st = int(self.status.item())
        if st:
            raise Bf1Error(-100, "device status 0x%x" % st)


def plan_route(cu_seqlens: torch.Tensor, max_seqlen: int, cfg: Optional[RouteCfg] = None,
               route: Optional[Route] = None, stream=None) -> Route:
    """bf1_plan_route: Eq. 1 lists for every query block of the packed batch."""
    cfg = cfg or RouteCfg()
    total = getattr(cu_seqlens, "_bf1_total", None)
    if total is None:
        total = int(cu_seqlens[-1].item())
    if route is None:
        cap, deg = route_capacity(cu_seqlens.numel() - 1, total, max_seqlen, cfg)
        route = Route.empty(cap, deg, cu_seqlens.device, cfg)
    _host().plan_route(cu_seqlens, total, max_seqlen, ctypes.addressof(cfg), ctypes.addressof(route.c), _stream_ptr(stream))
    route.cfg = cfg
    return route


def attn_fwd(q, k, v, cu_seqlens, max_seqlen: int, route: Route, scale: Optional[float] = None,
             out=None, lse=None, stream=None):
    """bf1_attn_fwd.  q [T, hq, d], k/v [T, hkv, d] bf16 CUDA -> (o [T, hq, d] bf16, lse [hq, T] fp32)."""
    return _host().forward(0, q, k, v, cu_seqlens, max_seqlen, scale, out, lse, _stream_ptr(stream),
                           ctypes.addressof(route.c), None, None)


def dense_causal_fwd(q, k, v, cu_seqlens, max_seqlen: int, scale: Optional[float] = None, out=None,
                     lse=None, work=None, stream=None):
    """bf1_dense_causal_fwd: plain causal attention through the same kernel.  `work`: optional
    zero-initialised int32[4] CUDA tensor (word 0 = device status, words 1..2 = hand-out counters)."""
    return _host().forward(1, q, k, v, cu_seqlens, max_seqlen, scale, out, lse, _stream_ptr(stream), work, None, None)


def attn_fwd_noalloc(q, k, v, cu_seqlens, max_seqlen: int, out, lse, cfg: Optional[RouteCfg] = None,
                     scale: Optional[float] = None, status=None, stream=None):
    """bf1_attn_fwd_noalloc: plan + attention using the library's built-in scratch array.

    For callers that must not allocate device memory, so `out` and `lse` are required here and
    the call itself allocates nothing (neither through torch nor through CUDA).  Up to 4096
    query blocks per batch; calls sharing a GPU must not overlap in time."""
    if out is None or lse is None:
        raise TypeError("attn_fwd_noalloc allocates nothing: out and lse are required")
    cfg = cfg or RouteCfg()
    return _host().forward(2, q, k, v, cu_seqlens, max_seqlen, scale, out, lse, _stream_ptr(stream),
                           getattr(cu_seqlens, "_bf1_total", None), ctypes.addressof(cfg), status)


@dataclass
class DecodePlan:
    """Device arrays of a decode plan (one page list per sequence) plus the C struct."""
    max_degree: int
    count: torch.Tensor
    page: torch.Tensor
    block: torch.Tensor
    status: torch.Tensor
    c: _DecodePlanC = None

    @staticmethod
    def empty(batch: int, max_degree: int, device) -> "DecodePlan":
        i32 = dict(dtype=torch.int32, device=device)
        p = DecodePlan(max_degree, torch.zeros(batch, **i32), torch.full((batch, max_degree), -1, **i32),
                       torch.zeros(batch, **i32), torch.zeros(1, **i32))
        p.c = _DecodePlanC(max_degree, p.count.data_ptr(), p.page.data_ptr(), p.block.data_ptr(), p.status.data_ptr())
        return p


def plan_decode(seqlens: torch.Tensor, page_table: torch.Tensor, cfg: Optional[RouteCfg] = None,
                plan: Optional[DecodePlan] = None, stream=None) -> DecodePlan:
    """bf1_plan_decode: page list of the newest token's block for every sequence."""
    cfg = cfg or RouteCfg()
    if plan is None:
        batch, max_pages = page_table.shape
        _, deg = route_capacity(1, max_pages * 64, max_pages * 64, cfg)
        plan = DecodePlan.empty(batch, deg, seqlens.device)
    _host().plan_decode(seqlens, page_table, ctypes.addressof(cfg), ctypes.addressof(plan.c), _stream_ptr(stream))
    return plan


def decode_workspace(batch: int, hq: int, hkv: int, max_degree: int, d: int, device) -> torch.Tensor:
    """Scratch for decode_fwd (reusable; its contents do not matter)."""
    nbytes = int(load().bf1_decode_workspace_bytes(batch, hq, hkv, max_degree, d))
    return torch.zeros(max(nbytes, 16), dtype=torch.uint8, device=device)


def decode_fwd(q, k_pages, v_pages, seqlens, plan: DecodePlan, workspace, scale: Optional[float] = None,
               out=None, lse=None, stream=None):
    """bf1_decode_fwd.  q [batch, hq, d]; k_pages / v_pages [pages, 64, hkv, d] bf16 CUDA."""
    return _host().decode(q, k_pages, v_pages, seqlens, ctypes.addressof(plan.c), workspace, scale, out, lse, _stream_ptr(stream))


def decode_fp8_workspace(batch: int, hq: int, hkv: int, max_degree: int, d: int, device) -> torch.Tensor:
    """Scratch for decode_fwd_fp8 (reusable; its contents do not matter; one for every call that may run at the same time)."""
    nbytes = int(load().bf1_decode_fp8_workspace_bytes(batch, hq, hkv, max_degree, d))
    if nbytes < 0:
        raise ValueError("decode_fp8_workspace: hq must be a multiple of hkv, all sizes positive")
    return torch.empty(max(nbytes, 16), dtype=torch.uint8, device=device)


def decode_fwd_fp8(q, k_pages, v_pages, k_scales, v_scales, seqlens, plan: DecodePlan, workspace, scale: Optional[float] = None,
                   out=None, lse=None, stream=None, cu_tokens=None):
    """bf1_decode_fwd_fp8: decode_fwd over a cache in 8 bits.  q [batch, hq, d] bf16; k_pages / v_pages [pages, 64, hkv, d]
    float8_e4m3fn, k_scales / v_scales [pages, hkv] fp32.  Page lists may be of any length: a dense layer's plan is
    plan_decode(seqlens, page_table, RouteCfg(64, page_table.shape[1], 0, 0)).

    With cu_tokens [batch + 1] (bf1_decode_fwd_fp8_packed) q and out are a step's packed rows [tokens, hq, d], as plan_cache numbers them and
    cache_write takes them, and lse is [hq, tokens]: the newest token of sequence s is row cu_tokens[s + 1] - 1, and a sequence without a
    token in the step is passed over.  Without it row s belongs to sequence s."""
    return _host().decode_fp8(q, k_pages, v_pages, k_scales, v_scales, seqlens, ctypes.addressof(plan.c), plan.count, workspace, scale,
                              out, lse, _stream_ptr(stream), cu_tokens)


def bwd_workspace(route: Route, total_tokens: int, hq: int, hkv: int, d: int, device) -> torch.Tensor:
    """Scratch for attn_bwd (reusable; its contents do not matter on entry)."""
    nbytes = int(load().bf1_attn_bwd_workspace_bytes(ctypes.byref(route.c), total_tokens, hq, hkv, d))
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def attn_bwd(q, k, v, o, lse, d_o, cu_seqlens, max_seqlen: int, route: Route, scale: Optional[float] = None,
             workspace=None, stream=None):
    """bf1_attn_bwd: (dq, dk, dv) in bf16 for the upstream gradient d_o."""
    if workspace is None:
        workspace = bwd_workspace(route, q.shape[0], q.shape[1], k.shape[1], q.shape[2], q.device)
    return _host().backward(q, k, v, o, lse, d_o, cu_seqlens, max_seqlen, ctypes.addressof(route.c), scale, workspace,
                            _stream_ptr(stream))


ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}


@dataclass(frozen=True)
class RopeCfg:
    """Rotary positions on the first `dim` dimensions of a head (a multiple of 16).

    layout      "half": pair i is (x[i], x[i + dim/2]); "interleaved": (x[2i], x[2i+1])
    scaling     "none", "linear" (angles / factor), "ntk" (the base times factor^(dim/(dim-2))), "yarn" (angles / factor for pairs
                that turn at most beta_slow times in original_len tokens, as they are for those that turn beta_fast times or
                more, linear in the number of turns between; values times 0.1 ln(factor) + 1)
    magnitude   factor on the rotated values in place of the scaling's own
    """
    dim: int
    base: float = 10000.0
    layout: str = "half"
    scaling: str = "none"
    factor: float = 1.0
    original_len: float = 0.0
    beta_fast: float = 32.0
    beta_slow: float = 1.0
    magnitude: Optional[float] = None


@dataclass
class Rope:
    """The device table of a rope: turns per position of every pair, in 64 bits."""
    dim: int
    layout: str
    magnitude: float
    turns: torch.Tensor
    c: _RopeC = None

    @staticmethod
    def from_turns(turns, layout: str, magnitude: float, device) -> "Rope":
        """A rope of the caller's own frequencies: `turns` of a pair per position (radians / 2 pi), [dim / 2]."""
        if layout not in ROPE_LAYOUTS:
            raise ValueError("layout %r: one of %s" % (layout, ", ".join(ROPE_LAYOUTS)))
        turns = torch.as_tensor(turns, dtype=torch.float64).to(device, copy=True).contiguous()
        if turns.dim() != 1 or turns.numel() < 8 or turns.numel() % 8:
            raise ValueError("turns must be 1-d, 8 pairs at a time")
        r = Rope(2 * turns.numel(), layout, float(magnitude), turns)
        r.c = _RopeC(r.dim, ROPE_LAYOUTS[layout], r.magnitude, turns.data_ptr())
        return r


def plan_rope(cfg: RopeCfg, device) -> Rope:
    """bf1_rope_turns: the table of a rope, made once and used by every layer."""
    if cfg.scaling not in ROPE_SCALINGS:
        raise ValueError("scaling %r: one of %s" % (cfg.scaling, ", ".join(ROPE_SCALINGS)))
    c = _RopeCfgC(cfg.dim, ROPE_SCALINGS[cfg.scaling], cfg.base, cfg.factor, cfg.original_len, cfg.beta_fast, cfg.beta_slow)
    turns, magnitude = (ctypes.c_double * max(cfg.dim // 2, 1))(), ctypes.c_double(1.0)
    _check(load().bf1_rope_turns(ctypes.byref(c), turns, ctypes.byref(magnitude)))
    return Rope.from_turns(list(turns), cfg.layout, magnitude.value if cfg.magnitude is None else cfg.magnitude, device)


def rope_fwd(q, k, positions, rope: Rope, out_q=None, out_k=None, stream=None):
    """bf1_rope_fwd: (q, k) with their heads rotated to `positions` (int32, one per token; negative: padding, whose output rows
    are not written).  q [T, hq, d], k [T, hkv, d] or None, bf16; rows and heads may be strided (parts of one projection's output), the
    outputs too, and they may be the inputs themselves.  Without out_q / out_k new contiguous tensors are made; out_k without k is
    refused."""
    return _host().rope(0, q, k, positions, ctypes.addressof(rope.c), rope.turns, out_q, out_k, _stream_ptr(stream))


def rope_bwd(d_q, d_k, positions, rope: Rope, out_q=None, out_k=None, stream=None):
    """bf1_rope_bwd: the gradients of q and k before the rotation, from those behind it.  Arguments as rope_fwd."""
    return _host().rope(1, d_q, d_k, positions, ctypes.addressof(rope.c), rope.turns, out_q, out_k, _stream_ptr(stream))


@dataclass
class CachePlan:
    """Device arrays of a serving step's tables plus the C struct: where the step's tokens stand in their sequences and in the pages."""
    batch: int
    tokens: int
    seqlens: torch.Tensor
    free_count: torch.Tensor
    cu_tokens: torch.Tensor
    positions: torch.Tensor
    slots: torch.Tensor
    units: torch.Tensor
    num_units: torch.Tensor
    starts: torch.Tensor
    status: torch.Tensor
    c: _CachePlanC = None

    @staticmethod
    def empty(batch: int, tokens: int, device) -> "CachePlan":
        """Arrays for steps of up to `tokens` tokens in `batch` sequences."""
        units = int(load().bf1_cache_plan_units(batch, tokens))
        if units < 0:
            raise ValueError("batch and tokens must not be negative")
        i32 = dict(dtype=torch.int32, device=device)
        p = CachePlan(batch, tokens, torch.zeros(batch, **i32), torch.zeros(1, **i32), torch.zeros(batch + 1, **i32),
                      torch.full((tokens,), -1, **i32), torch.full((tokens,), -1, **i32), torch.full((units, 4), -1, **i32),
                      torch.zeros(1, **i32), torch.zeros((max(batch, 1), 4), **i32), torch.zeros(1, **i32))
        some = p.status.data_ptr()     # (an array without entries has no address)
        at = lambda t: t.data_ptr() or some  # noqa: E731
        p.c = _CachePlanC(batch, tokens, units, at(p.seqlens), at(p.free_count), at(p.cu_tokens), at(p.positions), at(p.slots), at(p.units),
                          at(p.num_units), at(p.starts), at(p.status))
        return p

    def check_status(self):
        """Synchronising read of the device status word; raises if any BF1_DEV_* bit is set."""
        st = int(self.status.item())
        if st:
            raise Bf1Error(-100, "device status 0x%x" % st)


def plan_cache(seqlens: torch.Tensor, new_lens: torch.Tensor, page_table: torch.Tensor, num_pages: int, tokens: int, free_pages=None,
               free_count=None, plan: Optional[CachePlan] = None, seqlens_out=None, free_count_out=None, stream=None) -> CachePlan:
    """bf1_plan_cache: the tables of a step that adds new_lens[s] tokens (-1: releases the sequence) to seqlens[s] cached ones.

    page_table [batch, pages] is completed with pages from the stack free_pages [num_pages], of which free_count are there (without
    them it has to be complete).  `tokens`: rows of the step's packed tensors, at least the tokens it adds.  The lengths and the number
    of free pages after the step are in plan.seqlens and plan.free_count, or in seqlens_out / free_count_out, which may be the
    inputs themselves."""
    if plan is None:
        plan = CachePlan.empty(seqlens.numel(), tokens, seqlens.device)
    elif plan.tokens != tokens:
        raise ValueError("the plan is for %d tokens, not %d" % (plan.tokens, tokens))
    _host().plan_cache(seqlens, new_lens, page_table, num_pages, free_pages, free_count, ctypes.addressof(plan.c), plan.status,
                       plan.seqlens if seqlens_out is None else seqlens_out, plan.free_count if free_count_out is None else free_count_out,
                       _stream_ptr(stream))
    return plan


def cache_write(k, v, k_pages, v_pages, plan: CachePlan, k_scales=None, v_scales=None, rope: Optional[Rope] = None, q=None, out_q=None,
                stream=None):
    """bf1_cache_write: a step's keys and values [plan.tokens, hkv, d] bf16 (rows and heads may be strided) into the pages.

    k_pages / v_pages [pages, 64, hkv, d]: bf16, or float8_e4m3fn with k_scales / v_scales [pages, hkv] fp32.  With `rope` the keys are
    rotated to plan.positions on their way, and so are the queries q, into out_q (made if None), which is returned."""
    return _host().cache_write(k, v, k_pages, v_pages, ctypes.addressof(plan.c), plan.status, k_scales, v_scales,
                               None if rope is None else ctypes.addressof(rope.c), None if rope is None else rope.turns, q, out_q,
                               _stream_ptr(stream))


def shard_needed_blocks(n_tokens: int, lo_block: int, hi_block: int, cfg: Optional[RouteCfg] = None):
    """bf1_shard_needed_blocks: ascending global KV blocks the shard [lo_block, hi_block) reads but does not own (host only)."""
    cfg = cfg or RouteCfg()
    cap = max(lo_block, 1)
    buf = (ctypes.c_int32 * cap)()
    count = ctypes.c_int32(0)
    _check(load().bf1_shard_needed_blocks(n_tokens, ctypes.byref(cfg), lo_block, hi_block, buf, cap, ctypes.byref(count)))
    return list(buf[:count.value])


def plan_route_shard(n_tokens: int, lo_block: int, hi_block: int, needed_blocks: torch.Tensor,
                     cfg: Optional[RouteCfg] = None, route: Optional[Route] = None, stream=None):
    """bf1_plan_route_shard: the shard's route over its local [needed | own] key/value tensor.
    Returns (route, cu_seqlens [2] int32 device tensor of the shard's virtual sequence)."""
    cfg = cfg or RouteCfg()
    assert needed_blocks.dtype == torch.int32 and needed_blocks.is_cuda
    if route is None:
        _, deg = route_capacity(1, n_tokens, n_tokens, cfg)
        route = Route.empty(hi_block - lo_block, deg, needed_blocks.device, cfg)
    cu = torch.zeros(2, dtype=torch.int32, device=needed_blocks.device)
    _check(load().bf1_plan_route_shard(n_tokens, lo_block, hi_block, ctypes.byref(cfg),
                                       needed_blocks.data_ptr() if needed_blocks.numel() else None, needed_blocks.numel(),
                                       ctypes.byref(route.c), cu.data_ptr(), _raw_stream(stream)))
    own_tokens = min(n_tokens, hi_block * 64) - lo_block * 64
    cu._bf1_total = needed_blocks.numel() * 64 + own_tokens
    route.cfg = cfg
    return route, cu


def shard_needed_blocks_strided(n_tokens: int, first_block: int, stride: int, num_blocks: int,
                                cfg: Optional[RouteCfg] = None):
    """bf1_shard_needed_blocks_strided: ascending global KV blocks read but not owned by the shard
    first_block, first_block + stride, ... (num_blocks of them); host only."""
    cfg = cfg or RouteCfg()
    cap = max(first_block + (num_blocks - 1) * stride, 1)
    buf = (ctypes.c_int32 * cap)()
    count = ctypes.c_int32(0)
    _check(load().bf1_shard_needed_blocks_strided(n_tokens, ctypes.byref(cfg), first_block, stride, num_blocks, buf, cap,
                                                  ctypes.byref(count)))
    return list(buf[:count.value])


def plan_route_shard_strided(n_tokens: int, first_block: int, stride: int, num_blocks: int, needed_blocks: torch.Tensor,
                             cfg: Optional[RouteCfg] = None, route: Optional[Route] = None, stream=None):
    """bf1_plan_route_shard_strided: the strided shard's route over its local [needed | own] key/value tensor.
    Returns (route, cu_seqlens [2] int32 device tensor of the shard's virtual sequence)."""
    cfg = cfg or RouteCfg()
    assert needed_blocks.dtype == torch.int32 and needed_blocks.is_cuda
    if route is None:
        _, deg = route_capacity(1, n_tokens, n_tokens, cfg)
        route = Route.empty(num_blocks, deg, needed_blocks.device, cfg)
    cu = torch.zeros(2, dtype=torch.int32, device=needed_blocks.device)
    _check(load().bf1_plan_route_shard_strided(n_tokens, first_block, stride, num_blocks, ctypes.byref(cfg),
                                               needed_blocks.data_ptr() if needed_blocks.numel() else None,
                                               needed_blocks.numel(), ctypes.byref(route.c), cu.data_ptr(),
                                               _raw_stream(stream)))
    last = first_block + (num_blocks - 1) * stride
    own_tokens = (num_blocks - 1) * 64 + min(64, n_tokens - last * 64)
    cu._bf1_total = needed_blocks.numel() * 64 + own_tokens
    route.cfg = cfg
    return route, cu


def cu_seqlens_tensor(seqlens: Sequence[int], device) -> torch.Tensor:
    cu = [0]
    for n in seqlens:
        cu.append(cu[-1] + int(n))
    t = torch.tensor(cu, dtype=torch.int32, device=device)
    t._bf1_total = cu[-1]   # host copy of the total, saves a device sync in plan_route
    return t


def default_scale(d: int) -> float:
    return 1.0 / math.sqrt(d)
