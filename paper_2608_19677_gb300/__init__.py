"""GB300 (sm_103a) hot path of planned prefix-affinity routing (CacheRoute, arXiv 2608.19677).

Thin ctypes binding over the C ABI declared in ``include/cacheroute.h``: every
function below only marshals torch CUDA tensors into device pointers and calls
the library of the same name; every step of the path runs in the library's
CUDA kernels.  There is no CPU fallback: importing works without a GPU, but
creating a ``Context`` requires the compiled library and a CUDA device, and
fails loudly otherwise.

  hash_prefixes   request prefix spans -> routing keys          (cr_hash_prefixes)
  build_plans     one interval's keys -> plans (Eq. 1, Alg. 1)  (cr_build_plans)
  route_batch     keys -> destination per (request, replica)    (cr_route_batch)
  Ring            ring of the bounded-load policy               (cr_ring_create)
  plan_diff       churn between two plans                       (cr_plan_diff)
  shadow_replay   routed requests -> LRU hit / load counters    (cr_shadow_replay)

What a destination does with the prefixes it holds:

  KVPages         pages of a key/value cache, and pages_extend, pages_fork, pages_free, pages_compact
  Rotary, rope    rotary positions of queries and keys          (cr_rope)
  kv_write        keys and values of new tokens -> pages        (cr_kv_write)
  kv_append       the same, queries and keys rotated            (cr_kv_append)
  kv_read         pages -> keys and values                      (cr_kv_read)
  attn_packed     attention over whole prompts                  (cr_attn_packed)
  attn_paged      attention over cached pages                   (cr_attn_paged)
  attn_decode     of single tokens that share prefixes          (cr_attn_decode)
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import os
import struct
from typing import List, Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
# CR_DEBUG_LIB=1 loads the bounds-checking build (buildlib.build(debug=True)) instead
LIB_PATH = os.path.join(_HERE, "libcacheroute_debug.so" if os.environ.get("CR_DEBUG_LIB") == "1"
                        else "libcacheroute.so")

CR_OK, CR_EINVAL, CR_ENOMEM, CR_ECUDA, CR_ETIMEOUT, CR_EOVERFLOW = range(6)
STATUS_NAMES = {0: "CR_OK", 1: "CR_EINVAL", 2: "CR_ENOMEM", 3: "CR_ECUDA", 4: "CR_ETIMEOUT",
                5: "CR_EOVERFLOW"}
POLICY = {"CR": 0, "CR_NOLPT": 1, "CR_NOREPL": 2, "P2C": 3, "RR": 4, "HASH": 5, "CHWBL": 6}
VARIANT = {"LPT": 0, "RANDOM": 1, "NOREPL": 2, "SLOTCAP": 3}
MAX_R, MAX_CAP, MAX_CAPS, MAX_REPLICAS, CTR_FIELDS, MAX_VNODES = 8192, 1024, 8, 256, 5, 1024

# every symbol the header declares (checked by the CPU test suite)
EXPORTS = ("cr_create", "cr_destroy", "cr_set_stream", "cr_sync", "cr_last_error", "cr_launch_count",
           "cr_hash_prefixes", "cr_plan_create", "cr_plan_destroy", "cr_build_plans", "cr_build_plan",
           "cr_plan_get_info", "cr_plan_export", "cr_route_batch", "cr_replay_create", "cr_replay_reset",
           "cr_replay_destroy", "cr_shadow_replay", "cr_replay_export_state", "cr_key_histogram_noalloc",
           "cr_ring_create", "cr_ring_destroy", "cr_ring_export", "cr_plan_diff",
           "cr_replay_create_tokens", "cr_set_resolve_stream", "cr_partition_create", "cr_partition_destroy",
           "cr_profile_enable", "cr_profile_read", "cr_plan_import", "cr_replay_import_state",
           "cr_replay_input_create", "cr_replay_input_destroy", "cr_replay_partition", "cr_replay_simulate",
           "cr_pages_extend", "cr_pages_fork", "cr_pages_free", "cr_pages_compact", "cr_kv_write",
           "cr_attn_packed", "cr_attn_paged", "cr_attn_decode", "cr_rope", "cr_kv_append", "cr_kv_read")
PROF = {"hash": 0, "plan": 1, "route_cand": 2, "route_resolve": 3, "partition": 4, "replay": 5}
CR_NOALLOC_MAX_KEYS = 65536


class CacheRouteError(RuntimeError):
    def __init__(self, code: int, where: str, msg: str):
        super().__init__(f"{where}: {STATUS_NAMES.get(code, code)}: {msg}")
        self.code = code


class PlanParams(C.Structure):
    _fields_ = [("R", C.c_uint32), ("W", C.c_uint32), ("qcap_num", C.c_uint64),
                ("qcap_den", C.c_uint64), ("variant", C.c_uint32), ("reserved", C.c_uint32),
                ("seed", C.c_uint64), ("epoch", C.c_uint64), ("d_init_load", C.c_void_p)]


class PlanInfo(C.Structure):
    _fields_ = [("n", C.c_uint64), ("U", C.c_uint64), ("n_adm", C.c_uint64), ("sum_k", C.c_uint64),
                ("cold", C.c_uint64), ("max_k", C.c_uint64), ("R", C.c_uint32), ("W", C.c_uint32)]


class PlanDiff(C.Structure):
    _fields_ = [(f, C.c_uint64) for f in ("keys_a", "keys_b", "keys_common", "pairs_a", "pairs_b",
                                          "pairs_common", "adm_k_changed", "adm_set_changed", "hist_keys",
                                          "hist_kb_changed")]


class KVPagesDesc(C.Structure):
    _fields_ = ([(f, C.c_void_p) for f in ("d_cache", "d_ref", "d_table", "d_lens")] +
                [(f, C.c_uint32) for f in ("dtype", "layers", "n_pages", "page", "kv_heads", "head_dim", "n_seqs",
                                           "max_pages")] +
                [(f, C.c_uint64) for f in ("layer_stride", "kv_stride", "page_stride", "token_stride", "head_stride")] +
                [("d_scale", C.c_void_p), ("block", C.c_uint32), ("reserved", C.c_uint32)])


class RotaryDesc(C.Structure):
    _fields_ = [("d_turn", C.c_void_p), ("pairs", C.c_uint32), ("layout", C.c_uint32), ("inverse", C.c_uint32),
                ("scale", C.c_float)]


class Replica(C.Structure):
    _fields_ = [("policy", C.c_uint32), ("reserved", C.c_uint32), ("seed", C.c_uint64), ("ring", C.c_void_p)]


_lib = None


def build(force: bool = False) -> str:
    """Compile the CUDA library in-tree (nvcc, sm_103a)."""
    from . import buildlib
    return buildlib.build(force=force)


def lib() -> C.CDLL:
    """The loaded CUDA library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build the CUDA library first "
                          f"(python -c 'import __graft_entry__ as g; g.build()')")
    L = C.CDLL(LIB_PATH)
    vp, u64, u32, i32 = C.c_void_p, C.c_uint64, C.c_uint32, C.c_int
    sig = {
        "cr_create": ([C.POINTER(vp), i32, vp], i32),
        "cr_destroy": ([vp], i32),
        "cr_set_stream": ([vp, vp], i32),
        "cr_sync": ([vp], i32),
        "cr_last_error": ([vp], C.c_char_p),
        "cr_launch_count": ([vp], u64),
        "cr_hash_prefixes": ([vp, vp, vp, vp, u64, u64, vp], i32),
        "cr_plan_create": ([vp, C.POINTER(vp)], i32),
        "cr_plan_destroy": ([vp, vp], i32),
        "cr_build_plans": ([vp, vp, u64, C.POINTER(PlanParams), u32, C.POINTER(vp)], i32),
        "cr_build_plan": ([vp, vp, u64, C.POINTER(PlanParams), vp], i32),
        "cr_plan_get_info": ([vp, vp, C.POINTER(PlanInfo)], i32),
        "cr_plan_export": ([vp, vp] + [vp] * 9, i32),
        "cr_route_batch": ([vp, C.POINTER(vp), C.POINTER(Replica), u32, u32, vp, u64, u64, u32, vp, vp], i32),
        "cr_replay_create": ([vp, u32, u32, C.POINTER(C.c_uint32), u32, C.POINTER(vp)], i32),
        "cr_replay_create_tokens": ([vp, u32, u32, C.POINTER(C.c_uint32), u32, C.POINTER(vp)], i32),
        "cr_replay_reset": ([vp, vp], i32),
        "cr_replay_destroy": ([vp, vp], i32),
        "cr_shadow_replay": ([vp, vp, vp, vp, vp, vp, u64, vp], i32),
        "cr_replay_export_state": ([vp, vp, u32, u32, vp, C.POINTER(C.c_uint32)], i32),
        "cr_key_histogram_noalloc": ([vp, u64, vp, vp, vp, vp], i32),
        "cr_ring_create": ([vp, u32, u32, u64, C.POINTER(vp)], i32),
        "cr_ring_destroy": ([vp, vp], i32),
        "cr_ring_export": ([vp, vp, vp, vp], i32),
        "cr_plan_diff": ([vp, vp, vp, C.POINTER(PlanDiff)], i32),
        "cr_set_resolve_stream": ([vp, vp], i32),
        "cr_partition_create": ([i32, u32, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp)], i32),
        "cr_partition_destroy": ([vp], i32),
        "cr_plan_import": ([vp, vp, u32, u32, u64, vp, vp, vp, vp, vp, vp], i32),
        "cr_replay_import_state": ([vp, vp, u32, u32, vp, u32], i32),
        "cr_replay_input_create": ([vp, C.POINTER(vp)], i32),
        "cr_replay_input_destroy": ([vp, vp], i32),
        "cr_replay_partition": ([vp, vp, vp, vp, vp, vp, u64, vp], i32),
        "cr_replay_simulate": ([vp, vp, vp, vp], i32),
        "cr_profile_enable": ([vp, u32], i32),
        "cr_profile_read": ([vp, u32, C.POINTER(C.c_uint64), C.POINTER(C.c_double)], i32),
        "cr_pages_extend": ([vp, vp, vp, vp, u32], i32),
        "cr_pages_fork": ([vp, vp, vp, vp, vp, u32], i32),
        "cr_pages_free": ([vp, vp, vp, u32], i32),
        "cr_pages_compact": ([vp, vp, vp, vp, vp, vp], i32),
        "cr_kv_write": ([vp, vp, u32, vp, u64, u64, vp, u64, u64, vp, vp, u32, u32], i32),
        "cr_rope": ([vp, vp, vp], i32),
        "cr_kv_append": ([vp, vp, u32, vp, vp], i32),
        "cr_kv_read": ([vp, vp, u32, vp], i32),
        "cr_attn_packed": ([vp, vp, u32, u32, u32, vp, u64, u64, vp, u64, u64, vp, u32], i32),
        "cr_attn_paged": ([vp, vp, u32, vp], i32),
        "cr_attn_decode": ([vp, vp, u32, vp, vp, vp, u32], i32),
    }
    for name, (args, res) in sig.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = res
    _lib = L
    return L


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def _np_ptr(a: np.ndarray):
    return a.ctypes.data_as(C.c_void_p)


class Context:
    """A library context bound to one CUDA device and stream (torch's current stream by default)."""

    def __init__(self, device: int = 0, stream=None):
        import torch
        self.device = device
        self._stream_obj = stream if stream is not None else torch.cuda.current_stream(device)
        h = C.c_void_p()
        st = lib().cr_create(C.byref(h), device, C.c_void_p(self._stream_obj.cuda_stream))
        if st != CR_OK:
            raise CacheRouteError(st, "cr_create", lib().cr_last_error(None).decode())
        self._h = h
        self._raw_stream = self._stream_obj.cuda_stream
        _load_torch()

    @property
    def handle(self):
        return self._h

    @property
    def stream(self):
        """The torch stream that the library's work runs on."""
        return self._stream_obj

    def check(self, st: int, where: str):
        if st != CR_OK:
            raise CacheRouteError(st, where, lib().cr_last_error(self._h).decode())

    def sync(self):
        self.check(lib().cr_sync(self._h), "cr_sync")

    def set_stream(self, stream):
        """Later calls run on ``stream``, after what the context has enqueued so far."""
        self.check(lib().cr_set_stream(self._h, C.c_void_p(stream.cuda_stream)), "cr_set_stream")
        self._stream_obj, self._raw_stream = stream, stream.cuda_stream

    @property
    def launches(self) -> int:
        return int(lib().cr_launch_count(self._h))

    def profile_enable(self, max_launches: int):
        """Time the library's main kernels per launch with CUDA events (0: off); forgets earlier launches."""
        self.check(lib().cr_profile_enable(self._h, max_launches), "cr_profile_enable")

    def profile_read(self, tag: str):
        """(timed launches, summed milliseconds) of one kind of launch (blocking)."""
        n, ms = C.c_uint64(), C.c_double()
        self.check(lib().cr_profile_read(self._h, PROF[tag], C.byref(n), C.byref(ms)), "cr_profile_read")
        return int(n.value), float(ms.value)

    def close(self):
        if getattr(self, "_h", None):
            lib().cr_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _need_cuda(name, t, dtype=None):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")


def hash_prefixes(ctx: Context, tokens, off, plen, salt: int = 0, out=None):
    """Routing key per request (uint64 values in an int64 tensor)."""
    import torch
    n = int(off.shape[0])
    _need_cuda("tokens", tokens, torch.int32)
    _need_cuda("off", off, torch.int64)
    _need_cuda("plen", plen, torch.int32)
    if out is None:
        out = torch.empty(n, dtype=torch.int64, device=off.device)
    ctx.check(lib().cr_hash_prefixes(ctx.handle, _ptr(tokens), _ptr(off), _ptr(plen), n,
                                     salt & ((1 << 64) - 1), _ptr(out)), "cr_hash_prefixes")
    return out


class Plan:
    """A library-owned plan (device resident)."""

    def __init__(self, ctx: Context):
        self.ctx = ctx
        h = C.c_void_p()
        ctx.check(lib().cr_plan_create(ctx.handle, C.byref(h)), "cr_plan_create")
        self._h = h

    @property
    def handle(self):
        return self._h

    def info(self) -> PlanInfo:
        inf = PlanInfo()
        self.ctx.check(lib().cr_plan_get_info(self.ctx.handle, self._h, C.byref(inf)), "cr_plan_get_info")
        return inf

    def export(self) -> dict:
        inf = self.info()
        U, na, sk, R = int(inf.U), int(inf.n_adm), int(inf.sum_k), int(inf.R)
        a = dict(ukey=np.zeros(max(U, 1), np.uint64), ucnt=np.zeros(max(U, 1), np.uint64),
                 adm_key=np.zeros(max(na, 1), np.uint64), adm_cnt=np.zeros(max(na, 1), np.uint64),
                 adm_k=np.zeros(max(na, 1), np.uint32), koff=np.zeros(na + 1, np.uint32),
                 members=np.zeros(max(sk, 1), np.uint16), jobs=np.zeros(max(sk, 1), np.uint64),
                 load=np.zeros(R, np.uint64))
        self.ctx.check(lib().cr_plan_export(self.ctx.handle, self._h, *[_np_ptr(a[k]) for k in
                                                                        ("ukey", "ucnt", "adm_key", "adm_cnt",
                                                                         "adm_k", "koff", "members", "jobs",
                                                                         "load")]), "cr_plan_export")
        out = dict(U=U, n_adm=na, sum_k=sk, cold=int(inf.cold), max_k=int(inf.max_k), R=R, W=int(inf.W))
        out.update(ukey=a["ukey"][:U], ucnt=a["ucnt"][:U], adm_key=a["adm_key"][:na], adm_cnt=a["adm_cnt"][:na],
                   adm_k=a["adm_k"][:na], koff=a["koff"], members=a["members"][:sk], jobs=a["jobs"][:sk],
                   load=a["load"])
        return out

    def load(self, R: int, W: int, adm_key, adm_cnt, adm_k, members, jobs=None, load=None):
        """Install a plan given as host arrays in admission order (cr_plan_import)."""
        ak = np.ascontiguousarray(adm_key, np.uint64)
        ac = np.ascontiguousarray(adm_cnt, np.uint64)
        kk = np.ascontiguousarray(adm_k, np.uint32)
        mm = np.ascontiguousarray(members, np.uint16)
        jb = None if jobs is None else np.ascontiguousarray(jobs, np.uint64)
        ld = None if load is None else np.ascontiguousarray(load, np.uint64)
        self.ctx.check(lib().cr_plan_import(self.ctx.handle, self._h, R, W, ak.size, _np_ptr(ak), _np_ptr(ac),
                                            _np_ptr(kk), _np_ptr(mm), None if jb is None else _np_ptr(jb),
                                            None if ld is None else _np_ptr(ld)), "cr_plan_import")
        return self

    def close(self):
        if getattr(self, "_h", None):
            lib().cr_plan_destroy(self.ctx.handle, self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def plan_params(R: int, W: int, qcap_num: int, qcap_den: int, variant="LPT", seed: int = 0, epoch: int = 0,
                init_load=None) -> PlanParams:
    v = VARIANT[variant] if isinstance(variant, str) else int(variant)
    p = PlanParams(R, W, qcap_num, qcap_den, v, 0, seed & ((1 << 64) - 1), epoch, _ptr(init_load))
    p._init_load = init_load  # the device vector must outlive the parameters that point at it
    return p


def build_plans(ctx: Context, keys, params: Sequence[PlanParams], plans: Sequence[Plan]):
    import torch
    n = int(keys.shape[0])
    _need_cuda("keys", keys, torch.int64)
    arr = (PlanParams * len(params))(*params)
    hs = (C.c_void_p * len(plans))(*[p.handle for p in plans])
    ctx.check(lib().cr_build_plans(ctx.handle, _ptr(keys), n, arr, len(params), hs), "cr_build_plans")
    return plans


def build_plan(ctx: Context, keys, params: PlanParams, plan: Optional[Plan] = None) -> Plan:
    plan = plan or Plan(ctx)
    build_plans(ctx, keys, [params], [plan])
    return plan


def set_resolve_stream(ctx: Context, stream) -> None:
    """Route with the load-dependent resolution on ``stream`` (a torch stream; None: the context's)."""
    ctx.check(lib().cr_set_resolve_stream(ctx.handle, C.c_void_p(stream.cuda_stream) if stream is not None
                                          else None), "cr_set_resolve_stream")


class Partition:
    """Two streams whose kernels run on disjoint SM sets (green contexts): ``big`` and ``small``
    (torch external streams; ``small`` has ``small_sms`` SMs)."""

    def __init__(self, device: int, small_sms: int):
        import torch
        h, b, sm = C.c_void_p(), C.c_void_p(), C.c_void_p()
        st = lib().cr_partition_create(device, small_sms, C.byref(h), C.byref(b), C.byref(sm))
        if st != CR_OK:
            raise CacheRouteError(st, "cr_partition_create", lib().cr_last_error(None).decode())
        self._h = h
        dev = torch.device("cuda", device)
        self.big = torch.cuda.ExternalStream(b.value, device=dev)
        self.small = torch.cuda.ExternalStream(sm.value, device=dev)

    def close(self):
        if getattr(self, "_h", None):
            lib().cr_partition_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def plan_diff(ctx: Context, a: Plan, b: Plan) -> dict:
    """Counts of how plan b differs from plan a (blocking); see ``churn``."""
    out = PlanDiff()
    ctx.check(lib().cr_plan_diff(ctx.handle, a.handle, b.handle, C.byref(out)), "cr_plan_diff")
    return {f: int(getattr(out, f)) for f, _ in PlanDiff._fields_}


def churn(diff: dict):
    """(cache churn, count churn) as floats: 1 - Jaccard of the assignment sets, and the share of
    the keys of either histogram whose Eq. 1 k_b changed."""
    up = diff["pairs_a"] + diff["pairs_b"] - diff["pairs_common"]
    return (1.0 - diff["pairs_common"] / up if up else 0.0,
            diff["hist_kb_changed"] / diff["hist_keys"] if diff["hist_keys"] else 0.0)


class Ring:
    """Consistent-hashing ring of the bounded-load policy (R destinations x vnodes points), on the device."""

    def __init__(self, ctx: Context, R: int, vnodes: int, seed: int):
        self.ctx, self.R, self.vnodes, self.seed = ctx, R, vnodes, seed & ((1 << 64) - 1)
        h = C.c_void_p()
        ctx.check(lib().cr_ring_create(ctx.handle, R, vnodes, self.seed, C.byref(h)), "cr_ring_create")
        self._h = h

    @property
    def handle(self):
        return self._h

    def export(self):
        """(point uint64 [R*vnodes] ascending, owner uint16 [R*vnodes]) on the host."""
        M = self.R * self.vnodes
        pt = np.zeros(M, np.uint64)
        ow = np.zeros(M, np.uint16)
        self.ctx.check(lib().cr_ring_export(self.ctx.handle, self._h, _np_ptr(pt), _np_ptr(ow)), "cr_ring_export")
        return pt, ow

    def close(self):
        if getattr(self, "_h", None):
            lib().cr_ring_destroy(self.ctx.handle, self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def route_batch(ctx: Context, plans: Sequence[Optional[Plan]], policies: Sequence, seeds: Sequence[int],
                R: int, keys, first_req_index: int, batch_B: int, load, dest=None,
                rings: Optional[Sequence[Optional[Ring]]] = None):
    """Destinations (uint16 values in an int16 tensor [n_rep, n]); ``load`` [n_rep, R] is updated in place.

    ``rings[i]`` is the ring of replica i when its policy is CHWBL."""
    import torch
    n_rep = len(policies)
    n = int(keys.shape[0])
    _need_cuda("keys", keys, torch.int64)
    _need_cuda("load", load, torch.int64)
    if dest is None:
        dest = torch.empty((n_rep, n), dtype=torch.int16, device=keys.device)
    _need_cuda("dest", dest, torch.int16)
    rg = list(rings) if rings is not None else [None] * n_rep
    reps = (Replica * n_rep)(*[Replica(POLICY[p] if isinstance(p, str) else int(p), 0,
                                       int(s) & ((1 << 64) - 1), (g.handle.value if g is not None else None))
                               for p, s, g in zip(policies, seeds, rg)])
    hs = (C.c_void_p * n_rep)(*[(p.handle if p is not None else None) for p in plans])
    ctx.check(lib().cr_route_batch(ctx.handle, hs, reps, n_rep, R, _ptr(keys), n, first_req_index, batch_B,
                                   _ptr(load), _ptr(dest)), "cr_route_batch")
    return dest


class Replay:
    """Library-owned LRU state for n_rep x R destinations x len(caps) capacities.

    ``tokens``: capacities count prefix tokens (byte-aware variant, cr_replay_create_tokens)."""

    def __init__(self, ctx: Context, n_rep: int, R: int, caps: Sequence[int], tokens: bool = False):
        self.ctx, self.n_rep, self.R, self.caps, self.tokens = ctx, n_rep, R, list(caps), tokens
        cp = (C.c_uint32 * len(caps))(*caps)
        h = C.c_void_p()
        name = "cr_replay_create_tokens" if tokens else "cr_replay_create"
        ctx.check(getattr(lib(), name)(ctx.handle, n_rep, R, cp, len(caps), C.byref(h)), name)
        self._h = h

    @property
    def handle(self):
        return self._h

    def reset(self):
        self.ctx.check(lib().cr_replay_reset(self.ctx.handle, self._h), "cr_replay_reset")

    def set_state(self, rep: int, r: int, keys):
        """Resident keys of one simulator, most recent first (cr_replay_import_state)."""
        k = np.ascontiguousarray(keys, np.uint64)
        self.ctx.check(lib().cr_replay_import_state(self.ctx.handle, self._h, rep, r,
                                                    _np_ptr(k) if k.size else None, k.size), "cr_replay_import_state")

    def state(self, rep: int, r: int) -> np.ndarray:
        out = np.zeros(MAX_CAP, np.uint64)
        fill = C.c_uint32()
        self.ctx.check(lib().cr_replay_export_state(self.ctx.handle, self._h, rep, r, _np_ptr(out),
                                                    C.byref(fill)), "cr_replay_export_state")
        return out[:fill.value].copy()

    def close(self):
        if getattr(self, "_h", None):
            lib().cr_replay_destroy(self.ctx.handle, self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class ReplayInput:
    """A partitioned batch of routed requests (cr_replay_partition), read by replay_simulate."""

    def __init__(self, ctx: Context):
        self.ctx = ctx
        h = C.c_void_p()
        ctx.check(lib().cr_replay_input_create(ctx.handle, C.byref(h)), "cr_replay_input_create")
        self._h = h

    @property
    def handle(self):
        return self._h

    def close(self):
        if getattr(self, "_h", None):
            lib().cr_replay_input_destroy(self.ctx.handle, self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def replay_partition(ctx: Context, replay: Replay, keys, plen, slen, dest, inp: ReplayInput):
    """Partition routed requests for `replay` into `inp` (a8 alone), on ctx's stream."""
    import torch
    n = int(keys.shape[0])
    _need_cuda("keys", keys, torch.int64)
    _need_cuda("plen", plen, torch.int32)
    _need_cuda("slen", slen, torch.int32)
    _need_cuda("dest", dest, torch.int16)
    ctx.check(lib().cr_replay_partition(ctx.handle, replay.handle, _ptr(keys), _ptr(plen), _ptr(slen), _ptr(dest),
                                        n, inp.handle), "cr_replay_partition")
    return inp


def replay_simulate(ctx: Context, replay: Replay, inp: ReplayInput, ctr):
    """Run the simulators over a partitioned input (a9 alone), accumulating into ``ctr``."""
    import torch
    _need_cuda("ctr", ctr, torch.int64)
    ctx.check(lib().cr_replay_simulate(ctx.handle, replay.handle, inp.handle, _ptr(ctr)), "cr_replay_simulate")
    return ctr


def shadow_replay(ctx: Context, replay: Replay, keys, plen, slen, dest, ctr):
    """Accumulate counters into ``ctr`` (int64 [n_rep, n_caps, R, 5])."""
    import torch
    n = int(keys.shape[0])
    _need_cuda("keys", keys, torch.int64)
    _need_cuda("plen", plen, torch.int32)
    _need_cuda("slen", slen, torch.int32)
    _need_cuda("dest", dest, torch.int16)
    _need_cuda("ctr", ctr, torch.int64)
    ctx.check(lib().cr_shadow_replay(ctx.handle, replay.handle, _ptr(keys), _ptr(plen), _ptr(slen), _ptr(dest),
                                     n, _ptr(ctr)), "cr_shadow_replay")
    return ctr


# ---- what a destination does with the prefixes it holds ------------------------------------------------------------
# These calls are made once per layer and step: their checks take one look at each tensor.  They have no gradient, and
# refuse tensors that want one where gradients are recorded.
_torch = None        # set by the first Context
_codes = {}          # dtype -> CR_DTYPE_*


def _load_torch():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
        _codes.update({torch.bfloat16: 0, torch.float16: 1})
    return _torch


def _dtype_code(dtype) -> int:
    _load_torch()
    if dtype not in _codes:
        raise ValueError(f"keys, values and queries are bfloat16 or float16, got {dtype}")
    return _codes[dtype]


def _out(ctx: Context, shape, like, dtype):
    """An output of a call, in memory that ctx's stream has done with: on another stream's memory, that stream's earlier
    work might still read what is written here.  It is not handed out again before the current stream has passed it."""
    if ctx._raw_stream == _torch._C._cuda_getCurrentRawStream(ctx.device):
        return _torch.empty(shape, dtype=dtype, device=like.device)
    with _torch.cuda.stream(ctx._stream_obj):
        t = _torch.empty(shape, dtype=dtype, device=like.device)
    t.record_stream(_torch.cuda.current_stream(ctx.device))
    return t


def _int32(name, t, n=None):
    """Address of a contiguous int32 CUDA tensor, of n elements."""
    if t.dtype is not _torch.int32 or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 CUDA tensor")
    if n is not None and t.numel() != n:
        raise ValueError(f"{name} must have {n} elements, got {t.numel()}")
    return t.data_ptr()


def _heads(name, t, dtype, shape, tokens, heads, dim):
    """(address, token stride, head stride) of a tensor [tokens, heads, dim] of that shape, contiguous in its last
    dimension; ``shape``: t.shape; None: any."""
    if t.dtype is not dtype or not t.is_cuda or len(shape) != 3:
        raise ValueError(f"{name} must be a {dtype} CUDA tensor [tokens, heads, head_dim]")
    T, h, d = shape
    if (tokens is not None and T != tokens) or (heads is not None and h != heads) or (dim is not None and d != dim):
        raise ValueError(f"{name} must have shape {(tokens, heads, dim)} (None: any), got {tuple(shape)}")
    st, sh, sd = t.stride()
    if sd != 1:
        raise ValueError(f"{name} must be contiguous in head_dim")
    return t.data_ptr(), st, sh


def _no_gradient(*tensors):
    """These calls are for serving: a gradient that is asked for would be lost without a word."""
    for t in tensors:
        if t.requires_grad and _torch.is_grad_enabled():
            raise ValueError("the attention and cache calls have no gradient: call them under torch.no_grad(), or on "
                             "detached tensors")


class KVPages:
    """Pages of a destination's key/value cache, tables and lengths of its sequences (tensors the caller keeps).

    ``cache`` [layers, 2, n_pages, page, kv_heads, head_dim] (keys, values; bfloat16 or float16; a page's tokens and
    heads may be stored in either order), ``ref`` int32[n_pages] counts the table entries that name a page (0: free),
    ``table`` int32[n_seqs, max_pages] lists each sequence's pages (-1 behind them), ``lens`` int32[n_seqs] its
    tokens.  ``KVPages.empty`` makes an empty pool.

    In 8 bits ``cache`` is float8_e4m3fn, ``scale`` float32 [layers, 2, n_pages, kv_heads, page / block] holds the power
    of two of every block of tokens and head, and ``dtype`` (bfloat16 unless given) is the type of the keys, values and
    queries of the calls."""

    def __init__(self, cache, ref, table, lens, scale=None, dtype=None):
        _load_torch()
        if cache.dim() != 6 or cache.shape[1] != 2 or not cache.is_cuda or cache.stride(5) != 1:
            raise ValueError("cache must be a CUDA tensor [layers, 2, n_pages, page, kv_heads, head_dim]")
        layers, _, n_pages, page, heads, dim = cache.shape
        _int32("ref", ref, n_pages)
        _int32("table", table)
        if table.dim() != 2:
            raise ValueError("table must have two dimensions")
        _int32("lens", lens, table.shape[0])
        self.block = 0
        if cache.dtype is _torch.float8_e4m3fn:
            if scale is None:
                raise ValueError("a cache in 8 bits needs its blocks' scales")
            _need_cuda("scale", scale, _torch.float32)
            blocks = scale.shape[-1] if scale.dim() == 5 else 0
            if not blocks or page % blocks or tuple(scale.shape[:4]) != (layers, 2, n_pages, heads):
                raise ValueError(f"scale must have shape {(layers, 2, n_pages, heads)} and page / block, got {tuple(scale.shape)}")
            self.block = page // blocks
            dtype = dtype or _torch.bfloat16
        elif scale is not None or (dtype is not None and dtype is not cache.dtype):
            raise ValueError("scale, and a type of its own, are a cache's in 8 bits (float8_e4m3fn)")
        self.cache, self.ref, self.table, self.lens, self.scale = cache, ref, table, lens, scale
        self.layers, self.n_pages, self.page, self.kv_heads, self.head_dim = layers, n_pages, page, heads, dim
        self.dtype = dtype or cache.dtype
        self._code = _dtype_code(self.dtype) + (2 if self.block else 0)
        self._bind()

    def _bind(self):
        st = self.cache.stride()
        d = KVPagesDesc(_ptr(self.cache), _ptr(self.ref), _ptr(self.table), _ptr(self.lens), self._code, self.layers,
                        self.n_pages, self.page, self.kv_heads, self.head_dim, self.table.shape[0],
                        self.table.shape[1], st[0], st[1], st[2], st[3], st[4], _ptr(self.scale), self.block, 0)
        self._desc, self._addr = d, C.addressof(d)

    @classmethod
    def empty(cls, n_pages: int, page: int, n_seqs: int, max_pages: int, layers: int, kv_heads: int, head_dim: int,
              dtype=None, device="cuda", bits: int = 16, block: Optional[int] = None):
        """``bits``: 16, or 8: then with a scale for every ``block`` tokens (16 or the page, whichever is less) and head."""
        torch = _load_torch()
        if bits not in (8, 16) or (block is not None and bits != 8):
            raise ValueError("bits is 16 or 8; only a cache in 8 bits has blocks")
        cache = torch.zeros((layers, 2, n_pages, page, kv_heads, head_dim), device=device,
                            dtype=torch.float8_e4m3fn if bits == 8 else dtype or torch.bfloat16)
        scale = None
        if bits == 8:
            block = block or min(16, page)
            if not 8 <= block <= page or page % block:
                raise ValueError(f"blocks of {block} tokens in pages of {page}: a power of two, 8 to the page")
            scale = torch.ones((layers, 2, n_pages, kv_heads, page // block), dtype=torch.float32, device=device)
        return cls(cache, torch.zeros(n_pages, dtype=torch.int32, device=device),
                   torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device=device),
                   torch.zeros(n_seqs, dtype=torch.int32, device=device), scale=scale, dtype=dtype)

    def replace(self, ref, table):
        """Take the counts and tables that ``pages_compact`` gave (the cache's pages have moved already).  The old ones
        are let go: where the context has a stream of its own, after that stream's work."""
        _int32("ref", ref, self.n_pages)
        _int32("table", table)
        if table.shape != self.table.shape:
            raise ValueError("table must have the old table's shape")
        self.ref, self.table = ref, table
        self._bind()


def pages_extend(ctx: Context, pages: KVPages, seqs, add):
    """The sequences ``seqs`` get pages for ``add`` more tokens each (cr_pages_extend)."""
    n = seqs.numel()
    st = lib().cr_pages_extend(ctx._h, pages._addr, _int32("seqs", seqs), _int32("add", add, n), n)
    if st:
        ctx.check(st, "cr_pages_extend")


def pages_fork(ctx: Context, pages: KVPages, src, dst, keep):
    """The empty rows ``dst`` become the first ``keep`` tokens of the rows ``src`` (cr_pages_fork)."""
    n = src.numel()
    st = lib().cr_pages_fork(ctx._h, pages._addr, _int32("src", src), _int32("dst", dst, n), _int32("keep", keep, n), n)
    if st:
        ctx.check(st, "cr_pages_fork")


def pages_free(ctx: Context, pages: KVPages, seqs):
    """The rows ``seqs`` become empty (cr_pages_free)."""
    st = lib().cr_pages_free(ctx._h, pages._addr, _int32("seqs", seqs), seqs.numel())
    if st:
        ctx.check(st, "cr_pages_free")


def pages_compact(ctx: Context, pages: KVPages):
    """Move live pages to the front (cr_pages_compact): (ref, table, page_map, n_live), new tensors;
    ``pages.replace(ref, table)`` takes them."""
    int32 = _torch.int32
    ref = _out(ctx, pages.ref.shape, pages.ref, int32)
    table = _out(ctx, pages.table.shape, pages.table, int32)
    page_map = _out(ctx, pages.ref.shape, pages.ref, int32)
    live = _out(ctx, (1,), pages.ref, int32)
    st = lib().cr_pages_compact(ctx._h, pages._addr, ref.data_ptr(), table.data_ptr(), page_map.data_ptr(),
                                live.data_ptr())
    if st:
        ctx.check(st, "cr_pages_compact")
    return ref, table, page_map, live


def kv_write(ctx: Context, pages: KVPages, layer: int, k, v, cu, seqs=None):
    """Write the keys and values [tokens, kv_heads, head_dim] of every sequence's last tokens into its pages:
    entry i's tokens are cu[i] .. cu[i+1]-1, its row seqs[i] (None: i) (cr_kv_write).  Pages that other rows name are
    left alone: a row's tokens are written before it is forked."""
    n = max(cu.numel() - 1, 0)
    if k.requires_grad or v.requires_grad:
        _no_gradient(k, v)
    shape = k.shape
    T = shape[0]
    kp, kt, kh = _heads("k", k, pages.dtype, shape, None, pages.kv_heads, pages.head_dim)
    vp, vt, vh = _heads("v", v, pages.dtype, v.shape, T, pages.kv_heads, pages.head_dim)
    st = lib().cr_kv_write(ctx._h, pages._addr, layer, kp, kt, kh, vp, vt, vh, _int32("cu", cu),
                           None if seqs is None else _int32("seqs", seqs, n), n, T)
    if st:
        ctx.check(st, "cr_kv_write")


@functools.lru_cache(None)
def _pi(bits: int) -> int:
    """pi * 2^bits, off by a unit at most (Machin: pi = 16 atan(1/5) - 4 atan(1/239))."""
    def atan_inverse(n):
        total, power, k, sign = 0, (1 << bits + 32) // n, 1, 1
        while power:
            total += sign * (power // k)
            power, k, sign = power // (n * n), k + 2, -sign
        return total
    return (16 * atan_inverse(5) - 4 * atan_inverse(239)) >> 32


def _share(f: float) -> int:
    """f radians as a share of a full turn, times 2^64, whole turns left out: the nearest integer.  A double is below
    2^1024: with 1,280 bits of pi, the quotient is exact to 2^-190."""
    num, den = f.as_integer_ratio()
    num, den = num << 1280 + 64, 2 * den * _pi(1280)
    return (2 * num + den) // (2 * den) % 2 ** 64


class Rotary:
    """Rotary positions: pair i of the first ``dims`` elements of a head turns by position * f_i, f_i = base^(-2i/dims).

    ``layout``: "half" (pairs x[i], x[dims/2 + i]) or "interleaved" (x[2i], x[2i + 1]).  ``scaling`` stretches the
    positions ``factor`` times: "linear" divides every f_i; "ntk" takes the base times factor^(dims/(dims - 2)); "ramp"
    leaves pairs that turn more than ``fast`` times within ``original`` tokens, divides those that turn less than ``slow``
    times, and goes from one to the other linearly in the turns, and multiplies the rotated elements by
    0.1 ln(factor) + 1 (Peng et al., arXiv 2309.00071).  ``scale`` gives that multiplier instead.  ``frequencies`` gives
    the f_i (radians a token, ``dims`` / 2 of them) instead of the base.  ``inverse()`` turns back.

    The f_i are doubles (``frequencies``); at every position, angles are within 2^-31 turns of theirs."""

    def __init__(self, dims: int, base: float = 10000.0, layout: str = "half", scaling: Optional[str] = None,
                 factor: float = 1.0, original: int = 0, slow: float = 1.0, fast: float = 32.0,
                 scale: Optional[float] = None, frequencies: Optional[Sequence[float]] = None, device="cuda"):
        torch = _load_torch()
        if dims < 8 or dims % 8 or dims > 128:
            raise ValueError(f"{dims} rotated elements: a multiple of 8, 8..128")
        if layout not in ("half", "interleaved"):
            raise ValueError(f"layout {layout!r}: half or interleaved")
        if scaling not in (None, "linear", "ntk", "ramp"):
            raise ValueError(f"scaling {scaling!r}: linear, ntk or ramp")
        if not (base > 0 and factor > 0) or not (math.isfinite(base) and math.isfinite(factor)):
            raise ValueError("base and factor must be positive")
        if frequencies is None:
            try:
                if scaling == "ntk":
                    base *= factor ** (dims / (dims - 2))
                f = [base ** (-2.0 * i / dims) if math.isfinite(base) else math.inf for i in range(dims // 2)]
            except OverflowError:
                f = [math.inf]
        else:
            f = [float(x) for x in frequencies]
            if scaling == "ntk":
                raise ValueError("ntk scaling changes the base: give frequencies or that")
            if len(f) != dims // 2 or not all(map(math.isfinite, f)):
                raise ValueError(f"{len(f)} frequencies for {dims // 2} pairs")
        if scaling == "linear":
            f = [x / factor for x in f]
        elif scaling == "ramp":
            if original <= 0 or not fast > slow:
                raise ValueError("a ramp needs the original length, and fast > slow")
            keep = [min(1.0, max(0.0, (original * abs(x) / (2 * math.pi) - slow) / (fast - slow))) for x in f]
            f = [x * k + x / factor * (1.0 - k) for x, k in zip(f, keep)]
            if scale is None:
                scale = 0.1 * math.log(factor) + 1.0 if factor > 1.0 else 1.0
        scale = 1.0 if scale is None else float(scale)
        if not abs(scale) <= 3.4028234663852886e38:
            raise ValueError("scale must be finite")
        if not all(map(math.isfinite, f)):
            raise ValueError("base and factor give frequencies that are not finite")
        self.dims, self.layout, self.scale, self.frequencies = dims, layout, scale, f
        # position times share drops whole turns by itself
        turn = [_share(x) for x in f]
        self.turn = torch.tensor([t - 2 ** 64 if t >= 2 ** 63 else t for t in turn], dtype=torch.int64, device=device)
        self._bind(0)

    def _bind(self, inverse: int):
        d = RotaryDesc(_ptr(self.turn), self.dims // 2, 0 if self.layout == "half" else 1, inverse, self.scale)
        self._desc, self._addr, self._inverse = d, C.addressof(d), inverse
        self._device = self.turn.device.index if self.turn.is_cuda else None

    def _on(self, ctx: Context) -> int:
        """Address of cr_rotary, for a call on ctx's stream: the frequencies stay until that stream has passed it."""
        if self._device != ctx.device:
            raise ValueError(f"the rotation's frequencies are on {self.turn.device}, the context on GPU {ctx.device}")
        if ctx._raw_stream != _torch._C._cuda_getCurrentRawStream(ctx.device):
            self.turn.record_stream(ctx._stream_obj)
        return self._addr

    def inverse(self) -> "Rotary":
        """Turns by the opposite angles (and multiplies by the same scale): the gradient of the rotation."""
        r = object.__new__(Rotary)
        r.dims, r.layout, r.scale, r.frequencies, r.turn = self.dims, self.layout, self.scale, self.frequencies, self.turn
        r._bind(1 - self._inverse)
        return r


_pack_rope = struct.Struct("@3P4Q4I").pack    # cr_rope_args


def rope(ctx: Context, x, rotary: Rotary, pos, out=None):
    """Rotate tokens x [tokens, heads, head_dim] (bfloat16 or float16) to positions ``pos`` int32[tokens] (cr_rope).
    ``out`` may be ``x``."""
    dtype, shape = x.dtype, x.shape
    code = _codes.get(dtype)
    if code is None:
        code = _dtype_code(dtype)
    if x.requires_grad or (out is not None and out.requires_grad):
        _no_gradient(x, *(() if out is None else (out,)))
    xp, xt, xh = _heads("x", x, dtype, shape, None, None, None)
    T, heads, dim = shape
    if out is None:
        out = _out(ctx, shape, x, dtype)
        op, ot, oh = out.data_ptr(), heads * dim, dim
    else:
        op, ot, oh = _heads("out", out, dtype, out.shape, T, heads, dim)
    st = lib().cr_rope(ctx._h, rotary._on(ctx), _pack_rope(xp, op, _int32("pos", pos, T), xt, xh, ot, oh, T, heads, dim, code))
    if st:
        ctx.check(st, "cr_rope")
    return out


_pack_append = struct.Struct("@4P8Q2P4I").pack  # cr_append_args


def kv_append(ctx: Context, pages: KVPages, layer: int, q, k, v, rotary: Rotary, cu, seqs=None, out=None):
    """``kv_write`` with queries and keys rotated to the tokens' positions in their rows (cr_kv_append): returns the
    rotated queries [tokens, heads, head_dim] (``out`` may be ``q``; ``q`` None: keys and values only)."""
    n = max(cu.numel() - 1, 0)
    if k.requires_grad or v.requires_grad or (q is not None and q.requires_grad):
        _no_gradient(k, v, *(() if q is None else (q,)))
    dtype, dim = pages.dtype, pages.head_dim
    shape = k.shape
    T = shape[0]
    kp, kt, kh = _heads("k", k, dtype, shape, None, pages.kv_heads, dim)
    vp, vt, vh = _heads("v", v, dtype, v.shape, T, pages.kv_heads, dim)
    qp = qt = qh = op = ot = oh = heads = 0
    if q is not None:
        qp, qt, qh = _heads("q", q, dtype, q.shape, T, None, dim)
        heads = q.shape[1]
        if out is None:
            out = _out(ctx, q.shape, q, dtype)
            op, ot, oh = out.data_ptr(), heads * dim, dim
        else:
            op, ot, oh = _heads("out", out, dtype, out.shape, T, heads, dim)
    elif out is not None:
        raise ValueError("out without queries")
    a = _pack_append(qp, op, kp, vp, qt, qh, ot, oh, kt, kh, vt, vh, _int32("cu", cu),
                     0 if seqs is None else _int32("seqs", seqs, n), n, T, heads, 0)
    st = lib().cr_kv_append(ctx._h, pages._addr, layer, rotary._on(ctx), a)
    if st:
        ctx.check(st, "cr_kv_append")
    return out


_pack_read = struct.Struct("@5P4Q2I").pack    # cr_read_args


def kv_read(ctx: Context, pages: KVPages, layer: int, cu, seqs=None, start=None, tokens: Optional[int] = None, out=None):
    """Keys and values of cached tokens, [tokens, kv_heads, head_dim] each (cr_kv_read): entry i's are cu[i] .. cu[i+1]-1
    of them, and tokens start[i] .. of row seqs[i] (None: the row's last ones; row i).  ``tokens``: cu's last value, which
    is read from the GPU where neither it nor ``out`` (a pair of tensors) is given."""
    n = max(cu.numel() - 1, 0)
    heads, dim = pages.kv_heads, pages.head_dim
    if out is None:
        if tokens is None:
            tokens = int(cu[-1]) if n else 0
        T, kt, kh = tokens, heads * dim, dim
        k = _out(ctx, (T, heads, dim), pages.cache, pages.dtype)
        v = _out(ctx, (T, heads, dim), pages.cache, pages.dtype)
        kp, vp, vt, vh = k.data_ptr(), v.data_ptr(), kt, kh
    else:
        k, v = out
        if k.requires_grad or v.requires_grad:
            _no_gradient(k, v)
        kp, kt, kh = _heads("k", k, pages.dtype, k.shape, tokens, heads, dim)
        T = k.shape[0]
        vp, vt, vh = _heads("v", v, pages.dtype, v.shape, T, heads, dim)
    a = _pack_read(kp, vp, _int32("cu", cu), 0 if seqs is None else _int32("seqs", seqs, n),
                   0 if start is None else _int32("start", start, n), kt, kh, vt, vh, n, T)
    st = lib().cr_kv_read(ctx._h, pages._addr, layer, a)
    if st:
        ctx.check(st, "cr_kv_read")
    return k, v


_pack_attn = struct.Struct("@5P4IfI4Q").pack  # cr_attn_args


def _attn_args(ctx: Context, q, dtype, shape, dim, n, cu, seqs, causal, scale, out, lse):
    """cr_attn_args as bytes, and the outputs; ``shape``: q.shape, ``cu``: address or 0."""
    if q.requires_grad:
        _no_gradient(q)
    qp, qt, qh = _heads("q", q, dtype, shape, None, None, dim)
    T, heads, dim = shape
    if out is None:
        if ctx._raw_stream == _torch._C._cuda_getCurrentRawStream(ctx.device):
            out = _torch.empty_like(q, memory_format=_torch.contiguous_format)
        else:
            out = _out(ctx, shape, q, dtype)
        op, ot, oh = out.data_ptr(), heads * dim, dim
    else:
        op, ot, oh = _heads("out", out, dtype, out.shape, T, heads, dim)
    lp = 0
    if lse is not None and lse is not False:
        if lse is True:
            lse = _out(ctx, (T, heads), q, _torch.float32)
        _need_cuda("lse", lse, _torch.float32)
        if tuple(lse.shape) != (T, heads):
            raise ValueError(f"lse must have shape {(T, heads)}")
        lp = lse.data_ptr()
    a = _pack_attn(qp, op, lp, cu, 0 if seqs is None else _int32("seqs", seqs, n), n, T, heads, 1 if causal else 0,
                   dim ** -0.5 if scale is None else scale, 0, qt, qh, ot, oh)
    return a, out, lse


def attn_packed(ctx: Context, q, k, v, cu, cu_k=None, causal: bool = True, scale: Optional[float] = None, out=None,
                lse=None):
    """Attention over whole prompts packed back to back: q [tokens, heads, head_dim], k and v [tokens, kv_heads,
    head_dim]; sequence i's queries are cu[i] .. cu[i+1]-1, its keys cu_k[i] .. (None: the same) (cr_attn_packed).
    Returns the output, or (output, lse) with ``lse=True`` (or a tensor for it)."""
    n = max(cu.numel() - 1, 0)
    dtype, shape, kshape = q.dtype, q.shape, k.shape
    code = _codes.get(dtype)
    if code is None:
        code = _dtype_code(dtype)
    if len(shape) != 3 or len(kshape) != 3:
        raise ValueError("q and k must be [tokens, heads, head_dim]")
    if k.requires_grad or v.requires_grad:
        _no_gradient(k, v)
    S, heads, dim = kshape
    kp, kt, kh = _heads("k", k, dtype, kshape, None if cu_k is not None else shape[0], None, shape[2])
    vp, vt, vh = _heads("v", v, dtype, v.shape, S, heads, dim)
    a, out, lse = _attn_args(ctx, q, dtype, shape, dim, n, _int32("cu", cu), None, causal, scale, out, lse)
    st = lib().cr_attn_packed(ctx._h, a, code, heads, dim, kp, kt, kh, vp, vt, vh,
                              None if cu_k is None else _int32("cu_k", cu_k, n + 1), S)
    if st:
        ctx.check(st, "cr_attn_packed")
    return (out, lse) if lse is not None and lse is not False else out


def attn_paged(ctx: Context, q, pages: KVPages, layer: int, cu, seqs=None, causal: bool = True,
               scale: Optional[float] = None, out=None, lse=None):
    """Attention of every sequence's last tokens over its pages (cr_attn_paged): q [tokens, heads, head_dim], entry
    i's queries cu[i] .. cu[i+1]-1, its row seqs[i] (None: i).  Returns as ``attn_packed``."""
    a, out, lse = _attn_args(ctx, q, pages.dtype, q.shape, pages.head_dim, max(cu.numel() - 1, 0), _int32("cu", cu), seqs,
                             causal, scale, out, lse)
    st = lib().cr_attn_paged(ctx._h, pages._addr, layer, a)
    if st:
        ctx.check(st, "cr_attn_paged")
    return (out, lse) if lse is not None and lse is not False else out


def attn_decode(ctx: Context, q, pages: KVPages, layer: int, seqs=None, group_off=None, shared=None,
                scale: Optional[float] = None, out=None, lse=None):
    """Attention of one token per sequence, q [n, heads, head_dim], over its pages (cr_attn_decode).  Sequences
    group_off[g] .. group_off[g+1]-1 of the batch share their first shared[g] tokens' pages, which are read once for
    all of them.  Returns as ``attn_packed``."""
    ng = go = sh = 0
    if group_off is not None:
        if shared is None:
            raise ValueError("group_off without shared")
        ng = max(group_off.numel() - 1, 0)
        go, sh = _int32("group_off", group_off), _int32("shared", shared, ng)
    shape = q.shape
    a, out, lse = _attn_args(ctx, q, pages.dtype, shape, pages.head_dim, shape[0], 0, seqs, False, scale, out, lse)
    st = lib().cr_attn_decode(ctx._h, pages._addr, layer, a, go, sh, ng)
    if st:
        ctx.check(st, "cr_attn_decode")
    return (out, lse) if lse is not None and lse is not False else out
