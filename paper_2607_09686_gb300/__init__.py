"""GB300 routed-expert step of one MoE decoder layer (MawForge, arXiv 2607.09686), with the paged
attention, the sampling and the verification of drafts of a serving step around it.

Thin ctypes binding of ``libmawforge.so`` (declared in ``include/mawforge.h``).  Every
step of the path runs in the library's CUDA kernels; this module only marshals
arguments.  Device buffers may be given as torch CUDA tensors (anything with
``data_ptr()``) or as raw integer addresses; streams as ``torch.cuda.Stream`` objects,
raw handles, or ``None`` for torch's current stream.

There is no CPU fallback: importing this package fails if the library has not been built
(``python -c "import __graft_entry__ as g; g.build()"``).
"""
from __future__ import annotations

import ctypes
import os

__all__ = [
    "MFError", "Model", "PlanReq", "Plan", "Stats", "TunePoint", "Q8_0", "Q4_0", "LIB_PATH", "KERNEL_CLASSES",
    "mf_payload_bytes", "mf_plan", "mf_tune_cache", "mf_create", "mf_pack_put", "mf_load_pack", "mf_moe_forward",
    "mf_moe_forward_host", "mf_prefill_threshold", "mf_access_order", "mf_stats", "mf_reset", "mf_trace", "mf_timing", "mf_timing_read", "mf_check", "mf_wait_limit", "mf_test_hold", "mf_expert_ffn_noalloc",
    "mf_expert_ffn_noalloc_check", "mf_pack_save", "mf_create_from_file", "mf_pack_file_stats",
    "mf_pack_file_direct", "mf_destroy",
    "mf_strerror", "mf_last_cuda_error",
    "MF_F32", "MF_F16", "MF_BF16", "AttnShape", "KvCache", "Step", "Rope", "kv_cache", "step", "rope", "mf_kv_bytes",
    "mf_attn_create", "mf_kv_append", "mf_attn_forward", "mf_attn_check", "mf_attn_destroy", "mf_sample",
    "mf_sample_test_hold", "QkNorm", "Shared", "Cuts", "qk_norm", "shared", "cuts", "mf_kv_append_norm", "mf_attn_share",
    "mf_attn_forward_shared", "mf_verify_bytes", "mf_verify",
]

Q4_0 = 2
Q8_0 = 8
MF_F32, MF_F16, MF_BF16 = 0, 1, 30
MF_OK, MF_E_INVAL, MF_E_BUDGET, MF_E_OOM, MF_E_CUDA, MF_E_STATE, MF_E_TIMEOUT, MF_E_IO = 0, -1, -2, -3, -4, -5, -6, -7
KERNEL_CLASSES = ("router", "resolve", "materialize", "gateup_swiglu", "down_combine", "prefill_gemm", "ffn_fused")

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmawforge.so")
if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build the CUDA library first "
                      "(python -c 'import __graft_entry__ as g; g.build()')")
_lib = ctypes.CDLL(LIB_PATH)


class Model(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("hidden", ctypes.c_int32), ("n_experts", ctypes.c_int32),
                ("top_k", ctypes.c_int32), ("inter", ctypes.c_int32), ("qtype", ctypes.c_int32)]


class PlanReq(ctypes.Structure):
    _fields_ = [("cache_pct", ctypes.c_double), ("budget_bytes", ctypes.c_uint64), ("common_bytes", ctypes.c_uint64),
                ("kv_bytes", ctypes.c_uint64), ("max_tokens", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class Plan(ctypes.Structure):
    _fields_ = [("accepted", ctypes.c_int32), ("slots_per_layer", ctypes.c_int32),
                ("payload_bytes", ctypes.c_uint64), ("pool_bytes", ctypes.c_uint64),
                ("lower_bound_bytes", ctypes.c_uint64), ("overhead_bytes", ctypes.c_uint64),
                ("footprint_bytes", ctypes.c_uint64), ("max_tokens", ctypes.c_int32), ("reserved", ctypes.c_int32)]

    def as_dict(self) -> dict:
        return {name: getattr(self, name) for name, _ in self._fields_ if name != "reserved"}


class Stats(ctypes.Structure):
    _fields_ = [("accesses", ctypes.c_uint64), ("hits", ctypes.c_uint64), ("misses", ctypes.c_uint64),
                ("evictions", ctypes.c_uint64), ("bytes_materialized", ctypes.c_uint64)]

    def as_dict(self) -> dict:
        return {name: int(getattr(self, name)) for name, _ in self._fields_}


class TunePoint(ctypes.Structure):
    _fields_ = [("cache_pct", ctypes.c_double), ("accepted", ctypes.c_int32), ("slots_per_layer", ctypes.c_int32),
                ("pool_bytes", ctypes.c_uint64), ("footprint_bytes", ctypes.c_uint64), ("accesses", ctypes.c_uint64),
                ("hits", ctypes.c_uint64), ("misses", ctypes.c_uint64), ("bytes_materialized", ctypes.c_uint64),
                ("predicted_s", ctypes.c_double), ("predicted_tokens_per_s", ctypes.c_double)]

    def as_dict(self) -> dict:
        return {name: getattr(self, name) for name, _ in self._fields_}


class AttnShape(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class KvCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("page_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("n_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32)]
    kind = None  # kv heads, head_dim and type, where they are known (kv_cache)


class Step(ctypes.Structure):
    _fields_ = [("q_start", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("pages", ctypes.c_void_p),
                ("n_seqs", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("max_q", ctypes.c_int32),
                ("pages_per_seq", ctypes.c_int32)]


class Rope(ctypes.Structure):
    _fields_ = [("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("n_pos", ctypes.c_int32), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("n_axes", ctypes.c_int32), ("section", ctypes.c_int32 * 4)]
    tokens = None  # positions of each axis, where they are known (rope)


class _AppendArgs(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("q_out", ctypes.c_void_p),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
                ("q_out_stride", ctypes.c_int64)]


class _AttnArgs(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("out", ctypes.c_void_p), ("lse", ctypes.c_void_p),
                ("q_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64), ("scale", ctypes.c_float),
                ("window", ctypes.c_int32), ("causal", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class _SampleArgs(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("noise", ctypes.c_void_p), ("temperature", ctypes.c_void_p),
                ("top_p", ctypes.c_void_p), ("min_p", ctypes.c_void_p), ("top_k", ctypes.c_void_p),
                ("token", ctypes.c_void_p), ("logprob", ctypes.c_void_p), ("logits_stride", ctypes.c_int64),
                ("noise_stride", ctypes.c_int64), ("n_rows", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class QkNorm(ctypes.Structure):
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float), ("offset", ctypes.c_float),
                ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]
    dim = None  # head_dim of the weights, where it is known (qk_norm)


class Shared(ctypes.Structure):
    _fields_ = [("first", ctypes.c_void_p), ("len", ctypes.c_void_p), ("n_groups", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class Cuts(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_void_p), ("top_p", ctypes.c_void_p), ("min_p", ctypes.c_void_p), ("top_k", ctypes.c_void_p)]
    seqs = gpu = None  # sequences that all settings have, the GPU they are on (-1: several), where that is known (cuts)


class _VerifyArgs(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("draft_logits", ctypes.c_void_p), ("row_start", ctypes.c_void_p),
                ("tokens", ctypes.c_void_p), ("u", ctypes.c_void_p), ("noise", ctypes.c_void_p), ("cuts", Cuts), ("draft_cuts", Cuts),
                ("token", ctypes.c_void_p), ("accepted", ctypes.c_void_p), ("logprob", ctypes.c_void_p), ("work", ctypes.c_void_p),
                ("logits_stride", ctypes.c_int64), ("draft_stride", ctypes.c_int64), ("noise_stride", ctypes.c_int64),
                ("n_seqs", ctypes.c_int32), ("n_rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32)]


_vp, _i32, _u64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_uint64
_sig = {
    "mf_payload_bytes": (_i32, [ctypes.POINTER(Model), ctypes.POINTER(_u64)]),
    "mf_plan": (_i32, [ctypes.POINTER(Model), ctypes.POINTER(PlanReq), ctypes.POINTER(Plan)]),
    "mf_tune_cache": (_i32, [ctypes.POINTER(Model), ctypes.POINTER(PlanReq), _vp, _i32, _i32, _i32, ctypes.c_double,
                             ctypes.c_double, _vp, _i32, ctypes.POINTER(TunePoint), ctypes.POINTER(_i32)]),
    "mf_create": (_i32, [ctypes.POINTER(_vp), ctypes.POINTER(Model), ctypes.POINTER(Plan), _i32]),
    "mf_pack_put": (_i32, [_vp, _i32, _i32, _vp, _u64]),
    "mf_load_pack": (_i32, [ctypes.POINTER(_vp), ctypes.POINTER(Model), ctypes.POINTER(Plan), _vp, _i32]),
    "mf_moe_forward": (_i32, [_vp, _i32, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp]),
    "mf_moe_forward_host": (_i32, [_vp, _i32, _vp, _vp, _vp, _i32, _vp, _vp, _vp, _vp]),
    "mf_prefill_threshold": (_i32, [_vp, _i32]),
    "mf_access_order": (_i32, [_vp, _i32]),
    "mf_stats": (_i32, [_vp, _i32, ctypes.POINTER(Stats), _i32]),
    "mf_reset": (_i32, [_vp, _i32, _vp]),
    "mf_trace": (_i32, [_vp, _i32, _vp, _vp, _vp, _i32, ctypes.POINTER(_i32)]),
    "mf_timing": (_i32, [_vp, ctypes.c_uint]),
    "mf_timing_read": (_i32, [_vp, _vp, _vp]),
    "mf_check": (_i32, [_vp]),
    "mf_wait_limit": (_i32, [_vp, ctypes.c_double]),
    "mf_test_hold": (_i32, [_vp, _i32]),
    "mf_expert_ffn_noalloc": (_i32, [ctypes.POINTER(Model), _vp, _vp, _vp, _vp, _vp]),
    "mf_expert_ffn_noalloc_check": (_i32, []),
    "mf_pack_save": (_i32, [_vp, ctypes.c_char_p]),
    "mf_create_from_file": (_i32, [ctypes.POINTER(_vp), ctypes.POINTER(Model), ctypes.POINTER(Plan), ctypes.c_char_p,
                                   _i32]),
    "mf_pack_file_stats": (_i32, [_vp, ctypes.POINTER(_u64), ctypes.POINTER(_u64), ctypes.POINTER(ctypes.c_double)]),
    "mf_pack_file_direct": (_i32, [_vp]),
    "mf_destroy": (None, [_vp]),
    "mf_kv_bytes": (_i32, [ctypes.POINTER(AttnShape), _i32, ctypes.c_int64, _i32, ctypes.POINTER(_u64)]),
    "mf_attn_create": (_i32, [ctypes.POINTER(_vp), ctypes.POINTER(AttnShape), _i32, _i32, _i32]),
    "mf_kv_append": (_i32, [_vp, ctypes.POINTER(KvCache), ctypes.POINTER(Step), ctypes.POINTER(Rope),
                            ctypes.POINTER(_AppendArgs), _vp]),
    "mf_attn_forward": (_i32, [_vp, ctypes.POINTER(KvCache), ctypes.POINTER(Step), ctypes.POINTER(_AttnArgs), _vp]),
    "mf_attn_check": (_i32, [_vp]),
    "mf_attn_destroy": (None, [_vp]),
    "mf_sample": (_i32, [ctypes.POINTER(_SampleArgs), _vp]),
    "mf_sample_test_hold": (_i32, [_i32]),
    "mf_kv_append_norm": (_i32, [_vp, ctypes.POINTER(KvCache), ctypes.POINTER(Step), ctypes.POINTER(QkNorm), ctypes.POINTER(Rope),
                                 ctypes.POINTER(_AppendArgs), _vp]),
    "mf_attn_share": (_i32, [_vp, _i32]),
    "mf_attn_forward_shared": (_i32, [_vp, ctypes.POINTER(KvCache), ctypes.POINTER(Step), ctypes.POINTER(Shared),
                                      ctypes.POINTER(_AttnArgs), _vp]),
    "mf_verify_bytes": (_i32, [_i32, _i32, _i32, ctypes.POINTER(_u64)]),
    "mf_verify": (_i32, [ctypes.POINTER(_VerifyArgs), _vp]),
    "mf_strerror": (ctypes.c_char_p, [_i32]),
    "mf_last_cuda_error": (ctypes.c_char_p, []),
}
for _name, (_res, _args) in _sig.items():
    _f = getattr(_lib, _name)
    _f.restype, _f.argtypes = _res, _args


class MFError(RuntimeError):
    def __init__(self, status: int, where: str):
        msg = _lib.mf_strerror(status).decode()
        if status == MF_E_CUDA:
            msg += f" ({_lib.mf_last_cuda_error().decode()})"
        super().__init__(f"{where}: {msg} [{status}]")
        self.status = status


def _check(status: int, where: str) -> None:
    if status != MF_OK:
        raise MFError(status, where)


def _addr(buf):
    """Address of a buffer: None, an int, a torch tensor, or a numpy array."""
    if buf is None:
        return None
    if isinstance(buf, int):
        return buf
    if hasattr(buf, "data_ptr"):
        return buf.data_ptr()
    if hasattr(buf, "ctypes"):
        return buf.ctypes.data
    raise TypeError(f"cannot take the address of {type(buf).__name__}")


_raw_stream = None  # torch's current stream of a device as a handle, without making a Stream object


def _stream(stream):
    global _raw_stream
    if stream is None:
        if _raw_stream is None:
            import torch
            get, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
            if get is None or device is None:
                _raw_stream = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
            else:
                torch.cuda.current_stream()  # (initialises CUDA)
                _raw_stream = lambda: get(device())  # noqa: E731
        return _raw_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def mf_strerror(status: int) -> str:
    return _lib.mf_strerror(status).decode()


def mf_last_cuda_error() -> str:
    return _lib.mf_last_cuda_error().decode()


def mf_payload_bytes(model: Model) -> int:
    out = _u64()
    _check(_lib.mf_payload_bytes(ctypes.byref(model), ctypes.byref(out)), "mf_payload_bytes")
    return int(out.value)


def mf_plan(model: Model, req: PlanReq) -> Plan:
    """Static plan; a rejected plan is returned too (plan.accepted == 0), not raised."""
    out = Plan()
    rc = _lib.mf_plan(ctypes.byref(model), ctypes.byref(req), ctypes.byref(out))
    if rc not in (MF_OK, MF_E_BUDGET):
        _check(rc, "mf_plan")
    return out


def mf_tune_cache(model: Model, req: PlanReq, routes, T: int, t_token_s: float, t_miss_s: float, pcts,
                  order: int = 0):
    """Cache-size tuner (host only).  routes: int32 array [n_layers][n_tokens][top_k] (C order).
    Returns (list of per-candidate dicts, index of the best accepted candidate or -1)."""
    import numpy as np
    r = np.ascontiguousarray(routes, dtype=np.int32)
    if r.ndim != 3:
        raise ValueError("routes must be [n_layers][n_tokens][top_k]")
    n = len(pcts)
    cand = (ctypes.c_double * max(1, n))(*[float(p) for p in pcts])
    out = (TunePoint * max(1, n))()
    best = _i32(-1)
    rc = _lib.mf_tune_cache(ctypes.byref(model), ctypes.byref(req), r.ctypes.data, r.shape[1], T, order,
                            float(t_token_s), float(t_miss_s), cand, n, out, ctypes.byref(best))
    if rc not in (MF_OK, MF_E_BUDGET):
        _check(rc, "mf_tune_cache")
    return [out[i].as_dict() for i in range(n)], best.value


def mf_create(model: Model, plan: Plan, device: int = 0) -> int:
    h = _vp()
    _check(_lib.mf_create(ctypes.byref(h), ctypes.byref(model), ctypes.byref(plan), device), "mf_create")
    return h.value


def mf_pack_put(ctx: int, layer: int, expert: int, payload) -> None:
    n = payload.nbytes if hasattr(payload, "nbytes") else len(payload)
    _check(_lib.mf_pack_put(ctx, layer, expert, _addr(payload), n), "mf_pack_put")


def mf_pack_save(ctx: int, path: str) -> None:
    """Write the context's split-pack to a file (header, index, one record per payload)."""
    _check(_lib.mf_pack_save(ctx, os.fsencode(path)), "mf_pack_save")


def mf_create_from_file(model: Model, plan: Plan, path: str, device: int = 0) -> int:
    """A context whose split-pack is the file written by mf_pack_save (misses read from it)."""
    h = _vp()
    _check(_lib.mf_create_from_file(ctypes.byref(h), ctypes.byref(model), ctypes.byref(plan), os.fsencode(path),
                                    device), "mf_create_from_file")
    return h.value


def mf_pack_file_stats(ctx: int) -> dict:
    """{reads, bytes, seconds} of a file-backed context's reads so far."""
    r, b, t = _u64(), _u64(), ctypes.c_double()
    _check(_lib.mf_pack_file_stats(ctx, ctypes.byref(r), ctypes.byref(b), ctypes.byref(t)), "mf_pack_file_stats")
    return {"reads": int(r.value), "bytes": int(b.value), "seconds": float(t.value)}


def mf_pack_file_direct(ctx: int) -> bool:
    """True if the file-backed context reads its file unbuffered (O_DIRECT)."""
    rc = _lib.mf_pack_file_direct(ctx)
    if rc < 0:
        _check(rc, "mf_pack_file_direct")
    return rc == 1


def mf_load_pack(model: Model, plan: Plan, payloads, device: int = 0) -> int:
    """payloads: sequence of L*E host buffers (numpy uint8), layer-major."""
    arr = (_vp * len(payloads))(*[_addr(p) for p in payloads])
    h = _vp()
    _check(_lib.mf_load_pack(ctypes.byref(h), ctypes.byref(model), ctypes.byref(plan),
                             ctypes.cast(arr, _vp), device), "mf_load_pack")
    return h.value


def mf_moe_forward(ctx: int, layer: int, x, router_w, logit_bias, T: int, y, idx_out=None, w_out=None,
                   stream=None) -> None:
    _check(_lib.mf_moe_forward(ctx, layer, _addr(x), _addr(router_w), _addr(logit_bias), T, _addr(y),
                               _addr(idx_out), _addr(w_out), _stream(stream)), "mf_moe_forward")


def mf_moe_forward_host(ctx: int, layer: int, x, router_w, logit_bias, T: int, y, idx_out=None, w_out=None,
                        stream=None) -> None:
    _check(_lib.mf_moe_forward_host(ctx, layer, _addr(x), _addr(router_w), _addr(logit_bias), T, _addr(y),
                                    _addr(idx_out), _addr(w_out), _stream(stream)), "mf_moe_forward_host")


def mf_prefill_threshold(ctx: int, min_tokens: int) -> None:
    """Calls with T >= min_tokens use the tensor-core grouped GEMMs (0 = never)."""
    _check(_lib.mf_prefill_threshold(ctx, min_tokens), "mf_prefill_threshold")


MF_ORDER_FIRST_OCCURRENCE = 0
MF_ORDER_RESIDENT_FIRST = 1


def mf_access_order(ctx: int, order: int) -> None:
    """Order of a many-token call's accesses to the cache (MF_ORDER_*)."""
    _check(_lib.mf_access_order(ctx, order), "mf_access_order")


def mf_stats(ctx: int, layer: int = -1, reset: bool = False) -> dict:
    out = Stats()
    _check(_lib.mf_stats(ctx, layer, ctypes.byref(out), 1 if reset else 0), "mf_stats")
    return out.as_dict()


def mf_reset(ctx: int, slots_per_layer: int = 0, stream=None) -> None:
    _check(_lib.mf_reset(ctx, slots_per_layer, _stream(stream)), "mf_reset")


def mf_trace(ctx: int, layer: int, cap: int = 1024):
    """(experts, slots, hits) of the latest call of `layer`, as Python lists."""
    exp = (ctypes.c_int32 * cap)()
    slo = (ctypes.c_int32 * cap)()
    hit = (ctypes.c_uint8 * cap)()
    n = _i32()
    _check(_lib.mf_trace(ctx, layer, exp, slo, hit, cap, ctypes.byref(n)), "mf_trace")
    return list(exp[:n.value]), list(slo[:n.value]), [bool(v) for v in hit[:n.value]]


def mf_timing(ctx: int, classes=None) -> None:
    """Time the kernel classes named in `classes` (names from KERNEL_CLASSES; None = all, [] = off)."""
    if classes is None:
        mask = (1 << len(KERNEL_CLASSES)) - 1
    elif classes is False:
        mask = 0
    else:
        mask = 0
        for c in classes:
            mask |= 1 << KERNEL_CLASSES.index(c)
    _check(_lib.mf_timing(ctx, mask), "mf_timing")


def mf_timing_read(ctx: int) -> dict:
    """{kernel class: (summed ms, launches)} from the CUDA events of each launch."""
    ms = (ctypes.c_double * len(KERNEL_CLASSES))()
    n = (ctypes.c_int64 * len(KERNEL_CLASSES))()
    _check(_lib.mf_timing_read(ctx, ms, n), "mf_timing_read")
    return {KERNEL_CLASSES[i]: (float(ms[i]), int(n[i])) for i in range(len(KERNEL_CLASSES))}


def mf_check(ctx: int) -> int:
    """0, MF_E_TIMEOUT if a kernel of this context gave up a bounded wait, or MF_E_IO if a read of
    its split-pack file failed (returned, not raised)."""
    rc = _lib.mf_check(ctx)
    if rc not in (MF_OK, MF_E_TIMEOUT, MF_E_IO):
        _check(rc, "mf_check")
    return rc


def mf_wait_limit(ctx: int, seconds: float) -> None:
    """Time limit of every bounded wait inside the context's kernels."""
    _check(_lib.mf_wait_limit(ctx, float(seconds)), "mf_wait_limit")


def mf_test_hold(ctx: int, hold: int) -> None:
    """Test hold of the failure path: 1 = the one-token FFN's producer issues no copies."""
    _check(_lib.mf_test_hold(ctx, int(hold)), "mf_test_hold")


def mf_expert_ffn_noalloc_check() -> int:
    """0, or MF_E_TIMEOUT if a no-allocation call on the current device gave up a bounded wait since
    the last check (returned, not raised)."""
    rc = _lib.mf_expert_ffn_noalloc_check()
    if rc not in (MF_OK, MF_E_TIMEOUT):
        _check(rc, "mf_expert_ffn_noalloc_check")
    return rc


def mf_expert_ffn_noalloc(model: Model, experts, g, x, y, stream=None) -> None:
    """One-token expert FFN from caller-held expert slots, allocating nothing (see mawforge.h)."""
    _check(_lib.mf_expert_ffn_noalloc(ctypes.byref(model), _addr(experts), _addr(g), _addr(x), _addr(y),
                                      _stream(stream)), "mf_expert_ffn_noalloc")


def mf_destroy(ctx: int) -> None:
    if ctx:
        _lib.mf_destroy(ctx)


# ---- attention over a paged cache, and sampling (torch tensors; see mawforge.h for the layouts)

def mf_kv_bytes(shape: AttnShape, n_layers: int, n_tokens: int, page_size: int) -> int:
    """Cache bytes of one sequence over all layers, whole pages counted (PlanReq.kv_bytes per stream)."""
    out = _u64()
    _check(_lib.mf_kv_bytes(ctypes.byref(shape), n_layers, n_tokens, page_size, ctypes.byref(out)), "mf_kv_bytes")
    return int(out.value)


class _Types:
    """torch's types (torch is imported with the first call that takes tensors, not with this module)."""
    f32 = i32 = device = None
    codes: dict = {}
    of: dict = {}

    @classmethod
    def load(cls):
        import torch
        cls.f32, cls.i32, cls.device = torch.float32, torch.int32, torch.cuda.current_device
        cls.codes = {torch.float32: MF_F32, torch.float16: MF_F16, torch.bfloat16: MF_BF16}
        cls.of = {code: dtype for dtype, code in cls.codes.items()}


def _vector(t, dtype, n: int, where: str, device: int | None = None):
    """Address of n elements of a contiguous tensor that the GPU can reach, of `device` where that is given (None and plain addresses
    as they are)."""
    if t is None or isinstance(t, int):
        return t
    if t.dtype is not dtype or t.numel() < n or (n > 1 and not t.is_contiguous()) or \
            not ((t.is_cuda if device is None else t.get_device() == device) or t.is_pinned()):
        raise MFError(MF_E_INVAL, where)
    return t.data_ptr()


def kv_cache(k, v) -> KvCache:
    """Describe a layer's cache: k and v of shape [pages][lines][kv heads][head_dim] with the same strides, the
    last of them 1 (a page that holds its lines head by head is a transposed view)."""
    st = k.stride()
    if k.dim() != 4 or st != v.stride() or k.shape != v.shape or k.dtype != v.dtype or st[3] != 1:
        raise ValueError("k and v must be [pages][lines][heads][dim] of one dtype and stride, dim contiguous")
    _on_gpu(k, v)
    c = KvCache(k.data_ptr(), v.data_ptr(), st[0], st[1], st[2], k.shape[0], k.shape[1])
    c.held, c.kind = (k, v), (k.shape[2], k.shape[3], k.dtype)
    return c


def _on_gpu(*tensors) -> None:
    if not all(t.is_cuda or t.is_pinned() for t in tensors):
        raise ValueError("tensors must be on the GPU")


def _i32_tensor(t, name: str) -> None:
    if t is not None:
        if str(t.dtype) != "torch.int32" or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous int32 tensor")
        _on_gpu(t)


def step(q_start, kv_len, pages, n_tokens: int, max_q: int) -> Step:
    """Describe a step's sequences: q_start [n + 1] (None: one token each), kv_len [n], pages [n][pages a sequence],
    contiguous int32 tensors on the device."""
    for t, name in ((q_start, "q_start"), (kv_len, "kv_len"), (pages, "pages")):
        _i32_tensor(t, name)
    n = kv_len.shape[0]
    if pages.dim() != 2 or pages.shape[0] != n or (q_start is not None and q_start.shape[0] != n + 1):
        raise ValueError("q_start [n + 1], kv_len [n] and pages [n][...] must describe the same sequences")
    s = Step(_addr(q_start), kv_len.data_ptr(), pages.data_ptr(), n, n_tokens, max_q, pages.shape[1])
    s.held = (q_start, kv_len, pages)
    return s


def rope(cos, sin, pos=None, interleaved: bool = False, sections=None) -> Rope:
    """Describe the rotation: cos and sin float [positions][pairs]; pos int32 [axes][tokens] or None (the cache
    lines); sections: pairs of each axis."""
    if cos.shape != sin.shape or not (cos.is_contiguous() and sin.is_contiguous()) or \
            {str(cos.dtype), str(sin.dtype)} != {"torch.float32"}:
        raise ValueError("cos and sin must be contiguous float32 tensors of one shape")
    _on_gpu(cos, sin)
    _i32_tensor(pos, "pos")
    sections = tuple(sections) if sections is not None else (cos.shape[1],)
    axes = 1 if pos is None or pos.dim() == 1 else pos.shape[0]
    if len(sections) != axes or axes > 4:
        raise ValueError("one section for each of at most 4 axes")
    r = Rope(cos.data_ptr(), sin.data_ptr(), _addr(pos), cos.shape[0], 2 * cos.shape[1], int(interleaved), axes,
             (ctypes.c_int32 * 4)(*sections))
    r.held, r.tokens = (cos, sin, pos), None if pos is None else pos.shape[-1]
    return r


_attn_kinds: dict = {}  # by handle: query heads, kv heads, head_dim, type; the kind of its caches


def mf_attn_create(shape: AttnShape, max_seqs: int, max_tokens: int, device: int = 0) -> int:
    h = _vp()
    _check(_lib.mf_attn_create(ctypes.byref(h), ctypes.byref(shape), max_seqs, max_tokens, device), "mf_attn_create")
    if not _Types.codes:
        _Types.load()
    dtype = _Types.of[shape.dtype]
    _attn_kinds[h.value] = shape.n_heads, shape.n_kv_heads, shape.head_dim, dtype, (shape.n_kv_heads, shape.head_dim, dtype)
    return h.value


def _kind(attn: int, cache: KvCache, where: str):
    """What is known of a handle, which the cache has to fit."""
    kind = _attn_kinds.get(attn)
    if kind is None or (cache.kind != kind[4] and cache.kind is not None):
        raise MFError(MF_E_INVAL, where)
    return kind


def _rows(t, n: int, heads: int, dim: int, dtype, where: str):
    """(address, stride between tokens) of a [tokens][heads][head_dim] tensor of n tokens or more whose rows are contiguous."""
    try:
        (rows, h, d), (stride, head_stride, one) = t.shape, t.stride()
    except ValueError:  # not three dimensions
        raise MFError(MF_E_INVAL, where) from None
    if rows < n or h != heads or d != dim or one != 1 or (head_stride != d and h != 1) or t.dtype is not dtype or \
            not (t.is_cuda or t.is_pinned()):
        raise MFError(MF_E_INVAL, where)
    return t.data_ptr(), stride


def mf_kv_append(attn: int, cache: KvCache, step: Step, k, v, q=None, q_out=None, rope: Rope | None = None,
                 stream=None) -> None:
    """Rotate q (into q_out) and k by position, and store k and v into their lines of the cache.  q, q_out, k and v have
    the handle's heads and type and the step's tokens (or more rows, which are not touched)."""
    w = "mf_kv_append"
    a = _append_args(attn, cache, step, k, v, q, q_out, rope, w)
    rc = _lib.mf_kv_append(attn, cache, step, rope, a, _stream(stream))
    if rc:
        _check(rc, w)


def _append_args(attn, cache, step, k, v, q, q_out, rope, w: str) -> _AppendArgs:
    heads, kv_heads, dim, dtype, _ = _kind(attn, cache, w)
    n = step.n_tokens
    q_at, q_stride = _rows(q, n, heads, dim, dtype, w) if q is not None else (None, 0)
    o_at, o_stride = _rows(q_out, n, heads, dim, dtype, w) if q_out is not None else (None, 0)
    k_at, k_stride = _rows(k, n, kv_heads, dim, dtype, w)
    v_at, v_stride = _rows(v, n, kv_heads, dim, dtype, w)
    if rope is not None and rope.tokens is not None and (rope.tokens < n or (rope.n_axes > 1 and rope.tokens != n)):
        raise MFError(MF_E_INVAL, w)
    return _AppendArgs(q_at, k_at, v_at, o_at, q_stride, k_stride, v_stride, o_stride)


def qk_norm(q_weight, k_weight, eps: float, offset: float = 0.0) -> QkNorm:
    """Describe the norms of q and k: weights [head_dim], contiguous, both of one type (the handle's, or float32); None: that one is
    not normed."""
    given = [t for t in (q_weight, k_weight) if t is not None]
    if len({t.dtype for t in given}) > 1 or len({tuple(t.shape) for t in given}) > 1 or \
            any(t.dim() != 1 or not t.is_contiguous() for t in given):
        raise ValueError("weights must be contiguous [head_dim] tensors of one type")
    _on_gpu(*given)
    if not _Types.codes:
        _Types.load()
    if given and given[0].dtype not in _Types.codes:
        raise ValueError("weights must be float32, float16 or bfloat16")
    n = QkNorm(_addr(q_weight), _addr(k_weight), eps, offset, _Types.codes[given[0].dtype] if given else MF_F32, 0)
    n.held, n.dim = (q_weight, k_weight), given[0].shape[0] if given else None
    return n


def mf_kv_append_norm(attn: int, cache: KvCache, step: Step, norm: QkNorm, k, v, q=None, q_out=None, rope: Rope | None = None,
                      stream=None) -> None:
    """mf_kv_append with the norms of q and k, head by head, before the rotation."""
    w = "mf_kv_append_norm"
    a = _append_args(attn, cache, step, k, v, q, q_out, rope, w)
    if norm.dim is not None and norm.dim != _attn_kinds[attn][2]:
        raise MFError(MF_E_INVAL, w)
    rc = _lib.mf_kv_append_norm(attn, cache, step, norm, rope, a, _stream(stream))
    if rc:
        _check(rc, w)


def mf_attn_forward(attn: int, cache: KvCache, step: Step, q, out, lse=None, scale: float = 1.0, window: int = 0,
                    causal: bool = True, stream=None) -> None:
    """Attention of the step's tokens over the cache.  q and out as in mf_kv_append, lse contiguous float32 with an element for
    each token and head at least."""
    w = "mf_attn_forward"
    heads, _, dim, dtype, _ = _kind(attn, cache, w)
    n = step.n_tokens
    q_at, q_stride = _rows(q, n, heads, dim, dtype, w)
    o_at, o_stride = _rows(out, n, heads, dim, dtype, w)
    a = _AttnArgs(q_at, o_at, _vector(lse, _Types.f32, n * heads, w), q_stride, o_stride, scale, window, causal, 0)
    rc = _lib.mf_attn_forward(attn, cache, step, a, _stream(stream))
    if rc:
        _check(rc, w)


def mf_attn_share(attn: int, max_groups: int) -> None:
    """Make the handle ready for mf_attn_forward_shared with at most max_groups groups."""
    _check(_lib.mf_attn_share(attn, max_groups), "mf_attn_share")


def shared(first, lens) -> Shared:
    """Describe groups of sequences that share their first lines: first [groups + 1] (where each begins), lens [groups], contiguous
    int32 tensors on the device."""
    for t, name in ((first, "first"), (lens, "lens")):
        _i32_tensor(t, name)
    if first.dim() != 1 or lens.dim() != 1 or first.shape[0] != lens.shape[0] + 1:
        raise ValueError("first [groups + 1] and lens [groups] must describe the same groups")
    s = Shared(first.data_ptr(), lens.data_ptr(), lens.shape[0], 0)
    s.held = (first, lens)
    return s


def mf_attn_forward_shared(attn: int, cache: KvCache, step: Step, shared: Shared, q, out, lse=None, scale: float = 1.0,
                           causal: bool = True, stream=None) -> None:
    """mf_attn_forward for sequences that share their first lines, which are read once for a group."""
    w = "mf_attn_forward_shared"
    heads, _, dim, dtype, _ = _kind(attn, cache, w)
    n = step.n_tokens
    q_at, q_stride = _rows(q, n, heads, dim, dtype, w)
    o_at, o_stride = _rows(out, n, heads, dim, dtype, w)
    a = _AttnArgs(q_at, o_at, _vector(lse, _Types.f32, n * heads, w), q_stride, o_stride, scale, 0, causal, 0)
    rc = _lib.mf_attn_forward_shared(attn, cache, step, shared, a, _stream(stream))
    if rc:
        _check(rc, w)


def mf_attn_check(attn: int) -> int:
    """0, MF_E_TIMEOUT, or MF_E_INVAL for a length, page or position out of range (returned, not raised)."""
    rc = _lib.mf_attn_check(attn)
    if rc not in (MF_OK, MF_E_TIMEOUT, MF_E_INVAL):
        _check(rc, "mf_attn_check")
    return rc


def mf_attn_destroy(attn: int) -> None:
    if attn:
        _attn_kinds.pop(attn, None)
        _lib.mf_attn_destroy(attn)


def mf_sample(logits, noise, token, logprob=None, temperature=None, top_k=None, top_p=None, min_p=None,
              stream=None) -> None:
    """One token from each row of logits [rows][vocab], with Gumbel noise of the same shape (see mawforge.h).  noise,
    temperature, top_p, min_p and logprob are float32, top_k and token int32; all but logits and noise contiguous, with an
    element for each row at least."""
    w = "mf_sample"
    if not _Types.codes:
        _Types.load()
    f32, i32, shape, dtype = _Types.f32, _Types.i32, logits.shape, _Types.codes.get(logits.dtype)
    if dtype is None or len(shape) != 2 or noise.shape != shape or noise.dtype is not f32:
        raise MFError(MF_E_INVAL, w)
    ls, ns, n = logits.stride(), noise.stride(), shape[0]
    if ls[1] != 1 or ns[1] != 1 or not ((logits.is_cuda or logits.is_pinned()) and (noise.is_cuda or noise.is_pinned())):
        raise MFError(MF_E_INVAL, w)
    a = _SampleArgs(logits.data_ptr(), noise.data_ptr(), _vector(temperature, f32, n, w), _vector(top_p, f32, n, w),
                    _vector(min_p, f32, n, w), _vector(top_k, i32, n, w), _vector(token, i32, n, w), _vector(logprob, f32, n, w),
                    ls[0], ns[0], n, shape[1], dtype, 0)
    rc = _lib.mf_sample(a, _stream(stream))
    if rc:
        _check(rc, w)


def mf_sample_test_hold(hold: int) -> None:
    """1: sampling issues none of the copies its blocks wait for (a second at most), for tests; 0: as usual."""
    _check(_lib.mf_sample_test_hold(hold), "mf_sample_test_hold")


def cuts(temperature=None, top_k=None, top_p=None, min_p=None) -> Cuts:
    """Describe the settings of sequences' rows: float32 tensors, top_k int32, contiguous, with an element for each sequence."""
    if not _Types.codes:
        _Types.load()
    given = [t for t in (temperature, top_k, top_p, min_p) if t is not None]
    for t in given:
        if t.dim() != 1 or not t.is_contiguous() or t.dtype is not (_Types.i32 if t is top_k else _Types.f32):
            raise ValueError("settings must be contiguous vectors, float32 (top_k int32)")
    _on_gpu(*given)
    c = Cuts(_addr(temperature), _addr(top_p), _addr(min_p), _addr(top_k))
    c.held, c.seqs = (temperature, top_k, top_p, min_p), min((t.shape[0] for t in given), default=None)
    gpus = {t.get_device() for t in given if t.is_cuda}
    c.gpu = (gpus.pop() if len(gpus) == 1 else -1) if gpus else None
    return c


def mf_verify_bytes(n_seqs: int, n_rows: int, vocab: int) -> int:
    """Bytes of the workspace of mf_verify calls of at most these sizes."""
    out = _u64()
    _check(_lib.mf_verify_bytes(n_seqs, n_rows, vocab, ctypes.byref(out)), "mf_verify_bytes")
    return int(out.value)


_NO_CUTS = Cuts()


def mf_verify(logits, row_start, tokens, u, noise, token, accepted, work, logprob=None, cuts: Cuts | None = None, draft_logits=None,
              draft_cuts: Cuts | None = None, stream=None) -> None:
    """Drafted tokens taken or refused, and the token that ends each sequence (see mawforge.h).  All tensors are on the current
    device (or pinned), the settings' too: logits and draft_logits [rows][vocab] of one type, noise float32 [sequences][vocab], u and
    logprob float32, row_start, tokens, token and accepted int32, work uint8."""
    w = "mf_verify"
    if not _Types.codes:
        _Types.load()
    f32, i32, dtype = _Types.f32, _Types.i32, _Types.codes.get(logits.dtype)
    if dtype is None or logits.dim() != 2 or noise.dim() != 2 or noise.dtype is not f32 or noise.shape[1] != logits.shape[1]:
        raise MFError(MF_E_INVAL, w)
    (n, vocab), seqs = logits.shape, noise.shape[0]
    if not (logits.is_cuda or logits.is_pinned()):
        raise MFError(MF_E_INVAL, w)
    here = _Types.device()
    draft, draft_stride = None, 0
    if draft_logits is not None:
        if draft_logits.dtype is not logits.dtype or draft_logits.shape != logits.shape or draft_logits.stride(1) != 1 or \
                not (draft_logits.get_device() == here or draft_logits.is_pinned()):
            raise MFError(MF_E_INVAL, w)
        draft, draft_stride = draft_logits.data_ptr(), draft_logits.stride(0)
    ls, ns = logits.stride(), noise.stride()
    if ls[1] != 1 or ns[1] != 1 or not (logits.get_device() == here or logits.is_pinned()) or \
            not (noise.get_device() == here or noise.is_pinned()):
        raise MFError(MF_E_INVAL, w)
    cuts, draft_cuts = cuts or _NO_CUTS, draft_cuts or _NO_CUTS
    if cuts.gpu not in (None, here) or draft_cuts.gpu not in (None, here):
        raise MFError(MF_E_INVAL, w)
    need = _u64()
    if any(c.seqs is not None and c.seqs < seqs for c in (cuts, draft_cuts)) or \
            _lib.mf_verify_bytes(seqs, n, vocab, ctypes.byref(need)) or work.numel() * work.element_size() < need.value or \
            not work.is_contiguous() or work.get_device() != here:
        raise MFError(MF_E_INVAL, w)
    a = _VerifyArgs(logits.data_ptr(), draft, _vector(row_start, i32, seqs + 1, w, here), _vector(tokens, i32, n, w, here),
                    _vector(u, f32, n, w, here), noise.data_ptr(), cuts, draft_cuts, _vector(token, i32, n, w, here),
                    _vector(accepted, i32, seqs, w, here), _vector(logprob, f32, n, w, here), work.data_ptr(), ls[0], draft_stride, ns[0],
                    seqs, n, vocab, dtype)
    rc = _lib.mf_verify(a, _stream(stream))
    if rc:
        _check(rc, w)
