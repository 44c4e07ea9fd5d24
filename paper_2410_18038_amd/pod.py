"""Thin ctypes binding over ``libpod_attn.so`` (argument marshalling only).

Function names mirror the C ABI in ``include/pod_attn.h``.  Torch is used for device
memory and streams; every step of the attention path runs in the library's HIP kernels.
There is no fallback: if the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import dataclasses
import functools
import os
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpod_attn.so")

POD_OK = 0
F16, BF16 = 0, 1
MODE_FUSED, MODE_SERIAL, MODE_STREAMS, MODE_PREFILL_ONLY, MODE_DECODE_ONLY = range(5)
MODE_FLAG_NO_COMBINE = 0x100
MODE_FLAG_CTA_PARALLEL = 0x200
MODE_FLAG_PREFILL_HEAVY = 0x400
MODES = {"fused": MODE_FUSED, "serial": MODE_SERIAL, "streams": MODE_STREAMS,
         "prefill_only": MODE_PREFILL_ONLY, "decode_only": MODE_DECODE_ONLY,
         "fused_cta": MODE_FUSED | MODE_FLAG_CTA_PARALLEL,
         "fused_heavy": MODE_FUSED | MODE_FLAG_PREFILL_HEAVY,
         "prefill_only_heavy": MODE_PREFILL_ONLY | MODE_FLAG_PREFILL_HEAVY,
         "decode_only_lite": MODE_DECODE_ONLY | MODE_FLAG_PREFILL_HEAVY}
POLICY_AUTO, POLICY_ALTERNATE, POLICY_PROPORTIONAL = 0, 1, 2
KV_TOKEN_MAJOR, KV_HEAD_MAJOR = 0, 1

EXPORTS = ["pod_attn_plan_create", "pod_attn_plan_create_scored", "pod_attn_plan_destroy", "pod_attn_plan_info_get",
           "pod_attn_workspace_size", "pod_attn_plan_set_trace", "pod_attn_plan_set_event_log",
           "pod_attn_plan_upload", "pod_attn_forward", "pod_attn_forward_static",
           "pod_attn_build_tables", "pod_attn_rope_table", "pod_attn_append",
           "pod_attn_role_for_ticket", "pod_attn_simulate_launch", "pod_attn_plan_prefill_item", "pod_attn_plan_prefill_item_of_workgroup", "pod_attn_plan_decode_unit",
           "pod_attn_plan_decode_queue",
           "pod_attn_probe_hbm_read", "pod_attn_probe_mfma", "pod_attn_probe_issue", "pod_attn_probe_colocation",
           "pod_attn_last_error", "pod_attn_version"]


class PodError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"pod_attn status {status}: {message}")
        self.status = status


class Params(ctypes.Structure):
    _fields_ = [("n_prefill", ctypes.c_int32), ("n_decode", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("block_size", ctypes.c_int32),
                ("max_blocks_per_seq", ctypes.c_int32), ("n_cache_rows", ctypes.c_int32),
                ("n_blocks", ctypes.c_int32), ("kv_seq_stride", ctypes.c_int64),
                ("policy", ctypes.c_int32), ("max_prefill_waves", ctypes.c_int32),
                ("decode_chunk", ctypes.c_int32), ("prefill_split_len", ctypes.c_int32),
                ("n_compute_units", ctypes.c_int32), ("kv_order", ctypes.c_int32)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("n_prefill_items", ctypes.c_int32), ("n_decode_units", ctypes.c_int32),
                ("n_combine", ctypes.c_int32), ("max_prefill_splits", ctypes.c_int32),
                ("max_decode_splits", ctypes.c_int32), ("decode_chunk", ctypes.c_int32),
                ("prefill_ratio", ctypes.c_int32), ("decode_ratio", ctypes.c_int32),
                ("fused_grid", ctypes.c_int32), ("n_compute_units", ctypes.c_int32),
                ("n_prefill_rows", ctypes.c_int64), ("n_partial_rows", ctypes.c_int64),
                ("workspace_bytes", ctypes.c_int64), ("prefill_heavy_advised", ctypes.c_int32),
                ("prefill_heavy_chosen", ctypes.c_int32)]


class ScoresParams(ctypes.Structure):
    _fields_ = [("logit_cap", ctypes.c_float), ("window", ctypes.c_int32), ("slopes", ctypes.POINTER(ctypes.c_float)),
                ("doc_start", ctypes.POINTER(ctypes.c_int32)), ("prefix_len", ctypes.POINTER(ctypes.c_int32))]


class RopeParams(ctypes.Structure):
    _fields_ = [("layout", ctypes.c_int32), ("scaling", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
                ("cos_sin_scale", ctypes.c_float), ("theta", ctypes.c_double), ("factor", ctypes.c_double),
                ("trained_len", ctypes.c_double), ("low", ctypes.c_double), ("high", ctypes.c_double)]


class HeadNormParams(ctypes.Structure):
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float),
                ("weight_offset", ctypes.c_float), ("normalise_q", ctypes.c_int32), ("normalise_k", ctypes.c_int32)]


_lib = None


def lib():
    """The loaded C library; raises if it has not been built (no CPU fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2410_18038_amd.build` "
                "(hipcc, gfx950). This package has no fallback path.")
        # The library must share torch's HIP runtime (streams, events and device memory are torch's):
        # torch bundles its own libamdhip64 under the same soname, so it has to be loaded first.
        import torch
        bundled = os.path.join(os.path.dirname(torch.__file__), "lib", "libamdhip64.so")
        if os.path.exists(bundled):
            ctypes.CDLL(bundled, mode=ctypes.RTLD_GLOBAL)
        L = ctypes.CDLL(LIB_PATH)
        vp, i32p = ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32)
        L.pod_attn_plan_create.restype = ctypes.c_int
        L.pod_attn_plan_create.argtypes = [ctypes.POINTER(Params), i32p, ctypes.POINTER(vp)]
        L.pod_attn_plan_create_scored.restype = ctypes.c_int
        L.pod_attn_plan_create_scored.argtypes = [ctypes.POINTER(Params), ctypes.POINTER(ScoresParams), i32p, ctypes.POINTER(vp)]
        L.pod_attn_plan_destroy.restype = None
        L.pod_attn_plan_destroy.argtypes = [vp]
        L.pod_attn_plan_info_get.restype = ctypes.c_int
        L.pod_attn_plan_info_get.argtypes = [vp, ctypes.POINTER(PlanInfo)]
        L.pod_attn_plan_set_trace.restype = ctypes.c_int
        L.pod_attn_plan_set_trace.argtypes = [vp, vp, ctypes.c_size_t]
        L.pod_attn_plan_set_event_log.restype = ctypes.c_int
        L.pod_attn_plan_set_event_log.argtypes = [vp, vp, ctypes.c_size_t]
        L.pod_attn_workspace_size.restype = ctypes.c_size_t
        L.pod_attn_workspace_size.argtypes = [vp]
        L.pod_attn_plan_upload.restype = ctypes.c_int
        L.pod_attn_plan_upload.argtypes = [vp, vp, ctypes.c_size_t, vp]
        L.pod_attn_forward.restype = ctypes.c_int
        L.pod_attn_forward.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t,
                                       ctypes.c_int32, vp]
        L.pod_attn_forward_static.restype = ctypes.c_int
        L.pod_attn_forward_static.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int32, vp]
        L.pod_attn_build_tables.restype = ctypes.c_int
        L.pod_attn_build_tables.argtypes = [ctypes.POINTER(Params), vp, vp, ctypes.c_int32, vp, ctypes.c_int32, vp, vp, vp, vp]
        L.pod_attn_rope_table.restype = ctypes.c_int
        L.pod_attn_rope_table.argtypes = [ctypes.POINTER(RopeParams), ctypes.POINTER(ctypes.c_uint64)]
        L.pod_attn_append.restype = ctypes.c_int
        L.pod_attn_append.argtypes = [ctypes.POINTER(Params), ctypes.POINTER(RopeParams), vp, ctypes.POINTER(HeadNormParams),
                                      vp, ctypes.c_int64, vp, ctypes.c_int64, vp, ctypes.c_int64, vp, vp, ctypes.c_int32,
                                      vp, vp, vp, vp]
        L.pod_attn_role_for_ticket.restype = ctypes.c_int32
        L.pod_attn_role_for_ticket.argtypes = [ctypes.c_int32] * 4
        L.pod_attn_simulate_launch.restype = ctypes.c_int32
        L.pod_attn_simulate_launch.argtypes = [vp, i32p, ctypes.c_int32, i32p, ctypes.c_int32, i32p, i32p, i32p, i32p]
        L.pod_attn_plan_prefill_item.restype = ctypes.c_int
        L.pod_attn_plan_prefill_item.argtypes = [vp, ctypes.c_int32, i32p]
        L.pod_attn_plan_prefill_item_of_workgroup.restype = ctypes.c_int
        L.pod_attn_plan_prefill_item_of_workgroup.argtypes = [vp, ctypes.c_int32, i32p]
        L.pod_attn_plan_decode_unit.restype = ctypes.c_int
        L.pod_attn_plan_decode_unit.argtypes = [vp, ctypes.c_int32, i32p]
        L.pod_attn_plan_decode_queue.restype = ctypes.c_int
        L.pod_attn_plan_decode_queue.argtypes = [vp, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32),
                                                 ctypes.POINTER(ctypes.c_int32)]
        L.pod_attn_probe_hbm_read.restype = ctypes.c_int
        L.pod_attn_probe_hbm_read.argtypes = [vp, ctypes.c_size_t, vp, vp]
        L.pod_attn_probe_mfma.restype = ctypes.c_int
        L.pod_attn_probe_mfma.argtypes = [ctypes.c_int32, vp, ctypes.POINTER(ctypes.c_double), vp]
        L.pod_attn_probe_issue.restype = ctypes.c_int
        L.pod_attn_probe_issue.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp,
                                           ctypes.POINTER(ctypes.c_double), vp]
        L.pod_attn_probe_colocation.restype = ctypes.c_int
        L.pod_attn_probe_colocation.argtypes = [ctypes.c_int32, vp, vp, vp, ctypes.c_size_t, ctypes.c_int32,
                                                ctypes.c_int32, ctypes.c_int32, vp, vp, vp]
        L.pod_attn_last_error.restype = ctypes.c_char_p
        L.pod_attn_version.restype = ctypes.c_char_p
        _lib = L
    return _lib


def pod_attn_last_error() -> str:
    return lib().pod_attn_last_error().decode()


def pod_attn_version() -> str:
    return lib().pod_attn_version().decode()


def _check(status: int):
    if status != POD_OK:
        raise PodError(status, pod_attn_last_error())


def _i32(a):
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


class Plan:
    """Owner of one ``pod_attn_plan`` handle."""

    def __init__(self, handle: int, params: Params):
        self.handle = ctypes.c_void_p(handle)
        self.params = params

    def close(self):
        if self.handle:
            lib().pod_attn_plan_destroy(self.handle)
            self.handle = ctypes.c_void_p(None)

    def __del__(self):  # pragma: no cover - best effort
        try:
            self.close()
        except Exception:
            pass

    def info(self) -> PlanInfo:
        return pod_attn_plan_info_get(self)

    def prefill_items(self) -> np.ndarray:
        n = self.info().n_prefill_items
        return np.array([pod_attn_plan_prefill_item(self, i) for i in range(n)], dtype=np.int32).reshape(n, 8)

    def prefill_items_by_workgroup(self) -> np.ndarray:
        n = self.info().n_prefill_items
        return np.array([pod_attn_plan_prefill_item_of_workgroup(self, i) for i in range(n)], dtype=np.int32).reshape(n, 8)

    def decode_units(self) -> np.ndarray:
        n = self.info().n_decode_units
        return np.array([pod_attn_plan_decode_unit(self, i) for i in range(n)], dtype=np.int32).reshape(n, 8)

    def decode_queues(self) -> list:
        """[(begin, end)] of the 8 per-XCD decode queues; units before the first begin are fixed."""
        return [pod_attn_plan_decode_queue(self, q) for q in range(8)]


def make_params(*, n_prefill, n_decode, n_q_heads, n_kv_heads, head_dim, dtype, softmax_scale,
                block_size=0, max_blocks_per_seq=0, n_cache_rows=1, n_blocks=0, kv_seq_stride=0,
                policy=POLICY_AUTO, max_prefill_waves=0, decode_chunk=0, prefill_split_len=0,
                n_compute_units=0, kv_order=KV_TOKEN_MAJOR) -> Params:
    return Params(n_prefill, n_decode, n_q_heads, n_kv_heads, head_dim, dtype, softmax_scale,
                  block_size, max_blocks_per_seq, n_cache_rows, n_blocks, kv_seq_stride, policy,
                  max_prefill_waves, decode_chunk, prefill_split_len, n_compute_units, kv_order)


def pod_attn_plan_create(params: Params, seq_meta_host) -> Plan:
    meta, meta_p = _i32(np.asarray(seq_meta_host).reshape(-1, 4))
    handle = ctypes.c_void_p()
    _check(lib().pod_attn_plan_create(ctypes.byref(params), meta_p, ctypes.byref(handle)))
    return Plan(handle.value, params)


@dataclasses.dataclass
class Scores:
    """Scores other than plain causal ones (``pod_attn_scores``): capped by ``logit_cap * tanh(s / logit_cap)``, less
    ``slopes[head]`` times the distance to the key, and masked by a sliding ``window``, by the first key of each row's
    document (``doc_start``, one per output row) and by prefixes that are seen from everywhere in their request
    (``prefix_len``, one per request)."""
    logit_cap: float = 0.0
    window: int = 0
    slopes: Optional[Sequence[float]] = None
    doc_start: Optional[Sequence[int]] = None
    prefix_len: Optional[Sequence[int]] = None


def pod_attn_plan_create_scored(params: Params, scores: Optional[Scores], seq_meta_host) -> Plan:
    meta, meta_p = _i32(np.asarray(seq_meta_host).reshape(-1, 4))
    handle = ctypes.c_void_p()
    if scores is None:
        _check(lib().pod_attn_plan_create_scored(ctypes.byref(params), None, meta_p, ctypes.byref(handle)))
        return Plan(handle.value, params)
    if not -2**31 <= scores.window < 2**31:
        raise ValueError(f"window {scores.window} does not fit in 32 bits")
    if scores.logit_cap > 0 and not np.float32(scores.logit_cap) > 0:
        raise ValueError(f"logit_cap {scores.logit_cap} is 0 in 32 bits")
    n_rows = int(meta[:params.n_prefill, 1].clip(min=0).sum()) + params.n_decode
    kept, ptr = [], {}
    for name, size, dtype, ctype in (("slopes", params.n_q_heads, np.float32, ctypes.c_float),
                                     ("doc_start", n_rows, np.int32, ctypes.c_int32),
                                     ("prefix_len", meta.shape[0], np.int32, ctypes.c_int32)):
        value = getattr(scores, name)
        if value is None:
            continue
        given = np.asarray(value)
        with np.errstate(invalid="ignore", over="ignore"):
            a = np.ascontiguousarray(given, dtype=dtype)
        if a.shape != (size,):
            raise ValueError(f"{name} must hold {size} values, not {a.shape}")
        if dtype == np.int32 and not (a == given).all():                     # (numpy wraps and truncates without a word)
            raise ValueError(f"{name} holds values that are no 32-bit integers")
        kept.append(a)
        ptr[name] = a.ctypes.data_as(ctypes.POINTER(ctype))
    raw = ScoresParams(scores.logit_cap, scores.window, ptr.get("slopes"), ptr.get("doc_start"), ptr.get("prefix_len"))
    _check(lib().pod_attn_plan_create_scored(ctypes.byref(params), ctypes.byref(raw), meta_p, ctypes.byref(handle)))
    return Plan(handle.value, params)


def pod_attn_plan_destroy(plan: Plan):
    plan.close()


def pod_attn_plan_info_get(plan: Plan) -> PlanInfo:
    info = PlanInfo()
    _check(lib().pod_attn_plan_info_get(plan.handle, ctypes.byref(info)))
    return info


def pod_attn_plan_set_trace(plan: Plan, trace_ptr: int, trace_bytes: int):
    _check(lib().pod_attn_plan_set_trace(plan.handle, ctypes.c_void_p(trace_ptr), trace_bytes))


def pod_attn_plan_set_event_log(plan: Plan, log_ptr: int, log_bytes: int):
    _check(lib().pod_attn_plan_set_event_log(plan.handle, ctypes.c_void_p(log_ptr), log_bytes))


EVENT_DTYPE = np.dtype([("kind", np.int32), ("item", np.int32), ("cu", np.int32), ("wg", np.int32),
                        ("t_begin", np.uint64), ("t_end", np.uint64)])
TRACE_DTYPE = np.dtype([("cu", np.int32), ("first_role", np.int32), ("n_first", np.int32), ("n_second", np.int32),
                        ("t_begin", np.uint64), ("t_switch", np.uint64), ("t_end", np.uint64), ("pad", np.uint64)])


def pod_attn_workspace_size(plan: Plan) -> int:
    return int(lib().pod_attn_workspace_size(plan.handle))


def pod_attn_plan_prefill_item_of_workgroup(plan: Plan, workgroup: int):
    out = (ctypes.c_int32 * 8)()
    _check(lib().pod_attn_plan_prefill_item_of_workgroup(plan.handle, workgroup, out))
    return list(out)


def pod_attn_plan_prefill_item(plan: Plan, index: int):
    out = (ctypes.c_int32 * 8)()
    _check(lib().pod_attn_plan_prefill_item(plan.handle, index, out))
    return list(out)


def pod_attn_plan_decode_unit(plan: Plan, index: int):
    out = (ctypes.c_int32 * 8)()
    _check(lib().pod_attn_plan_decode_unit(plan.handle, index, out))
    return list(out)


def pod_attn_plan_decode_queue(plan: Plan, q: int):
    b, e = ctypes.c_int32(), ctypes.c_int32()
    _check(lib().pod_attn_plan_decode_queue(plan.handle, q, ctypes.byref(b), ctypes.byref(e)))
    return int(b.value), int(e.value)


def pod_attn_plan_upload(plan: Plan, workspace_ptr: int, workspace_bytes: int, stream: int = 0):
    _check(lib().pod_attn_plan_upload(plan.handle, ctypes.c_void_p(workspace_ptr), workspace_bytes,
                                      ctypes.c_void_p(stream)))


def pod_attn_forward(prefill_q: int, decode_q: int, k_cache: int, v_cache: int, seq_meta: int,
                     block_table: int, out: int, plan: Plan, workspace: int, workspace_bytes: int,
                     mode: int = MODE_FUSED, stream: int = 0):
    """All tensor arguments are raw device addresses (``tensor.data_ptr()``), 0 for NULL."""
    vp = ctypes.c_void_p
    _check(lib().pod_attn_forward(vp(prefill_q), vp(decode_q), vp(k_cache), vp(v_cache), vp(seq_meta),
                                  vp(block_table), vp(out), plan.handle, vp(workspace), workspace_bytes,
                                  mode, vp(stream)))


def pod_attn_build_tables(params: Params, seq_meta: int, free_blocks: int, n_free: int, block_table: int, n_rows: int,
                          slots: int, positions: int, report: int, stream: int = 0):
    """Blocks, slots and positions of a batch's new tokens; all tensor arguments are raw device addresses."""
    _check(lib().pod_attn_build_tables(ctypes.byref(params), seq_meta, free_blocks, n_free, block_table, n_rows, slots,
                                       positions, report, stream))


def pod_attn_rope_table(rope: RopeParams) -> np.ndarray:
    """uint64 [rot_dim / 2]: each pair's turns per position modulo 1, times 2^64 (host)."""
    table = np.zeros(max(int(rope.rot_dim) // 2, 1), dtype=np.uint64)
    _check(lib().pod_attn_rope_table(ctypes.byref(rope), table.ctypes.data_as(ctypes.POINTER(ctypes.c_uint64))))
    return table


def pod_attn_append(params: Params, rope: Optional[RopeParams], rope_table: int, norm: Optional[HeadNormParams], q: int,
                    q_stride: int, k: int, k_stride: int, v: int, v_stride: int, slots: int, positions: int, n_rows: int,
                    q_out: int, k_cache: int, v_cache: int, stream: int = 0):
    """Normalise, rotate and write a batch's new tokens; all tensor arguments are raw device addresses."""
    _check(lib().pod_attn_append(ctypes.byref(params), None if rope is None else ctypes.byref(rope), rope_table,
                                 None if norm is None else ctypes.byref(norm), q, q_stride, k, k_stride, v, v_stride, slots,
                                 positions, n_rows, q_out, k_cache, v_cache, stream))


STATIC_SCRATCH_BYTES = 64 << 20


def pod_attn_forward_static(prefill_q: int, decode_q: int, k_cache: int, v_cache: int, seq_meta: int,
                            block_table: int, out: int, plan: Plan, mode: int = MODE_FUSED, stream: int = 0):
    """pod_attn_forward on the library's own static scratch: no workspace argument, no allocation."""
    vp = ctypes.c_void_p
    _check(lib().pod_attn_forward_static(vp(prefill_q), vp(decode_q), vp(k_cache), vp(v_cache), vp(seq_meta),
                                         vp(block_table), vp(out), plan.handle, mode, vp(stream)))


def pod_attn_probe_hbm_read(buf: int, nbytes: int, sink: int, stream: int = 0):
    vp = ctypes.c_void_p
    status = lib().pod_attn_probe_hbm_read(vp(buf), nbytes, vp(sink), vp(stream))
    if status != POD_OK:
        raise PodError(status, "pod_attn_probe_hbm_read failed")


def pod_attn_probe_mfma(iters: int, sink: int, stream: int = 0) -> float:
    """Enqueue the MFMA issue loop; returns the flop count of the launch."""
    flops = ctypes.c_double(0.0)
    status = lib().pod_attn_probe_mfma(iters, ctypes.c_void_p(sink), ctypes.byref(flops), ctypes.c_void_p(stream))
    if status != POD_OK:
        raise PodError(status, "pod_attn_probe_mfma failed")
    return float(flops.value)


ISSUE_PROBE_VARIANTS = ["4 matrix instructions", "each + one 2^x", "each + the work of one softmax score (no dot product)",
                        "that + one 2-element dot product", "each + one 2-element dot product only",
                        "pipelined turn: LDS read, 1 matrix instruction, staged softmax of 1 score",
                        "pipelined turn: LDS read, 2 matrix instructions, staged softmax of 2 scores",
                        "no matrix instruction: 8 independent v_fma_f32 (ns per vector instruction)",
                        "no matrix instruction: 8 independent v_exp_f32 (ns per vector instruction)"]


def pod_attn_probe_issue(variant: int, iters: int, wgs_per_unit: int, sink: int, stream: int = 0) -> float:
    """Enqueue one instruction-mix probe; returns the matrix instructions (for the last two variants:
    the vector instructions) one wavefront issues."""
    n = ctypes.c_double(0.0)
    status = lib().pod_attn_probe_issue(variant, iters, wgs_per_unit, ctypes.c_void_p(sink), ctypes.byref(n),
                                        ctypes.c_void_p(stream))
    if status != POD_OK:
        raise PodError(status, "pod_attn_probe_issue failed")
    return float(n.value)


def pod_attn_probe_colocation(variant: int, a: int, b: int, c: int, bytes_per_item: int, n_memory_items: int,
                              n_compute_items: int, compute_iters: int, counters: int, sink: int, stream: int = 0):
    _check(lib().pod_attn_probe_colocation(variant, ctypes.c_void_p(a), ctypes.c_void_p(b), ctypes.c_void_p(c),
                                           bytes_per_item, n_memory_items, n_compute_items, compute_iters,
                                           ctypes.c_void_p(counters), ctypes.c_void_p(sink), ctypes.c_void_p(stream)))


def pod_attn_role_for_ticket(ticket: int, prefill_ratio: int, decode_ratio: int, unit: int = 0) -> int:
    return int(lib().pod_attn_role_for_ticket(ticket, prefill_ratio, decode_ratio, unit))


def pod_attn_simulate_launch(plan: Plan, unit_of_wg, order):
    """Host model of one fused launch; returns (steps, first_role, seat_of_wg, item_owner, unit_owner)."""
    units, units_p = _i32(np.asarray(unit_of_wg))
    order, order_p = _i32(np.asarray(order))
    info = plan.info()
    first = np.full(max(units.size, 1), -2, dtype=np.int32)
    seat = np.full(max(units.size, 1), -1, dtype=np.int32)
    items = np.full(max(info.n_prefill_items, 1), -2, dtype=np.int32)
    dunits = np.full(max(info.n_decode_units, 1), -2, dtype=np.int32)
    p = lambda a: a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
    steps = lib().pod_attn_simulate_launch(plan.handle, units_p, int(units.size), order_p, int(order.size),
                                           p(first), p(seat), p(items), p(dunits))
    return (int(steps), first[:units.size], seat[:units.size], items[:info.n_prefill_items],
            dunits[:info.n_decode_units])


# ----------------------------------------------------------------------------------------------
# Convenience wrapper for torch tensors (marshalling only).
# ----------------------------------------------------------------------------------------------
def _stream_of(device) -> int:
    """The hipStream_t of torch's current stream on a device.  (As an object it costs 1.8 us to ask for, as a number 0.1.)"""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device.index) if raw is not None else torch.cuda.current_stream(device).cuda_stream


def _call(device, function, *args):
    """function(*args) with `device` as the current one, which is where its tensors are."""
    import torch
    if torch.cuda.current_device() == device.index:
        status = function(*args)
    else:
        with torch.cuda.device(device):
            status = function(*args)
    if status != POD_OK:
        _check(status)


def _apart(t, strides):
    """Whether the elements of t lie this far apart in each dimension (one of size 1 has no next element)."""
    return all(n == 1 or is_ == ought for n, is_, ought in zip(t.shape, t.stride(), strides))


def _need(t, what, dtype, shape, device, strided=False, strides=None):
    """Raises ValueError unless t is a tensor of this type and shape on this device, in one piece (with `strided`, of two
    dimensions, whose rows are; with `strides`, with elements that far apart).  A None in the shape is any size."""
    if t.dtype is dtype and t.shape == shape and t.device == device and strides is None and (t.stride(1) == 1 if strided else t.is_contiguous()):
        return
    if t.dtype != dtype:
        raise ValueError(f"{what} must be {dtype}, not {t.dtype}")
    if t.device != device:
        raise ValueError(f"{what} must be on {device}, not {t.device}")
    if t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise ValueError(f"{what} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
    if strides is not None:
        if not _apart(t, strides):
            raise ValueError(f"{what} must have the strides {tuple(strides)}, not {tuple(t.stride())}")
        return
    if not (t.is_contiguous() or (strided and t.stride(1) == 1)):
        raise ValueError(f"{what} must lie in one piece" + (" row by row" if strided else ""))


def _device(device):
    import torch
    device = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device()) if device.type == "cuda" and device.index is None else device


_KIND = ("dtype", "n_q_heads", "n_kv_heads", "head_dim", "block_size", "kv_order", "n_blocks or n_cache_rows", "kv_seq_stride")


def _kind(p: Params):
    """What the calls of one layer have to have in common, as _KIND names it: the heads, and the cache that a slot names a place
    of (blocks of a paged one, rows and their length of a contiguous one)."""
    cache = (p.n_blocks, 0) if p.block_size > 0 else (p.n_cache_rows, p.kv_seq_stride)
    return (p.dtype, p.n_q_heads, p.n_kv_heads, p.head_dim, p.block_size, p.kv_order) + cache


class Rope:
    """Rotary positions: which channels turn together, how fast, and how that is stretched for long contexts.

    ``scaling`` is "none", "linear", "parts" or "index" (``pod_rope_scaling``); ``trained_len``, ``low`` and ``high`` are read
    by the last two."""
    LAYOUTS = {"half": 0, "interleaved": 1}
    SCALINGS = {"none": 0, "linear": 1, "parts": 2, "index": 3}

    def __init__(self, rot_dim, *, layout="half", theta=10000.0, scaling="none", factor=1.0, trained_len=8192, low=1.0,
                 high=4.0, cos_sin_scale=1.0):
        if layout not in self.LAYOUTS or scaling not in self.SCALINGS:
            raise ValueError(f"unknown rope layout {layout!r} or scaling {scaling!r}")
        self.params = RopeParams(self.LAYOUTS[layout], self.SCALINGS[scaling], rot_dim, cos_sin_scale, theta, factor, trained_len,
                                 low, high)
        self.table = pod_attn_rope_table(self.params)


class HeadNorm:
    """RMS normalisation of each query and key head; a weight of None is 1, ``q`` or ``k`` False leaves those heads alone."""

    def __init__(self, q_weight=None, k_weight=None, *, eps=1e-6, weight_offset=0.0, q=True, k=True):
        self.q_weight, self.k_weight, self.eps, self.weight_offset, self.q, self.k = q_weight, k_weight, eps, weight_offset, q, k


class TokenTables:
    """Slots and positions of the new tokens of batches of one shape, and the blocks they take.

    ``build`` may be called once per step and recorded into a graph; it fills ``slots`` and ``positions`` (int32 [n_rows],
    rows behind the batch are padding) and ``report`` (blocks taken, blocks missing, requests refused, rows).  A batch of which
    blocks are missing, requests refused or rows more than ``n_rows`` must not go on to the attention: its block table lacks
    blocks."""

    def __init__(self, params: Params, n_rows: int, *, device="cuda"):
        import torch
        self.params, self.n_rows, self.device, self.kind = params, int(n_rows), _device(device), _kind(params)
        self.requests = params.n_prefill, params.n_decode
        self.slots = torch.empty(self.n_rows, dtype=torch.int32, device=self.device)
        self.positions = torch.empty(self.n_rows, dtype=torch.int32, device=self.device)
        self.report = torch.zeros(4, dtype=torch.int32, device=self.device)
        self._args = ctypes.byref(params), self.n_rows, self.slots.data_ptr(), self.positions.data_ptr(), self.report.data_ptr()

    def build(self, seq_meta, free_blocks=None, block_table=None):
        """From seq_meta (int32 [requests, 4]); a paged cache also takes its free blocks and its block table, which is
        written."""
        import torch
        p, dev = self.params, self.device
        _need(seq_meta, "seq_meta", torch.int32, (p.n_prefill + p.n_decode, 4), dev)
        free = table = n_free = 0
        if p.block_size > 0:
            _need(free_blocks, "free_blocks", torch.int32, (None,), dev)
            _need(block_table, "block_table", torch.int32, (p.n_cache_rows, p.max_blocks_per_seq), dev)
            free, n_free, table = free_blocks.data_ptr(), free_blocks.numel(), block_table.data_ptr()
        ref, n_rows, slots, positions, report = self._args
        _call(dev, lib().pod_attn_build_tables, ref, seq_meta.data_ptr(), free, n_free, table, n_rows, slots, positions, report,
              _stream_of(dev))
        return self


class TokenAppend:
    """New tokens normalised, rotated and written: queries to rows for the attention, keys and values to the cache."""

    def __init__(self, params: Params, *, rope: Optional[Rope] = None, norm: Optional[HeadNorm] = None, device="cuda"):
        import torch
        self.params, self.device = params, _device(device)
        self.index, self.kind = self.device.index if self.device.type == "cuda" else -1, _kind(params)
        self.dtype = {F16: torch.float16, BF16: torch.bfloat16}[params.dtype]
        self.rope, self.table, self.norm = None, None, None
        if rope is not None:
            if rope.params.rot_dim > params.head_dim:
                raise ValueError(f"rot_dim {rope.params.rot_dim} is more than head_dim {params.head_dim}")
            self.rope = rope.params
            self.table = torch.from_numpy(rope.table.view(np.int64)).to(self.device)
        if norm is not None:
            for name in ("q_weight", "k_weight"):
                if getattr(norm, name) is not None:
                    _need(getattr(norm, name), name, self.dtype, (params.head_dim,), self.device)
            self.weights = (norm.q_weight, norm.k_weight)                # kept alive
            ptr = lambda w: None if w is None else w.data_ptr()
            self.norm = HeadNormParams(ptr(norm.q_weight), ptr(norm.k_weight), norm.eps, norm.weight_offset, int(norm.q), int(norm.k))
        p = params
        n, tokens = (p.n_blocks, p.block_size) if p.block_size > 0 else (p.n_cache_rows, p.kv_seq_stride // max(p.n_kv_heads * p.head_dim, 1))
        self.cache_shape = (n, p.n_kv_heads, tokens, p.head_dim) if p.kv_order == KV_HEAD_MAJOR else (n, tokens, p.n_kv_heads, p.head_dim)
        # Rows of a contiguous cache may lie further apart than their tokens; such a cache is a view with gaps.
        row, stride = p.n_kv_heads * p.head_dim, int(p.kv_seq_stride)
        self.cache_strides = (stride, row, p.head_dim, 1) if p.block_size <= 0 and stride != tokens * row else None
        self._rows = p.n_q_heads * p.head_dim, p.n_kv_heads * p.head_dim, p.n_q_heads, p.head_dim
        ref = lambda x: None if x is None else ctypes.byref(x)
        self._args = ref(params), ref(self.rope), 0 if self.table is None else self.table.data_ptr(), ref(self.norm)

    def __call__(self, q, k, v, slots, positions, k_cache, v_cache, q_out=None):
        """q, k, v: [rows, heads * head_dim] (or views of one projection); returns q_out, [rows, Hq, d].  The caches are in one
        piece, or, where kv_seq_stride is no whole number of tokens, views whose rows lie kv_seq_stride elements apart."""
        import torch
        dev, dtype, i, i32 = self.device, self.dtype, self.index, torch.int32
        q_row, kv_row, heads, d = self._rows
        cache_strides = self.cache_strides
        flat = slots.shape
        rows = flat[0] if flat else 0
        if q_out is None:
            q_out = torch.empty((rows, heads, d), dtype=dtype, device=dev)
        kv_shape, cache_shape, q_strides, k_strides, v_strides = (rows, kv_row), self.cache_shape, q.stride(), k.stride(), v.stride()
        # What _need asks of each tensor, written out: a decode step of few rows waits for this call (8 of its 8.7 us with a call of
        # _need for each).  Where something does not fit, _need says what.
        if not (q.dtype is dtype and k.dtype is dtype and v.dtype is dtype and k_cache.dtype is dtype and v_cache.dtype is dtype and
                q_out.dtype is dtype and slots.dtype is i32 and positions.dtype is i32 and
                q.shape == (rows, q_row) and k.shape == kv_shape and v.shape == kv_shape and k_cache.shape == cache_shape and
                v_cache.shape == cache_shape and q_out.shape == (rows, heads, d) and len(flat) == 1 and positions.shape == flat and
                q.get_device() == i and k.get_device() == i and v.get_device() == i and k_cache.get_device() == i and
                v_cache.get_device() == i and q_out.get_device() == i and slots.get_device() == i and positions.get_device() == i and
                q_strides[1] == 1 and k_strides[1] == 1 and v_strides[1] == 1 and cache_strides is None and
                k_cache.is_contiguous() and v_cache.is_contiguous() and q_out.is_contiguous() and slots.is_contiguous() and positions.is_contiguous()):
            _need(slots, "slots", i32, (rows,), dev)
            _need(positions, "positions", i32, (rows,), dev)
            _need(q, "q", dtype, (rows, q_row), dev, strided=True)
            _need(k, "k", dtype, kv_shape, dev, strided=True)
            _need(v, "v", dtype, kv_shape, dev, strided=True)
            _need(k_cache, "k_cache", dtype, cache_shape, dev, strides=cache_strides)
            _need(v_cache, "v_cache", dtype, cache_shape, dev, strides=cache_strides)
            _need(q_out, "q_out", dtype, (rows, heads, d), dev)
        # (a single row has no distance to a next one: torch may name any)
        q_stride, k_stride, v_stride = (q_strides[0], k_strides[0], v_strides[0]) if rows > 1 else (q_row, kv_row, kv_row)
        ref, rope, table, norm = self._args
        _call(dev, lib().pod_attn_append, ref, rope, table, norm, q.data_ptr(), q_stride, k.data_ptr(), k_stride, v.data_ptr(),
              v_stride, slots.data_ptr(), positions.data_ptr(), rows, q_out.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
              _stream_of(dev))
        return q_out


class HybridAttention:
    """Plan + workspace for one batch shape; ``forward`` may be called once per layer.  ``scores``: scores other than plain
    causal ones."""

    def __init__(self, batch, *, scores: Optional[Scores] = None, policy=POLICY_AUTO, max_prefill_waves=0, decode_chunk=0,
                 prefill_split_len=0, n_compute_units=0):
        import torch
        self.torch = torch
        self.batch_meta = np.ascontiguousarray(batch.seq_meta, dtype=np.int32)
        self.params = make_params(
            n_prefill=batch.n_prefill, n_decode=batch.n_decode, n_q_heads=batch.n_q_heads,
            n_kv_heads=batch.n_kv_heads, head_dim=batch.head_dim, dtype=batch.dtype,
            softmax_scale=batch.softmax_scale, block_size=batch.block_size,
            max_blocks_per_seq=batch.max_blocks_per_seq, n_cache_rows=batch.n_cache_rows,
            n_blocks=batch.n_blocks, kv_seq_stride=batch.kv_seq_stride, policy=policy,
            max_prefill_waves=max_prefill_waves, decode_chunk=decode_chunk,
            prefill_split_len=prefill_split_len, n_compute_units=n_compute_units,
            kv_order=KV_HEAD_MAJOR if batch.head_major else KV_TOKEN_MAJOR)
        self.plan = (pod_attn_plan_create(self.params, self.batch_meta) if scores is None
                     else pod_attn_plan_create_scored(self.params, scores, self.batch_meta))
        self.info = self.plan.info()
        dev = batch.k_cache.device
        self.ws_bytes = pod_attn_workspace_size(self.plan)
        self.workspace = torch.empty(self.ws_bytes + 256, dtype=torch.uint8, device=dev)
        base = self.workspace.data_ptr()
        self.ws_ptr = (base + 255) & ~255
        self.seq_meta_dev = torch.from_numpy(self.batch_meta).to(dev)
        stream = torch.cuda.current_stream(dev).cuda_stream
        pod_attn_plan_upload(self.plan, self.ws_ptr, self.ws_bytes, stream)

    def forward(self, batch, out=None, mode=MODE_FUSED):
        ptr = lambda t: 0 if t is None else t.data_ptr()                   # (0 of an empty tensor)
        return self._forward(ptr(batch.prefill_q), ptr(batch.decode_q), batch, out, mode)

    def _forward(self, prefill_q, decode_q, batch, out, mode):
        torch = self.torch
        dev = batch.k_cache.device
        if out is None:
            out = torch.empty((batch.n_rows, batch.n_q_heads, batch.head_dim), dtype=batch.torch_dtype,
                              device=dev)
        table = batch.block_table
        _call(dev, lib().pod_attn_forward, prefill_q, decode_q, batch.k_cache.data_ptr(), batch.v_cache.data_ptr(),
              self.seq_meta_dev.data_ptr(), 0 if table is None else table.data_ptr(), out.data_ptr(), self.plan.handle,
              self.ws_ptr, self.ws_bytes, mode, _stream_of(dev))
        return out

    @functools.cached_property
    def _shape(self):
        return _kind(self.params), (self.params.n_prefill, self.params.n_decode)

    @functools.cached_property
    def _row_counts(self):
        return self.info.n_prefill_rows, self.params.n_decode

    def forward_tokens(self, batch, append: TokenAppend, tables: TokenTables, q, k, v, out=None, mode=MODE_FUSED):
        """One layer of the batch from its projections: the new tokens are put into the cache at ``tables``' slots, then the
        attention reads them.  q, k, v: [rows, heads * head_dim] in the order of the output rows; rows behind the batch are
        padding.  The queries of ``batch`` are not read.  Returns the output rows."""
        n = batch.n_rows
        kind, requests = self._shape
        if append.kind != kind or tables.kind != kind:
            differing = [name for name, *of in zip(_KIND, kind, append.kind, tables.kind) if len(set(of)) > 1]
            raise ValueError(f"{', '.join(differing)} in the plan, {kind}, differ from those of the append, {append.kind}, or the tables, {tables.kind}")
        if tables.requests != requests:
            raise ValueError(f"tables for {tables.requests} prefill and decode requests beside a plan for {requests}")
        rows = batch.n_prefill_rows, batch.n_decode
        if rows != self._row_counts:
            raise ValueError(f"a batch of {rows} prefill and decode rows beside a plan for {self._row_counts}")
        if q.shape[0] < n:
            raise ValueError(f"{q.shape[0]} rows of projections for a batch of {n}")
        rows = append(q, k, v, tables.slots, tables.positions, batch.k_cache, batch.v_cache)
        first = rows.data_ptr()
        return self._forward(first, first + batch.n_prefill_rows * rows.stride(0) * rows.element_size(), batch, out, mode)

    def enable_trace(self):
        """Allocate a trace buffer (one record per workgroup) and switch tracing on."""
        n = max(self.info.n_prefill_items + (self.info.n_decode_units + 3) // 4, self.info.fused_grid, 1)
        self.trace = self.torch.zeros(n * 48, dtype=self.torch.uint8, device=self.workspace.device)
        pod_attn_plan_set_trace(self.plan, self.trace.data_ptr(), self.trace.numel())

    def read_trace(self) -> np.ndarray:
        """Records of the last fused launch: one per workgroup.  A batch of prompts alone runs the prefill
        kernel there, which has a workgroup per item."""
        self.torch.cuda.synchronize()
        n = self.info.fused_grid if self.info.n_decode_units > 0 else self.info.n_prefill_items
        return self.trace.cpu().numpy().view(TRACE_DTYPE)[:n].copy()

    def disable_trace(self):
        pod_attn_plan_set_trace(self.plan, 0, 0)

    def enable_event_log(self):
        """Allocate an event log (one record per prefill item and decode unit) and switch it on."""
        n = self.info.n_prefill_items + self.info.n_decode_units + 1
        self.evlog = self.torch.zeros(16 + n * 32, dtype=self.torch.uint8, device=self.workspace.device)
        pod_attn_plan_set_event_log(self.plan, self.evlog.data_ptr(), self.evlog.numel())

    def read_event_log(self) -> np.ndarray:
        """Records of the forward call made since the log was last read; clears the log."""
        self.torch.cuda.synchronize()
        raw = self.evlog.cpu().numpy()
        n = min(int(raw[:4].view(np.uint32)[0]), (raw.size - 16) // 32)
        ev = raw[16:16 + n * 32].view(EVENT_DTYPE).copy()
        self.evlog[:16].zero_()
        return ev

    def disable_event_log(self):
        pod_attn_plan_set_event_log(self.plan, 0, 0)

    def close(self):
        self.plan.close()
