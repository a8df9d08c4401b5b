"""ctypes binding of libapril.so: same names as include/april.h, argument marshalling only.

Every step of the rollout path runs in the library's HIP kernels; nothing here
computes.  Loading fails loudly when the library is missing: there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass, field
from typing import Dict, List, NamedTuple, Optional, Sequence

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libapril.so")

APRIL_OK, APRIL_EINVAL, APRIL_ENOMEM, APRIL_ESTARVED, APRIL_EHANDLE, APRIL_EDEVICE = 0, -1, -2, -3, -4, -5
APRIL_DTYPE_FP32, APRIL_DTYPE_BF16, APRIL_DTYPE_BF16_KV4 = 0, 1, 2
APRIL_SAMPLER_GREEDY, APRIL_SAMPLER_TOPK, APRIL_SAMPLER_CATEGORICAL = 0, 1, 2
APRIL_MEM_KV, APRIL_MEM_WEIGHTS = 1, 2
APRIL_KERNEL_CLASSES = 24

EXPORTS = [
    "april_init", "april_rollout_step", "april_resume", "april_buffer_size", "april_buffer_export",
    "april_buffer_import", "april_buffer_drop_kv", "april_buffer_free", "april_update_weights", "april_memory_pause", "april_memory_resume", "april_debug_watch",
    "april_debug_logits", "april_sample_rows", "april_sample_rows_logprobs", "april_sample_rows_noalloc", "april_profile_enable", "april_profile_get",
    "april_profile_reset", "april_get_info", "april_last_error", "april_destroy",
    "april_cache_block_bytes", "april_cache_extend", "april_cache_append", "april_cache_attention", "april_cache_attention_workspace",
    "april_logprobs", "april_logprobs_workspace", "april_logprobs_grad", "april_embed", "april_embed_grad", "april_embed_grad_workspace",
    "april_expert_sort", "april_expert_sort_workspace", "april_expert_gather", "april_expert_combine", "april_expert_combine_grad",
]
APRIL_CACHE_PAGE = 16


class AprilError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"april error {code}: {msg}")
        self.code = code


class april_model_cfg(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("d_ffn", C.c_int32), ("vocab", C.c_int32),
        ("n_experts", C.c_int32), ("experts_per_tok", C.c_int32), ("d_expert_ffn", C.c_int32),
        ("dtype", C.c_int32), ("rope_theta", C.c_float), ("rms_eps", C.c_float),
        ("kv_block_tokens", C.c_int32), ("kv_pool_bytes", C.c_int64),
        ("max_inflight", C.c_int32), ("max_ctx", C.c_int32),
        ("sampler", C.c_int32), ("top_k", C.c_int32), ("temperature", C.c_float), ("seed", C.c_uint64),
        ("eos_token", C.c_int32), ("debug_logits", C.c_int32), ("top_p", C.c_float), ("logprobs", C.c_int32),
        ("n_samples_per_prompt", C.c_int32), ("pausable", C.c_int32), ("stream", C.c_void_p),
    ]


class april_tensor(C.Structure):
    _fields_ = [("name", C.c_char_p), ("data", C.c_void_p), ("nbytes", C.c_int64), ("on_device", C.c_int32)]


class april_request(C.Structure):
    _fields_ = [("request_id", C.c_int64), ("tokens", C.POINTER(C.c_int32)), ("n_tokens", C.c_int32),
                ("forced_len", C.c_int32), ("forced_tokens", C.POINTER(C.c_int32)), ("n_forced_tokens", C.c_int32),
                ("group_id", C.c_int64)]


class april_step_result(C.Structure):
    _fields_ = [
        ("n_completed", C.c_int32), ("request_id", C.POINTER(C.c_int64)),
        ("tokens", C.POINTER(C.POINTER(C.c_int32))), ("n_tokens", C.POINTER(C.c_int32)),
        ("n_resumes", C.POINTER(C.c_int32)), ("logprobs", C.POINTER(C.POINTER(C.c_float))),
        ("group_id", C.POINTER(C.c_int64)), ("buffer", C.c_void_p), ("n_new_consumed", C.c_int32),
        ("decode_iters", C.c_int64), ("tokens_generated", C.c_int64), ("prefill_tokens", C.c_int64),
        ("reprefill_tokens", C.c_int64), ("n_preempted", C.c_int64), ("sum_live", C.c_int64), ("sum_ctx", C.c_int64),
        ("dec_sum_live", C.c_int64), ("dec_sum_ctx", C.c_int64), ("dec_sum_experts", C.c_int64),
        ("t_prefill_s", C.c_double), ("t_decode_s", C.c_double), ("t_total_s", C.c_double),
    ]


class april_partial(C.Structure):
    _fields_ = [("request_id", C.c_int64), ("prompt", C.POINTER(C.c_int32)), ("n_prompt", C.c_int32),
                ("generated", C.POINTER(C.c_int32)), ("n_generated", C.c_int32), ("limit", C.c_int32),
                ("n_resumes", C.c_int32), ("done", C.c_int32), ("kv_resident", C.c_int32),
                ("logprobs", C.POINTER(C.c_float)), ("group_id", C.c_int64)]


class april_kernel_stat(C.Structure):
    _fields_ = [("name", C.c_char_p), ("launches", C.c_int64), ("total_ms", C.c_double),
                ("alg_bytes", C.c_double), ("alg_flops", C.c_double)]


class april_info(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("hbm_total", "hbm_free", "kv_pool_bytes", "kv_blocks_total",
                                         "kv_blocks_free", "weight_bytes", "decode_weight_bytes",
                                         "kv_bytes_per_token", "expert_bytes")]


class april_cache_extend_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_seqs", "max_pages", "n_pages", "n_rows")] + [("table_stride", C.c_int64)] + [
        (n, C.c_void_p) for n in ("lens", "new_lens", "free_top", "block_table", "free_pages", "lens_out", "free_top_out", "q_start",
                                  "slot_map", "positions", "status", "stream")]


class april_cache_append_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_pages", "n_kv_heads", "head_dim", "n_rows", "dtype", "reserved")] + [
        (n, C.c_int64) for n in ("k_row", "k_head", "v_row", "v_head")] + [
        (n, C.c_void_p) for n in ("k", "v", "k_values", "v_values", "slot_map", "pool", "stream")]


class april_cache_attention_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_q_heads", "n_kv_heads", "head_dim", "n_pages", "n_seqs", "max_pages", "n_rows", "max_q",
                                         "max_len")] + [("scale", C.c_float)] + [
        (n, C.c_int64) for n in ("table_stride", "q_row", "q_head", "out_row", "out_head")] + [
        (n, C.c_void_p) for n in ("q", "pool", "block_table", "lens", "q_start", "out", "lse", "workspace")] + [
        ("workspace_bytes", C.c_int64), ("stream", C.c_void_p)]


class april_logprobs_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_rows", "vocab", "dtype", "index_bits", "n_top")] + [("temperature", C.c_float), ("logits_row", C.c_int64)] + [
        (n, C.c_void_p) for n in ("logits", "tokens", "logprob", "entropy", "lse", "norm", "top_logprobs", "top_ids", "workspace")] + [
        ("workspace_bytes", C.c_int64), ("stream", C.c_void_p)]


class april_logprobs_grad_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_rows", "vocab", "dtype", "index_bits")] + [("temperature", C.c_float), ("reserved", C.c_int32)] + [
        (n, C.c_int64) for n in ("logits_row", "grad_row")] + [
        (n, C.c_void_p) for n in ("logits", "tokens", "norm", "entropy", "grad_logprob", "grad_entropy", "grad_lse", "grad", "stream")]


class april_embed_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_rows", "vocab", "d", "table_dtype", "out_dtype", "index_bits")] + [
        ("scale", C.c_float), ("reserved", C.c_int32), ("table_row", C.c_int64), ("out_row", C.c_int64)] + [
        (n, C.c_void_p) for n in ("table", "tokens", "out", "stream")]


class april_embed_grad_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_rows", "vocab", "d", "out_dtype", "table_dtype", "index_bits")] + [
        ("scale", C.c_float), ("accumulate", C.c_int32), ("out_row", C.c_int64), ("table_row", C.c_int64)] + [
        (n, C.c_void_p) for n in ("grad_out", "tokens", "grad_table", "workspace")] + [("workspace_bytes", C.c_int64), ("stream", C.c_void_p)]


class april_expert_sort_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_rows", "k", "n_experts", "align", "n_packed", "index_bits")] + [
        (n, C.c_void_p) for n in ("ids", "starts", "source", "position", "workspace")] + [("workspace_bytes", C.c_int64), ("stream", C.c_void_p)]


class april_expert_gather_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_rows", "k", "d", "n_packed", "dtype", "reserved")] + [
        ("x_row", C.c_int64), ("packed_row", C.c_int64)] + [(n, C.c_void_p) for n in ("x", "source", "position", "packed", "stream")]


class april_expert_combine_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_rows", "k", "d", "n_packed", "dtype", "reserved")] + [
        ("packed_row", C.c_int64), ("out_row", C.c_int64)] + [(n, C.c_void_p) for n in ("packed", "position", "weights", "out", "stream")]


class april_expert_combine_grad_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_rows", "k", "d", "n_packed", "dtype", "reserved")] + [
        (n, C.c_int64) for n in ("out_row", "packed_row", "grad_packed_row")] + [
        (n, C.c_void_p) for n in ("grad_out", "packed", "source", "position", "weights", "grad_packed", "grad_weights", "stream")]


# The same structs as bytes: packing them is a third of the time of filling a ctypes structure.
_PACK_EXTEND = struct.Struct("4iq12Q").pack
_PACK_APPEND = struct.Struct("6i4q7Q").pack
_PACK_ATTENTION = struct.Struct("9if5q8QqQ").pack
_PACK_LOGPROBS = struct.Struct("5ifq9QqQ").pack
_PACK_LOGPROBS_GRAD = struct.Struct("4ifi2q9Q").pack
_PACK_EMBED = struct.Struct("6ifi2q4Q").pack
_PACK_EMBED_GRAD = struct.Struct("6ifi2q4QqQ").pack
_PACK_EXPERT_SORT = struct.Struct("6i5QqQ").pack
_PACK_EXPERT_GATHER = struct.Struct("6i2q5Q").pack
_PACK_EXPERT_COMBINE = struct.Struct("6i2q5Q").pack
_PACK_EXPERT_COMBINE_GRAD = struct.Struct("6i3q8Q").pack

_lib = None
_calls = {}


def _call(name):
    """A library function that takes its struct as bytes."""
    f = _calls.get(name)
    if f is None:
        f = load_library()[name]
        f.argtypes, f.restype = [C.c_char_p], C.c_int64 if name.endswith("workspace") else C.c_int
        _calls[name] = f
    return f


def load_library():
    """dlopen libapril.so (built in-tree by build.py) and declare the prototypes."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} is missing: build it with `python -m paper_2509_18521_amd.build` "
                                "(there is no CPU fallback)")
    lib = C.CDLL(LIB_PATH)
    vp = C.c_void_p
    lib.april_init.argtypes = [C.POINTER(april_model_cfg), C.POINTER(april_tensor), C.c_int32, C.POINTER(vp)]
    lib.april_rollout_step.argtypes = [vp, C.POINTER(april_request), C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                       C.POINTER(april_step_result)]
    lib.april_resume.argtypes = [vp, vp]
    lib.april_buffer_size.argtypes = [vp, vp]
    lib.april_buffer_export.argtypes = [vp, vp, C.POINTER(april_partial), C.c_int32]
    lib.april_buffer_import.argtypes = [vp, C.POINTER(april_partial), C.c_int32, C.POINTER(vp)]
    lib.april_buffer_drop_kv.argtypes = [vp, vp]
    lib.april_buffer_free.argtypes = [vp, vp]
    lib.april_buffer_free.restype = None
    lib.april_update_weights.argtypes = [vp, C.POINTER(april_tensor), C.c_int32, C.c_int32]
    lib.april_memory_pause.argtypes = [vp, C.c_int32]
    lib.april_memory_resume.argtypes = [vp, C.c_int32]
    lib.april_debug_watch.argtypes = [vp, C.c_int64, C.c_int32, C.c_int32]
    lib.april_debug_logits.argtypes = [vp, C.c_int64, C.c_int32, C.POINTER(C.c_float), C.POINTER(C.c_int32)]
    lib.april_sample_rows.argtypes = [vp, vp, C.c_int32, C.POINTER(C.c_int64), C.POINTER(C.c_int32),
                                      C.POINTER(C.c_int32)]
    lib.april_sample_rows_noalloc.argtypes = lib.april_sample_rows.argtypes
    lib.april_sample_rows_logprobs.argtypes = lib.april_sample_rows.argtypes + [C.POINTER(C.c_float)]
    lib.april_profile_enable.argtypes = [vp, C.c_int32]
    lib.april_profile_get.argtypes = [vp, C.POINTER(april_kernel_stat), C.c_int32]
    lib.april_profile_reset.argtypes = [vp]
    lib.april_get_info.argtypes = [vp, C.POINTER(april_info)]
    lib.april_last_error.argtypes = [vp]
    lib.april_last_error.restype = C.c_char_p
    lib.april_destroy.argtypes = [vp]
    lib.april_destroy.restype = None
    lib.april_cache_block_bytes.argtypes = [C.c_int32]
    lib.april_cache_extend.argtypes = [C.POINTER(april_cache_extend_args)]
    lib.april_cache_append.argtypes = [C.POINTER(april_cache_append_args)]
    lib.april_cache_attention.argtypes = [C.POINTER(april_cache_attention_args)]
    lib.april_cache_attention_workspace.argtypes = [C.POINTER(april_cache_attention_args)]
    for name in ("logprobs", "logprobs_grad", "embed", "embed_grad", "expert_sort", "expert_gather", "expert_combine", "expert_combine_grad"):
        for call in ("april_" + name, "april_%s_workspace" % name):
            if call in EXPORTS:
                getattr(lib, call).argtypes = [C.POINTER(globals()["april_%s_args" % name])]
    for name in EXPORTS:
        if name not in ("april_buffer_free", "april_destroy", "april_last_error"):
            getattr(lib, name).restype = C.c_int64 if name.endswith("_workspace") else C.c_int
    _lib = lib
    return lib


def _check(ctx, rc):
    if rc < 0:
        msg = load_library().april_last_error(ctx)
        raise AprilError(rc, msg.decode() if msg else "")
    return rc


def _i32ptr(a: np.ndarray):
    return a.ctypes.data_as(C.POINTER(C.c_int32))


# ---------------------------------------------------------------------------
# same-name wrappers
# ---------------------------------------------------------------------------
def _tensor_table(weights: Dict[str, object]):
    """name -> numpy array (host) or an object with .data_ptr() / .numel() / .element_size() on
    the GPU (e.g. a torch CUDA tensor)  ->  (april_tensor array, objects to keep alive)."""
    arr = (april_tensor * len(weights))()
    keep = []
    for i, (name, w) in enumerate(weights.items()):
        name = name.encode()
        keep.append(name)
        if isinstance(w, np.ndarray):
            w = np.ascontiguousarray(w)
            keep.append(w)
            arr[i] = april_tensor(name, w.ctypes.data, w.nbytes, 0)
        else:
            keep.append(w)
            arr[i] = april_tensor(name, w.data_ptr(), w.numel() * w.element_size(), 1)
    return arr, keep


def april_init(cfg: april_model_cfg, weights: Dict[str, object]) -> C.c_void_p:
    """weights: see _tensor_table.  Arrays are borrowed for the duration of the call."""
    lib = load_library()
    arr, keep = _tensor_table(weights)
    out = C.c_void_p()
    _check(None, lib.april_init(C.byref(cfg), arr, len(weights), C.byref(out)))
    return out


def april_update_weights(ctx, weights: Dict[str, object], keep_kv: bool = False):
    arr, keep = _tensor_table(weights)
    _check(ctx, load_library().april_update_weights(ctx, arr, len(weights), 1 if keep_kv else 0))


def april_destroy(ctx):
    load_library().april_destroy(ctx)


@dataclass
class StepResult:
    request_id: List[int]
    tokens: List[np.ndarray]
    n_resumes: List[int]
    buffer: C.c_void_p
    n_new_consumed: int
    decode_iters: int
    tokens_generated: int
    prefill_tokens: int
    reprefill_tokens: int
    n_preempted: int
    sum_live: int
    sum_ctx: int
    dec_sum_live: int
    dec_sum_ctx: int
    dec_sum_experts: int
    t_prefill_s: float
    t_decode_s: float
    t_total_s: float
    logprobs: Optional[List[np.ndarray]] = None      # per completed rollout (contexts created with logprobs)
    group_id: Optional[List[int]] = None             # per completed rollout (n_samples_per_prompt > 1)


def april_rollout_step(ctx, requests: Sequence[dict], n_target: int, n_overprovision: int, max_new: int) -> StepResult:
    """requests: dicts with request_id, tokens (int32 array), forced_len, optional forced_tokens."""
    lib = load_library()
    n = len(requests)
    arr = (april_request * max(n, 1))()
    keep = []
    for i, r in enumerate(requests):
        t = np.ascontiguousarray(r["tokens"], dtype=np.int32)
        keep.append(t)
        ft = r.get("forced_tokens")
        if ft is not None:
            ft = np.ascontiguousarray(ft, dtype=np.int32)
            keep.append(ft)
        arr[i] = april_request(int(r["request_id"]), _i32ptr(t), t.shape[0], int(r.get("forced_len", 0)),
                               _i32ptr(ft) if ft is not None else None, 0 if ft is None else ft.shape[0],
                               int(r.get("group_id", -1)))
    res = april_step_result()
    _check(ctx, lib.april_rollout_step(ctx, arr, n, n_target, n_overprovision, max_new, C.byref(res)))
    ids, toks, nres = [], [], []
    lps = [] if res.logprobs else None
    for i in range(res.n_completed):
        ids.append(int(res.request_id[i]))
        nt = int(res.n_tokens[i])
        toks.append(np.ctypeslib.as_array(res.tokens[i], shape=(nt,)).copy() if nt > 0 else np.zeros(0, np.int32))
        nres.append(int(res.n_resumes[i]))
        if lps is not None:
            lps.append(np.ctypeslib.as_array(res.logprobs[i], shape=(nt,)).copy() if nt > 0 else np.zeros(0, np.float32))
    return StepResult(ids, toks, nres, C.c_void_p(res.buffer), res.n_new_consumed, res.decode_iters,
                      res.tokens_generated, res.prefill_tokens, res.reprefill_tokens, res.n_preempted, res.sum_live, res.sum_ctx, res.dec_sum_live, res.dec_sum_ctx, res.dec_sum_experts,
                      res.t_prefill_s, res.t_decode_s, res.t_total_s, lps,
                      [int(res.group_id[i]) for i in range(res.n_completed)] if res.group_id else None)


def april_resume(ctx, buffer):
    _check(ctx, load_library().april_resume(ctx, buffer))


def april_buffer_size(ctx, buffer) -> int:
    return _check(ctx, load_library().april_buffer_size(ctx, buffer))


def april_buffer_export(ctx, buffer) -> List[dict]:
    lib = load_library()
    n = april_buffer_size(ctx, buffer)
    arr = (april_partial * max(n, 1))()
    _check(ctx, lib.april_buffer_export(ctx, buffer, arr, n))
    out = []
    for i in range(n):
        p = arr[i]
        out.append(dict(
            request_id=int(p.request_id),
            prompt=np.ctypeslib.as_array(p.prompt, shape=(p.n_prompt,)).copy(),
            generated=(np.ctypeslib.as_array(p.generated, shape=(p.n_generated,)).copy()
                       if p.n_generated > 0 else np.zeros(0, np.int32)),
            limit=int(p.limit), n_resumes=int(p.n_resumes), done=int(p.done), kv_resident=int(p.kv_resident),
            logprobs=(np.ctypeslib.as_array(p.logprobs, shape=(p.n_generated,)).copy()
                      if p.logprobs and p.n_generated > 0 else None), group_id=int(p.group_id)))
    return out


def april_buffer_import(ctx, partials: Sequence[dict]):
    lib = load_library()
    n = len(partials)
    arr = (april_partial * max(n, 1))()
    keep = []
    for i, p in enumerate(partials):
        pr = np.ascontiguousarray(p["prompt"], dtype=np.int32)
        ge = np.ascontiguousarray(p["generated"], dtype=np.int32)
        lp = p.get("logprobs")
        if lp is not None:
            lp = np.ascontiguousarray(lp, dtype=np.float32)
        keep += [pr, ge, lp]
        arr[i] = april_partial(int(p["request_id"]), _i32ptr(pr), pr.shape[0],
                               _i32ptr(ge) if ge.shape[0] else None, ge.shape[0], int(p["limit"]),
                               int(p.get("n_resumes", 0)), int(p.get("done", 0)), 0,
                               lp.ctypes.data_as(C.POINTER(C.c_float)) if lp is not None and lp.shape[0] else None,
                               int(p.get("group_id", -1)))
    out = C.c_void_p()
    _check(ctx, lib.april_buffer_import(ctx, arr, n, C.byref(out)))
    return out


def april_memory_pause(ctx, tags: int):
    _check(ctx, load_library().april_memory_pause(ctx, tags))


def april_memory_resume(ctx, tags: int):
    _check(ctx, load_library().april_memory_resume(ctx, tags))


def april_buffer_drop_kv(ctx, buffer):
    _check(ctx, load_library().april_buffer_drop_kv(ctx, buffer))


def april_buffer_free(ctx, buffer):
    load_library().april_buffer_free(ctx, buffer)


def april_debug_watch(ctx, request_id: int, first_gen: int, n_gen: int):
    _check(ctx, load_library().april_debug_watch(ctx, request_id, first_gen, n_gen))


def april_debug_logits(ctx, request_id: int, gen_index: int, vocab: int):
    out = np.empty(vocab, dtype=np.float32)
    sampled = C.c_int32(-1)
    _check(ctx, load_library().april_debug_logits(ctx, request_id, gen_index,
                                                  out.ctypes.data_as(C.POINTER(C.c_float)), C.byref(sampled)))
    return out, int(sampled.value)


def april_sample_rows(ctx, logits_device_ptr: int, n_rows: int, request_ids, gen_index) -> np.ndarray:
    rid = np.ascontiguousarray(request_ids, dtype=np.int64)
    gi = np.ascontiguousarray(gen_index, dtype=np.int32)
    out = np.empty(n_rows, dtype=np.int32)
    _check(ctx, load_library().april_sample_rows(ctx, C.c_void_p(logits_device_ptr), n_rows,
                                                 rid.ctypes.data_as(C.POINTER(C.c_int64)), _i32ptr(gi), _i32ptr(out)))
    return out


def april_sample_rows_logprobs(ctx, logits_device_ptr: int, n_rows: int, request_ids, gen_index):
    rid = np.ascontiguousarray(request_ids, dtype=np.int64)
    gi = np.ascontiguousarray(gen_index, dtype=np.int32)
    out = np.empty(n_rows, dtype=np.int32)
    lp = np.empty(n_rows, dtype=np.float32)
    _check(ctx, load_library().april_sample_rows_logprobs(ctx, C.c_void_p(logits_device_ptr), n_rows,
                                                          rid.ctypes.data_as(C.POINTER(C.c_int64)), _i32ptr(gi),
                                                          _i32ptr(out), lp.ctypes.data_as(C.POINTER(C.c_float))))
    return out, lp


def april_sample_rows_noalloc(ctx, logits_device_ptr: int, n_rows: int, request_ids, gen_index) -> np.ndarray:
    rid = np.ascontiguousarray(request_ids, dtype=np.int64)
    gi = np.ascontiguousarray(gen_index, dtype=np.int32)
    out = np.empty(n_rows, dtype=np.int32)
    _check(ctx, load_library().april_sample_rows_noalloc(ctx, C.c_void_p(logits_device_ptr), n_rows,
                                                         rid.ctypes.data_as(C.POINTER(C.c_int64)), _i32ptr(gi),
                                                         _i32ptr(out)))
    return out


def april_profile_enable(ctx, every: int):
    _check(ctx, load_library().april_profile_enable(ctx, every))


def april_profile_reset(ctx):
    _check(ctx, load_library().april_profile_reset(ctx))


def april_profile_get(ctx) -> List[dict]:
    arr = (april_kernel_stat * APRIL_KERNEL_CLASSES)()
    n = _check(ctx, load_library().april_profile_get(ctx, arr, APRIL_KERNEL_CLASSES))
    return [dict(name=arr[i].name.decode(), launches=int(arr[i].launches), total_ms=float(arr[i].total_ms),
                 alg_bytes=float(arr[i].alg_bytes), alg_flops=float(arr[i].alg_flops)) for i in range(n)]


def april_get_info(ctx) -> dict:
    info = april_info()
    _check(ctx, load_library().april_get_info(ctx, C.byref(info)))
    return {n: int(getattr(info, n)) for n, _ in april_info._fields_}


# ---------------------------------------------------------------------------
# Operators of the 4-bit KV cache, on torch tensors of one GPU.  They are enqueued on torch's current stream of the tensors' device and return at once; what they
# allocate (results that were not handed in, attention's workspace) comes from torch on that stream, so they may be
# captured into a graph.
# ---------------------------------------------------------------------------
class CacheTables(NamedTuple):
    """What april_cache_extend leaves, see april.h: all int32 but slot_map (int64)."""
    lens: object
    free_top: object
    q_start: object
    slot_map: object
    positions: object
    status: object


_torch = None               # imported by the first of these calls (the engine's calls need none)
_forward = None             # its forward-mode differentiation


def _need_torch():
    global _torch, _forward
    import torch
    import torch.autograd.forward_ad
    _torch, _forward = torch, torch.autograd.forward_ad


def _refuse(text, *args):
    raise AprilError(APRIL_EINVAL, text % args if args else text)


def _refuse_tensor(name, t, dtype, shape, dev, contiguous):
    if t.dtype is not dtype:
        _refuse("%s: %s wanted, not %s", name, dtype, t.dtype)
    if t.shape != shape:
        _refuse("%s: shape %s wanted, not %s", name, tuple(shape), tuple(t.shape))
    if t.get_device() != dev:
        _refuse("%s is on %s, not on GPU %d", name, t.device, dev)
    _refuse("%s has to be contiguous" if contiguous else "%s: the dimensions of a head have to be adjacent", name)


def _ptr(name, t, dtype, shape, dev):
    """Pointer of a contiguous tensor of that type and shape on GPU `dev`, or a refusal.  (One test: a call is a few microseconds.)"""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        _refuse_tensor(name, t, dtype, shape, dev, True)
    return t.data_ptr()


def _rows(name, t, dtype, shape, dev):
    """(pointer, strides of rows and heads) of a tensor [rows][heads][head_dim] whose heads may lie apart."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        _refuse_tensor(name, t, dtype, shape, dev, False)
    row, head, dim = t.stride()
    if dim != 1:
        _refuse_tensor(name, t, dtype, shape, dev, False)
    return t.data_ptr(), row, head


def _table(t, rows, dev):
    """(pointer, columns, stride) of a block table; its rows may lie apart."""
    if len(t.shape) != 2 or t.shape[0] != rows:
        _refuse("block_table: %d rows wanted, not %s", rows, tuple(t.shape))
    cols, stride = t.shape[1], t.stride()
    if stride[1] != 1 and cols > 1:
        _refuse("block_table: the pages of a sequence have to be adjacent")
    if t.dtype is not _torch.int32 or t.get_device() != dev:
        _refuse_tensor("block_table", t, _torch.int32, t.shape, dev, True)
    return t.data_ptr(), cols, max(stride[0], cols) if rows == 1 else stride[0]


def _differentiable(name):
    """A tensor that asks for a gradient: refused where one would be recorded, since none is."""
    if _torch is None:
        _need_torch()
    if _torch.is_grad_enabled():
        _refuse("%s requires a gradient, and the operator has none: call it under torch.no_grad(), or on %s.detach()", name, name)


def _duals():
    """Whether tensors may carry forward-mode tangents now."""
    if _torch is None:
        _need_torch()
    return _forward._current_level >= 0


def _no_tangent(**tensors):
    """Refuses tensors with a forward-mode tangent, which a result would be without: its derivative would be zero in silence."""
    for name, t in tensors.items():
        if t is not None and _forward.unpack_dual(t).tangent is not None:
            _refuse("%s has a tangent, and the operator has no forward-mode derivative: call it on torch.autograd.forward_ad.unpack_dual(%s).primal", name, name)


def _gpu(name, t):
    dev = t.get_device()
    if dev < 0:
        _refuse("%s is on %s, not on a GPU", name, t.device)
    return dev


def _pool(pool):
    """(pointer, pages, KV heads, head_dim, GPU)."""
    if _torch is None:
        _need_torch()
    if len(pool.shape) != 3 or pool.shape[2] not in (544, 1088, 2176):
        _refuse("pool: [pages][KV heads][17 * head_dim] wanted for a head_dim of 32, 64 or 128, not %s", tuple(pool.shape))
    dev = _gpu("pool", pool)
    pages, heads, size = pool.shape
    return _ptr("pool", pool, _torch.uint8, pool.shape, dev), pages, heads, size // 17, dev


def _bytes(pack, *fields):
    try:
        return pack(*fields)
    except struct.error as e:
        _refuse("an argument is outside its type's range: %s", e)


def _enqueue(call, dev, pack, *fields):
    """Call with the fields' struct, the stream that torch works on for GPU `dev` last; that GPU is the current one meanwhile."""
    if _torch._C._cuda_getDevice() == dev:                   # (torch.cuda.current_device() makes sure first that there is a GPU; the tensors are on it)
        return _check(None, call(_bytes(pack, *fields, _torch._C._cuda_getCurrentRawStream(dev))))
    with _torch.cuda.device(dev):
        return _check(None, call(_bytes(pack, *fields, _torch._C._cuda_getCurrentRawStream(dev))))


def april_cache_block_bytes(head_dim: int) -> int:
    return _check(None, load_library().april_cache_block_bytes(head_dim))


def make_cache_pool(n_pages: int, n_kv_heads: int, head_dim: int, device="cuda"):
    """A pool of n_pages pages of 16 tokens, uninitialised: nothing reads what has not been stored."""
    if _torch is None:
        _need_torch()
    return _torch.empty((n_pages, n_kv_heads, april_cache_block_bytes(head_dim)), dtype=_torch.uint8, device=device)


def april_cache_extend(lens, new_lens, block_table, free_pages, free_top, n_rows: int, out: Optional[Sequence] = None) -> CacheTables:
    """Tables of one iteration from the requests' lengths: sequences of new_lens < 0 give their pages back, the others grow.

    lens, new_lens [n_seqs], free_pages [n_pages], free_top [1]: int32; block_table [n_seqs, max_pages]: int32, in place, as
    free_pages.  out: an earlier call's result (or six tensors in its order) to write into; its lens and free_top may be
    the arguments themselves.
    """
    if _torch is None:
        _need_torch()
    i32 = _torch.int32
    if n_rows < 0:
        _refuse("n_rows: %d is below zero", n_rows)
    dev = _gpu("lens", lens)
    if len(lens.shape) != 1 or len(free_pages.shape) != 1:
        _refuse("lens and free_pages: one dimension wanted")
    n, n_pages = lens.shape[0], free_pages.shape[0]
    table, cols, stride = _table(block_table, n, dev)
    if out is None:
        e = lambda size, t=i32: _torch.empty(size, dtype=t, device=lens.device)  # noqa: E731
        out = CacheTables(e(n), e(1), e(n + 1), e(n_rows, _torch.int64), e(n_rows), e(1))
    o_lens, o_top, q_start, slots, positions, status = out
    _enqueue(_call("april_cache_extend"), dev, _PACK_EXTEND, n, cols, n_pages, n_rows, stride, _ptr("lens", lens, i32, (n,), dev),
             _ptr("new_lens", new_lens, i32, (n,), dev), _ptr("free_top", free_top, i32, (1,), dev), table,
             _ptr("free_pages", free_pages, i32, (n_pages,), dev), _ptr("out.lens", o_lens, i32, (n,), dev), _ptr("out.free_top", o_top, i32, (1,), dev),
             _ptr("out.q_start", q_start, i32, (n + 1,), dev), _ptr("out.slot_map", slots, _torch.int64, (n_rows,), dev),
             _ptr("out.positions", positions, i32, (n_rows,), dev), _ptr("out.status", status, i32, (1,), dev))
    return out if isinstance(out, CacheTables) else CacheTables(*out)


def april_cache_append(pool, k, v, slot_map, k_values=None, v_values=None) -> None:
    """Store k and v [n_rows, n_kv_heads, head_dim] (bf16 or fp32) in the pool at slot_map [n_rows] (int64); rows whose slot lies
    outside the pool are left out.  k_values, v_values: contiguous, of k's type: what the cache now stands for.  Not differentiable: refused
    where autograd would record a gradient of one of them."""
    if k.requires_grad:
        _differentiable("k")
    if v.requires_grad:
        _differentiable("v")
    if k_values is not None and k_values.requires_grad:
        _differentiable("k_values")
    if v_values is not None and v_values.requires_grad:
        _differentiable("v_values")
    if _duals():
        _no_tangent(k=k, v=v, k_values=k_values, v_values=v_values)
    p, pages, heads, dh, dev = _pool(pool)
    t = k.dtype
    if t is not _torch.bfloat16 and t is not _torch.float32:
        _refuse("k: bfloat16 or float32 wanted, not %s", t)
    if len(slot_map.shape) != 1:
        _refuse("slot_map: one dimension wanted")
    n = slot_map.shape[0]
    shape = (n, heads, dh)
    kp, k_row, k_head = _rows("k", k, t, shape, dev)
    vp, v_row, v_head = _rows("v", v, t, shape, dev)
    _enqueue(_call("april_cache_append"), dev, _PACK_APPEND, pages, heads, dh, n, APRIL_DTYPE_BF16 if t is _torch.bfloat16 else APRIL_DTYPE_FP32, 0,
             k_row, k_head, v_row, v_head, kp, vp, 0 if k_values is None else _ptr("k_values", k_values, t, shape, dev),
             0 if v_values is None else _ptr("v_values", v_values, t, shape, dev), _ptr("slot_map", slot_map, _torch.int64, (n,), dev), p)


def april_cache_attention(q, pool, block_table, lens, max_len: int, *, q_start=None, max_q: int = 1, scale: float = 0.0, out=None, lse=None,
                          workspace=None):
    """Causal attention of q [n_rows, n_q_heads, head_dim] (bf16) over the cache: rows q_start[b] .. q_start[b + 1] - 1 are the last tokens
    of sequence b (q_start None: row b).  lens [n_seqs]: tokens in the cache, those of the rows included; max_len, max_q: bounds on
    lens and on a sequence's rows.  lse: fp32 [n_rows, n_q_heads], written if given.  Returns out (rows of no sequence are left as
    they were; in a new `out` they are undefined).  Not differentiable: refused where autograd would record a gradient of q,
    out or lse."""
    if q.requires_grad:
        _differentiable("q")
    if out is not None and out.requires_grad:
        _differentiable("out")
    if lse is not None and lse.requires_grad:
        _differentiable("lse")
    if _duals():
        _no_tangent(q=q, out=out, lse=lse)
    p, pages, heads, dh, dev = _pool(pool)
    bf16, i32 = _torch.bfloat16, _torch.int32
    shape = q.shape
    if len(shape) != 3 or shape[2] != dh or len(lens.shape) != 1:
        _refuse("q: [rows][heads][%d] wanted, not %s, and lens of one dimension", dh, tuple(shape))
    n, (rows, q_heads, _) = lens.shape[0], shape
    qp, q_row, q_head = _rows("q", q, bf16, shape, dev)
    table, cols, stride = _table(block_table, n, dev)
    if out is None:
        out = _torch.empty(shape, dtype=bf16, device=q.device)
    op, o_row, o_head = _rows("out", out, bf16, shape, dev)
    fields = (q_heads, heads, dh, pages, n, cols, rows, max_q, max_len, scale, stride, q_row, q_head, o_row, o_head, qp, p, table,
              _ptr("lens", lens, i32, (n,), dev), 0 if q_start is None else _ptr("q_start", q_start, i32, (n + 1,), dev), op,
              0 if lse is None else _ptr("lse", lse, _torch.float32, (rows, q_heads), dev))
    need = _check(None, _call("april_cache_attention_workspace")(_bytes(_PACK_ATTENTION, *fields, 0, 0, 0)))
    if workspace is None:
        workspace = _torch.empty(need, dtype=_torch.uint8, device=q.device) if need else None
    elif len(workspace.shape) != 1:
        _refuse("workspace: one dimension wanted")
    size = 0 if workspace is None else workspace.shape[0]
    _enqueue(_call("april_cache_attention"), dev, _PACK_ATTENTION, *fields, _ptr("workspace", workspace, _torch.uint8, (size,), dev) if size else 0, size)
    return out


# ---------------------------------------------------------------------------
# Operators that score rollouts and train on them, on torch tensors of one GPU, each with its gradient: where autograd would record one of
# logits, table, x, packed or weights, the result carries it, else the call is the library's alone.  They run on torch's current stream and may
# be captured into a graph.  Forward-mode derivatives there are none: a tensor with a tangent is refused.  What torch itself asks of a captured
# backward pass holds here too: no autograd graph of the same leaf tensors that was recorded outside the capture may be alive meanwhile.  The
# gradients' own calls (april_*_grad) have no such bound.
# ---------------------------------------------------------------------------
class Logprobs(NamedTuple):
    """What april_logprobs leaves, see april.h (None: not asked for)."""
    logprob: object
    entropy: object
    lse: object
    top_logprobs: object
    top_ids: object
    norm: object


class ExpertRows(NamedTuple):
    """What april_expert_sort leaves, see april.h (int32)."""
    starts: object
    source: object
    position: object


_functions = {}             # autograd's classes, made by the first call that records a gradient (torch is imported late)


def _dtype(name, t):
    if t is _torch.bfloat16:
        return APRIL_DTYPE_BF16
    if t is _torch.float32:
        return APRIL_DTYPE_FP32
    _refuse("%s: bfloat16 or float32 wanted, not %s", name, t)


def _matrix(name, t, dtype, shape, dev):
    """(pointer, stride of rows) of a tensor [rows][columns] whose rows may lie apart or be one."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        _refuse_tensor(name, t, dtype, shape, dev, True)
    row, col = t.stride()
    if col != 1 and shape[1] > 1:
        _refuse("%s: the elements of a row have to be adjacent", name)
    return t.data_ptr(), row


def _first(name, t):
    """(rows, columns, GPU, type, pointer, stride of rows) of a call's first matrix.  (One call: in a backward pass, on a thread of torch's, each costs twice its time.)"""
    shape, of, dev = t.shape, t.dtype, t.get_device()
    if len(shape) != 2 or dev < 0:
        _two(name, t)
        _gpu(name, t)
    n, d = shape
    row, col = t.stride()
    if col != 1 and d > 1:
        _refuse("%s: the elements of a row have to be adjacent", name)
    return n, d, dev, APRIL_DTYPE_BF16 if of is _torch.bfloat16 else _dtype(name, of), t.data_ptr(), row


def _index(name, t, shape, dev):
    """(pointer, bits) of a contiguous tensor of int32 or int64."""
    if t.dtype is _torch.int64:
        return _ptr(name, t, _torch.int64, shape, dev), 64
    return _ptr(name, t, _torch.int32, shape, dev), 32


def _float_ptr(name, t, shape, dev):
    return 0 if t is None else _ptr(name, t, _torch.float32, shape, dev)


def _two(name, t):
    if _torch is None:
        _need_torch()
    if len(t.shape) != 2:
        _refuse("%s: two dimensions wanted, not %s", name, tuple(t.shape))
    return t.shape


def _records(**tensors):
    """Whether autograd would record a gradient of one of them (one with a tangent is refused)."""
    if _duals():
        _no_tangent(**tensors)
    for t in tensors.values():
        if t is not None and t.requires_grad:
            return _torch.is_grad_enabled()
    return False


def _no_gradient(**tensors):
    if _duals():
        _no_tangent(**tensors)
    for name, t in tensors.items():
        if t is not None and t.requires_grad:
            _differentiable(name)


def _wrote(out):
    """The caller's `out`, which autograd now knows to be changed: where it was kept for a gradient, that backward pass is refused."""
    _torch.autograd.graph.increment_version(out)
    return out


def _space(call, pack, fields, device):
    """(tensor, pointer, bytes) of the workspace that the call asks for."""
    need = _check(None, _call(call)(_bytes(pack, *fields, 0, 0, 0)))
    space = _torch.empty(need, dtype=_torch.uint8, device=device) if need else None
    return space, (space.data_ptr() if need else 0), need


def _function(name):
    """autograd's class of an operator.  (A backward pass checks what it gets back of its tensors: hooks for saved ones may return others.)"""
    if not _functions:
        t = _torch
        once = t.autograd.function.once_differentiable
        whole = lambda g: None if g is None else g.contiguous()  # noqa: E731
        adjacent = lambda g: g if g.stride(1) == 1 or g.shape[1] == 1 else g.contiguous()  # noqa: E731

        class AprilLogprobs(t.autograd.Function):
            @staticmethod
            def forward(ctx, logits, tokens, temperature, entropy, lse, top):
                got = _logprobs(logits, tokens, temperature, entropy, lse, top)
                ctx.set_materialize_grads(False)
                ctx.mark_non_differentiable(*(x for x in got[3:] if x is not None))
                ctx.save_for_backward(logits, tokens, got.norm, got.entropy)
                ctx.temperature = temperature
                return tuple(got)

            @staticmethod
            @once
            def backward(ctx, g, h, z, *_):
                if g is None and h is None and z is None:
                    return (None,) * 6
                if _forward._current_level >= 0:
                    _no_tangent(grad_logprob=g, grad_entropy=h, grad_lse=z)
                logits, tokens, norm, entropy = ctx.saved_tensors
                return _logprobs_grad(logits, tokens, norm, None if h is None else entropy, whole(g), whole(h), whole(z), ctx.temperature), None, None, None, None, None

        class AprilEmbed(t.autograd.Function):
            @staticmethod
            def forward(ctx, table, tokens, scale, dtype):
                ctx.save_for_backward(tokens)
                ctx.of = table.shape[0], table.dtype, scale
                return _embed(table, tokens, scale, dtype, None)

            @staticmethod
            @once
            def backward(ctx, g):
                vocab, dtype, scale = ctx.of
                return april_embed_grad(adjacent(g), *ctx.saved_tensors, vocab, scale=scale, dtype=dtype), None, None, None

        class AprilExpertGather(t.autograd.Function):
            @staticmethod
            def forward(ctx, x, source, position):
                ctx.save_for_backward(position)
                return _expert_gather(x, source, position, None)

            @staticmethod
            @once
            def backward(ctx, g):
                if _forward._current_level >= 0:
                    _no_tangent(grad_out=g)
                position, = ctx.saved_tensors
                return _combine(adjacent(g), position, None, None), None, None

        class AprilExpertCombine(t.autograd.Function):
            @staticmethod
            def forward(ctx, packed, source, position, weights):
                # (the values of packed matter to the weights' gradient alone)
                ctx.save_for_backward(packed if ctx.needs_input_grad[3] else None, source, position, weights)
                return _expert_combine(packed, source, position, weights, None)

            @staticmethod
            @once
            def backward(ctx, g):
                if _forward._current_level >= 0:
                    _no_tangent(grad_out=g)
                packed, source, position, weights = ctx.saved_tensors
                of_packed, _, _, of_weights = ctx.needs_input_grad
                of_packed, of_weights = _combine_grad(adjacent(g), packed, source, position, weights, of_packed, of_weights)
                return of_packed, None, None, of_weights

        _functions.update(logprobs=AprilLogprobs, embed=AprilEmbed, gather=AprilExpertGather, combine=AprilExpertCombine)
    return _functions[name]


def _logprobs(logits, tokens, temperature, entropy, lse, top):
    n, vocab, dev, dtype, p, row = _first("logits", logits)
    if top < 0:
        _refuse("top: %d is below zero", top)
    tp, bits = _index("tokens", tokens, (n,), dev)
    empty, f32, device = _torch.empty, _torch.float32, logits.device
    logprob, norm = empty(n, dtype=f32, device=device), empty((n, 2), dtype=f32, device=device)
    entropy = empty(n, dtype=f32, device=device) if entropy else None
    lse = empty(n, dtype=f32, device=device) if lse else None
    best = empty((n, top), dtype=f32, device=device) if top else None
    ids = empty((n, top), dtype=_torch.int32, device=device) if top else None
    fields = (n, vocab, dtype, bits, top, temperature, row, p, tp, logprob.data_ptr(), 0 if entropy is None else entropy.data_ptr(), 0 if lse is None else lse.data_ptr(),
              norm.data_ptr(), best.data_ptr() if top else 0, ids.data_ptr() if top else 0)
    space, at, need = _space("april_logprobs_workspace", _PACK_LOGPROBS, fields, device)
    _enqueue(_call("april_logprobs"), dev, _PACK_LOGPROBS, *fields, at, need)
    return Logprobs(logprob, entropy, lse, best, ids, norm)


def april_logprobs(logits, tokens, *, temperature: float = 1.0, entropy: bool = False, lse: bool = False, top: int = 0) -> Logprobs:
    """log softmax(logits / temperature)[token] of each row of logits [n_rows, vocab] (bf16 or fp32), tokens [n_rows] (int32 or int64; below zero: a
    padding row, zeros), and as asked for the entropy, the log of the sum of exponentials, and the `top` (at most 64) most likely tokens with their
    log-probabilities.  Differentiable: logprob, entropy, lse."""
    if _records(logits=logits):
        return Logprobs(*_function("logprobs").apply(logits, tokens, temperature, entropy, lse, top))
    return _logprobs(logits, tokens, temperature, entropy, lse, top)


def _logprobs_grad(logits, tokens, norm, entropy, g, h, z, temperature, out=None):
    """(g, h and z are checked.)"""
    n, vocab, dev, dtype, p, row = _first("logits", logits)
    f32, i64 = _torch.float32, _torch.int64
    wide = tokens.dtype is i64
    tp, np_ = _ptr("tokens", tokens, i64 if wide else _torch.int32, (n,), dev), _ptr("made.norm", norm, f32, (n, 2), dev)
    if out is None:
        out = _torch.empty((n, vocab), dtype=logits.dtype, device=logits.device)
        op, o_row = out.data_ptr(), vocab
    else:
        op, o_row = _matrix("out", out, logits.dtype, (n, vocab), dev)
    _enqueue(_call("april_logprobs_grad"), dev, _PACK_LOGPROBS_GRAD, n, vocab, dtype, 64 if wide else 32, temperature, 0, row, o_row, p, tp, np_,
             0 if entropy is None else _ptr("made.entropy", entropy, f32, (n,), dev), 0 if g is None else g.data_ptr(), 0 if h is None else h.data_ptr(),
             0 if z is None else z.data_ptr(), op)
    return out


def april_logprobs_grad(logits, tokens, made: Logprobs, *, grad_logprob=None, grad_entropy=None, grad_lse=None, temperature: float = 1.0, out=None):
    """Gradient of the logits, of their type.  made: april_logprobs' of the same arguments (its norm, and its entropy for grad_entropy); grad_*
    [n_rows]: fp32, None is zero.  out may be the logits themselves, which are then overwritten.  Not differentiable."""
    _no_gradient(logits=logits, grad_logprob=grad_logprob, grad_entropy=grad_entropy, grad_lse=grad_lse, out=out)
    n, dev = _two("logits", logits)[0], _gpu("logits", logits)
    if grad_entropy is not None and made.entropy is None:
        _refuse("grad_entropy: april_logprobs was not asked for the entropy")
    for name, t in (("grad_logprob", grad_logprob), ("grad_entropy", grad_entropy), ("grad_lse", grad_lse)):
        _float_ptr(name, t, (n,), dev)
    got = _logprobs_grad(logits, tokens, made.norm, None if grad_entropy is None else made.entropy, grad_logprob, grad_entropy, grad_lse, temperature, out)
    return got if out is None else _wrote(out)


def _embed(table, tokens, scale, dtype, out):
    vocab, d = _two("table", table)
    dev, of = _gpu("table", table), _dtype("table", table.dtype)
    if len(tokens.shape) != 1:
        _refuse("tokens: one dimension wanted, not %s", tuple(tokens.shape))
    n = tokens.shape[0]
    if out is None:
        out = _torch.empty((n, d), dtype=table.dtype if dtype is None else dtype, device=table.device)
    elif dtype is not None and out.dtype is not dtype:
        _refuse("out: %s wanted, not %s", dtype, out.dtype)
    to = _dtype("out", out.dtype)
    p, row = _matrix("table", table, table.dtype, (vocab, d), dev)
    op, o_row = _matrix("out", out, out.dtype, (n, d), dev)
    tp, bits = _index("tokens", tokens, (n,), dev)
    _enqueue(_call("april_embed"), dev, _PACK_EMBED, n, vocab, d, of, to, bits, scale, 0, row, o_row, p, tp, op)
    return out


def april_embed(table, tokens, *, scale: float = 1.0, dtype=None, out=None):
    """scale * table[tokens] [n_rows, d] (bf16 or fp32, as dtype or out says; else of the table's type) for tokens [n_rows] (int32 or int64; below zero:
    padding, zeros).  Differentiable in the table, but not into an `out`."""
    if _records(table=table, out=out):
        if out is not None:
            _differentiable("table" if table.requires_grad else "out")
        return _function("embed").apply(table, tokens, scale, dtype)
    got = _embed(table, tokens, scale, dtype, out)
    return got if out is None else _wrote(out)


def april_embed_grad(grad_out, tokens, vocab: int, *, scale: float = 1.0, dtype=None, out=None, accumulate: bool = False):
    """Gradient [vocab, d] of april_embed's table (of type dtype or out's; else of grad_out's) for the gradient [n_rows, d] of its result.  accumulate: added to
    `out`, of which the rows of no token are not touched.  Not differentiable."""
    _no_gradient(grad_out=grad_out, out=out)
    given = out is not None
    n, d = _two("grad_out", grad_out)
    dev, of = _gpu("grad_out", grad_out), _dtype("grad_out", grad_out.dtype)
    if out is None:
        if accumulate:
            _refuse("accumulate: no `out` to add to")
        if vocab < 1:
            _refuse("vocab: %d is below one", vocab)
        out = _torch.empty((vocab, d), dtype=grad_out.dtype if dtype is None else dtype, device=grad_out.device)
    elif dtype is not None and out.dtype is not dtype:
        _refuse("out: %s wanted, not %s", dtype, out.dtype)
    to = _dtype("out", out.dtype)
    p, row = _matrix("grad_out", grad_out, grad_out.dtype, (n, d), dev)
    op, o_row = _matrix("out", out, out.dtype, (vocab, d), dev)
    tp, bits = _index("tokens", tokens, (n,), dev)
    fields = n, vocab, d, of, to, bits, scale, 1 if accumulate else 0, row, o_row, p, tp, op
    space, at, need = _space("april_embed_grad_workspace", _PACK_EMBED_GRAD, fields, grad_out.device)
    _enqueue(_call("april_embed_grad"), dev, _PACK_EMBED_GRAD, *fields, at, need)
    return _wrote(out) if given else out


def april_expert_sort(ids, n_experts: int, *, align: int = 1) -> ExpertRows:
    """The assignments ids [n_rows, k] (int32 or int64; outside 0..n_experts - 1: left out) sorted by expert, each expert's packed rows from a multiple of
    `align` on.  The packed arrays have as many rows as the largest shares of the experts could take: source.shape[0]."""
    n, k = _two("ids", ids)
    dev = _gpu("ids", ids)
    p, bits = _index("ids", ids, (n, k), dev)
    if n_experts < 1 or align < 1:
        _refuse("n_experts and align: at least one wanted")
    m = (n * k + min(n_experts, n * k) * (align - 1)) // align * align
    e = lambda *shape: _torch.empty(shape, dtype=_torch.int32, device=ids.device)  # noqa: E731
    rows = ExpertRows(e(n_experts + 1), e(m), e(n, k))
    fields = n, k, n_experts, align, m, bits, p, rows.starts.data_ptr(), rows.source.data_ptr(), rows.position.data_ptr()
    space, at, need = _space("april_expert_sort_workspace", _PACK_EXPERT_SORT, fields, ids.device)
    _enqueue(_call("april_expert_sort"), dev, _PACK_EXPERT_SORT, *fields, at, need)
    return rows


def _packed_rows(source, dev):
    """(pointer, packed rows)."""
    if len(source.shape) != 1:
        _refuse("rows.source: one dimension wanted")
    m = source.shape[0]
    return _ptr("rows.source", source, _torch.int32, (m,), dev), m


def _positions(position, dev):
    """(pointer, rows, experts of a row)."""
    shape = position.shape
    if len(shape) != 2:
        _two("rows.position", position)
    return (_ptr("rows.position", position, _torch.int32, shape, dev), *shape)


def _expert_gather(x, source, position, out):
    rows, d, dev, dtype, p, row = _first("x", x)
    sp, m = _packed_rows(source, dev)
    at, n, k = _positions(position, dev)
    if rows != n:
        _refuse("x: %d rows wanted, not %d", n, rows)
    if out is None:
        out = _torch.empty((m, d), dtype=x.dtype, device=x.device)
        op, o_row = out.data_ptr(), d
    else:
        op, o_row = _matrix("out", out, x.dtype, (m, d), dev)
    _enqueue(_call("april_expert_gather"), dev, _PACK_EXPERT_GATHER, n, k, d, m, dtype, 0, row, o_row, p, sp, at, op)
    return out


def april_expert_gather(x, rows: ExpertRows, *, out=None):
    """The tokens' rows x [n_rows, d] (bf16 or fp32) in the order of their experts; packed rows of no assignment are zeros.  Differentiable in x, but not
    into an `out`."""
    if _records(x=x, out=out):
        if out is not None:
            _differentiable("x" if x.requires_grad else "out")
        return _function("gather").apply(x, rows.source, rows.position)
    got = _expert_gather(x, rows.source, rows.position, out)
    return got if out is None else _wrote(out)


def _combine(packed, position, weights, out):
    m, d, dev, dtype, p, row = _first("packed", packed)
    at, n, k = _positions(position, dev)
    if out is None:
        out = _torch.empty((n, d), dtype=packed.dtype, device=packed.device)
        op, o_row = out.data_ptr(), d
    else:
        op, o_row = _matrix("out", out, packed.dtype, (n, d), dev)
    _enqueue(_call("april_expert_combine"), dev, _PACK_EXPERT_COMBINE, n, k, d, m, dtype, 0, row, o_row, p, at,
             0 if weights is None else _ptr("weights", weights, _torch.float32, (n, k), dev), op)
    return out


def _expert_combine(packed, source, position, weights, out):
    if _two("packed", packed)[0] != _packed_rows(source, _gpu("packed", packed))[1]:
        _refuse("packed: %d rows wanted, not %d", source.shape[0], packed.shape[0])
    return _combine(packed, position, weights, out)


def april_expert_combine(packed, rows: ExpertRows, weights=None, *, out=None):
    """What the experts made of their rows, packed [source.shape[0], d] (bf16 or fp32), summed for each token by weights [n_rows, k] (fp32; None: 1), in the order
    of the token's experts.  Differentiable in packed and weights, but not into an `out`."""
    if _records(packed=packed, weights=weights, out=out):
        if out is not None:
            _differentiable("packed" if packed.requires_grad else "weights" if weights is not None and weights.requires_grad else "out")
        return _function("combine").apply(packed, rows.source, rows.position, weights)
    got = _expert_combine(packed, rows.source, rows.position, weights, out)
    return got if out is None else _wrote(out)


def _combine_grad(grad_out, packed, source, position, weights, of_packed, of_weights):
    """(packed may be None where of_weights is false.)"""
    rows, d, dev, dtype, g, row = _first("grad_out", grad_out)
    sp, m = _packed_rows(source, dev)
    at, n, k = _positions(position, dev)
    if rows != n:
        _refuse("grad_out: %d rows wanted, not %d", n, rows)
    p, p_row = (0, 0) if packed is None else _matrix("packed", packed, grad_out.dtype, (m, d), dev)
    wp = 0 if weights is None else _ptr("weights", weights, _torch.float32, (n, k), dev)
    g_packed = _torch.empty((m, d), dtype=grad_out.dtype, device=grad_out.device) if of_packed else None
    g_weights = _torch.empty((n, k), dtype=_torch.float32, device=grad_out.device) if of_weights else None
    _enqueue(_call("april_expert_combine_grad"), dev, _PACK_EXPERT_COMBINE_GRAD, n, k, d, m, dtype, 0, row, p_row, d, g, p, sp, at, wp,
             g_packed.data_ptr() if of_packed else 0, g_weights.data_ptr() if of_weights else 0)
    return g_packed, g_weights


def april_expert_combine_grad(grad_out, packed, rows: ExpertRows, weights=None, *, of_packed: bool = True, of_weights: bool = True):
    """(gradient of packed, gradient of weights) for the gradient [n_rows, d] of april_expert_combine's result; None where not asked for.  Not differentiable."""
    _no_gradient(grad_out=grad_out, packed=packed, weights=weights)
    return _combine_grad(grad_out, packed, rows.source, rows.position, weights, of_packed, of_weights)


# ---------------------------------------------------------------------------
# helpers to build the configuration and weight table from the synthetic inputs
# ---------------------------------------------------------------------------
def make_cfg(shape, *, max_inflight, max_ctx, sampler=APRIL_SAMPLER_GREEDY, top_k=1, temperature=1.0, seed=0,
             eos_token=-1, debug_logits=False, kv_pool_bytes=0, stream=None, top_p=0.0,
             logprobs=False, n_samples_per_prompt=0, pausable=False) -> april_model_cfg:
    return april_model_cfg(
        shape.n_layers, shape.d_model, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.d_ffn,
        shape.vocab, shape.n_experts, shape.experts_per_tok, shape.d_expert_ffn, shape.dtype,
        shape.rope_theta, shape.rms_eps, 16, kv_pool_bytes, max_inflight, max_ctx, sampler, top_k,
        temperature, seed, eos_token, 1 if debug_logits else 0, top_p, 1 if logprobs else 0,
        n_samples_per_prompt, 1 if pausable else 0, stream)


def pack_weights(shape, weights_fp32: Dict[str, np.ndarray]) -> Dict[str, np.ndarray]:
    """fp32-valued arrays -> the element type the library expects: matrices and the
    embedding as bf16 bit patterns for a bf16 model (the values are already exactly
    representable), gains always float32."""
    out = {}
    for name, a in weights_fp32.items():
        is_gain = name.startswith(("attn_norm", "mlp_norm", "final_norm"))
        if shape.dtype != APRIL_DTYPE_FP32 and not is_gain:
            bits = np.ascontiguousarray(a, dtype=np.float32).view(np.uint32)
            if np.any(bits & np.uint32(0xFFFF)):
                raise ValueError(f"{name}: values are not exactly representable in bf16")
            out[name] = (bits >> np.uint32(16)).astype(np.uint16)
        else:
            out[name] = np.ascontiguousarray(a, dtype=np.float32)
    return out
