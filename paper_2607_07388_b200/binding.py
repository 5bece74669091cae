"""ctypes binding of libtfe.so: the same entry points as include/tfe.h.

Argument marshalling only -- every step of the path runs in the library's CUDA
kernels.  Device buffers are ``torch`` CUDA tensors (or raw integer addresses);
host buffers are numpy arrays or pinned CPU tensors.  Loading fails loudly when
the shared library has not been built; there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("TFE_LIB") or os.path.join(_HERE, "libtfe.so")   # TFE_LIB: a tuning build

TFE_OK = 0
STATUS_NAMES = ["TFE_OK", "TFE_ERR_INVALID_ARG", "TFE_ERR_DUPLICATE_PHRASE", "TFE_ERR_KEY_COLLISION",
                "TFE_ERR_CAPACITY", "TFE_ERR_SLOT_RANGE", "TFE_ERR_UNKNOWN_PHRASE",
                "TFE_ERR_ALREADY_RESIDENT", "TFE_ERR_MISS_OVERFLOW", "TFE_ERR_PROBE_LIMIT",
                "TFE_ERR_CUDA", "TFE_ERR_INTERNAL"]
(TFE_ERR_INVALID_ARG, TFE_ERR_DUPLICATE_PHRASE, TFE_ERR_KEY_COLLISION, TFE_ERR_CAPACITY,
 TFE_ERR_SLOT_RANGE, TFE_ERR_UNKNOWN_PHRASE, TFE_ERR_ALREADY_RESIDENT, TFE_ERR_MISS_OVERFLOW,
 TFE_ERR_PROBE_LIMIT, TFE_ERR_CUDA, TFE_ERR_INTERNAL) = range(1, 12)
POLICY_LONGEST, POLICY_ALL = 0, 1
GATE_CONST, GATE_COSINE = 0, 1
HIDDEN_BF16, HIDDEN_F32 = 0, 1
NO_PHRASE = 0xFFFFFFFF

EXPORTS = ["tfe_index_build", "tfe_index_build_device", "tfe_cache_install", "tfe_cache_install_device", "tfe_lookup_inject", "tfe_lookup_inject_host",
           "tfe_miss_list", "tfe_miss_list_device", "tfe_destroy", "tfe_status_string",
           "tfe_last_cuda_error", "tfe_index_geometry", "tfe_phrase_key64", "tfe_home_bucket",
           "tfe_launch_geometry", "tfe_set_tuning", "tfe_lookup_inject_noalloc", "tfe_prefetch_candidates",
           "tfe_cache_policy_enable", "tfe_cache_select_victims", "tfe_cache_select_victims_device",
           "tfe_cache_stats", "tfe_head_create", "tfe_head_destroy", "tfe_head_topk", "tfe_head_buffers",
           "tfe_head_status", "tfe_head_geometry", "tfe_mine_ngrams", "tfe_mine_workspace_bytes", "tfe_assign_residency", "tfe_stream_copy",
           "tfe_cache_select_tuning", "tfe_distill_forward", "tfe_distill_backward", "tfe_sample_tokens",
           "tfe_quantize_fp8", "tfe_quantize_fp8_ld", "tfe_matmul_fp8", "tfe_matmul_fp8_status", "tfe_matmul_fp8_give_up",
           "tfe_xent_forward_workspace_bytes", "tfe_xent_backward_workspace_bytes", "tfe_xent_forward", "tfe_xent_backward",
           "tfe_xent_status", "tfe_xent_give_up", "tfe_inject_norm_forward", "tfe_inject_norm_backward", "tfe_inject_norm_workspace_bytes",
           "tfe_grad_norm", "tfe_clip_grad_norm", "tfe_clip_workspace_bytes", "tfe_describe_tensors"]


class TfeConfig(C.Structure):
    _fields_ = [("d", C.c_int32), ("vocab", C.c_int32), ("n_orders", C.c_int32),
                ("orders", C.c_int32 * 4), ("n_phrases", C.c_int64), ("gpu_slots", C.c_int64),
                ("load_factor", C.c_float), ("hidden_dtype", C.c_int32),
                ("max_kicks", C.c_int32)]


class TfeInjectParams(C.Structure):
    _fields_ = [("policy", C.c_int32), ("gate", C.c_int32), ("lam", C.c_float)]


class TfePrefetchParams(C.Structure):
    _fields_ = [("benefit_host", C.c_float), ("benefit_ssd", C.c_float), ("budget", C.c_int32)]


class TfeSampleParams(C.Structure):
    _fields_ = [("temperature", C.c_void_p), ("top_k", C.c_void_p), ("top_p", C.c_void_p), ("min_p", C.c_void_p)]


class TfeInjectNormParams(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("Q", C.c_int32), ("d", C.c_int32), ("gate_kind", C.c_int32), ("sigmoid", C.c_int32),
                ("weight_dtype", C.c_int32), ("h", C.c_void_p), ("m", C.c_void_p), ("gate", C.c_void_p), ("ld_h", C.c_int64),
                ("ld_m", C.c_int64), ("ld_gate", C.c_int64), ("post_weight", C.c_void_p), ("next_weight", C.c_void_p),
                ("lam", C.c_float), ("eps", C.c_float)]


class TfeInjectNormGrads(C.Structure):
    _fields_ = [("grad_out", C.c_void_p), ("grad_normed", C.c_void_p), ("ld_grad_out", C.c_int64), ("ld_grad_normed", C.c_int64),
                ("grad_h", C.c_void_p), ("grad_m", C.c_void_p), ("grad_gate", C.c_void_p), ("ld_grad_h", C.c_int64),
                ("ld_grad_m", C.c_int64), ("ld_grad_gate", C.c_int64), ("grad_post", C.c_void_p), ("grad_next", C.c_void_p)]


class TfeError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        detail = ""
        if status == TFE_ERR_CUDA:
            detail = ": " + lib().tfe_last_cuda_error().decode()
        super().__init__(f"{where}: {STATUS_NAMES[status]} ({lib().tfe_status_string(status).decode()}){detail}")


_lib = None


def lib() -> C.CDLL:
    """The loaded library.  Raises if it is not built: this package has no other compute path."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2607_07388_b200.build` (needs nvcc); there is no fallback")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64
        L.tfe_index_build.argtypes = [C.POINTER(TfeConfig), vp, vp, vp, vp, vp, C.POINTER(vp)]
        L.tfe_index_build_device.argtypes = L.tfe_index_build.argtypes
        L.tfe_cache_install.argtypes = [vp, i32, vp, vp, vp, vp]
        L.tfe_cache_install_device.argtypes = [vp, i32, vp, vp, vp, vp, vp, vp]
        L.tfe_lookup_inject.argtypes = [vp, vp, i32, i32, i32, vp, vp, C.POINTER(TfeInjectParams), vp, vp, vp, vp]
        L.tfe_lookup_inject_host.argtypes = L.tfe_lookup_inject.argtypes
        L.tfe_lookup_inject_noalloc.argtypes = [vp, vp, i32, i32, i32, vp, vp, C.POINTER(TfeInjectParams), vp, vp, vp,
                                                vp, vp, vp, vp, vp]
        L.tfe_miss_list.argtypes = [vp, vp, vp, vp, i64, C.POINTER(i64), vp]
        L.tfe_prefetch_candidates.argtypes = [vp, vp, i32, i32, vp, vp, i32, vp, C.POINTER(TfePrefetchParams),
                                              vp, vp, vp, vp, vp, vp]
        L.tfe_miss_list_device.argtypes = [vp, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp)]
        L.tfe_destroy.argtypes = [vp]
        L.tfe_destroy.restype = None
        L.tfe_status_string.argtypes = [C.c_int]
        L.tfe_status_string.restype = C.c_char_p
        L.tfe_last_cuda_error.restype = C.c_char_p
        L.tfe_index_geometry.argtypes = [vp, C.POINTER(i64), C.POINTER(i64), C.POINTER(i64)]
        L.tfe_phrase_key64.argtypes = [i32, vp, i32, C.POINTER(i32)]
        L.tfe_phrase_key64.restype = u64
        L.tfe_home_bucket.argtypes = [u64, u64]
        L.tfe_home_bucket.restype = u64
        L.tfe_launch_geometry.argtypes = [vp, C.POINTER(i32), C.POINTER(i32), C.POINTER(i32)]
        L.tfe_set_tuning.argtypes = [vp, i32]
        L.tfe_cache_policy_enable.argtypes = [vp, vp]
        L.tfe_cache_select_victims.argtypes = [vp, i32, i32, vp, vp, C.POINTER(i32), vp]
        L.tfe_cache_select_victims_device.argtypes = [vp, C.POINTER(vp), C.POINTER(vp)]
        L.tfe_cache_stats.argtypes = [vp, vp, C.POINTER(C.c_uint32), vp]
        L.tfe_head_create.argtypes = [vp, i32, i32, i32, C.POINTER(vp)]
        L.tfe_head_destroy.argtypes = [vp]
        L.tfe_head_destroy.restype = None
        L.tfe_head_topk.argtypes = [vp, vp, i32, i32, vp, vp, vp]
        L.tfe_head_buffers.argtypes = [vp, C.POINTER(vp), C.POINTER(i64), C.POINTER(vp)]
        L.tfe_head_status.argtypes = [vp, C.POINTER(C.c_uint32), vp]
        L.tfe_head_geometry.argtypes = [vp, C.POINTER(i32), C.POINTER(i32), C.POINTER(i32)]
        L.tfe_mine_ngrams.argtypes = [vp, i64, i32, i32, vp, C.c_uint32, i64, vp, vp, vp, C.POINTER(i64), vp, vp, vp, i64, vp]
        L.tfe_mine_workspace_bytes.argtypes = [i64, i32]
        L.tfe_assign_residency.argtypes = [vp, i64, i64, C.c_uint32, vp, vp, vp]
        L.tfe_mine_workspace_bytes.restype = i64
        L.tfe_stream_copy.argtypes = [vp, vp, i64, vp]
        L.tfe_cache_select_tuning.argtypes = [vp, i32, i32, i32]
        f32 = C.c_float
        L.tfe_quantize_fp8.argtypes = [vp, i32, i32, i32, i64, i32, vp, vp, vp]
        L.tfe_quantize_fp8_ld.argtypes = [vp, i32, i32, i32, i64, i32, vp, i64, vp, vp]
        L.tfe_matmul_fp8.argtypes = [vp, i64, vp, i32, vp, i64, vp, i32, i32, vp, i32, i64, vp]
        L.tfe_matmul_fp8_status.argtypes = [C.POINTER(C.c_uint32), vp]
        L.tfe_matmul_fp8_give_up.argtypes = [i32]
        L.tfe_xent_forward_workspace_bytes.argtypes = L.tfe_xent_backward_workspace_bytes.argtypes = [i32, i32, i32]
        L.tfe_xent_forward_workspace_bytes.restype = L.tfe_xent_backward_workspace_bytes.restype = i64
        L.tfe_xent_forward.argtypes = [vp, i64, i32, vp, i64, i32, i32, vp, vp, vp, vp, i64, vp]
        L.tfe_xent_backward.argtypes = [vp, i64, i32, vp, i64, i32, i32, vp, vp, vp, vp, i64, vp, i64, vp, i64, vp]
        L.tfe_xent_status.argtypes = [C.POINTER(C.c_uint32), vp]
        L.tfe_xent_give_up.argtypes = [i32]
        L.tfe_inject_norm_forward.argtypes = [C.POINTER(TfeInjectNormParams), vp, i64, vp, i64, vp]
        L.tfe_inject_norm_backward.argtypes = [C.POINTER(TfeInjectNormParams), C.POINTER(TfeInjectNormGrads), vp, i64, vp]
        L.tfe_inject_norm_workspace_bytes.argtypes = [i32, i32]
        L.tfe_grad_norm.argtypes = [vp, vp, vp, i32, vp, vp, i64, vp]
        L.tfe_clip_grad_norm.argtypes = [vp, vp, vp, vp, i32, f32, vp, vp, i64, vp]
        L.tfe_clip_workspace_bytes.argtypes = [i32]
        L.tfe_describe_tensors.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp]
        L.tfe_inject_norm_workspace_bytes.restype = L.tfe_clip_workspace_bytes.restype = i64
        L.tfe_sample_tokens.argtypes = [vp, i32, i32, i32, i64, C.POINTER(TfeSampleParams), vp, vp, vp, vp]
        L.tfe_distill_forward.argtypes = [vp, i32, i32, i32, i64, vp, vp, i32, f32, vp, vp, vp]
        L.tfe_distill_backward.argtypes = [vp, i32, i32, i32, i64, vp, vp, i32, f32, vp, vp, vp, i64, vp]
        for name in ("tfe_index_build", "tfe_index_build_device", "tfe_cache_install", "tfe_cache_install_device", "tfe_lookup_inject", "tfe_lookup_inject_host",
                     "tfe_miss_list", "tfe_miss_list_device", "tfe_index_geometry", "tfe_launch_geometry",
                     "tfe_set_tuning", "tfe_lookup_inject_noalloc", "tfe_prefetch_candidates",
                     "tfe_cache_policy_enable", "tfe_cache_select_victims", "tfe_cache_select_victims_device",
                     "tfe_cache_stats", "tfe_head_create", "tfe_head_topk", "tfe_head_buffers", "tfe_head_status",
                     "tfe_head_geometry", "tfe_mine_ngrams", "tfe_assign_residency", "tfe_cache_select_tuning",
                     "tfe_distill_forward", "tfe_distill_backward", "tfe_sample_tokens", "tfe_quantize_fp8", "tfe_quantize_fp8_ld",
                     "tfe_matmul_fp8", "tfe_matmul_fp8_status", "tfe_matmul_fp8_give_up", "tfe_xent_forward", "tfe_xent_backward",
                     "tfe_xent_status", "tfe_xent_give_up", "tfe_inject_norm_forward", "tfe_inject_norm_backward", "tfe_grad_norm",
                     "tfe_clip_grad_norm"):
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def _addr(x):
    """Address of a device tensor, host tensor, numpy array, int or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if isinstance(x, np.ndarray):
        assert x.flags["C_CONTIGUOUS"]
        return x.ctypes.data
    assert x.is_contiguous()
    return x.data_ptr()


_raw_stream = None      # torch's current stream of a device as a plain address: (device index) -> int


def current_stream_address(device: int) -> int:
    """Address of torch's current stream of that device; torch's own shortcut makes no stream object (0.1 us, not 3 us)."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda index: torch.cuda.current_stream(index).cuda_stream)
    return _raw_stream(device)


def _stream(stream):
    if stream is None:
        import torch
        return current_stream_address(torch.cuda.current_device())
    return stream if isinstance(stream, int) else stream.cuda_stream


def _check(status: int, where: str):
    if status != TFE_OK:
        raise TfeError(status, where)


def make_config(*, d, vocab, orders, n_phrases, gpu_slots, load_factor=0.7, hidden_dtype=HIDDEN_BF16,
                max_kicks=0) -> TfeConfig:
    cfg = TfeConfig()
    cfg.d, cfg.vocab, cfg.n_orders = int(d), int(vocab), len(orders)
    for i in range(4):
        cfg.orders[i] = int(orders[i]) if i < len(orders) else 0
    cfg.n_phrases, cfg.gpu_slots = int(n_phrases), int(gpu_slots)
    cfg.load_factor, cfg.hidden_dtype, cfg.max_kicks = float(load_factor), int(hidden_dtype), int(max_kicks)
    return cfg


# ---- the C entry points, same names -------------------------------------------------------


def tfe_index_build(cfg: TfeConfig, phrase_tokens, phrase_len, init_slot, gpu_rows, stream=None) -> int:
    """Returns the context handle (an integer address)."""
    pt = np.ascontiguousarray(phrase_tokens, dtype=np.int32)
    pl = np.ascontiguousarray(phrase_len, dtype=np.uint8)
    sl = np.ascontiguousarray(init_slot, dtype=np.int32)
    out = C.c_void_p()
    _check(lib().tfe_index_build(C.byref(cfg), _addr(pt), _addr(pl), _addr(sl), _addr(gpu_rows),
                                 _stream(stream), C.byref(out)), "tfe_index_build")
    return out.value


def tfe_index_build_device(cfg: TfeConfig, phrase_tokens, phrase_len, init_slot, gpu_rows, stream=None) -> int:
    """As tfe_index_build, with the three phrase arrays on the device (int32 [N,4], uint8 [N], int32 [N])."""
    out = C.c_void_p()
    _check(lib().tfe_index_build_device(C.byref(cfg), _addr(phrase_tokens), _addr(phrase_len), _addr(init_slot),
                                        _addr(gpu_rows), _stream(stream), C.byref(out)), "tfe_index_build_device")
    return out.value


def tfe_cache_install(ctx: int, phrase_ids, src_rows, dst_slots, stream=None) -> None:
    ids = np.ascontiguousarray(phrase_ids, dtype=np.uint32)
    dst = np.ascontiguousarray(dst_slots, dtype=np.int32)
    _check(lib().tfe_cache_install(ctx, len(ids), _addr(ids), _addr(src_rows), _addr(dst), _stream(stream)),
           "tfe_cache_install")


def _params(policy, gate, lam):
    p = TfeInjectParams()
    p.policy, p.gate, p.lam = int(policy), int(gate), float(lam)
    return p


def tfe_lookup_inject(ctx: int, tokens, B, T, q_start, h, out, *, policy=POLICY_LONGEST, gate=GATE_CONST,
                      lam=1.0, sel_phrase=None, sel_slot=None, flags=None, stream=None) -> None:
    p = _params(policy, gate, lam)
    _check(lib().tfe_lookup_inject(ctx, _addr(tokens), B, T, q_start, _addr(h), _addr(out), C.byref(p),
                                   _addr(sel_phrase), _addr(sel_slot), _addr(flags), _stream(stream)),
           "tfe_lookup_inject")


def tfe_lookup_inject_host(ctx: int, tokens, B, T, q_start, h, out, *, policy=POLICY_LONGEST,
                           gate=GATE_CONST, lam=1.0, sel_phrase=None, sel_slot=None, flags=None,
                           stream=None) -> None:
    p = _params(policy, gate, lam)
    _check(lib().tfe_lookup_inject_host(ctx, _addr(tokens), B, T, q_start, _addr(h), _addr(out), C.byref(p),
                                        _addr(sel_phrase), _addr(sel_slot), _addr(flags), _stream(stream)),
           "tfe_lookup_inject_host")


NOALLOC_MAX_ENTRIES = 262_144


def tfe_lookup_inject_noalloc(ctx: int, tokens, B, T, q_start, h, out, *, miss_q, miss_phrase, miss_tier,
                              miss_count, policy=POLICY_LONGEST, gate=GATE_CONST, lam=1.0, sel_phrase=None,
                              sel_slot=None, flags=None, stream=None) -> None:
    """The lookup for callers that must not allocate: scratch is a fixed area of the library image,
    the miss list goes to caller-owned device buffers.  At most NOALLOC_MAX_ENTRIES (query, order)
    entries per call."""
    p = _params(policy, gate, lam)
    _check(lib().tfe_lookup_inject_noalloc(ctx, _addr(tokens), B, T, q_start, _addr(h), _addr(out), C.byref(p),
                                           _addr(sel_phrase), _addr(sel_slot), _addr(flags), _addr(miss_q),
                                           _addr(miss_phrase), _addr(miss_tier), _addr(miss_count),
                                           _stream(stream)), "tfe_lookup_inject_noalloc")


PREFETCH_MAX_BUDGET = 4096


def tfe_prefetch_candidates(ctx: int, history, B, H, cand_tokens, cand_prob, K, *, out_phrase, out_tier, out_score,
                            out_src, out_count, usefulness=None, benefit_host=1.0, benefit_ssd=2.0, budget=4096,
                            stream=None) -> None:
    p = TfePrefetchParams(float(benefit_host), float(benefit_ssd), int(budget))
    _check(lib().tfe_prefetch_candidates(ctx, _addr(history), B, H, _addr(cand_tokens), _addr(cand_prob), K,
                                         _addr(usefulness), C.byref(p), _addr(out_phrase), _addr(out_tier),
                                         _addr(out_score), _addr(out_src), _addr(out_count), _stream(stream)),
           "tfe_prefetch_candidates")


VICTIMS_MAX = 4096
INSTALL_DEVICE_MAX = 4096


def tfe_cache_install_device(ctx: int, n: int, phrase_ids, src_rows, dst_slots, applied=None, applied_count=None,
                             stream=None) -> None:
    """All arrays on the device; entries that cannot be applied are skipped."""
    _check(lib().tfe_cache_install_device(ctx, int(n), _addr(phrase_ids), _addr(src_rows), _addr(dst_slots),
                                          _addr(applied), _addr(applied_count), _stream(stream)),
           "tfe_cache_install_device")


def tfe_cache_policy_enable(ctx: int, stream=None) -> None:
    _check(lib().tfe_cache_policy_enable(ctx, _stream(stream)), "tfe_cache_policy_enable")


def tfe_cache_select_victims(ctx: int, n: int, half_life: int = 0, stream=None):
    """(slots int32[m], keys uint32[m]), m = min(n, gpu_slots), ascending (retention key, slot)."""
    slots, keys = np.empty(max(n, 1), np.int32), np.empty(max(n, 1), np.uint32)
    cnt = C.c_int32(0)
    _check(lib().tfe_cache_select_victims(ctx, int(n), int(half_life), _addr(slots), _addr(keys), C.byref(cnt),
                                          _stream(stream)), "tfe_cache_select_victims")
    return slots[:cnt.value], keys[:cnt.value]


def tfe_cache_select_tuning(ctx: int, list_cap: int = 0, final_cap: int = 0, n_samples: int = 0) -> None:
    _check(lib().tfe_cache_select_tuning(ctx, int(list_cap), int(final_cap), int(n_samples)), "tfe_cache_select_tuning")


def tfe_cache_select_victims_async(ctx: int, n: int, half_life: int = 0, stream=None) -> int:
    """Selection left on the device (see tfe_cache_select_victims_device); returns min(n, gpu_slots)."""
    cnt = C.c_int32(0)
    _check(lib().tfe_cache_select_victims(ctx, int(n), int(half_life), None, None, C.byref(cnt), _stream(stream)),
           "tfe_cache_select_victims")
    return cnt.value


def tfe_cache_select_victims_device(ctx: int):
    a, b = C.c_void_p(), C.c_void_p()
    _check(lib().tfe_cache_select_victims_device(ctx, C.byref(a), C.byref(b)), "tfe_cache_select_victims_device")
    return a.value, b.value


def tfe_cache_stats(ctx: int, gpu_slots: int, stream=None):
    """(freq uint32[C], last uint32[C], epoch)."""
    fl = np.empty((max(gpu_slots, 1), 2), np.uint32)
    ep = C.c_uint32(0)
    _check(lib().tfe_cache_stats(ctx, _addr(fl), C.byref(ep), _stream(stream)), "tfe_cache_stats")
    return fl[:gpu_slots, 0].copy(), fl[:gpu_slots, 1].copy(), ep.value


def tfe_miss_list(ctx: int, cap: int, stream=None, allow_overflow=False):
    """(q_idx uint32[n], phrase_id uint32[n], tier uint8[n], count) of the most recent lookup."""
    q = np.empty(max(cap, 1), np.uint32)
    ph = np.empty(max(cap, 1), np.uint32)
    tr = np.empty(max(cap, 1), np.uint8)
    cnt = C.c_int64(0)
    st = lib().tfe_miss_list(ctx, _addr(q), _addr(ph), _addr(tr), cap, C.byref(cnt), _stream(stream))
    if not (allow_overflow and st == TFE_ERR_MISS_OVERFLOW):
        _check(st, "tfe_miss_list")
    n = min(cnt.value, cap)
    return q[:n], ph[:n], tr[:n], cnt.value


def tfe_miss_list_device(ctx: int):
    """Device addresses (q_idx, phrase_id, tier, count) owned by the context."""
    a, b, c_, d = C.c_void_p(), C.c_void_p(), C.c_void_p(), C.c_void_p()
    _check(lib().tfe_miss_list_device(ctx, C.byref(a), C.byref(b), C.byref(c_), C.byref(d)),
           "tfe_miss_list_device")
    return a.value, b.value, c_.value, d.value


def tfe_destroy(ctx: int) -> None:
    if ctx:
        lib().tfe_destroy(ctx)


def tfe_index_geometry(ctx: int):
    a, b, c_ = C.c_int64(), C.c_int64(), C.c_int64()
    _check(lib().tfe_index_geometry(ctx, C.byref(a), C.byref(b), C.byref(c_)), "tfe_index_geometry")
    return a.value, b.value, c_.value


def tfe_launch_geometry(ctx: int):
    """(grid, block, queries per warp batch) of the most recent lookup."""
    g, b, t = C.c_int32(), C.c_int32(), C.c_int32()
    _check(lib().tfe_launch_geometry(ctx, C.byref(g), C.byref(b), C.byref(t)), "tfe_launch_geometry")
    return g.value, b.value, t.value


def tfe_set_tuning(ctx: int, batch_queries: int = 0) -> None:
    _check(lib().tfe_set_tuning(ctx, int(batch_queries)), "tfe_set_tuning")


def tfe_phrase_key64(vocab: int, tokens) -> tuple[int, bool]:
    t = np.ascontiguousarray(tokens, dtype=np.int32)
    ex = C.c_int32(0)
    k = lib().tfe_phrase_key64(vocab, _addr(t), len(t), C.byref(ex))
    return int(k), bool(ex.value)


def tfe_home_bucket(key: int, n_buckets: int) -> int:
    return int(lib().tfe_home_bucket(key, n_buckets))


# -- early-exit prefetch head -------------------------------------------------------------------
HEAD_MAX_K = 128
HEAD_MAX_BATCH = 256


def tfe_head_create(w_pref, V: int, d: int, max_batch: int) -> int:
    out = C.c_void_p()
    _check(lib().tfe_head_create(_addr(w_pref), int(V), int(d), int(max_batch), C.byref(out)), "tfe_head_create")
    return out.value


def tfe_head_destroy(head: int) -> None:
    lib().tfe_head_destroy(head)


def tfe_head_topk(head: int, hidden, B: int, K: int, cand_tokens, cand_prob, stream=None) -> None:
    _check(lib().tfe_head_topk(head, _addr(hidden), int(B), int(K), _addr(cand_tokens), _addr(cand_prob),
                               _stream(stream)), "tfe_head_topk")


def tfe_head_buffers(head: int):
    """Device addresses (logits fp32 [B][ld], ld, lse fp32 [B]) of the most recent call."""
    a, ld, b = C.c_void_p(), C.c_int64(0), C.c_void_p()
    _check(lib().tfe_head_buffers(head, C.byref(a), C.byref(ld), C.byref(b)), "tfe_head_buffers")
    return a.value, ld.value, b.value


def tfe_head_status(head: int, stream=None) -> int:
    """Synchronises; returns the device status word (0 = no wait ran out)."""
    flags = C.c_uint32(0)
    st = lib().tfe_head_status(head, C.byref(flags), _stream(stream))
    if st not in (TFE_OK, TFE_ERR_INTERNAL):
        _check(st, "tfe_head_status")
    return flags.value


def tfe_head_geometry(head: int):
    g, r, t = C.c_int32(0), C.c_int32(0), C.c_int32(0)
    _check(lib().tfe_head_geometry(head, C.byref(g), C.byref(r), C.byref(t)), "tfe_head_geometry")
    return g.value, r.value, t.value


MINE_HIST_BINS = 1024
MINE_MAX_TOKENS = 1 << 30


def tfe_mine_workspace_bytes(L: int, n_orders: int) -> int:
    return int(lib().tfe_mine_workspace_bytes(int(L), int(n_orders)))


def tfe_mine_ngrams(tokens, L: int, vocab: int, orders, min_count: int, cap: int, phrase_tokens=None, phrase_len=None,
                    phrase_count=None, want_hist: bool = True, workspace=None, workspace_bytes: int = 0, stream=None):
    """tokens and the three outputs on the device; returns (n_found, distinct int64 [n_orders], hist int64 [1024] or None)."""
    o = np.ascontiguousarray(orders, np.int32)
    found = C.c_int64(0)
    distinct = np.zeros(len(o), np.int64)
    hist = np.zeros(MINE_HIST_BINS, np.int64) if want_hist else None
    _check(lib().tfe_mine_ngrams(_addr(tokens), int(L), int(vocab), len(o), _addr(o), int(min_count), int(cap),
                                 _addr(phrase_tokens), _addr(phrase_len), _addr(phrase_count), C.byref(found),
                                 _addr(distinct), _addr(hist), _addr(workspace), int(workspace_bytes), _stream(stream)),
           "tfe_mine_ngrams")
    return found.value, distinct, hist


def tfe_assign_residency(count, N: int, gpu_slots: int, host_min_count: int, init_slot, stream=None):
    """count and init_slot on the device; returns (n_gpu, n_host, n_ssd)."""
    tiers = np.zeros(3, np.int64)
    _check(lib().tfe_assign_residency(_addr(count), int(N), int(gpu_slots), int(host_min_count), _addr(init_slot),
                                      _addr(tiers), _stream(stream)), "tfe_assign_residency")
    return tuple(int(x) for x in tiers)


def tfe_stream_copy(dst, src, nbytes: int, stream=None):
    """Streaming device copy of nbytes (a multiple of 16) bytes: the benchmark's same-footprint yardstick."""
    _check(lib().tfe_stream_copy(_addr(dst), _addr(src), int(nbytes), _stream(stream)), "tfe_stream_copy")


# -- rows of logits -----------------------------------------------------------------------------
DTYPE_BF16, DTYPE_F32 = 0, 1
ROWS_MAX = 1 << 27
DISTILL_MAX_TOP = 1024
SAMPLE_MAX_VOCAB = 1 << 24


# The calls below take addresses (integers, or None where the header allows NULL): they are made for every decoded token.


def tfe_sample_tokens(logits, dtype: int, B: int, V: int, ld: int, u, tokens, prob=None, *, temperature=None, top_k=None,
                      top_p=None, min_p=None, stream=None) -> None:
    st = lib().tfe_sample_tokens(logits, dtype, B, V, ld, C.byref(TfeSampleParams(temperature, top_k, top_p, min_p)), u,
                                 tokens, prob, _stream(stream))
    if st:
        raise TfeError(st, "tfe_sample_tokens")


def tfe_distill_forward(logits, dtype: int, N: int, V: int, ld: int, teacher_ids, teacher_logits, K: int, tau: float,
                        loss, lse, stream=None) -> None:
    st = lib().tfe_distill_forward(logits, dtype, N, V, ld, teacher_ids, teacher_logits, K, tau, loss, lse, _stream(stream))
    if st:
        raise TfeError(st, "tfe_distill_forward")


def tfe_distill_backward(logits, dtype: int, N: int, V: int, ld: int, teacher_ids, teacher_logits, K: int, tau: float,
                         lse, grad_loss, grad_logits, ld_grad: int, stream=None) -> None:
    st = lib().tfe_distill_backward(logits, dtype, N, V, ld, teacher_ids, teacher_logits, K, tau, lse, grad_loss,
                                    grad_logits, ld_grad, _stream(stream))
    if st:
        raise TfeError(st, "tfe_distill_backward")


# -- the vocabulary product in 8 bits -----------------------------------------------------------
FP8_MAX_COLS = 1 << 16


def tfe_quantize_fp8(x, dtype: int, R: int, C_: int, ld: int, block_rows: int, q, scale, stream=None) -> None:
    st = lib().tfe_quantize_fp8(x, dtype, R, C_, ld, block_rows, q, scale, _stream(stream))
    if st:
        raise TfeError(st, "tfe_quantize_fp8")


def tfe_quantize_fp8_ld(x, dtype: int, R: int, C_: int, ld: int, block_rows: int, q, ldq: int, scale, stream=None) -> None:
    st = lib().tfe_quantize_fp8_ld(x, dtype, R, C_, ld, block_rows, q, ldq, scale, _stream(stream))
    if st:
        raise TfeError(st, "tfe_quantize_fp8_ld")


def tfe_matmul_fp8(a, lda: int, a_scale, M: int, w, ldw: int, w_scale, N: int, K: int, out, out_dtype: int, ldo: int,
                   stream=None) -> None:
    st = lib().tfe_matmul_fp8(a, lda, a_scale, M, w, ldw, w_scale, N, K, out, out_dtype, ldo, _stream(stream))
    if st:
        raise TfeError(st, "tfe_matmul_fp8")


def tfe_matmul_fp8_status(stream=None) -> int:
    """Synchronises; returns the device status word and clears it (0 = no wait ran out since the last report)."""
    flags = C.c_uint32(0)
    st = lib().tfe_matmul_fp8_status(C.byref(flags), _stream(stream))
    if st not in (TFE_OK, TFE_ERR_INTERNAL):
        _check(st, "tfe_matmul_fp8_status")
    return flags.value


def tfe_matmul_fp8_give_up(how: int) -> None:
    """1 (True): the waits of the products that follow count as run out from the start; 2: those of the MMA issuers after their first
    tile; 0 (False): as usual again."""
    _check(lib().tfe_matmul_fp8_give_up(int(how)), "tfe_matmul_fp8_give_up")


# -- cross entropy from hidden states -----------------------------------------------------------
XENT_MAX_ROWS = 1 << 24
XENT_MAX_COLS = 1 << 16


def tfe_xent_forward_workspace_bytes(N: int, V: int, d: int) -> int:
    return lib().tfe_xent_forward_workspace_bytes(N, V, d)


def tfe_xent_backward_workspace_bytes(N: int, V: int, d: int) -> int:
    return lib().tfe_xent_backward_workspace_bytes(N, V, d)


def tfe_xent_forward(hidden, ld_hidden: int, N: int, weight, ld_weight: int, V: int, d: int, target, loss, lse, workspace,
                     workspace_bytes: int, stream=None) -> None:
    st = lib().tfe_xent_forward(hidden, ld_hidden, N, weight, ld_weight, V, d, target, loss, lse, workspace, workspace_bytes,
                                _stream(stream))
    if st:
        raise TfeError(st, "tfe_xent_forward")


def tfe_xent_backward(hidden, ld_hidden: int, N: int, weight, ld_weight: int, V: int, d: int, target, lse, grad_loss, grad_hidden,
                      ld_grad_hidden: int, grad_weight, ld_grad_weight: int, workspace, workspace_bytes: int, stream=None) -> None:
    st = lib().tfe_xent_backward(hidden, ld_hidden, N, weight, ld_weight, V, d, target, lse, grad_loss, grad_hidden, ld_grad_hidden,
                                 grad_weight, ld_grad_weight, workspace, workspace_bytes, _stream(stream))
    if st:
        raise TfeError(st, "tfe_xent_backward")


def tfe_xent_status(stream=None) -> int:
    """Synchronises; returns the device status word and clears it (0 = no wait ran out since the last report)."""
    flags = C.c_uint32(0)
    st = lib().tfe_xent_status(C.byref(flags), _stream(stream))
    if st not in (TFE_OK, TFE_ERR_INTERNAL):
        _check(st, "tfe_xent_status")
    return flags.value


def tfe_xent_give_up(how: int) -> None:
    """1 (True): the waits of the cross entropy calls that follow count as run out from the start; 2: those of the MMA issuers after
    their first sum; 0 (False): as usual again."""
    _check(lib().tfe_xent_give_up(int(how)), "tfe_xent_give_up")


# -- injection between two norms ----------------------------------------------------------------
INJECT_NORM_MAX_COLS = 8192
GATE_NONE, GATE_SCALAR, GATE_VECTOR = 0, 1, 2


def tfe_inject_norm_workspace_bytes(Q: int, d: int) -> int:
    return lib().tfe_inject_norm_workspace_bytes(Q, d)


def tfe_inject_norm_forward(params: TfeInjectNormParams, out, ld_out: int, normed, ld_normed: int, stream=None) -> None:
    st = lib().tfe_inject_norm_forward(C.byref(params), out, ld_out, normed, ld_normed, _stream(stream))
    if st:
        raise TfeError(st, "tfe_inject_norm_forward")


def tfe_inject_norm_backward(params: TfeInjectNormParams, grads: TfeInjectNormGrads, workspace, workspace_bytes: int, stream=None) -> None:
    st = lib().tfe_inject_norm_backward(C.byref(params), C.byref(grads), workspace, workspace_bytes, _stream(stream))
    if st:
        raise TfeError(st, "tfe_inject_norm_backward")


# -- the norm of many gradients, and clipping by it ---------------------------------------------
CLIP_MAX_TENSORS = 1 << 20


def tfe_clip_workspace_bytes(n: int) -> int:
    return lib().tfe_clip_workspace_bytes(n)


_describe = None        # (the library with the interpreter's lock held, PyList_GetItem, the tensors' describing function), on first use


class _DlpackExchange(C.Structure):     # DLPackExchangeAPI of the DLPack standard, version 1.3
    _fields_ = [("major", C.c_uint32), ("minor", C.c_uint32), ("previous", C.c_void_p), ("allocator", C.c_void_p), ("managed_from_object", C.c_void_p),
                ("managed_to_object", C.c_void_p), ("tensor_from_object", C.c_void_p), ("work_stream", C.c_void_p)]


def _describer():
    global _describe
    if _describe is None:
        import torch
        lib()
        pointer = C.pythonapi.PyCapsule_GetPointer
        pointer.restype, pointer.argtypes = C.c_void_p, [C.py_object, C.c_char_p]
        offered = getattr(torch.Tensor, "__dlpack_c_exchange_api__", None)
        exchange = None if offered is None else _DlpackExchange.from_address(pointer(offered, b"dlpack_exchange_api"))
        if exchange is None or exchange.major != 1 or not exchange.tensor_from_object:
            raise NotImplementedError(f"torch {torch.__version__}: its tensors do not offer the DLPack exchange interface, version 1")
        f = C.PyDLL(LIB_PATH).tfe_describe_tensors
        f.restype, f.argtypes = C.c_int, [C.py_object, C.c_void_p, C.c_void_p, C.c_int32] + [C.c_void_p] * 5
        _describe = (f, C.cast(C.pythonapi.PyList_GetItem, C.c_void_p).value, exchange.tensor_from_object)
    return _describe


def tfe_describe_tensors(tensors: list):
    """(addresses, sizes, the library's type numbers, CUDA device, reason) of a list of torch tensors, the first three as array.array
    objects; the reason is 0, or why a tensor is refused (see the header).  NotImplementedError: a torch whose tensors cannot be asked."""
    f, item, describe = _describe or _describer()
    n = len(tensors)
    at, numel, kinds, told = array("Q", bytes(8 * n)), array("q", bytes(8 * n)), array("i", bytes(4 * n)), array("i", (0, 0))
    device = told.buffer_info()[0]
    f(tensors, item, describe, n, at.buffer_info()[0], numel.buffer_info()[0], kinds.buffer_info()[0], device, device + 4)
    return at, numel, kinds, told[0], told[1]


def _list(x, code: str):
    """Address of a host list for the length of a call: the caller holds the object meanwhile."""
    if x is None:
        return None
    assert x.typecode == code
    return x.buffer_info()[0]


def tfe_grad_norm(tensors, numel, dtype, n: int, norm, workspace, workspace_bytes: int, stream=None) -> None:
    """The lists are array.array objects: tensors "Q", numel "q", dtype "i"."""
    st = lib().tfe_grad_norm(_list(tensors, "Q"), _list(numel, "q"), _list(dtype, "i"), n, norm, workspace, workspace_bytes, _stream(stream))
    if st:
        raise TfeError(st, "tfe_grad_norm")


def tfe_clip_grad_norm(tensors, results, numel, dtype, n: int, max_norm: float, norm, workspace, workspace_bytes: int, stream=None) -> None:
    """As tfe_grad_norm; results: "Q" too, or None for in place."""
    st = lib().tfe_clip_grad_norm(_list(tensors, "Q"), _list(results, "Q"), _list(numel, "q"), _list(dtype, "i"), n, max_norm, norm,
                                  workspace, workspace_bytes, _stream(stream))
    if st:
        raise TfeError(st, "tfe_clip_grad_norm")
