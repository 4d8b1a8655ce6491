"""ctypes binding of ``libvtoken.so``: same names as the C ABI in ``include/vtoken.h``,
argument marshalling only.  Device pointers may be given as ints or as anything with a
``data_ptr()`` method (torch tensors); streams as ints or objects with ``cuda_stream``.

There is no CPU fallback: importing the library fails loudly when it has not been built.
"""
from __future__ import annotations

import ctypes
import os

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libvtoken.so")
CHECKED_LIB_PATH = os.path.join(_PKG, "libvtoken_checked.so")     # same ABI, every index range-checked

OK, EINVAL, ECAPACITY, ECUDA, ENOMEM, ESTATE = 0, -1, -2, -3, -4, -5
NOT_SELECTED, REPACKED, NO_GAIN, DEFERRED_NO_FREE = 0, 1, 2, 3
FLAG_BAD_SLOT, FLAG_BAD_BLOCK, FLAG_BAD_FREE, FLAG_CAPACITY, FLAG_TIMEOUT, FLAG_GATHER_OVERFLOW = 1, 2, 4, 8, 16, 32
FLAG_BAD_VICTIM, FLAG_APPEND_STOPPED, FLAG_CHECK_FAILED, FLAG_BAD_POSITION = 64, 128, 256, 512
KV_BF16, KV_FP16, KV_FP4 = 0, 1, 2
PROB_BF16, PROB_FP16, PROB_F32 = 0, 1, 2

SYMBOLS = ["vtoken_create", "vtoken_destroy", "vtoken_plan", "vtoken_repack", "vtoken_gather_logical",
           "vtoken_read_counts", "vtoken_repack_host", "vtoken_strerror", "vtoken_last_cuda_error",
           "vtoken_copy_grid", "vtoken_scratch_bytes", "vtoken_plan_form", "vtoken_gather_logical_noalloc", "vtoken_evict_tokens",
           "vtoken_sync_new_tokens", "vtoken_build_slot_mapping", "vtoken_apply_moves",
           "vtoken_block_liveness", "vtoken_plan_partial", "vtoken_digest_logical",
           "vtoken_waves_workspace_bytes", "vtoken_repack_waves", "vtoken_slot_cache_mark",
           "vtoken_slot_cache_update", "vtoken_repack_host_partial", "vtoken_check_tables",
           "vtoken_evict_tokens_counted", "vtoken_sync_new_tokens_counted", "vtoken_checked_build",
           "vtoken_debug_probe", "vtoken_kv_row_bytes", "vtoken_write_tokens", "vtoken_read_tokens",
           "vtoken_attention_workspace_bytes", "vtoken_attention", "vtoken_token_weights_workspace_bytes",
           "vtoken_token_weights", "vtoken_select_victims", "vtoken_verify_drafts",
           "vtoken_attention_shared_workspace_bytes", "vtoken_attention_shared"]


class VtokenError(RuntimeError):
    def __init__(self, code: int, where: str, cuda_error: int = 0):
        self.code = code
        self.cuda_error = cuda_error
        msg = f"{where}: {strerror(code)} (code {code})"
        if cuda_error:
            msg += f", cudaError {cuda_error}"
        super().__init__(msg)


class CopyTuning(ctypes.Structure):
    _fields_ = [("enabled", ctypes.c_int32), ("warps", ctypes.c_int32), ("stages", ctypes.c_int32),
                ("rows", ctypes.c_int32), ("depth", ctypes.c_int32), ("ahead", ctypes.c_int32),
                ("fixed_shares", ctypes.c_int32), ("chunk", ctypes.c_int32), ("ctas", ctypes.c_int32)]


class Config(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_int32), ("num_blocks", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("elem_bytes", ctypes.c_int32),
                ("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p),
                ("layer_stride_bytes", ctypes.c_int64), ("max_requests", ctypes.c_int32),
                ("max_tokens", ctypes.c_int64), ("max_table_blocks", ctypes.c_int64),
                ("max_free_blocks", ctypes.c_int32), ("max_ctas", ctypes.c_int32),
                ("copy_variant", ctypes.c_int32), ("wait_limit_ms", ctypes.c_int32),
                ("plain_launches", ctypes.c_int32), ("plan_variant", ctypes.c_int32), ("tuning", CopyTuning),
                ("debug_stall_item", ctypes.c_int64)]


class PlanIn(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_void_p), ("bt_offsets", ctypes.c_void_p), ("bt_blocks", ctypes.c_void_p),
                ("tt_offsets", ctypes.c_void_p), ("tt_slots", ctypes.c_void_p), ("keep", ctypes.c_void_p),
                ("select", ctypes.c_void_p), ("thr_num", ctypes.c_uint32), ("thr_den", ctypes.c_uint32),
                ("free_blocks", ctypes.c_void_p), ("num_free", ctypes.c_void_p)]


class Counts(ctypes.Structure):
    _fields_ = [("num_moves", ctypes.c_int32), ("num_dst_blocks", ctypes.c_int32), ("num_freed", ctypes.c_int32),
                ("num_free_consumed", ctypes.c_int32), ("num_admitted", ctypes.c_int32),
                ("num_deferred", ctypes.c_int32), ("error_flags", ctypes.c_uint32), ("num_released", ctypes.c_int32)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class PlanOut(ctypes.Structure):
    _fields_ = [("new_bt_offsets", ctypes.c_void_p), ("new_bt_blocks", ctypes.c_void_p),
                ("new_tt_slots", ctypes.c_void_p), ("freed_blocks", ctypes.c_void_p),
                ("req_status", ctypes.c_void_p), ("counts", ctypes.c_void_p), ("released_blocks", ctypes.c_void_p)]


class PartialOpts(ctypes.Structure):
    _fields_ = [("protect", ctypes.c_void_p), ("util_num", ctypes.c_uint32), ("util_den", ctypes.c_uint32),
                ("max_source_blocks", ctypes.c_int32), ("theta_num", ctypes.c_uint32), ("theta_den", ctypes.c_uint32),
                ("detach_num", ctypes.c_uint32), ("detach_den", ctypes.c_uint32),
                ("detach_rule", ctypes.c_uint32)]


class WavesOut(ctypes.Structure):
    _fields_ = [("new_bt_offsets", ctypes.c_void_p), ("new_bt_blocks", ctypes.c_void_p),
                ("new_tt_slots", ctypes.c_void_p), ("req_status", ctypes.c_void_p), ("req_wave", ctypes.c_void_p),
                ("req_append_pos", ctypes.c_void_p), ("free_out", ctypes.c_void_p), ("num_free_out", ctypes.c_void_p), ("wave_counts", ctypes.c_void_p),
                ("free_capacity", ctypes.c_int32), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_int64), ("released_blocks", ctypes.c_void_p),
                ("num_released", ctypes.c_void_p)]


class HostTables(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_int32),
                ("bt_offsets", ctypes.c_void_p), ("bt_blocks", ctypes.c_void_p),
                ("tt_offsets", ctypes.c_void_p), ("tt_slots", ctypes.c_void_p),
                ("keep", ctypes.c_void_p), ("select", ctypes.c_void_p),
                ("thr_num", ctypes.c_uint32), ("thr_den", ctypes.c_uint32),
                ("free_blocks", ctypes.c_void_p), ("num_free", ctypes.c_int32),
                ("new_bt_offsets", ctypes.c_void_p), ("new_bt_blocks", ctypes.c_void_p),
                ("new_tt_slots", ctypes.c_void_p), ("freed_blocks", ctypes.c_void_p),
                ("req_status", ctypes.c_void_p), ("counts", ctypes.c_void_p), ("released_blocks", ctypes.c_void_p)]


class Heads(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("kv_type", ctypes.c_int32), ("act_type", ctypes.c_int32), ("k_exponent", ctypes.c_int32),
                ("v_exponent", ctypes.c_int32)]


class WriteIn(ctypes.Structure):
    _fields_ = [("num_tokens", ctypes.c_void_p), ("max_tokens", ctypes.c_int32), ("q", ctypes.c_void_p),
                ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64), ("positions", ctypes.c_void_p),
                ("slots", ctypes.c_void_p), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p),
                ("eps", ctypes.c_float), ("cos_sin", ctypes.c_void_p), ("max_position", ctypes.c_int32),
                ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("q_out", ctypes.c_void_p),
                ("q_out_stride", ctypes.c_int64)]


class AttentionIn(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_void_p), ("q_offsets", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("q", ctypes.c_void_p), ("q_stride", ctypes.c_int64), ("max_query_tokens", ctypes.c_int32),
                ("max_query_len", ctypes.c_int32), ("tt_offsets", ctypes.c_void_p), ("cache_slots", ctypes.c_void_p),
                ("cache_ids", ctypes.c_void_p), ("cache_len", ctypes.c_void_p), ("sm_scale", ctypes.c_float),
                ("window", ctypes.c_int32), ("sinks", ctypes.c_int32), ("out", ctypes.c_void_p),
                ("out_stride", ctypes.c_int64), ("lse", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_int64)]


class WeightsIn(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_void_p), ("q_offsets", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("q", ctypes.c_void_p), ("q_stride", ctypes.c_int64), ("max_query_tokens", ctypes.c_int32),
                ("max_query_len", ctypes.c_int32), ("tt_offsets", ctypes.c_void_p), ("cache_slots", ctypes.c_void_p),
                ("cache_ids", ctypes.c_void_p), ("cache_len", ctypes.c_void_p), ("lse", ctypes.c_void_p),
                ("sm_scale", ctypes.c_float), ("window", ctypes.c_int32), ("sinks", ctypes.c_int32),
                ("decay", ctypes.c_float), ("prev", ctypes.c_void_p), ("scores", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_int64)]


class SelectIn(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_void_p), ("tt_offsets", ctypes.c_void_p), ("cache_ids", ctypes.c_void_p),
                ("cache_len", ctypes.c_void_p), ("scores", ctypes.c_void_p), ("budget", ctypes.c_void_p),
                ("shared_len", ctypes.c_void_p), ("sinks", ctypes.c_int32), ("recent", ctypes.c_int32),
                ("max_cache_len", ctypes.c_int32), ("victim_req", ctypes.c_void_p), ("victim_tok", ctypes.c_void_p),
                ("max_victims", ctypes.c_int32), ("num_victims", ctypes.c_void_p)]


class VerifyIn(ctypes.Structure):
    _fields_ = [("num_requests", ctypes.c_void_p), ("draft_offsets", ctypes.c_void_p), ("max_drafts", ctypes.c_int32),
                ("draft_tokens", ctypes.c_void_p), ("prob_type", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("target_probs", ctypes.c_void_p), ("target_stride", ctypes.c_int64), ("draft_probs", ctypes.c_void_p),
                ("draft_stride", ctypes.c_int64), ("accept_random", ctypes.c_void_p),
                ("sample_random", ctypes.c_void_p), ("first_id", ctypes.c_void_p), ("accepted", ctypes.c_void_p),
                ("next_tokens", ctypes.c_void_p), ("out_tokens", ctypes.c_void_p), ("victim_req", ctypes.c_void_p),
                ("victim_tok", ctypes.c_void_p), ("max_victims", ctypes.c_int32), ("num_victims", ctypes.c_void_p)]


class SharedIn(ctypes.Structure):
    _fields_ = [("num_groups", ctypes.c_void_p), ("group_offsets", ctypes.c_void_p), ("shared_len", ctypes.c_void_p)]


_lib = None
_libs = {}
_flavour = "production"


def _build_if_needed():
    """Compiles the CUDA libraries in-tree when they are missing or older than their sources and
    nvcc is available; a build failure is reported, never papered over."""
    from . import build as _build
    try:
        _build._nvcc()
    except RuntimeError:
        return                      # no compiler here: use the library as shipped (or fail below)
    _build.build()


def load():
    """Loads libvtoken.so (once), building it first when needed.  Raises when it cannot be had:
    there is no fallback."""
    global _lib
    if _lib is None:
        _build_if_needed()
        path = LIB_PATH if _flavour == "production" else CHECKED_LIB_PATH
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: run `python -m paper_2608_13263_b200.build` "
                              "(needs nvcc); this package has no CPU fallback")
        if path in _libs:
            _lib = _libs[path]
            return _lib
        lib = ctypes.CDLL(path)
        lib.vtoken_create.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(ctypes.c_void_p)]
        lib.vtoken_destroy.argtypes = [ctypes.c_void_p]
        lib.vtoken_destroy.restype = None
        lib.vtoken_plan.argtypes = [ctypes.c_void_p, ctypes.POINTER(PlanIn), ctypes.POINTER(PlanOut), ctypes.c_void_p]
        lib.vtoken_repack.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
        lib.vtoken_gather_logical.argtypes = [ctypes.c_void_p] * 6 + [ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                                                                       ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                                                       ctypes.c_void_p]
        lib.vtoken_read_counts.argtypes = [ctypes.c_void_p, ctypes.POINTER(Counts), ctypes.c_void_p]
        lib.vtoken_repack_host.argtypes = [ctypes.c_void_p, ctypes.POINTER(HostTables), ctypes.c_void_p]
        lib.vtoken_repack_host_partial.argtypes = [ctypes.c_void_p, ctypes.POINTER(HostTables),
                                                   ctypes.POINTER(PartialOpts), ctypes.c_void_p]
        lib.vtoken_check_tables.argtypes = [ctypes.c_void_p, ctypes.POINTER(PlanIn), ctypes.c_void_p, ctypes.c_void_p,
                                            ctypes.c_void_p]
        lib.vtoken_evict_tokens_counted.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32] + \
                                                   [ctypes.c_void_p] * 10
        lib.vtoken_sync_new_tokens_counted.argtypes = [ctypes.c_void_p] * 13
        lib.vtoken_strerror.argtypes = [ctypes.c_int]
        lib.vtoken_strerror.restype = ctypes.c_char_p
        lib.vtoken_last_cuda_error.argtypes = [ctypes.c_void_p]
        lib.vtoken_copy_grid.argtypes = [ctypes.c_void_p] + [ctypes.POINTER(ctypes.c_int32)] * 4
        lib.vtoken_scratch_bytes.argtypes = [ctypes.c_void_p]
        lib.vtoken_scratch_bytes.restype = ctypes.c_int64
        lib.vtoken_plan_form.argtypes = [ctypes.c_void_p]
        lib.vtoken_plan_form.restype = ctypes.c_int
        lib.vtoken_gather_logical_noalloc.argtypes = (
            [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64,
             ctypes.c_int64, ctypes.c_void_p, ctypes.c_int32] + [ctypes.c_void_p] * 4 +
            [ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
             ctypes.c_void_p, ctypes.c_void_p])
        lib.vtoken_evict_tokens.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32] + [ctypes.c_void_p] * 7
        lib.vtoken_sync_new_tokens.argtypes = [ctypes.c_void_p] * 11
        lib.vtoken_build_slot_mapping.argtypes = [ctypes.c_void_p] * 8 + [ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p]
        lib.vtoken_apply_moves.argtypes = [ctypes.c_void_p] * 11
        lib.vtoken_block_liveness.argtypes = [ctypes.c_void_p] * 11
        lib.vtoken_digest_logical.argtypes = [ctypes.c_void_p] * 6 + [ctypes.c_int32, ctypes.c_int32] + [ctypes.c_void_p] * 3
        lib.vtoken_plan_partial.argtypes = [ctypes.c_void_p, ctypes.POINTER(PlanIn), ctypes.POINTER(PartialOpts),
                                            ctypes.POINTER(PlanOut), ctypes.c_void_p]
        lib.vtoken_waves_workspace_bytes.argtypes = [ctypes.c_void_p, ctypes.c_int32]
        lib.vtoken_waves_workspace_bytes.restype = ctypes.c_int64
        lib.vtoken_repack_waves.argtypes = [ctypes.c_void_p, ctypes.POINTER(PlanIn), ctypes.POINTER(PartialOpts),
                                            ctypes.c_int32, ctypes.POINTER(WavesOut), ctypes.c_void_p]
        lib.vtoken_slot_cache_mark.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32] + \
                                              [ctypes.c_void_p] * 4
        lib.vtoken_slot_cache_update.argtypes = [ctypes.c_void_p] * 13
        lib.vtoken_checked_build.argtypes = []
        lib.vtoken_debug_probe.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p]
        lib.vtoken_kv_row_bytes.argtypes = [ctypes.POINTER(Heads)]
        lib.vtoken_kv_row_bytes.restype = ctypes.c_int64
        lib.vtoken_write_tokens.argtypes = [ctypes.c_void_p, ctypes.POINTER(Heads), ctypes.c_int32,
                                            ctypes.POINTER(WriteIn), ctypes.c_void_p]
        lib.vtoken_read_tokens.argtypes = [ctypes.c_void_p, ctypes.POINTER(Heads), ctypes.c_int32, ctypes.c_void_p,
                                           ctypes.c_int32] + [ctypes.c_void_p] * 4
        lib.vtoken_attention_workspace_bytes.argtypes = [ctypes.c_void_p, ctypes.POINTER(Heads), ctypes.c_int32]
        lib.vtoken_attention_workspace_bytes.restype = ctypes.c_int64
        lib.vtoken_attention.argtypes = [ctypes.c_void_p, ctypes.POINTER(Heads), ctypes.c_int32,
                                         ctypes.POINTER(AttentionIn), ctypes.c_void_p]
        for name in ("vtoken_token_weights_workspace_bytes", "vtoken_attention_shared_workspace_bytes"):
            getattr(lib, name).argtypes = [ctypes.c_void_p, ctypes.POINTER(Heads), ctypes.c_int32]
            getattr(lib, name).restype = ctypes.c_int64
        lib.vtoken_token_weights.argtypes = [ctypes.c_void_p, ctypes.POINTER(Heads), ctypes.c_int32,
                                             ctypes.POINTER(WeightsIn), ctypes.c_void_p]
        lib.vtoken_select_victims.argtypes = [ctypes.c_void_p, ctypes.POINTER(SelectIn), ctypes.c_void_p]
        lib.vtoken_verify_drafts.argtypes = [ctypes.c_void_p, ctypes.POINTER(VerifyIn), ctypes.c_void_p]
        lib.vtoken_attention_shared.argtypes = [ctypes.c_void_p, ctypes.POINTER(Heads), ctypes.c_int32,
                                                ctypes.POINTER(AttentionIn), ctypes.POINTER(SharedIn), ctypes.c_void_p]
        _libs[path] = lib
        _lib = lib
    return _lib


def use_library(flavour: str) -> str:
    """Selects the build every later call of this module goes to: "production" (libvtoken.so) or
    "checked" (libvtoken_checked.so: the same sources compiled with -DVTOKEN_CHECKED, every index
    into scratch, tables and pools range-checked, an out-of-range access skipped and reported as
    VTOKEN_FLAG_CHECK_FAILED).  Returns the previous flavour.  Contexts belong to the library that
    created them: destroy them before switching."""
    global _lib, _flavour
    if flavour not in ("production", "checked"):
        raise ValueError(flavour)
    prev, _flavour = _flavour, flavour
    _lib = None
    return prev


def _ptr(x):
    try:
        return x.data_ptr()           # (first: a call marshals a dozen tensors)
    except AttributeError:
        pass
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "ctypes"):          # numpy array (host pointers of vtoken_repack_host)
        return x.ctypes.data
    raise TypeError(f"cannot take a pointer from {type(x)}")


def _stream(s):
    if s is None:
        return None
    if isinstance(s, int):
        return s
    return s.cuda_stream


def strerror(code: int) -> str:
    return load().vtoken_strerror(code).decode()


def _check(rc, where, ctx=None):
    if rc != OK:
        cuda = load().vtoken_last_cuda_error(ctx) if (ctx and rc in (ECUDA, ENOMEM)) else 0
        raise VtokenError(rc, where, cuda)


def vtoken_create(num_layers, num_blocks, block_size, num_kv_heads, head_dim, k_pool, v_pool, max_requests,
                  max_tokens, max_table_blocks, max_free_blocks, elem_bytes=2, layer_stride_bytes=0, max_ctas=0,
                  copy_variant=0, wait_limit_ms=0, plain_launches=0, tuning=None, plan_variant=0,
                  debug_stall_item=0) -> int:
    """``tuning``: dict with any of warps, stages, rows, depth, ahead, fixed_shares, chunk, ctas (the fields of
    vtoken_copy_tuning; giving it sets ``enabled``)."""
    t = CopyTuning()
    if tuning:
        t.enabled = 1
        t.depth, t.ahead = 2, 2                   # the defaults of the two fields whose zero means something
        for k, v in tuning.items():
            setattr(t, k, int(v))
    cfg = Config(num_layers, num_blocks, block_size, num_kv_heads, head_dim, elem_bytes, _ptr(k_pool), _ptr(v_pool),
                 layer_stride_bytes, max_requests, max_tokens, max_table_blocks, max_free_blocks, max_ctas,
                 copy_variant, wait_limit_ms, plain_launches, plan_variant, t, debug_stall_item)
    ctx = ctypes.c_void_p()
    _check(load().vtoken_create(ctypes.byref(cfg), ctypes.byref(ctx)), "vtoken_create")
    return ctx.value


def vtoken_destroy(ctx) -> None:
    load().vtoken_destroy(ctx)


def vtoken_plan(ctx, *, num_requests, bt_offsets, bt_blocks, tt_offsets, tt_slots, keep, free_blocks, num_free,
                new_bt_offsets, new_bt_blocks, new_tt_slots, freed_blocks, req_status, counts,
                select=None, thr_num=0, thr_den=0, stream=None) -> None:
    pin = PlanIn(_ptr(num_requests), _ptr(bt_offsets), _ptr(bt_blocks), _ptr(tt_offsets), _ptr(tt_slots), _ptr(keep),
                 _ptr(select), thr_num, thr_den, _ptr(free_blocks), _ptr(num_free))
    pout = PlanOut(_ptr(new_bt_offsets), _ptr(new_bt_blocks), _ptr(new_tt_slots), _ptr(freed_blocks),
                   _ptr(req_status), _ptr(counts))
    _check(load().vtoken_plan(ctx, ctypes.byref(pin), ctypes.byref(pout), _stream(stream)), "vtoken_plan", ctx)


def vtoken_repack(ctx, stream=None) -> None:
    _check(load().vtoken_repack(ctx, _stream(stream)), "vtoken_repack", ctx)


def vtoken_gather_logical(ctx, *, num_requests, tt_offsets, tt_slots, keep, select, layer_begin, layer_end,
                          out_k, out_v, out_capacity_tokens, out_offsets, stream=None) -> None:
    _check(load().vtoken_gather_logical(ctx, _ptr(num_requests), _ptr(tt_offsets), _ptr(tt_slots), _ptr(keep),
                                        _ptr(select), layer_begin, layer_end, _ptr(out_k), _ptr(out_v),
                                        out_capacity_tokens, _ptr(out_offsets), _stream(stream)),
           "vtoken_gather_logical", ctx)


def vtoken_read_counts(ctx, stream=None) -> dict:
    c = Counts()
    _check(load().vtoken_read_counts(ctx, ctypes.byref(c), _stream(stream)), "vtoken_read_counts", ctx)
    return c.as_dict()


def vtoken_repack_host(ctx, *, num_requests, bt_offsets, bt_blocks, tt_offsets, tt_slots, keep, free_blocks,
                       num_free, new_bt_offsets, new_bt_blocks, new_tt_slots, freed_blocks, req_status,
                       select=None, thr_num=0, thr_den=0, stream=None) -> dict:
    """All table arguments are HOST arrays (numpy or pinned torch tensors)."""
    c = Counts()
    h = HostTables(num_requests, _ptr(bt_offsets), _ptr(bt_blocks), _ptr(tt_offsets), _ptr(tt_slots), _ptr(keep),
                   _ptr(select), thr_num, thr_den, _ptr(free_blocks), num_free, _ptr(new_bt_offsets),
                   _ptr(new_bt_blocks), _ptr(new_tt_slots), _ptr(freed_blocks), _ptr(req_status),
                   ctypes.addressof(c))
    _check(load().vtoken_repack_host(ctx, ctypes.byref(h), _stream(stream)), "vtoken_repack_host", ctx)
    return c.as_dict()


def vtoken_repack_host_partial(ctx, *, num_requests, bt_offsets, bt_blocks, tt_offsets, tt_slots, keep, free_blocks,
                               num_free, new_bt_offsets, new_bt_blocks, new_tt_slots, freed_blocks, req_status,
                               select=None, thr_num=0, thr_den=0, protect=None, util=(0, 0), max_source_blocks=0,
                               theta=(0, 0), detach=(0, 0), released_blocks=None, detach_rule=0,
                               stream=None) -> dict:
    """vtoken_repack_host with the partial planner; ``protect`` is a HOST array of num_blocks bytes,
    ``released_blocks`` a HOST array of bt_offsets[R] entries (needed with a detach threshold)."""
    c = Counts()
    h = HostTables(num_requests, _ptr(bt_offsets), _ptr(bt_blocks), _ptr(tt_offsets), _ptr(tt_slots), _ptr(keep),
                   _ptr(select), thr_num, thr_den, _ptr(free_blocks), num_free, _ptr(new_bt_offsets),
                   _ptr(new_bt_blocks), _ptr(new_tt_slots), _ptr(freed_blocks), _ptr(req_status),
                   ctypes.addressof(c), _ptr(released_blocks))
    po = PartialOpts(_ptr(protect), util[0], util[1], max_source_blocks, theta[0], theta[1], detach[0], detach[1],
                     int(detach_rule))
    _check(load().vtoken_repack_host_partial(ctx, ctypes.byref(h), ctypes.byref(po), _stream(stream)),
           "vtoken_repack_host_partial", ctx)
    return c.as_dict()


def vtoken_check_tables(ctx, *, num_requests, bt_offsets, bt_blocks, tt_offsets, tt_slots, free_blocks, num_free,
                        out_bits, protect=None, stream=None) -> None:
    """Bit set of violated input preconditions into ``out_bits`` (device uint32); 0 = valid."""
    pin = PlanIn(_ptr(num_requests), _ptr(bt_offsets), _ptr(bt_blocks), _ptr(tt_offsets), _ptr(tt_slots), None,
                 None, 0, 0, _ptr(free_blocks), _ptr(num_free))
    _check(load().vtoken_check_tables(ctx, ctypes.byref(pin), _ptr(protect), _ptr(out_bits), _stream(stream)),
           "vtoken_check_tables", ctx)


def vtoken_copy_grid(ctx) -> dict:
    v = [ctypes.c_int32() for _ in range(4)]
    _check(load().vtoken_copy_grid(ctx, *[ctypes.byref(x) for x in v]), "vtoken_copy_grid")
    return dict(ctas=v[0].value, threads=v[1].value, smem_bytes=v[2].value, variant=v[3].value)


def vtoken_checked_build() -> int:
    return int(load().vtoken_checked_build())


def vtoken_debug_probe(ctx, index: int, out_value, stream=None) -> None:
    _check(load().vtoken_debug_probe(ctx, index, _ptr(out_value), _stream(stream)), "vtoken_debug_probe", ctx)


def vtoken_scratch_bytes(ctx) -> int:
    return load().vtoken_scratch_bytes(ctx)


def vtoken_plan_form(ctx) -> int:
    return load().vtoken_plan_form(ctx)


NOALLOC_MAX_REQUESTS = 4096
NOALLOC_MAX_TOKENS = 262144


def vtoken_gather_logical_noalloc(*, k_pool, v_pool, num_layers, num_blocks, block_size, row_bytes, num_requests,
                                  max_requests, tt_offsets, tt_slots, keep, select, layer_begin, layer_end, out_k,
                                  out_v, out_capacity_tokens, out_offsets, error_flags=None, layer_stride_bytes=0,
                                  stream=None) -> None:
    """The logical gather without a context and without any device allocation: for callers
    whose memory is fully committed to the KV pool or who may not call the allocator.  Limits:
    max_requests <= 4096 and out_capacity_tokens <= 262144 (VtokenError ECAPACITY beyond).  Calls
    on one device share a fixed scratch array, so they must not overlap on the GPU."""
    _check(load().vtoken_gather_logical_noalloc(
        _ptr(k_pool), _ptr(v_pool), num_layers, num_blocks, block_size, row_bytes, layer_stride_bytes,
        _ptr(num_requests), max_requests, _ptr(tt_offsets), _ptr(tt_slots), _ptr(keep), _ptr(select), layer_begin,
        layer_end, _ptr(out_k), _ptr(out_v), out_capacity_tokens, _ptr(out_offsets), _ptr(error_flags),
        _stream(stream)), "vtoken_gather_logical_noalloc")


# ---- token-table runtime ------------------------------------------------------------------
def vtoken_evict_tokens(ctx, *, num_victims, max_victims, victim_req, victim_tok, num_requests, tt_offsets, tt_len,
                        keep, stream=None) -> None:
    _check(load().vtoken_evict_tokens(ctx, _ptr(num_victims), max_victims, _ptr(victim_req), _ptr(victim_tok),
                                      _ptr(num_requests), _ptr(tt_offsets), _ptr(tt_len), _ptr(keep),
                                      _stream(stream)), "vtoken_evict_tokens", ctx)


def vtoken_sync_new_tokens(ctx, *, num_requests, tt_offsets, tt_slots, keep, tt_len, phys_len, bt_offsets, bt_blocks,
                           new_len, stream=None) -> None:
    _check(load().vtoken_sync_new_tokens(ctx, _ptr(num_requests), _ptr(tt_offsets), _ptr(tt_slots), _ptr(keep),
                                         _ptr(tt_len), _ptr(phys_len), _ptr(bt_offsets), _ptr(bt_blocks),
                                         _ptr(new_len), _stream(stream)), "vtoken_sync_new_tokens", ctx)


def vtoken_evict_tokens_counted(ctx, *, num_victims, max_victims, victim_req, victim_tok, num_requests, tt_offsets,
                                tt_len, tt_slots, keep, n_b, live_total=None, stream=None) -> None:
    _check(load().vtoken_evict_tokens_counted(ctx, _ptr(num_victims), max_victims, _ptr(victim_req), _ptr(victim_tok),
                                              _ptr(num_requests), _ptr(tt_offsets), _ptr(tt_len), _ptr(tt_slots),
                                              _ptr(keep), _ptr(n_b), _ptr(live_total), _stream(stream)),
           "vtoken_evict_tokens_counted", ctx)


def vtoken_sync_new_tokens_counted(ctx, *, num_requests, tt_offsets, tt_slots, keep, tt_len, phys_len, bt_offsets,
                                   bt_blocks, new_len, n_b, live_total=None, stream=None) -> None:
    _check(load().vtoken_sync_new_tokens_counted(ctx, _ptr(num_requests), _ptr(tt_offsets), _ptr(tt_slots),
                                                 _ptr(keep), _ptr(tt_len), _ptr(phys_len), _ptr(bt_offsets),
                                                 _ptr(bt_blocks), _ptr(new_len), _ptr(n_b), _ptr(live_total),
                                                 _stream(stream)), "vtoken_sync_new_tokens_counted", ctx)


def vtoken_build_slot_mapping(ctx, *, num_requests, tt_offsets, tt_slots, keep, select, out_slots, out_token_ids,
                              out_capacity, out_offsets, stream=None) -> None:
    _check(load().vtoken_build_slot_mapping(ctx, _ptr(num_requests), _ptr(tt_offsets), _ptr(tt_slots), _ptr(keep),
                                            _ptr(select), _ptr(out_slots), _ptr(out_token_ids), out_capacity,
                                            _ptr(out_offsets), _stream(stream)), "vtoken_build_slot_mapping", ctx)


def vtoken_apply_moves(ctx, *, num_requests, tt_offsets, tt_slots, keep, phys_len, new_tt_slots, req_status,
                       new_bt_offsets=None, append_pos=None, stream=None) -> None:
    _check(load().vtoken_apply_moves(ctx, _ptr(num_requests), _ptr(tt_offsets), _ptr(tt_slots), _ptr(keep),
                                     _ptr(phys_len), _ptr(new_tt_slots), _ptr(req_status), _ptr(new_bt_offsets),
                                     _ptr(append_pos), _stream(stream)),
           "vtoken_apply_moves", ctx)


def vtoken_slot_cache_mark(ctx, *, dirty, num_requests, num_victims=None, max_victims=0, victim_req=None,
                           req_status=None, stream=None) -> None:
    _check(load().vtoken_slot_cache_mark(ctx, _ptr(dirty), _ptr(num_victims), max_victims, _ptr(victim_req),
                                         _ptr(req_status), _ptr(num_requests), _stream(stream)),
           "vtoken_slot_cache_mark", ctx)


def vtoken_slot_cache_update(ctx, *, num_requests, tt_offsets, tt_slots, keep, tt_len, dirty, cache_slots, cache_len,
                             cache_seen, cache_ids=None, stats=None, stream=None) -> None:
    _check(load().vtoken_slot_cache_update(ctx, _ptr(num_requests), _ptr(tt_offsets), _ptr(tt_slots), _ptr(keep),
                                           _ptr(tt_len), _ptr(dirty), _ptr(cache_slots), _ptr(cache_ids),
                                           _ptr(cache_len), _ptr(cache_seen), _ptr(stats), _stream(stream)),
           "vtoken_slot_cache_update", ctx)


# ---- eligibility metadata and partial plans ---------------------------------------------------
def vtoken_block_liveness(ctx, *, num_requests, bt_offsets, bt_blocks, tt_offsets, tt_slots, keep, n_b, hist=None,
                          summary=None, stream=None) -> None:
    _check(load().vtoken_block_liveness(ctx, _ptr(num_requests), _ptr(bt_offsets), _ptr(bt_blocks), _ptr(tt_offsets),
                                        _ptr(tt_slots), _ptr(keep), _ptr(n_b), _ptr(hist), _ptr(summary),
                                        _stream(stream)), "vtoken_block_liveness", ctx)


def vtoken_plan_partial(ctx, *, num_requests, bt_offsets, bt_blocks, tt_offsets, tt_slots, keep, free_blocks, num_free,
                        new_bt_offsets, new_bt_blocks, new_tt_slots, freed_blocks, req_status, counts, select=None,
                        thr_num=0, thr_den=0, protect=None, util=(0, 0), max_source_blocks=0, theta=(0, 0),
                        detach=(0, 0), released_blocks=None, detach_rule=0, stream=None) -> None:
    pin = PlanIn(_ptr(num_requests), _ptr(bt_offsets), _ptr(bt_blocks), _ptr(tt_offsets), _ptr(tt_slots), _ptr(keep),
                 _ptr(select), thr_num, thr_den, _ptr(free_blocks), _ptr(num_free))
    pout = PlanOut(_ptr(new_bt_offsets), _ptr(new_bt_blocks), _ptr(new_tt_slots), _ptr(freed_blocks),
                   _ptr(req_status), _ptr(counts), _ptr(released_blocks))
    po = PartialOpts(_ptr(protect), util[0], util[1], max_source_blocks, theta[0], theta[1], detach[0], detach[1],
                     int(detach_rule))
    _check(load().vtoken_plan_partial(ctx, ctypes.byref(pin), ctypes.byref(po), ctypes.byref(pout), _stream(stream)),
           "vtoken_plan_partial", ctx)


def vtoken_digest_logical(ctx, *, num_requests, tt_offsets, tt_slots, keep, select, layer_begin, layer_end, out_digest,
                          out_offsets=None, stream=None) -> None:
    _check(load().vtoken_digest_logical(ctx, _ptr(num_requests), _ptr(tt_offsets), _ptr(tt_slots), _ptr(keep),
                                        _ptr(select), layer_begin, layer_end, _ptr(out_digest), _ptr(out_offsets),
                                        _stream(stream)), "vtoken_digest_logical", ctx)


# ---- repack in waves --------------------------------------------------------------------------
def vtoken_waves_workspace_bytes(ctx, free_capacity: int) -> int:
    return load().vtoken_waves_workspace_bytes(ctx, free_capacity)


def vtoken_repack_waves(ctx, *, num_requests, bt_offsets, bt_blocks, tt_offsets, tt_slots, keep, free_blocks, num_free,
                        num_waves, new_bt_offsets, new_bt_blocks, new_tt_slots, req_status, req_wave, free_out,
                        num_free_out, wave_counts, free_capacity, workspace, workspace_bytes, select=None, thr_num=0,
                        thr_den=0, partial=None, req_append_pos=None, released_blocks=None, num_released=None,
                        stream=None) -> None:
    """``partial``: None for the whole-request planner, else a dict with the option keywords of
    vtoken_plan_partial (protect, util, max_source_blocks, theta, detach)."""
    pin = PlanIn(_ptr(num_requests), _ptr(bt_offsets), _ptr(bt_blocks), _ptr(tt_offsets), _ptr(tt_slots), _ptr(keep),
                 _ptr(select), thr_num, thr_den, _ptr(free_blocks), _ptr(num_free))
    wout = WavesOut(_ptr(new_bt_offsets), _ptr(new_bt_blocks), _ptr(new_tt_slots), _ptr(req_status), _ptr(req_wave),
                    _ptr(req_append_pos), _ptr(free_out), _ptr(num_free_out), _ptr(wave_counts), free_capacity, _ptr(workspace),
                    workspace_bytes, _ptr(released_blocks), _ptr(num_released))
    po = None
    if partial is not None:
        util, theta = partial.get("util", (0, 0)), partial.get("theta", (0, 0))
        detach = partial.get("detach", (0, 0))
        po = ctypes.byref(PartialOpts(_ptr(partial.get("protect")), util[0], util[1],
                                      partial.get("max_source_blocks", 0), theta[0], theta[1], detach[0], detach[1],
                                      int(partial.get("detach_rule", 0))))
    _check(load().vtoken_repack_waves(ctx, ctypes.byref(pin), po, num_waves, ctypes.byref(wout), _stream(stream)),
           "vtoken_repack_waves", ctx)


# ---- the attention step around the relocation ------------------------------------------------
def vtoken_kv_row_bytes(heads) -> int:
    """Bytes of a pool row of this geometry; VtokenError EINVAL when it is not supported."""
    n = load().vtoken_kv_row_bytes(ctypes.byref(heads))
    if n < 0:
        raise VtokenError(int(n), "vtoken_kv_row_bytes")
    return n


def vtoken_write_tokens(ctx, *, heads, layer, max_tokens, k, v, slots, positions=None, num_tokens=None, q=None,
                        q_out=None, q_weight=None, k_weight=None, eps=0.0, cos_sin=None, max_position=0, rot_dim=0,
                        interleaved=False, q_stride=0, k_stride=0, v_stride=0, q_out_stride=0, stream=None) -> None:
    """Queries and keys normalised per head and rotated, keys and values written to their slots."""
    a = WriteIn(_ptr(num_tokens), max_tokens, _ptr(q), _ptr(k), _ptr(v), q_stride, k_stride, v_stride,
                _ptr(positions), _ptr(slots), _ptr(q_weight), _ptr(k_weight), eps, _ptr(cos_sin), max_position,
                rot_dim, interleaved, _ptr(q_out), q_out_stride)
    rc = load().vtoken_write_tokens(ctx, heads, layer, a, _stream(stream))
    if rc != OK:
        _check(rc, "vtoken_write_tokens", ctx)


def vtoken_read_tokens(ctx, *, heads, layer, max_tokens, slots, out_k=None, out_v=None, num_tokens=None,
                       stream=None) -> None:
    """K and V rows of the given slots as 16-bit values."""
    rc = load().vtoken_read_tokens(ctx, heads, layer, _ptr(num_tokens), max_tokens, _ptr(slots), _ptr(out_k),
                                   _ptr(out_v), _stream(stream))
    if rc != OK:
        _check(rc, "vtoken_read_tokens", ctx)


def vtoken_attention_workspace_bytes(ctx, heads, max_query_tokens) -> int:
    n = load().vtoken_attention_workspace_bytes(ctx, ctypes.byref(heads), max_query_tokens)
    if n < 0:
        raise VtokenError(int(n), "vtoken_attention_workspace_bytes")
    return n


def vtoken_attention(ctx, *, heads, layer, num_requests, q_offsets, positions, q, max_query_tokens, max_query_len,
                     tt_offsets, cache_slots, cache_len, out, sm_scale, workspace, workspace_bytes, cache_ids=None,
                     lse=None, window=0, sinks=0, q_stride=0, out_stride=0, stream=None) -> None:
    """Queries of every request against the active tokens of its slot cache."""
    a = AttentionIn(_ptr(num_requests), _ptr(q_offsets), _ptr(positions), _ptr(q), q_stride, max_query_tokens,
                    max_query_len, _ptr(tt_offsets), _ptr(cache_slots), _ptr(cache_ids), _ptr(cache_len), sm_scale,
                    window, sinks, _ptr(out), out_stride, _ptr(lse), _ptr(workspace), workspace_bytes)
    rc = load().vtoken_attention(ctx, heads, layer, a, _stream(stream))
    if rc != OK:
        _check(rc, "vtoken_attention", ctx)


# ---- which tokens leave the cache --------------------------------------------------------------
def vtoken_token_weights_workspace_bytes(ctx, heads, max_query_tokens) -> int:
    n = load().vtoken_token_weights_workspace_bytes(ctx, ctypes.byref(heads), max_query_tokens)
    if n < 0:
        raise VtokenError(int(n), "vtoken_token_weights_workspace_bytes")
    return n


def vtoken_token_weights(ctx, *, heads, layer, num_requests, q_offsets, positions, q, max_query_tokens, max_query_len,
                         tt_offsets, cache_slots, cache_len, lse, sm_scale, scores, workspace, workspace_bytes,
                         cache_ids=None, window=0, sinks=0, decay=1.0, prev=None, q_stride=0, stream=None) -> None:
    """The attention weight that every active token received from the queries, added to its decayed score."""
    a = WeightsIn(_ptr(num_requests), _ptr(q_offsets), _ptr(positions), _ptr(q), q_stride, max_query_tokens,
                  max_query_len, _ptr(tt_offsets), _ptr(cache_slots), _ptr(cache_ids), _ptr(cache_len), _ptr(lse), sm_scale,
                  window, sinks, decay, _ptr(prev), _ptr(scores), _ptr(workspace), workspace_bytes)
    rc = load().vtoken_token_weights(ctx, heads, layer, a, _stream(stream))
    if rc != OK:
        _check(rc, "vtoken_token_weights", ctx)


def vtoken_select_victims(ctx, *, num_requests, tt_offsets, cache_len, scores, budget, victim_req, victim_tok, max_victims,
                          num_victims, max_cache_len, cache_ids=None, shared_len=None, sinks=0, recent=0, stream=None) -> None:
    """The tokens that leave when every request is cut back to its budget: the lowest scores."""
    a = SelectIn(_ptr(num_requests), _ptr(tt_offsets), _ptr(cache_ids), _ptr(cache_len), _ptr(scores), _ptr(budget),
                 _ptr(shared_len), sinks, recent, max_cache_len, _ptr(victim_req), _ptr(victim_tok), max_victims,
                 _ptr(num_victims))
    rc = load().vtoken_select_victims(ctx, a, _stream(stream))
    if rc != OK:
        _check(rc, "vtoken_select_victims", ctx)


def vtoken_verify_drafts(ctx, *, num_requests, draft_offsets, max_drafts, draft_tokens, prob_type, vocab, target_probs,
                         accept_random, sample_random, accepted, next_tokens, draft_probs=None, target_stride=0,
                         draft_stride=0, first_id=None, out_tokens=None, victim_req=None, victim_tok=None, max_victims=0,
                         num_victims=None, stream=None) -> None:
    """Drafted tokens accepted or refused by the target's probabilities, and the token behind the accepted ones."""
    a = VerifyIn(_ptr(num_requests), _ptr(draft_offsets), max_drafts, _ptr(draft_tokens), prob_type, vocab,
                 _ptr(target_probs), target_stride, _ptr(draft_probs), draft_stride, _ptr(accept_random),
                 _ptr(sample_random), _ptr(first_id), _ptr(accepted), _ptr(next_tokens), _ptr(out_tokens), _ptr(victim_req),
                 _ptr(victim_tok), max_victims, _ptr(num_victims))
    rc = load().vtoken_verify_drafts(ctx, a, _stream(stream))
    if rc != OK:
        _check(rc, "vtoken_verify_drafts", ctx)


# ---- attention behind shared prefixes -----------------------------------------------------------
def vtoken_attention_shared_workspace_bytes(ctx, heads, max_query_tokens) -> int:
    n = load().vtoken_attention_shared_workspace_bytes(ctx, ctypes.byref(heads), max_query_tokens)
    if n < 0:
        raise VtokenError(int(n), "vtoken_attention_shared_workspace_bytes")
    return n


def vtoken_attention_shared(ctx, *, heads, layer, num_requests, q_offsets, positions, q, max_query_tokens, max_query_len,
                            tt_offsets, cache_slots, cache_len, out, sm_scale, num_groups, group_offsets, shared_len,
                            workspace, workspace_bytes, cache_ids=None, lse=None, window=0, sinks=0, q_stride=0,
                            out_stride=0, stream=None) -> None:
    """vtoken_attention for groups of requests whose caches begin with the same entries."""
    a = AttentionIn(_ptr(num_requests), _ptr(q_offsets), _ptr(positions), _ptr(q), q_stride, max_query_tokens,
                    max_query_len, _ptr(tt_offsets), _ptr(cache_slots), _ptr(cache_ids), _ptr(cache_len), sm_scale,
                    window, sinks, _ptr(out), out_stride, _ptr(lse), _ptr(workspace), workspace_bytes)
    b = SharedIn(_ptr(num_groups), _ptr(group_offsets), _ptr(shared_len))
    rc = load().vtoken_attention_shared(ctx, heads, layer, a, b, _stream(stream))
    if rc != OK:
        _check(rc, "vtoken_attention_shared", ctx)
