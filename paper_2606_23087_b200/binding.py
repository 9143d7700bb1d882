"""ctypes binding of libflowpool.so: the same calls as include/flowpool.h, argument marshalling only.

Device buffers are passed as integer addresses (torch tensors' data_ptr()); host arrays as numpy.
There is no fallback: if the shared library is missing or cannot be loaded, importing this module fails.
"""
import ctypes as C
import os

import numpy as np

from .build import SO, build

FT_BF16, FT_F32 = 0, 1
FT_RING_SORTED, FT_RING_SHUFFLED = 0, 1
FT_BIND_IDENTITY, FT_BIND_PERMUTED = 0, 1
FT_PLAN_ALLOW_UNWRITTEN, FT_PLAN_SORT_DECREASING, FT_PLAN_COST_SUMSQ, FT_PLAN_ZIGZAG_CARRY, FT_PLAN_AUTO_K = 1, 2, 4, 8, 16
FT_NOALLOC_MAX_SPANS = 4096

STATUS = {
    0: "OK", -1: "INVALID_ARG", -2: "POOL_EXHAUSTED", -3: "UNKNOWN_SAMPLE", -4: "ALREADY_WRITTEN",
    -5: "NOT_READY", -6: "TOO_LONG", -7: "BAD_GVA", -8: "PLACEHOLDER_MISMATCH", -9: "BAD_TOKEN_ID",
    -10: "SLOT_IN_USE", -11: "CAPACITY", -12: "CUDA", -13: "TIMEOUT",
}

EXPORTS = (
    "pool_create", "pool_register_samples", "pool_write_embeddings", "pool_write_embeddings_noalloc",
    "pool_plan_microbatches", "plan_summary",
    "plan_arrays", "plan_destroy", "pool_gather_packed", "pool_gather_list", "pool_set_span_grids", "pool_gather_padded", "pool_embed_grad", "pool_layer_norm", "pool_layer_norm_grad", "pool_layer_norm_grad_workspace", "pool_token_loss",
    "pool_token_loss_grad", "pool_token_loss_workspace", "pool_adamw_step",
    "pool_rotary", "pool_rms_norm", "pool_rms_norm_grad", "pool_rms_norm_grad_workspace", "pool_grad_norm", "pool_grad_norm_workspace",
    "pool_token_logprobs", "pool_token_logprobs_workspace", "pool_free", "pool_status", "pool_stats",
    "pool_ready_count", "pool_take_ready", "pool_backing", "pool_ipc_export", "pool_ipc_open", "pool_ipc_close", "pool_export_mapping", "pool_import_mapping", "pool_export_samples", "pool_import_samples",
    "pool_get_tuning", "pool_set_tuning", "pool_profile_enable", "pool_profile_read", "pool_debug_span_pages", "pool_debug_ring", "pool_debug_translate", "pool_destroy", "flowpool_last_cuda_error",
)


class FlowpoolError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        detail = ""
        if code == -12:
            detail = ": " + (lib().flowpool_last_cuda_error() or b"").decode()
        super().__init__(f"{where}: FT_ERR_{STATUS.get(code, code)}{detail}")


class PoolConfig(C.Structure):
    _fields_ = [
        ("page_bytes", C.c_uint64), ("hbm_pages", C.c_uint64), ("host_pages", C.c_uint64),
        ("max_text_tokens", C.c_uint64), ("ring_seed", C.c_uint64), ("bind_seed", C.c_uint64),
        ("gva_hbm_start", C.c_uint64), ("gva_host_start", C.c_uint64), ("max_size", C.c_uint64),
        ("hidden", C.c_uint32), ("max_samples", C.c_uint32), ("max_spans_per_sample", C.c_uint32),
        ("max_pages_per_span", C.c_uint32), ("max_seq_len", C.c_uint32),
        ("placeholder_id", C.c_int32), ("ring_order", C.c_uint32), ("bind_order", C.c_uint32),
        ("world_size", C.c_uint32), ("rank", C.c_uint32), ("max_imported_pages", C.c_uint64),
    ]


class PlanConfig(C.Structure):
    _fields_ = [
        ("coef_A", C.c_uint64), ("coef_B", C.c_uint64), ("budget_L", C.c_uint32),
        ("n_buckets_K", C.c_uint32), ("n_ranks_N", C.c_uint32), ("flags", C.c_uint32),
    ]


class PoolStats(C.Structure):
    _fields_ = [(k, C.c_uint64) for k in (
        "pages_total", "pages_free", "hbm_pages", "host_pages", "text_pages_total", "text_pages_free",
        "live_samples", "live_spans", "bytes_written", "bytes_gathered", "gpu_launches")]


class AdamwTensor(C.Structure):
    _fields_ = [
        ("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p),
        ("v_scale", C.c_void_p), ("copy", C.c_void_p), ("n", C.c_uint64), ("weight_decay", C.c_double),
        ("param_dtype", C.c_uint32), ("grad_dtype", C.c_uint32), ("state_bits", C.c_uint32), ("reserved", C.c_uint32),
    ]


class AdamwConfig(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("grad_scale", C.c_void_p), ("step", C.c_uint64)]


class RotaryConfig(C.Structure):
    _fields_ = [("freq", C.c_void_p), ("axis", C.c_void_p), ("pairs", C.c_uint32), ("head_dim", C.c_uint32),
                ("interleaved", C.c_uint32), ("inverse", C.c_uint32)]


class RotaryTensor(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("src_row", C.c_uint64), ("src_head", C.c_uint64),
                ("dst_row", C.c_uint64), ("dst_head", C.c_uint64), ("heads", C.c_uint32), ("dtype", C.c_uint32)]


class GradTensor(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("n", C.c_uint64), ("dtype", C.c_uint32), ("reserved", C.c_uint32)]


def rotary_config(freqs, axes, head_dim, interleaved=False, inverse=False):
    """A RotaryConfig that keeps its host arrays alive; `axes` None = one axis."""
    f = np.ascontiguousarray(freqs, dtype=np.float64)
    a = None if axes is None else np.ascontiguousarray(axes, dtype=np.uint8)
    if a is not None and len(a) != len(f):
        raise ValueError("one axis for each frequency")
    cfg = RotaryConfig(freq=f.ctypes.data, axis=None if a is None else a.ctypes.data, pairs=len(f), head_dim=head_dim,
                       interleaved=1 if interleaved else 0, inverse=1 if inverse else 0)
    cfg.keep = (f, a)
    return cfg


TUNING_FIELDS = ("dev_ctas_per_sm", "scatter_ctas_per_sm", "scatter_group", "chunk_shift", "host_ctas", "host_store_ctas",
                 "gather_unroll", "grad_ctas_per_sm", "grad_hot_threshold", "remote_ctas", "peers_remote", "scatter_smem_carveout", "gather_smem_carveout",
                 "bulk_wait_limit_us", "bulk_timeout_test", "host_copy_engine")


class Tuning(C.Structure):
    _fields_ = [(k, C.c_uint32) for k in TUNING_FIELDS]


class KernelTime(C.Structure):
    _fields_ = [("ms", C.c_double), ("launches", C.c_uint64)]


KERNEL_CLASSES = ("gather_device", "gather_host", "scatter_device", "scatter_host", "embed_grad", "gather_remote")

IPC_HANDLES_BYTES = 2 * 64 + 8   # ft_ipc_handles


def ipc_open(handles: bytes):
    """Maps a peer process's slabs into this process: (rc, hbm_base, text_base)."""
    buf = (C.c_uint8 * IPC_HANDLES_BYTES).from_buffer_copy(handles)
    a, b = C.c_void_p(), C.c_void_p()
    rc = lib().pool_ipc_open(buf, C.byref(a), C.byref(b))
    return rc, a.value or 0, b.value or 0


def ipc_close(hbm_base: int, text_base: int):
    return lib().pool_ipc_close(hbm_base or None, text_base or None)


_lib = None


def lib():
    """The loaded shared library (built in-tree on first use when nvcc is available)."""
    global _lib
    if _lib is None:
        if not os.path.exists(SO):
            build()
        _lib = C.CDLL(SO)
        P, u32, u64, i32, f32, f64 = C.c_void_p, C.c_uint32, C.c_uint64, C.c_int32, C.c_float, C.c_double
        sig = {
            "pool_create": [P, P, P, P],
            "pool_register_samples": [P, u32, P, P, P, P, P, P, P],
            "pool_write_embeddings": [P, u32, P, P, P, P, u32, P],
            "pool_write_embeddings_noalloc": [P, u32, P, P, P, P, u32, P],
            "pool_plan_microbatches": [P, P, u32, P, P, P],
            "plan_summary": [P, P, P, P],
            "plan_arrays": [P] * 13,
            "plan_destroy": [P],
            "pool_gather_packed": [P, P, u32, u32, P, u32, P, P, P, P],
            "pool_gather_list": [P, P, P, u32, P, u32, P, P, P, P],
            "pool_set_span_grids": [P, u32, P, P, P, P],
            "pool_gather_padded": [P, P, u32, u32, P, u32, i32, P, P, P, P, P, P, P],
            "pool_embed_grad": [P, P, u32, u32, u32, P, P, u32, P],
            "pool_layer_norm": [P, u64, u32, P, u64, u32, P, P, u32, f32, P, u64, P, P, P],
            "pool_layer_norm_grad_workspace": [P, u64, u32, P],
            "pool_layer_norm_grad": [P, u64, u32, P, u64, P, u64, u32, P, u32, P, P, P, u64, P, P, u32, P, u64, P],
            "pool_token_loss_workspace": [P, u64, u32, u32, u32, u32, P, P],
            "pool_token_loss": [P, u64, u32, u32, P, u64, P, u64, P, P, P, P, u64, P],
            "pool_token_loss_grad": [P, u64, u32, u32, P, u64, P, u64, P, P, u32, P, P, P, u64, P, u32, u32, P, u64, P],
            "pool_adamw_step": [P, P, u32, P, P],
            "pool_rotary": [P, u64, P, u64, P, P, u32, P],
            "pool_rms_norm": [P, u64, u32, P, u64, P, u64, u32, P, u32, f32, P, u64, P, u64, P, u64, P, u64, P, P],
            "pool_rms_norm_grad_workspace": [P, u64, u32, P],
            "pool_rms_norm_grad": [P, u64, u32, P, u64, P, u64, P, u64, u32, P, u32, P, P, u64, P, u32, P, u64, P],
            "pool_grad_norm_workspace": [P, P],
            "pool_grad_norm": [P, P, u32, f64, P, P, P, P, P, u64, P],
            "pool_token_logprobs_workspace": [P, u64, u32, u32, u32, P, P],
            "pool_token_logprobs": [P, u64, u32, u32, P, u64, P, u64, P, f32, P, P, u32, P, P, P, u64, P],
            "pool_free": [P, P, u32, P],
            "pool_status": [P, P, P],
            "pool_stats": [P, P],
            "pool_ready_count": [P, P, P],
            "pool_take_ready": [P, u64, u32, P, P, P],
            "pool_backing": [P, P, P, P],
            "pool_export_mapping": [P, P, u64, P],
            "pool_import_mapping": [P, P, u64, P, P, P],
            "pool_export_samples": [P, P, u32, P, u64, P, P],
            "pool_import_samples": [P, P, u32, P, u64, P],
            "pool_ipc_export": [P, P],
            "pool_ipc_open": [P, P, P],
            "pool_ipc_close": [P, P],
            "pool_get_tuning": [P, P],
            "pool_set_tuning": [P, P],
            "pool_profile_enable": [P, i32],
            "pool_profile_read": [P, P],
            "pool_debug_span_pages": [P, u32, u32, P, u32, P],
            "pool_debug_ring": [P, P, u64, P],
            "pool_debug_translate": [P, P, u32, P, P, P, P],
            "pool_destroy": [P],
        }
        for name, argtypes in sig.items():
            fn = getattr(_lib, name)
            fn.argtypes, fn.restype = argtypes, i32
        _lib.flowpool_last_cuda_error.restype = C.c_char_p
        _lib.flowpool_last_cuda_error.argtypes = []
    return _lib


def _u32(a):
    return np.ascontiguousarray(a, dtype=np.uint32)


def _p(a):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


class Plan:
    def __init__(self, handle, n, n_ranks):
        self.h, self.n, self.n_ranks = handle, n, n_ranks

    def summary(self):
        n_mb, tot, mx = C.c_uint32(), C.c_uint64(), C.c_uint32()
        rc = lib().plan_summary(self.h, C.byref(n_mb), C.byref(tot), C.byref(mx))
        if rc:
            raise FlowpoolError(rc, "plan_summary")
        return n_mb.value, tot.value, mx.value

    def arrays(self):
        n_mb = self.summary()[0]
        n, N = self.n, self.n_ranks
        a = {
            "mb_sample_off": np.zeros(n_mb + 1, np.uint32), "mb_samples": np.zeros(n, np.uint32),
            "mb_tokens": np.zeros(n_mb, np.uint32), "mb_lmax": np.zeros(n_mb, np.uint32),
            "mb_residual": np.zeros(n_mb, np.uint32), "mb_cost": np.zeros(n_mb, np.uint64),
            "mb_bucket": np.zeros(n_mb, np.uint32), "mb_rank": np.zeros(n_mb, np.uint32),
            "rank_mb_off": np.zeros(N + 1, np.uint32), "rank_mbs": np.zeros(n_mb, np.uint32),
            "sample_cost": np.zeros(n, np.uint64), "sample_mb": np.zeros(n, np.uint32),
        }
        rc = lib().plan_arrays(self.h, *[_p(v) for v in a.values()])
        if rc:
            raise FlowpoolError(rc, "plan_arrays")
        a["n_mb"] = n_mb
        return a

    def destroy(self):
        if self.h:
            lib().plan_destroy(self.h)
            self.h = None


class Pool:
    """Thin handle around ft_pool.  Every method returns the library's int32 status unchanged
    (0 = OK); nothing is computed on the Python side."""

    def __init__(self, cfg: PoolConfig, hbm_base: int = 0, host_base: int = 0):
        self.cfg = cfg
        self.h = C.c_void_p()
        self.rc = lib().pool_create(C.byref(cfg), hbm_base or None, host_base or None, C.byref(self.h))
        if self.rc != 0:
            self.h = None

    def destroy(self):
        if self.h:
            lib().pool_destroy(self.h)
            self.h = None

    def register_samples(self, slots, seq_len, n_spans, span_pos, span_tokens, input_ids_ptr: int, stream: int = 0):
        slots, seq_len, n_spans = _u32(slots), _u32(seq_len), _u32(n_spans)
        span_pos, span_tokens = _u32(span_pos), _u32(span_tokens)
        return lib().pool_register_samples(self.h, len(slots), _p(slots), _p(seq_len), _p(n_spans), _p(span_pos),
                                           _p(span_tokens), input_ids_ptr or None, stream or None)

    def write_embeddings(self, slots, span_idx, n_tokens, src_ptrs, dtype, stream: int = 0):
        slots, span_idx, n_tokens = _u32(slots), _u32(span_idx), _u32(n_tokens)
        src = np.ascontiguousarray(src_ptrs, dtype=np.uint64)
        return lib().pool_write_embeddings(self.h, len(slots), _p(slots), _p(span_idx), _p(n_tokens), _p(src),
                                           dtype, stream or None)

    def write_embeddings_noalloc(self, slots, span_idx, n_tokens, src_ptrs, dtype, stream: int = 0):
        """pool_write_embeddings_noalloc: same scatter, per-call scratch in the library's fixed device array
        (for callers that may not allocate); at most FT_NOALLOC_MAX_SPANS spans per call."""
        slots, span_idx, n_tokens = _u32(slots), _u32(span_idx), _u32(n_tokens)
        src = np.ascontiguousarray(src_ptrs, dtype=np.uint64)
        return lib().pool_write_embeddings_noalloc(self.h, len(slots), _p(slots), _p(span_idx), _p(n_tokens), _p(src),
                                                   dtype, stream or None)

    def plan_microbatches(self, slots, cfg: PlanConfig, stream: int = 0):
        slots = _u32(slots)
        h = C.c_void_p()
        rc = lib().pool_plan_microbatches(self.h, _p(slots), len(slots), C.byref(cfg), C.byref(h), stream or None)
        return rc, (Plan(h, len(slots), cfg.n_ranks_N) if rc == 0 else None)

    def gather_packed(self, plan: Plan, mb_begin, mb_end, table_ptr: int, vocab: int, out_ptr: int, cu_ptr: int,
                      pos_ptr: int, stream: int = 0):
        return lib().pool_gather_packed(self.h, plan.h, mb_begin, mb_end, table_ptr or None, vocab, out_ptr or None,
                                        cu_ptr or None, pos_ptr or None, stream or None)

    def gather_list(self, plan: Plan, mb_list, table_ptr: int, vocab: int, out_ptr: int, cu_ptr: int, pos_ptr: int,
                    stream: int = 0):
        mb_list = _u32(mb_list)
        return lib().pool_gather_list(self.h, plan.h, _p(mb_list), len(mb_list), table_ptr or None, vocab, out_ptr or None,
                                      cu_ptr or None, pos_ptr or None, stream or None)

    def set_span_grids(self, slots, span_idx, grids, stream: int = 0):
        slots, span_idx = _u32(slots), _u32(span_idx)
        grids = np.ascontiguousarray(np.asarray(grids, dtype=np.uint32).reshape(-1, 3))
        return lib().pool_set_span_grids(self.h, len(slots), _p(slots), _p(span_idx), _p(grids), stream or None)

    def gather_padded(self, plan: Plan, mb_begin, mb_end, table_ptr: int, vocab: int, pad_id: int, out_ptr: int,
                      cu_ptr: int, pos3_ptr: int, ids_ptr: int, labels_ptr: int, mask_ptr: int, stream: int = 0):
        return lib().pool_gather_padded(self.h, plan.h, mb_begin, mb_end, table_ptr or None, vocab, pad_id, out_ptr or None,
                                        cu_ptr or None, pos3_ptr or None, ids_ptr or None, labels_ptr or None,
                                        mask_ptr or None, stream or None)

    def embed_grad(self, plan: Plan, mb_begin, mb_end, padded, grad_out_ptr: int, grad_table_ptr: int, vocab: int,
                   stream: int = 0):
        return lib().pool_embed_grad(self.h, plan.h, mb_begin, mb_end, 1 if padded else 0, grad_out_ptr or None,
                                     grad_table_ptr or None, vocab, stream or None)

    def layer_norm(self, rows, cols, x_ptr: int, ldx, dtype, weight_ptr: int, bias_ptr: int, param_dtype, eps, y_ptr: int, ldy,
                   mean_ptr: int = 0, rstd_ptr: int = 0, stream: int = 0):
        return lib().pool_layer_norm(self.h, rows, cols, x_ptr or None, ldx, dtype, weight_ptr or None, bias_ptr or None,
                                     param_dtype, eps, y_ptr or None, ldy, mean_ptr or None, rstd_ptr or None, stream or None)

    def layer_norm_grad_workspace(self, rows, cols):
        n = C.c_uint64()
        rc = lib().pool_layer_norm_grad_workspace(self.h, rows, cols, C.byref(n))
        if rc:
            raise FlowpoolError(rc, "pool_layer_norm_grad_workspace")
        return n.value

    def layer_norm_grad(self, rows, cols, dy_ptr: int, lddy, x_ptr: int, ldx, dtype, weight_ptr: int, param_dtype, mean_ptr: int,
                        rstd_ptr: int, dx_ptr: int, lddx, dweight_ptr: int, dbias_ptr: int, accumulate, ws_ptr: int, ws_bytes,
                        stream: int = 0):
        return lib().pool_layer_norm_grad(self.h, rows, cols, dy_ptr or None, lddy, x_ptr or None, ldx, dtype, weight_ptr or None,
                                          param_dtype, mean_ptr or None, rstd_ptr or None, dx_ptr or None, lddx,
                                          dweight_ptr or None, dbias_ptr or None, 1 if accumulate else 0, ws_ptr or None, ws_bytes,
                                          stream or None)

    def token_loss_workspace(self, rows, hidden, vocab, with_grad, dw_dtype=FT_F32):
        """(least, best) workspace bytes of token_loss (with_grad false) or token_loss_grad."""
        a, b = C.c_uint64(), C.c_uint64()
        rc = lib().pool_token_loss_workspace(self.h, rows, hidden, vocab, 1 if with_grad else 0, dw_dtype, C.byref(a), C.byref(b))
        if rc:
            raise FlowpoolError(rc, "pool_token_loss_workspace")
        return a.value, b.value

    def token_loss(self, rows, hidden, vocab, x_ptr: int, ldx, w_ptr: int, ldw, labels_ptr: int, loss_ptr: int, lse_ptr: int,
                   ws_ptr: int, ws_bytes, stream: int = 0):
        return lib().pool_token_loss(self.h, rows, hidden, vocab, x_ptr or None, ldx, w_ptr or None, ldw, labels_ptr or None,
                                     loss_ptr or None, lse_ptr or None, ws_ptr or None, ws_bytes, stream or None)

    def token_loss_grad(self, rows, hidden, vocab, x_ptr: int, ldx, w_ptr: int, ldw, labels_ptr: int, grad_loss_ptr: int, grad_stride,
                        loss_ptr: int, lse_ptr: int, dx_ptr: int, lddx, dw_ptr: int, dw_dtype, accumulate, ws_ptr: int, ws_bytes,
                        stream: int = 0):
        return lib().pool_token_loss_grad(self.h, rows, hidden, vocab, x_ptr or None, ldx, w_ptr or None, ldw, labels_ptr or None,
                                          grad_loss_ptr or None, grad_stride, loss_ptr or None, lse_ptr or None, dx_ptr or None, lddx,
                                          dw_ptr or None, dw_dtype, 1 if accumulate else 0, ws_ptr or None, ws_bytes, stream or None)

    def adamw_step(self, tensors, cfg: AdamwConfig, stream: int = 0):
        """pool_adamw_step; `tensors` is a ctypes array of AdamwTensor (kept by the caller from step to step) or a list of them."""
        if not isinstance(tensors, C.Array):
            tensors = (AdamwTensor * len(tensors))(*tensors)
        return lib().pool_adamw_step(self.h, tensors, len(tensors), C.byref(cfg), stream or None)

    def rotary(self, rows, pos_ptr: int, pos_ld, cfg: RotaryConfig, tensors, stream: int = 0):
        """pool_rotary; `tensors` is a ctypes array of RotaryTensor or a list of them."""
        if not isinstance(tensors, C.Array):
            tensors = (RotaryTensor * len(tensors))(*tensors)
        return lib().pool_rotary(self.h, rows, pos_ptr or None, pos_ld, C.byref(cfg), tensors, len(tensors), stream or None)

    def rms_norm(self, rows, cols, x_ptr: int, ldx, residual_ptr: int, ldr, dtype, weight_ptr: int, param_dtype, eps, sum_ptr: int, lds,
                 y_ptr: int, ldy, q_ptr: int = 0, ldq=0, q_scale_ptr: int = 0, ldqs=0, rstd_ptr: int = 0, stream: int = 0):
        return lib().pool_rms_norm(self.h, rows, cols, x_ptr or None, ldx, residual_ptr or None, ldr, dtype, weight_ptr or None, param_dtype,
                                   eps, sum_ptr or None, lds, y_ptr or None, ldy, q_ptr or None, ldq, q_scale_ptr or None, ldqs,
                                   rstd_ptr or None, stream or None)

    def rms_norm_grad_workspace(self, rows, cols):
        n = C.c_uint64()
        rc = lib().pool_rms_norm_grad_workspace(self.h, rows, cols, C.byref(n))
        if rc:
            raise FlowpoolError(rc, "pool_rms_norm_grad_workspace")
        return n.value

    def rms_norm_grad(self, rows, cols, dy_ptr: int, lddy, s_ptr: int, lds, dsum_ptr: int, lddsum, dtype, weight_ptr: int, param_dtype,
                      rstd_ptr: int, dx_ptr: int, lddx, dweight_ptr: int, accumulate, ws_ptr: int, ws_bytes, stream: int = 0):
        return lib().pool_rms_norm_grad(self.h, rows, cols, dy_ptr or None, lddy, s_ptr or None, lds, dsum_ptr or None, lddsum, dtype,
                                        weight_ptr or None, param_dtype, rstd_ptr or None, dx_ptr or None, lddx, dweight_ptr or None,
                                        1 if accumulate else 0, ws_ptr or None, ws_bytes, stream or None)

    def grad_norm_workspace(self):
        n = C.c_uint64()
        rc = lib().pool_grad_norm_workspace(self.h, C.byref(n))
        if rc:
            raise FlowpoolError(rc, "pool_grad_norm_workspace")
        return n.value

    def grad_norm(self, tensors, max_norm, more_ptr: int, sumsq_ptr: int, norm_ptr: int, factor_ptr: int, ws_ptr: int, ws_bytes,
                  stream: int = 0):
        """pool_grad_norm; `tensors` is a ctypes array of GradTensor (kept by the caller from step to step) or a list of them."""
        if not isinstance(tensors, C.Array):
            tensors = (GradTensor * len(tensors))(*tensors)
        return lib().pool_grad_norm(self.h, tensors, len(tensors), max_norm, more_ptr or None, sumsq_ptr or None, norm_ptr or None,
                                    factor_ptr or None, ws_ptr or None, ws_bytes, stream or None)

    def token_logprobs_workspace(self, rows, hidden, vocab, top=0):
        """(least, best) workspace bytes of token_logprobs."""
        a, b = C.c_uint64(), C.c_uint64()
        rc = lib().pool_token_logprobs_workspace(self.h, rows, hidden, vocab, top, C.byref(a), C.byref(b))
        if rc:
            raise FlowpoolError(rc, "pool_token_logprobs_workspace")
        return a.value, b.value

    def token_logprobs(self, rows, hidden, vocab, x_ptr: int, ldx, w_ptr: int, ldw, tokens_ptr: int, logit_scale, logprob_ptr: int,
                       entropy_ptr: int, top, top_ids_ptr: int, top_logprobs_ptr: int, ws_ptr: int, ws_bytes, stream: int = 0):
        return lib().pool_token_logprobs(self.h, rows, hidden, vocab, x_ptr or None, ldx, w_ptr or None, ldw, tokens_ptr or None,
                                         logit_scale, logprob_ptr or None, entropy_ptr or None, top, top_ids_ptr or None,
                                         top_logprobs_ptr or None, ws_ptr or None, ws_bytes, stream or None)

    def free(self, slots, stream: int = 0):
        slots = _u32(slots)
        return lib().pool_free(self.h, _p(slots), len(slots), stream or None)

    def status(self):
        code, detail = C.c_int32(), C.c_uint64()
        rc = lib().pool_status(self.h, C.byref(code), C.byref(detail))
        if rc:
            raise FlowpoolError(rc, "pool_status")
        return code.value, detail.value

    def stats(self):
        s = PoolStats()
        rc = lib().pool_stats(self.h, C.byref(s))
        if rc:
            raise FlowpoolError(rc, "pool_stats")
        return {k: getattr(s, k) for k, _ in PoolStats._fields_}

    def ready_count(self):
        n, t = C.c_uint32(), C.c_uint64()
        rc = lib().pool_ready_count(self.h, C.byref(n), C.byref(t))
        if rc:
            raise FlowpoolError(rc, "pool_ready_count")
        return n.value, t.value

    def take_ready(self, min_tokens, max_samples):
        out = np.zeros(max(1, max_samples), np.uint32)
        n, t = C.c_uint32(), C.c_uint64()
        rc = lib().pool_take_ready(self.h, min_tokens, max_samples, _p(out), C.byref(n), C.byref(t))
        return rc, out[: n.value].copy(), t.value

    def backing(self):
        """(hbm_base, host_base as the device sees it, text_base) of this pool's slabs."""
        a, b, c = C.c_void_p(), C.c_void_p(), C.c_void_p()
        rc = lib().pool_backing(self.h, C.byref(a), C.byref(b), C.byref(c))
        if rc:
            raise FlowpoolError(rc, "pool_backing")
        return a.value or 0, b.value or 0, c.value or 0

    def ipc_export(self):
        """Shareable handles (bytes) of this pool's HBM slab and text frames, for a consumer in another process."""
        buf = (C.c_uint8 * IPC_HANDLES_BYTES)()
        rc = lib().pool_ipc_export(self.h, buf)
        return rc, bytes(buf)

    def export_mapping(self):
        n = C.c_uint64()
        rc = lib().pool_export_mapping(self.h, None, 0, C.byref(n))
        if rc:
            return rc, None
        buf = np.zeros(n.value, np.uint8)
        rc = lib().pool_export_mapping(self.h, _p(buf), n.value, C.byref(n))
        return rc, buf

    def import_mapping(self, blob, peer_hbm_base, peer_host_base, peer_text_base):
        blob = np.ascontiguousarray(blob, dtype=np.uint8)
        return lib().pool_import_mapping(self.h, _p(blob), len(blob), peer_hbm_base or None, peer_host_base or None,
                                         peer_text_base or None)

    def export_samples(self, slots, stream: int = 0):
        slots = _u32(slots)
        n = C.c_uint64()
        rc = lib().pool_export_samples(self.h, _p(slots), len(slots), None, 0, C.byref(n), stream or None)
        if rc:
            return rc, None
        buf = np.zeros(n.value, np.uint8)
        rc = lib().pool_export_samples(self.h, _p(slots), len(slots), _p(buf), n.value, C.byref(n), stream or None)
        return rc, buf

    def import_samples(self, local_slots, blob, stream: int = 0):
        local_slots = _u32(local_slots)
        blob = np.ascontiguousarray(blob, dtype=np.uint8)
        return lib().pool_import_samples(self.h, _p(local_slots), len(local_slots), _p(blob), len(blob), stream or None)

    def get_tuning(self):
        t = Tuning()
        rc = lib().pool_get_tuning(self.h, C.byref(t))
        if rc:
            raise FlowpoolError(rc, "pool_get_tuning")
        return {k: getattr(t, k) for k in TUNING_FIELDS}

    def set_tuning(self, **fields):
        """pool_set_tuning: the named knobs, every other one at its default."""
        t = Tuning()
        for k, v in fields.items():
            if k not in TUNING_FIELDS:
                raise KeyError(k)
            setattr(t, k, int(v))
        return lib().pool_set_tuning(self.h, C.byref(t))

    def profile_enable(self, on=True):
        return lib().pool_profile_enable(self.h, 1 if on else 0)

    def profile_read(self):
        out = (KernelTime * len(KERNEL_CLASSES))()
        rc = lib().pool_profile_read(self.h, out)
        if rc:
            raise FlowpoolError(rc, "pool_profile_read")
        return {k: {"ms": out[i].ms, "launches": out[i].launches} for i, k in enumerate(KERNEL_CLASSES)}

    def span_pages(self, slot, span, cap=1 << 16):
        out = np.zeros(cap, np.uint64)
        n = C.c_uint32()
        rc = lib().pool_debug_span_pages(self.h, slot, span, _p(out), cap, C.byref(n))
        return rc, out[: n.value].copy()

    def ring(self):
        total = self.cfg.hbm_pages + self.cfg.host_pages
        out = np.zeros(total, np.uint32)
        n = C.c_uint64()
        rc = lib().pool_debug_ring(self.h, _p(out), total, C.byref(n))
        if rc:
            raise FlowpoolError(rc, "pool_debug_ring")
        return out[: n.value].copy()

    def translate(self, gvas):
        g = np.ascontiguousarray(gvas, dtype=np.uint64)
        kind, frame = np.zeros(len(g), np.uint32), np.zeros(len(g), np.uint64)
        off, st = np.zeros(len(g), np.uint64), np.zeros(len(g), np.int32)
        rc = lib().pool_debug_translate(self.h, _p(g), len(g), _p(kind), _p(frame), _p(off), _p(st))
        if rc:
            raise FlowpoolError(rc, "pool_debug_translate")
        return st, kind, frame, off
