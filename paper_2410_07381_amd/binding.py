"""Thin ctypes binding of libtally.so: argument marshalling only.

Every step of the path (the three launch forms, preemption, resume, profiling, the
scheduling loop) runs inside the library.  PyTorch appears only as the owner of
device memory and streams.  There is no CPU fallback: if the library is missing the
import fails.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import NamedTuple

import numpy as np

# Hardware queues.  HIP folds a process's streams onto GPU_MAX_HW_QUEUES hardware queues
# (4 unless the environment says otherwise) and reads the variable when it initialises;
# streams that share a queue run in order.  The scheduler needs one queue each for the
# high-priority stream, the best-effort stream and the relay stream beside the null
# stream's, and two more per further best-effort client (2 + 2n for n clients).  This
# module does not touch the environment: a program that wants several clients sets the
# variable itself before its first GPU call, and the library refuses a run whose clients
# would not get queues of their own.
def hw_queues():
    """The number of hardware queues this process asked HIP for (its default is 4)."""
    try:
        return int(os.environ.get("GPU_MAX_HW_QUEUES", "4"))
    except ValueError:
        return 4


_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtally.so")

# ---------------------------------------------------------------- enums
K_SAXPY, K_REDUCE_SUM, K_REDUCE_FINAL, K_GEMM_BF16, K_GEMV_BF16 = 0, 1, 2, 3, 4
K_SOFTMAX_F32, K_LAYERNORM_F32, K_ATTN_DECODE_BF16, K_GEMM_BF16_SMALL = 5, 6, 7, 8
K_GEMM_BF16_N128, K_ATTN_PROMPT_BF16, K_ATTN_PREFIX_BF16, K_GEMV_W4_BF16 = 9, 10, 11, 12
K_ROPE_BF16, K_KV_APPEND_FP8, K_ATTN_PAGED_FP8 = 13, 14, 15
ROPE_INTERLEAVED, ROPE_INVERSE = 1, 2
JOB_QUEUED, JOB_RUNNING, JOB_STOPPED, JOB_COMPLETE = 0, 1, 2, 3
OK, ERR_INVALID_ARG, ERR_BAD_STATE, ERR_HIP, ERR_NOMEM, ERR_UNSUPPORTED = 0, -1, -2, -3, -4, -5
CFG_PTB, CFG_SLICED, CFG_NATIVE, CFG_AUTO = 0, 1, 2, 3
SUBMIT_LOOP, SUBMIT_END_OF_STEP = 1, 2
SCHED_NO_PAUSE = 1
POLICY_TALLY, POLICY_PRIORITY_NATIVE, POLICY_NONE = 0, 1, 2

EXPORTS = [
    "tally_create", "tally_destroy", "tally_logical_grid", "tally_attn_decode_scratch_bytes",
    "tally_attn_prefix_scratch_bytes", "tally_attn_paged_scratch_bytes",
    "tally_launch_native", "tally_launch_sliced", "tally_launch_ptb", "tally_preempt",
    "tally_resume", "tally_progress", "tally_pump", "tally_wait", "tally_job_free",
    "tally_launch_ptb_until", "tally_resume_until", "tally_coverage", "tally_marker",
    "tally_marker_read", "tally_last_preempt_latency_us", "tally_last_hip_error",
    "tally_strerror", "tally_max_workers", "tally_kernel_footprint", "tally_mfma_ceiling_tflops", "tally_device_info", "tally_stream_report", "tally_ptb_turnaround_ms", "tally_select_config",
    "tally_profile", "tally_lookup_config", "tally_sched_run", "tally_set_yield_bound_us",
    "tally_launch_attn_decode_static", "tally_preempt_pausing", "tally_end_pause",
    "tally_candidate_configs", "tally_profile_table", "tally_profile_reset",
    "tally_sched_create", "tally_sched_destroy", "tally_sched_submit_be", "tally_sched_submit_hi",
    "tally_sched_poll", "tally_sched_enable_be", "tally_sched_stats",
    "tally_sched_take_preempt_latencies", "tally_set_yield_every", "tally_parts_executions",
]


class Dim3(C.Structure):
    _fields_ = [("x", C.c_uint32), ("y", C.c_uint32), ("z", C.c_uint32)]


class SaxpyArgs(C.Structure):
    _fields_ = [("x", C.c_void_p), ("y", C.c_void_p), ("a", C.c_float), ("n", C.c_uint32)]


class ReduceSumArgs(C.Structure):
    _fields_ = [("x", C.c_void_p), ("partial", C.c_void_p), ("n", C.c_uint64)]


class ReduceFinalArgs(C.Structure):
    _fields_ = [("partial", C.c_void_p), ("total", C.c_void_p), ("count", C.c_uint32)]


class GemmArgs(C.Structure):
    _fields_ = [("A", C.c_void_p), ("Bt", C.c_void_p), ("C", C.c_void_p),
                ("m", C.c_uint32), ("n", C.c_uint32), ("k", C.c_uint32), ("batch", C.c_uint32),
                ("stride_a", C.c_uint64), ("stride_b", C.c_uint64), ("stride_c", C.c_uint64),
                ("lda", C.c_uint32), ("ldb", C.c_uint32)]


class GemvArgs(C.Structure):
    _fields_ = [("x", C.c_void_p), ("W", C.c_void_p), ("y", C.c_void_p),
                ("n", C.c_uint32), ("k", C.c_uint32)]


class SoftmaxArgs(C.Structure):
    _fields_ = [("x", C.c_void_p), ("y", C.c_void_p), ("rows", C.c_uint32), ("cols", C.c_uint32)]


class LayerNormArgs(C.Structure):
    _fields_ = [("x", C.c_void_p), ("gamma", C.c_void_p), ("beta", C.c_void_p), ("y", C.c_void_p),
                ("rows", C.c_uint32), ("cols", C.c_uint32), ("eps", C.c_float)]


class AttnDecodeArgs(C.Structure):
    _fields_ = [("q", C.c_void_p), ("K", C.c_void_p), ("V", C.c_void_p), ("out", C.c_void_p),
                ("scratch", C.c_void_p), ("tokens", C.c_uint32), ("heads", C.c_uint32),
                ("dim", C.c_uint32)]


class AttnPromptArgs(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("out", C.c_void_p),
                ("cu_seqlens", C.c_void_p), ("total", C.c_uint32), ("n_seqs", C.c_uint32),
                ("heads", C.c_uint32), ("kv_heads", C.c_uint32), ("dim", C.c_uint32),
                ("ld_q", C.c_uint32), ("ld_k", C.c_uint32), ("ld_v", C.c_uint32),
                ("ld_out", C.c_uint32), ("scale", C.c_float)]


class AttnPrefixArgs(C.Structure):
    _fields_ = [("q", C.c_void_p), ("K", C.c_void_p), ("V", C.c_void_p), ("Ko", C.c_void_p),
                ("Vo", C.c_void_p), ("own_len", C.c_void_p), ("out", C.c_void_p), ("scratch", C.c_void_p),
                ("stride_own", C.c_uint64), ("batch", C.c_uint32), ("prefix", C.c_uint32),
                ("own_cap", C.c_uint32), ("heads", C.c_uint32), ("kv_heads", C.c_uint32),
                ("dim", C.c_uint32), ("ld_q", C.c_uint32), ("ld_prefix", C.c_uint32),
                ("ld_own", C.c_uint32), ("ld_out", C.c_uint32), ("scale", C.c_float)]


class GemvW4Args(C.Structure):
    _fields_ = [("x", C.c_void_p), ("W", C.c_void_p), ("scales", C.c_void_p), ("zeros", C.c_void_p),
                ("y", C.c_void_p), ("m", C.c_uint32), ("n", C.c_uint32), ("k", C.c_uint32),
                ("group", C.c_uint32), ("ld_x", C.c_uint32), ("ld_y", C.c_uint32)]


class RopeArgs(C.Structure):
    _fields_ = [("x", C.c_void_p), ("out", C.c_void_p), ("freqs", C.c_void_p), ("positions", C.c_void_p),
                ("total", C.c_uint32), ("heads", C.c_uint32), ("dim", C.c_uint32), ("rot", C.c_uint32),
                ("ld_x", C.c_uint32), ("ld_out", C.c_uint32), ("flags", C.c_uint32), ("magnitude", C.c_float)]


class KvAppendArgs(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("cu_seqlens", C.c_void_p), ("lens", C.c_void_p),
                ("table", C.c_void_p), ("freqs", C.c_void_p), ("positions", C.c_void_p),
                ("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("k_exps", C.c_void_p), ("v_exps", C.c_void_p),
                ("total", C.c_uint32), ("n_seqs", C.c_uint32), ("kv_heads", C.c_uint32), ("dim", C.c_uint32),
                ("page", C.c_uint32), ("n_pages", C.c_uint32), ("seq_pages", C.c_uint32), ("ld_table", C.c_uint32),
                ("ld_k", C.c_uint32), ("ld_v", C.c_uint32), ("rot", C.c_uint32), ("flags", C.c_uint32),
                ("magnitude", C.c_float)]


class AttnPagedArgs(C.Structure):
    _fields_ = [("q", C.c_void_p), ("out", C.c_void_p), ("k_pages", C.c_void_p), ("v_pages", C.c_void_p),
                ("k_exps", C.c_void_p), ("v_exps", C.c_void_p), ("table", C.c_void_p), ("lens", C.c_void_p),
                ("scratch", C.c_void_p), ("batch", C.c_uint32), ("heads", C.c_uint32), ("kv_heads", C.c_uint32),
                ("dim", C.c_uint32), ("page", C.c_uint32), ("n_pages", C.c_uint32), ("seq_pages", C.c_uint32),
                ("ld_table", C.c_uint32), ("ld_q", C.c_uint32), ("ld_out", C.c_uint32), ("scale", C.c_float)]


class KernelDesc(C.Structure):
    _fields_ = [("kernel_id", C.c_uint32), ("grid", Dim3), ("block", Dim3),
                ("args", C.c_void_p), ("args_size", C.c_size_t)]


class CoverRec(C.Structure):
    _fields_ = [("count", C.c_uint32), ("bx", C.c_uint32), ("by", C.c_uint32), ("bz", C.c_uint32),
                ("segment", C.c_uint32), ("worker", C.c_uint32)]


COVER_DTYPE = np.dtype([("count", "<u4"), ("bx", "<u4"), ("by", "<u4"), ("bz", "<u4"),
                        ("segment", "<u4"), ("worker", "<u4")])


class Config(C.Structure):
    _fields_ = [("kind", C.c_uint32), ("param", C.c_uint32), ("chunk", C.c_uint32),
                ("latency_ms", C.c_float), ("turnaround_ms", C.c_float)]


class BeItem(C.Structure):
    _fields_ = [("kernel", C.POINTER(KernelDesc)), ("config", Config)]


class SchedRun(C.Structure):
    _fields_ = [("hi_kernels", C.POINTER(KernelDesc)), ("n_hi_kernels", C.c_uint32),
                ("arrivals_us", C.POINTER(C.c_double)), ("n_arrivals", C.c_uint32),
                ("be_items", C.POINTER(BeItem)), ("n_be_items", C.c_uint32),
                ("policy", C.c_uint32), ("tail_us", C.c_double),
                ("latency_us", C.POINTER(C.c_double)),
                ("preempt_latency_us", C.POINTER(C.c_double)), ("preempt_cap", C.c_uint32),
                ("n_preempts", C.c_uint32),
                ("be_kernels_done", C.c_uint64), ("be_steps_done", C.c_uint64),
                ("window_us", C.c_double), ("issue_us", C.POINTER(C.c_double)),
                ("be_client_items", C.POINTER(C.c_uint32)), ("n_be_clients", C.c_uint32),
                ("be_client_kernels_done", C.POINTER(C.c_uint64)),
                ("threshold_ms", C.c_double), ("profile_runs", C.c_uint32),
                ("sched_flags", C.c_uint32),
                ("profile_samples", C.c_uint64), ("configs_fixed", C.c_uint64),
                ("be_toggle_every", C.c_uint32), ("be_enabled_us", C.c_double)]


class SchedOpts(C.Structure):
    _fields_ = [("policy", C.c_uint32), ("n_be_clients", C.c_uint32), ("threshold_ms", C.c_double),
                ("profile_runs", C.c_uint32), ("flags", C.c_uint32)]


class SchedStats(C.Structure):
    _fields_ = [("hi_requests_done", C.c_uint64), ("be_kernels_done", C.c_uint64),
                ("be_steps_done", C.c_uint64), ("be_client_kernels_done", C.c_uint64 * 8),
                ("n_preempts", C.c_uint64), ("profile_samples", C.c_uint64),
                ("configs_fixed", C.c_uint64)]


class TallyError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        msg = _lib.tally_strerror(status).decode() if _lib is not None else str(status)
        hip = _lib.tally_last_hip_error() if (_lib is not None and status == ERR_HIP) else 0
        super().__init__(f"{what}: {msg} (status {status}" + (f", hip error {hip})" if hip else ")"))


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it first (python -m paper_2410_07381_amd.build). "
            "There is no fallback path.")
    lib = C.CDLL(LIB_PATH)
    vp, u32, u64, i32, dbl = C.c_void_p, C.c_uint32, C.c_uint64, C.c_int, C.c_double
    P = C.POINTER
    sig = {
        "tally_create": ([P(vp), vp, vp], i32),
        "tally_destroy": ([vp], i32),
        "tally_logical_grid": ([u32, vp, C.c_size_t, P(Dim3), P(Dim3)], i32),
        "tally_attn_decode_scratch_bytes": ([u32], C.c_size_t),
        "tally_attn_prefix_scratch_bytes": ([u32] * 6, C.c_size_t),
        "tally_attn_paged_scratch_bytes": ([u32] * 6, C.c_size_t),
        "tally_launch_native": ([vp, P(KernelDesc), i32], i32),
        "tally_launch_attn_decode_static": ([vp, P(AttnDecodeArgs), i32], i32),
        "tally_launch_sliced": ([vp, P(KernelDesc), u32, u32, i32, P(vp)], i32),
        "tally_launch_ptb": ([vp, P(KernelDesc), u32, u32, i32, P(vp)], i32),
        "tally_preempt": ([vp], i32),
        "tally_resume": ([vp], i32),
        "tally_progress": ([vp, P(u64), P(u64), P(i32)], i32),
        "tally_pump": ([vp], i32),
        "tally_wait": ([vp, P(i32)], i32),
        "tally_job_free": ([vp], i32),
        "tally_launch_ptb_until": ([vp, P(KernelDesc), u32, u32, u64, i32, P(vp)], i32),
        "tally_resume_until": ([vp, u64], i32),
        "tally_coverage": ([vp, vp, C.c_size_t], i32),
        "tally_marker": ([vp, i32, u32], i32),
        "tally_marker_read": ([vp, i32, P(u32)], i32),
        "tally_last_preempt_latency_us": ([vp, P(dbl)], i32),
        "tally_last_hip_error": ([], i32),
        "tally_strerror": ([i32], C.c_char_p),
        "tally_device_info": ([P(u32), P(u32), P(u32)], i32),
        "tally_stream_report": ([vp, P(i32), P(u32)], i32),
        "tally_parts_executions": ([u32, u64], u32),
        "tally_ptb_turnaround_ms": ([dbl, u32, u32, u64], dbl),
        "tally_select_config": ([P(Config), u32, dbl], i32),
        "tally_profile": ([vp, P(KernelDesc), P(Config), u32, u32, dbl, P(u32)], i32),
        "tally_lookup_config": ([vp, P(KernelDesc), P(Config)], i32),
        "tally_sched_run": ([vp, P(SchedRun)], i32),
        "tally_set_yield_bound_us": ([vp, u32], i32),
        "tally_max_workers": ([vp, P(KernelDesc), P(u32)], i32),
        "tally_kernel_footprint": ([vp, u32, i32, P(u32), P(u32), P(u32)], i32),
        "tally_mfma_ceiling_tflops": ([vp, u32, P(dbl)], i32),
        "tally_set_yield_every": ([vp, u32], i32),
        "tally_preempt_pausing": ([vp], i32),
        "tally_end_pause": ([vp], i32),
        "tally_candidate_configs": ([vp, P(KernelDesc), P(Config), u32, P(u32)], i32),
        "tally_profile_table": ([vp, P(KernelDesc), P(Config), u32, P(u32), P(u32), P(i32)], i32),
        "tally_profile_reset": ([vp], i32),
        "tally_sched_create": ([vp, P(SchedOpts), P(vp)], i32),
        "tally_sched_destroy": ([vp], i32),
        "tally_sched_submit_be": ([vp, u32, P(KernelDesc), P(Config), u32], i32),
        "tally_sched_submit_hi": ([vp, P(KernelDesc), u32], i32),
        "tally_sched_poll": ([vp, i32, P(i32)], i32),
        "tally_sched_enable_be": ([vp, i32], i32),
        "tally_sched_stats": ([vp, P(SchedStats)], i32),
        "tally_sched_take_preempt_latencies": ([vp, P(dbl), u32, P(u32)], i32),
    }
    assert set(sig) == set(EXPORTS), set(sig) ^ set(EXPORTS)
    for name, (argtypes, restype) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = argtypes
        fn.restype = restype
    return lib


_lib = None
_lib = _load()


def lib():
    return _lib


def _check(rc, what):
    if rc != OK:
        raise TallyError(rc, what)


# ---------------------------------------------------------------- descriptors
_ARGS_FOR = {
    K_SAXPY: SaxpyArgs, K_REDUCE_SUM: ReduceSumArgs, K_REDUCE_FINAL: ReduceFinalArgs,
    K_GEMM_BF16: GemmArgs, K_GEMM_BF16_SMALL: GemmArgs, K_GEMM_BF16_N128: GemmArgs,
    K_GEMV_BF16: GemvArgs,
    K_SOFTMAX_F32: SoftmaxArgs, K_LAYERNORM_F32: LayerNormArgs, K_ATTN_DECODE_BF16: AttnDecodeArgs,
    K_ATTN_PROMPT_BF16: AttnPromptArgs, K_ATTN_PREFIX_BF16: AttnPrefixArgs, K_GEMV_W4_BF16: GemvW4Args,
    K_ROPE_BF16: RopeArgs, K_KV_APPEND_FP8: KvAppendArgs, K_ATTN_PAGED_FP8: AttnPagedArgs,
}


class Kernel:
    """A kernel descriptor plus the objects that must outlive it (args struct, tensors)."""

    def __init__(self, kernel_id, args, keep=()):
        assert isinstance(args, _ARGS_FOR[kernel_id])
        self.kernel_id = kernel_id
        self.args = args
        self.keep = tuple(keep)
        g, b = Dim3(), Dim3()
        _check(_lib.tally_logical_grid(kernel_id, C.addressof(args), C.sizeof(args),
                                       C.byref(g), C.byref(b)), "tally_logical_grid")
        self.desc = KernelDesc(kernel_id, g, b, C.addressof(args), C.sizeof(args))

    @property
    def grid(self):
        return (self.desc.grid.x, self.desc.grid.y, self.desc.grid.z)

    @property
    def total_blocks(self):
        g = self.grid
        return g[0] * g[1] * g[2]


def logical_grid(kernel_id, args):
    g, b = Dim3(), Dim3()
    _check(_lib.tally_logical_grid(kernel_id, C.addressof(args), C.sizeof(args), C.byref(g),
                                   C.byref(b)), "tally_logical_grid")
    return (g.x, g.y, g.z), (b.x, b.y, b.z)


def saxpy(x, y, a):
    return Kernel(K_SAXPY, SaxpyArgs(x.data_ptr(), y.data_ptr(), float(a), x.numel()), (x, y))


def reduce_sum(x, partial):
    return Kernel(K_REDUCE_SUM, ReduceSumArgs(x.data_ptr(), partial.data_ptr(), x.numel()),
                  (x, partial))


def reduce_final(partial, total, count=None):
    n = partial.numel() if count is None else count
    return Kernel(K_REDUCE_FINAL, ReduceFinalArgs(partial.data_ptr(), total.data_ptr(), n),
                  (partial, total))


def gemm_bf16(A, Bt, Cout, small=False, n128=False):
    """A [batch,m,k], Bt [batch,n,k], C [batch,m,n]; 16-bit storage tensors.  Tiles of
    256 x 256 outputs, 256 x 128 with n128, 32 x 32 (ragged edges allowed) with small.
    A and Bt may be views with padded rows (last dimension contiguous): their row and
    batch pitches are taken from the tensors; C must be contiguous."""
    batch, m, k = A.shape
    n = Bt.shape[1]
    assert A.stride(2) == 1 and Bt.stride(2) == 1 and Cout.is_contiguous()
    args = GemmArgs(A.data_ptr(), Bt.data_ptr(), Cout.data_ptr(), m, n, k, batch,
                    A.stride(0), Bt.stride(0), m * n, A.stride(1), Bt.stride(1))
    kid = K_GEMM_BF16_SMALL if small else (K_GEMM_BF16_N128 if n128 else K_GEMM_BF16)
    return Kernel(kid, args, (A, Bt, Cout))


def gemv_bf16(x, W, y):
    n, k = W.shape
    return Kernel(K_GEMV_BF16, GemvArgs(x.data_ptr(), W.data_ptr(), y.data_ptr(), n, k), (x, W, y))


def softmax_f32(x, y):
    rows, cols = x.shape
    return Kernel(K_SOFTMAX_F32, SoftmaxArgs(x.data_ptr(), y.data_ptr(), rows, cols), (x, y))


def layernorm_f32(x, gamma, beta, y, eps):
    rows, cols = x.shape
    return Kernel(K_LAYERNORM_F32,
                  LayerNormArgs(x.data_ptr(), gamma.data_ptr(), beta.data_ptr(), y.data_ptr(),
                                rows, cols, float(eps)), (x, gamma, beta, y))


def attn_decode_bf16(q, Kc, Vc, out, scratch):
    tokens, heads, dim = Kc.shape
    return Kernel(K_ATTN_DECODE_BF16,
                  AttnDecodeArgs(q.data_ptr(), Kc.data_ptr(), Vc.data_ptr(), out.data_ptr(),
                                 scratch.data_ptr(), tokens, heads, dim), (q, Kc, Vc, out, scratch))


def attn_decode_scratch_bytes(heads):
    return int(_lib.tally_attn_decode_scratch_bytes(heads))


def _rows(t, dim=None):
    """Elements between the rows of a tensor: its outermost stride but one if `dim` is None, else
    that of the tokens of a [..., tokens, heads, dim] tensor whose heads lie side by side."""
    if dim is None:
        n, row, width = t.shape[-2], t.stride(-2), t.shape[-1]
    else:
        n, row, width = t.shape[-3], t.stride(-3), t.shape[-2] * dim
        assert t.shape[-1] == dim and (t.shape[-2] == 1 or t.stride(-2) == dim)
    assert t.stride(-1) == 1 or t.shape[-1] == 1
    row = row if n > 1 else width
    assert row >= width, "rows overlap"
    assert row < 1 << 32, "rows too far apart"             # (it would wrap)
    return row


def _is_bf16(*tensors):
    """bf16, or any 16 bits that hold one; fp16, which would be taken for one, is none."""
    import torch
    return all(t.element_size() == 2 and t.dtype != torch.float16 for t in tensors)


def _is_int32(t):
    import torch
    return t.dtype == torch.int32 and t.dim() == 1 and t.is_contiguous()


def attn_prompt_bf16(q, k, v, out, cu_seqlens, scale=None):
    """Causal attention over prompts packed one behind the other: q, out [total, heads, dim]; k, v
    [total, kv_heads, dim]; 16-bit storage tensors that may be views with padded tokens (one
    fused projection's output).  cu_seqlens: int32 [sequences + 1] on the device, where each begins and
    the last one ends.  scale: None for dim ** -0.5."""
    total, heads, dim = q.shape
    kv_heads = k.shape[1]
    assert out.shape == q.shape and k.shape == v.shape == (total, kv_heads, dim)
    assert _is_bf16(q, k, v, out)
    assert _is_int32(cu_seqlens) and cu_seqlens.numel() >= 2
    args = AttnPromptArgs(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), cu_seqlens.data_ptr(),
                          total, cu_seqlens.numel() - 1, heads, kv_heads, dim,
                          _rows(q, dim), _rows(k, dim), _rows(v, dim), _rows(out, dim), _scale(scale))
    return Kernel(K_ATTN_PROMPT_BF16, args, (q, k, v, out, cu_seqlens))


def attn_prefix_bf16(q, K, V, Ko, Vo, own_len, out, scratch, scale=None):
    """One query per head and sequence of a batch behind a shared prefix: q, out [batch, heads, dim];
    K, V [prefix, kv_heads, dim]; Ko, Vo [batch, own_cap, kv_heads, dim], of which own_len (int32 [batch]
    on the device) tokens count; 16-bit storage tensors, padded tokens allowed.  K and V (or Ko and Vo) with
    no tokens, or None, where there is no prefix (no cache).  scratch: attn_prefix_scratch_bytes() bytes."""
    batch, heads, dim = q.shape
    held = lambda t, tokens: t is not None and t.shape[tokens] > 0
    prefix, own_cap, ld_prefix, ld_own, stride = 0, 0, 0, 0, 0
    kv_heads = K.shape[1] if K is not None else Ko.shape[2]
    if held(K, 0):
        prefix, ld_prefix = K.shape[0], _rows(K, dim)
        assert V.shape == K.shape == (prefix, kv_heads, dim) and _rows(V, dim) == ld_prefix
        assert _is_bf16(K, V)
    if held(Ko, 1):
        own_cap, ld_own = Ko.shape[1], _rows(Ko, dim)
        assert Vo.shape == Ko.shape == (batch, own_cap, kv_heads, dim) and _rows(Vo, dim) == ld_own
        assert _is_bf16(Ko, Vo)
        assert _is_int32(own_len) and own_len.numel() == batch
        stride = Ko.stride(0) if batch > 1 else 0
        assert batch == 1 or (stride == Vo.stride(0) and stride > 0)
    assert out.shape == q.shape and _is_bf16(q, out)
    assert scratch.is_contiguous() and (scratch.numel() * scratch.element_size() >=
                                        attn_prefix_scratch_bytes(batch, heads, kv_heads, dim, prefix, own_cap))
    ptr = lambda t, n: t.data_ptr() if n else None
    args = AttnPrefixArgs(q.data_ptr(), ptr(K, prefix), ptr(V, prefix), ptr(Ko, own_cap), ptr(Vo, own_cap),
                          ptr(own_len, own_cap), out.data_ptr(), scratch.data_ptr(), stride,
                          batch, prefix, own_cap, heads, kv_heads, dim, _rows(q, dim), ld_prefix, ld_own,
                          _rows(out, dim), _scale(scale))
    return Kernel(K_ATTN_PREFIX_BF16, args, (q, K, V, Ko, Vo, own_len, out, scratch))


def attn_prefix_scratch_bytes(batch, heads, kv_heads, dim, prefix, own_cap):
    return int(_lib.tally_attn_prefix_scratch_bytes(batch, heads, kv_heads, dim, prefix, own_cap))


def _scale(scale):
    """0 stands for the usual scale in the C structs, so it is no scale of its own."""
    if scale is None:
        return 0.0
    assert scale > 0
    return float(scale)


def gemv_w4_bf16(x, W, scales, y, zeros=None, group=128):
    """y = x (codes - zeros)^T with a scale per row and group: x [m, k], y [m, n], m <= 16, 16-bit storage
    tensors whose rows may be padded; W, scales and zeros as pack_w4() and pack_w4_groups() lay them out."""
    (m, k), n = x.shape, y.shape[1]
    assert group > 0
    tiles, blocks, groups = -(-n // 16), -(-k // 128), -(-k // group)
    assert y.shape[0] == m and _is_bf16(x, y, scales)
    assert W.shape == (tiles, blocks, 64, 4) and W.element_size() == 4 and W.is_contiguous()
    assert scales.shape == (tiles, groups, 16) and scales.is_contiguous()
    assert zeros is None or (zeros.shape == scales.shape and zeros.element_size() == 1 and zeros.is_contiguous())
    args = GemvW4Args(x.data_ptr(), W.data_ptr(), scales.data_ptr(), zeros.data_ptr() if zeros is not None else None,
                      y.data_ptr(), m, n, k, group, _rows(x), _rows(y))
    return Kernel(K_GEMV_W4_BF16, args, (x, W, scales, y) + (() if zeros is None else (zeros,)))


def pack_w4(codes):
    """4-bit codes [n, k] (any integer tensor of values 0 .. 15) as gemv_w4_bf16 reads them: int32 tiles
    [ceil(n / 16), ceil(k / 128), 64, 4] of 16 rows by 128 columns, filled up with zeros."""
    import torch
    n, k = codes.shape
    assert not codes.is_floating_point()
    tiles, blocks = -(-n // 16), -(-k // 128)
    full = torch.zeros((tiles * 16, blocks * 128), dtype=torch.int64, device=codes.device)
    full[:n, :k] = codes
    # (a code of more bits would change its neighbours)
    assert full.numel() == 0 or (int(full.min()) >= 0 and int(full.max()) <= 15)
    at = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], device=codes.device)
    words = (full.view(tiles, 16, blocks, 4, 4, 8) << at).sum(-1)      # tile, row, block, word, quarter
    words = words.permute(0, 2, 4, 1, 3).reshape(tiles, blocks, 64, 4)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32).contiguous()


def pack_w4_groups(t):
    """Scales or zero points (bytes 0 .. 128) [n, groups] as gemv_w4_bf16 reads them: [ceil(n / 16), groups, 16]."""
    import torch
    n, groups = t.shape
    assert t.element_size() != 1 or t.numel() == 0 or (int(t.min()) >= 0 and int(t.max()) <= 128)
    full = torch.zeros((-(-n // 16) * 16, groups), dtype=t.dtype, device=t.device)
    full[:n] = t
    return full.view(-1, 16, groups).transpose(1, 2).contiguous()


# ---------------------------------------------------------------- rotary positions and the paged cache
def rope_freqs(rot, base=10000.0, factor=1.0, scaling="positions", context=None, turns=(1.0, 32.0), device=None):
    """Frequencies of the rot / 2 pairs, base ** (-2 i / rot) radians a position, as rope_bf16 and kv_append_fp8 take
    them: (fp32 tensor, on the host unless `device` is given; magnitude).  For contexts `factor` times as long as those of training:
      "positions"  every frequency is divided by factor (arXiv 2306.15595);
      "base"       the base is raised so that the slowest pair turns factor times slower and the fastest as before;
      "parts"      pairs that make fewer than turns[0] turns within `context` positions (those of training) are divided by
                   factor, those that make more than turns[1] stay, in between both are mixed in proportion to the number of turns (not to
                   the pair's index, which gives other frequencies); q and k grow by 0.1 ln(factor) + 1 (arXiv 2309.00071)."""
    import math

    import torch
    assert rot > 0 and rot % 2 == 0 and base > 0 and factor >= 1 and scaling in ("positions", "base", "parts")
    i = torch.arange(rot // 2, dtype=torch.float64)
    if scaling == "base":
        assert rot > 2
        base = base * factor ** (rot / (rot - 2))
    freqs, magnitude = base ** (-2 * i / rot), 1.0
    if scaling == "positions":
        freqs = freqs / factor
    elif scaling == "parts":
        assert context and turns[1] > turns[0]
        keep = ((context * freqs / (2 * math.pi) - turns[0]) / (turns[1] - turns[0])).clamp(0, 1)
        freqs = freqs * keep + freqs / factor * (1 - keep)
        magnitude = 0.1 * math.log(factor) + 1.0
    return freqs.to(torch.float32).to(device), magnitude


def _together(first, *others):
    """All on the device of the first one (or in pinned host memory, which the device reads too): a host pointer ends the process."""
    return all(t is None or t.device == first.device or t.device.type == "cpu" and t.is_pinned() for t in others)


def _floats(t):
    import torch
    return t.dtype == torch.float32 and t.dim() == 1 and t.is_contiguous()


def rope_bf16(x, out, freqs, positions, interleaved=False, inverse=False, magnitude=None):
    """Rotary positions: x, out [total, heads, dim], 16-bit storage tensors that may be views with padded tokens (the first
    heads of a fused projection); out may be x.  The first 2 x len(freqs) dims of each head are turned by positions
    (int32 [total]) times freqs (fp32, radians; both on x's device): pairs (i, i + len(freqs)), or (2 i, 2 i + 1) with interleaved.  inverse: by the negative
    angle, the operator's transpose, for gradients.  magnitude: what the turned dims are multiplied with, None for 1."""
    total, heads, dim = x.shape
    assert out.shape == x.shape and _is_bf16(x, out) and _floats(freqs)
    assert _is_int32(positions) and positions.numel() == total
    assert _together(x, out, freqs, positions), "on different devices"
    args = RopeArgs(x.data_ptr(), out.data_ptr(), freqs.data_ptr(), positions.data_ptr(), total, heads, dim,
                    2 * freqs.numel(), _rows(x, dim), _rows(out, dim),
                    (ROPE_INTERLEAVED if interleaved else 0) | (ROPE_INVERSE if inverse else 0), _scale(magnitude))
    return Kernel(K_ROPE_BF16, args, (x, out, freqs, positions))


class PagedCache(NamedTuple):
    """Keys and values in pages of 8-bit numbers (include/tally.h has the layout): k [pages, kv_heads, page, dim], v [pages,
    kv_heads, page / 16, dim, 16], uint8 or float8_e4m3fn; k_exps, v_exps uint8 [pages, kv_heads]."""
    k: object
    v: object
    k_exps: object
    v_exps: object

    @classmethod
    def empty(cls, pages, kv_heads, page, dim, device="cuda"):
        import torch
        assert page in (16, 32, 64, 128) and dim in (64, 128)
        z = lambda *s: torch.zeros(s, dtype=torch.uint8, device=device)
        return cls(z(pages, kv_heads, page, dim), z(pages, kv_heads, page // 16, dim, 16), z(pages, kv_heads), z(pages, kv_heads))

    def values(self):
        """What the pages stand for, fp32: keys and values [pages, kv_heads, page, dim]."""
        import torch

        def of(codes, exps):
            scale = torch.exp2(exps.to(torch.float64) - 127).to(torch.float32)
            return codes.view(torch.float8_e4m3fn).to(torch.float32) * scale.view(*exps.shape, *[1] * (codes.dim() - 2))
        pages, heads, page, dim = self.k.shape
        return of(self.k, self.k_exps), of(self.v, self.v_exps).transpose(3, 4).reshape(pages, heads, page, dim)


def _pages(cache, dim):
    """(pages, kv_heads, page) of a cache for heads of `dim`."""
    import torch
    pages, heads, page, width = cache.k.shape
    assert width == dim and page > 0 and page % 16 == 0 and cache.v.shape == (pages, heads, page // 16, dim, 16)
    assert cache.k_exps.shape == cache.v_exps.shape == (pages, heads)
    assert all(t.dtype in (torch.uint8, torch.float8_e4m3fn) and t.is_contiguous() for t in cache[:2])
    assert all(t.dtype == torch.uint8 and t.is_contiguous() for t in cache[2:])
    return pages, heads, page


def _table(table, seqs):
    """(pages per sequence, entries between rows) of a table of pages."""
    import torch
    assert table.dtype == torch.int32 and table.dim() == 2 and table.shape[0] == seqs and table.shape[1] > 0
    return table.shape[1], _rows(table)


def kv_append_fp8(k, v, cu_seqlens, lens, table, cache, freqs=None, positions=None, interleaved=False, magnitude=None):
    """Keys and values of packed tokens go to a paged cache: k, v [total, kv_heads, dim], 16-bit storage tensors that may be views
    with padded tokens; cu_seqlens int32 [sequences + 1]: where each sequence's tokens begin and the last one's end; lens int32
    [sequences]: how many tokens each has WITH these, its last ones; table int32 [sequences, pages of one]; cache a PagedCache.
    With freqs, keys are turned on the way as rope_bf16 does, by their place in the sequence or by positions (int32
    [total]).  All but freqs=None and positions=None on the device."""
    total, kv_heads, dim = k.shape
    assert v.shape == k.shape and _is_bf16(k, v)
    assert _is_int32(cu_seqlens) and cu_seqlens.numel() >= 2
    seqs = cu_seqlens.numel() - 1
    assert _is_int32(lens) and lens.numel() == seqs
    pages, heads, page = _pages(cache, dim)
    assert heads == kv_heads
    seq_pages, ld_table = _table(table, seqs)
    assert freqs is None or _floats(freqs)
    assert positions is None or (freqs is not None and _is_int32(positions) and positions.numel() == total)
    assert _together(k, v, cu_seqlens, lens, table, *cache, freqs, positions), "on different devices"
    ptr = lambda t: None if t is None else t.data_ptr()
    args = KvAppendArgs(k.data_ptr(), v.data_ptr(), cu_seqlens.data_ptr(), lens.data_ptr(), table.data_ptr(), ptr(freqs),
                        ptr(positions), *(t.data_ptr() for t in cache), total, seqs, kv_heads, dim, page, pages, seq_pages, ld_table,
                        _rows(k, dim), _rows(v, dim), 0 if freqs is None else 2 * freqs.numel(),
                        ROPE_INTERLEAVED if interleaved else 0, _scale(magnitude))
    return Kernel(K_KV_APPEND_FP8, args, (k, v, cu_seqlens, lens, table, *cache, freqs, positions))


def attn_paged_fp8(q, cache, table, lens, out, scratch=None, scale=None):
    """One query per head and sequence over a paged cache: q, out [batch, heads, dim], 16-bit storage tensors, padded sequences
    allowed; table int32 [batch, pages of one], of whose tokens lens (int32 [batch]) count; scratch:
    attn_paged_scratch_bytes() bytes, None where that is 0.  scale: None for dim ** -0.5."""
    batch, heads, dim = q.shape
    assert out.shape == q.shape and _is_bf16(q, out)
    pages, kv_heads, page = _pages(cache, dim)
    seq_pages, ld_table = _table(table, batch)
    assert _is_int32(lens) and lens.numel() == batch
    assert _together(q, out, *cache, table, lens, scratch), "on different devices"
    size = attn_paged_scratch_bytes(batch, heads, kv_heads, dim, page, seq_pages)
    assert size == 0 if scratch is None else scratch.is_contiguous() and scratch.numel() * scratch.element_size() >= size
    args = AttnPagedArgs(q.data_ptr(), out.data_ptr(), *(t.data_ptr() for t in cache), table.data_ptr(), lens.data_ptr(),
                         None if scratch is None else scratch.data_ptr(), batch, heads, kv_heads, dim, page, pages, seq_pages,
                         ld_table, _rows(q, dim), _rows(out, dim), _scale(scale))
    return Kernel(K_ATTN_PAGED_FP8, args, (q, out, *cache, table, lens, scratch))


def attn_paged_scratch_bytes(batch, heads, kv_heads, dim, page, seq_pages):
    return int(_lib.tally_attn_paged_scratch_bytes(batch, heads, kv_heads, dim, page, seq_pages))


# ---------------------------------------------------------------- context / jobs
class Job:
    def __init__(self, handle, kernel):
        self.h = handle
        self.kernel = kernel

    def preempt(self, pause=False):
        """Raise the preemption signal; with pause, also ask workers to pause inside long blocks."""
        if pause:
            _check(_lib.tally_preempt_pausing(self.h), "tally_preempt_pausing")
        else:
            _check(_lib.tally_preempt(self.h), "tally_preempt")

    def end_pause(self):
        _check(_lib.tally_end_pause(self.h), "tally_end_pause")

    def resume(self, stop_at=None):
        if stop_at is None:
            _check(_lib.tally_resume(self.h), "tally_resume")
        else:
            _check(_lib.tally_resume_until(self.h, int(stop_at)), "tally_resume_until")

    def progress(self):
        d, t, s = C.c_uint64(), C.c_uint64(), C.c_int()
        _check(_lib.tally_progress(self.h, C.byref(d), C.byref(t), C.byref(s)), "tally_progress")
        return d.value, t.value, s.value

    def pump(self):
        _check(_lib.tally_pump(self.h), "tally_pump")

    def wait(self):
        s = C.c_int()
        _check(_lib.tally_wait(self.h, C.byref(s)), "tally_wait")
        return s.value

    def coverage(self):
        rec = np.zeros(self.kernel.total_blocks, dtype=COVER_DTYPE)
        _check(_lib.tally_coverage(self.h, rec.ctypes.data, rec.nbytes), "tally_coverage")
        return rec

    def preempt_latency_us(self):
        v = C.c_double()
        _check(_lib.tally_last_preempt_latency_us(self.h, C.byref(v)), "preempt latency")
        return v.value

    def free(self):
        if self.h is not None:
            _check(_lib.tally_job_free(self.h), "tally_job_free")
            self.h = None


class Context:
    def __init__(self, stream_hi, stream_be):
        """stream_hi / stream_be: torch.cuda.Stream objects (default priority)."""
        self._streams = (stream_hi, stream_be)
        h = C.c_void_p()
        _check(_lib.tally_create(C.byref(h), C.c_void_p(stream_hi.cuda_stream),
                                 C.c_void_p(stream_be.cuda_stream)), "tally_create")
        self.h = h

    def close(self):
        if self.h is not None:
            _check(_lib.tally_destroy(self.h), "tally_destroy")
            self.h = None

    def launch_native(self, kernel, hi=False):
        _check(_lib.tally_launch_native(self.h, C.byref(kernel.desc), 1 if hi else 0),
               "tally_launch_native")

    def launch_attn_decode_static(self, q, Kc, Vc, out, hi=False):
        """Decode attention with the library's own static split records (allocates nothing)."""
        tokens, heads, dim = Kc.shape
        args = AttnDecodeArgs(q.data_ptr(), Kc.data_ptr(), Vc.data_ptr(), out.data_ptr(), None,
                              tokens, heads, dim)
        _check(_lib.tally_launch_attn_decode_static(self.h, C.byref(args), 1 if hi else 0),
               "tally_launch_attn_decode_static")

    def launch_sliced(self, kernel, slice_blocks, max_in_flight=1, coverage=False):
        j = C.c_void_p()
        _check(_lib.tally_launch_sliced(self.h, C.byref(kernel.desc), slice_blocks, max_in_flight,
                                        int(coverage), C.byref(j)), "tally_launch_sliced")
        return Job(j, kernel)

    def launch_ptb(self, kernel, workers, chunk=1, coverage=False, stop_at=None):
        j = C.c_void_p()
        if stop_at is None:
            _check(_lib.tally_launch_ptb(self.h, C.byref(kernel.desc), workers, chunk,
                                         int(coverage), C.byref(j)), "tally_launch_ptb")
        else:
            _check(_lib.tally_launch_ptb_until(self.h, C.byref(kernel.desc), workers, chunk,
                                               int(stop_at), int(coverage), C.byref(j)),
                   "tally_launch_ptb_until")
        return Job(j, kernel)

    def set_yield_bound_us(self, us):
        _check(_lib.tally_set_yield_bound_us(self.h, int(us)), "tally_set_yield_bound_us")

    def stream_report(self):
        """Whether the caller's best-effort stream delays the high-priority one, and how many
        streams the library created and set aside because they would."""
        a, b = C.c_int(), C.c_uint32()
        _check(_lib.tally_stream_report(self.h, C.byref(a), C.byref(b)), "tally_stream_report")
        return {"be_delays_hi": bool(a.value & 1), "crowded": bool(a.value & 2), "set_aside": b.value}

    def set_yield_every(self, steps):
        _check(_lib.tally_set_yield_every(self.h, int(steps)), "tally_set_yield_every")

    def marker(self, value, hi=True):
        _check(_lib.tally_marker(self.h, 1 if hi else 0, value), "tally_marker")

    def marker_read(self, hi=True):
        v = C.c_uint32()
        _check(_lib.tally_marker_read(self.h, 1 if hi else 0, C.byref(v)), "tally_marker_read")
        return v.value

    def profile(self, kernel, candidates, runs=10, threshold_ms=0.0316):
        """candidates: list of (kind, param, chunk).  Returns (list of dicts, chosen index)."""
        arr = (Config * len(candidates))(*[Config(k, p, c, 0.0, 0.0) for k, p, c in candidates])
        chosen = C.c_uint32()
        _check(_lib.tally_profile(self.h, C.byref(kernel.desc), arr, len(candidates), runs,
                                  threshold_ms, C.byref(chosen)), "tally_profile")
        out = [dict(kind=c.kind, param=c.param, chunk=c.chunk, latency_ms=c.latency_ms,
                    turnaround_ms=c.turnaround_ms) for c in arr]
        return out, chosen.value

    def candidate_configs(self, kernel, cap=64):
        """The Section 4.2 candidate set of a kernel as a list of (kind, param, chunk)."""
        arr = (Config * cap)()
        n = C.c_uint32()
        _check(_lib.tally_candidate_configs(self.h, C.byref(kernel.desc), arr, cap, C.byref(n)),
               "tally_candidate_configs")
        return [(arr[i].kind, arr[i].param, arr[i].chunk) for i in range(n.value)]

    def profile_table(self, kernel, cap=64):
        """(list of candidate dicts with their sample counts, index of the fixed choice or -1)."""
        arr = (Config * cap)()
        smp = (C.c_uint32 * cap)()
        n, chosen = C.c_uint32(), C.c_int()
        _check(_lib.tally_profile_table(self.h, C.byref(kernel.desc), arr, cap, C.byref(n), smp,
                                        C.byref(chosen)), "tally_profile_table")
        rows = [dict(kind=arr[i].kind, param=arr[i].param, chunk=arr[i].chunk,
                     latency_ms=arr[i].latency_ms, turnaround_ms=arr[i].turnaround_ms,
                     samples=smp[i]) for i in range(min(n.value, cap))]
        return rows, chosen.value

    def profile_reset(self):
        _check(_lib.tally_profile_reset(self.h), "tally_profile_reset")

    def scheduler(self, policy=POLICY_TALLY, be_clients=1, threshold_ms=0.0, profile_runs=0, flags=0):
        return Scheduler(self, policy, be_clients, threshold_ms, profile_runs, flags)

    def mfma_ceiling_tflops(self, reps=10):
        """Measured bf16 matrix-pipe ceiling (register-only MFMA loop on every compute unit)."""
        v = C.c_double()
        _check(_lib.tally_mfma_ceiling_tflops(self.h, reps, C.byref(v)), "tally_mfma_ceiling_tflops")
        return v.value

    def kernel_footprint(self, kernel_id, form):
        """(LDS bytes, waves, registers per lane) of one workgroup; form 0 = persistent
        workers, 1 = original form."""
        a, b, c = C.c_uint32(), C.c_uint32(), C.c_uint32()
        _check(_lib.tally_kernel_footprint(self.h, kernel_id, form, C.byref(a), C.byref(b), C.byref(c)),
               "tally_kernel_footprint")
        return a.value, b.value, c.value

    def max_workers(self, kernel):
        """Largest worker count whose workgroups are all resident at once."""
        n = C.c_uint32()
        _check(_lib.tally_max_workers(self.h, C.byref(kernel.desc), C.byref(n)), "tally_max_workers")
        return n.value

    def lookup_config(self, kernel):
        c = Config()
        rc = _lib.tally_lookup_config(self.h, C.byref(kernel.desc), C.byref(c))
        if rc == ERR_BAD_STATE:
            return None
        _check(rc, "tally_lookup_config")
        return dict(kind=c.kind, param=c.param, chunk=c.chunk, latency_ms=c.latency_ms,
                    turnaround_ms=c.turnaround_ms)

    def sched_run(self, hi_kernels, arrivals_us, be_items, policy=POLICY_TALLY, tail_us=0.0,
                  be_clients=None, threshold_ms=0.0, profile_runs=0, flags=0, be_toggle_every=0):
        """hi_kernels: list of Kernel (one request).  be_items: list of (Kernel, (kind, param,
        chunk)).  be_clients: optional list of item counts, one per best-effort client (the
        items are the concatenation of the clients' steps).  Returns a dict of numpy arrays
        and counters."""
        n_hi = len(hi_kernels)
        hi_arr = (KernelDesc * max(n_hi, 1))(*[k.desc for k in hi_kernels])
        arrivals = np.ascontiguousarray(arrivals_us, dtype=np.float64)
        lat = np.zeros(len(arrivals), dtype=np.float64)
        cap = max(len(arrivals), 1)
        pre = np.zeros(cap, dtype=np.float64)
        items = (BeItem * max(len(be_items), 1))()
        for i, (k, cfg) in enumerate(be_items):
            items[i].kernel = C.pointer(k.desc)
            items[i].config = Config(cfg[0], cfg[1], cfg[2] if len(cfg) > 2 else 1, 0.0, 0.0)
        run = SchedRun()
        run.hi_kernels = hi_arr
        run.n_hi_kernels = n_hi
        run.arrivals_us = arrivals.ctypes.data_as(C.POINTER(C.c_double))
        run.n_arrivals = len(arrivals)
        run.be_items = items
        run.n_be_items = len(be_items)
        run.policy = policy
        run.tail_us = float(tail_us)
        run.threshold_ms = float(threshold_ms)
        run.profile_runs = int(profile_runs)
        run.sched_flags = int(flags)
        run.be_toggle_every = int(be_toggle_every)
        run.latency_us = lat.ctypes.data_as(C.POINTER(C.c_double))
        run.preempt_latency_us = pre.ctypes.data_as(C.POINTER(C.c_double))
        run.preempt_cap = cap
        per_client = None
        if be_clients is not None:
            counts = (C.c_uint32 * len(be_clients))(*be_clients)
            per_client = np.zeros(len(be_clients), dtype=np.uint64)
            run.be_client_items = counts
            run.n_be_clients = len(be_clients)
            run.be_client_kernels_done = per_client.ctypes.data_as(C.POINTER(C.c_uint64))
        issue = np.zeros(len(arrivals), dtype=np.float64)
        run.issue_us = issue.ctypes.data_as(C.POINTER(C.c_double))
        _check(_lib.tally_sched_run(self.h, C.byref(run)), "tally_sched_run")
        return {
            "latency_us": lat,
            "issue_us": issue,
            "preempt_latency_us": pre[: min(run.n_preempts, cap)].copy(),
            "n_preempts": run.n_preempts,
            "be_kernels_done": run.be_kernels_done,
            "be_steps_done": run.be_steps_done,
            "window_us": run.window_us,
            "be_client_kernels_done": per_client,
            "be_enabled_us": run.be_enabled_us,
            "profile_samples": run.profile_samples,
            "configs_fixed": run.configs_fixed,
        }


class Scheduler:
    """The priority scheduler as a running service (tally_sched_*)."""

    def __init__(self, ctx, policy, be_clients, threshold_ms, profile_runs, flags):
        self.ctx = ctx
        self._keep = []
        opts = SchedOpts(policy, be_clients, float(threshold_ms), int(profile_runs), int(flags))
        h = C.c_void_p()
        _check(_lib.tally_sched_create(ctx.h, C.byref(opts), C.byref(h)), "tally_sched_create")
        self.h = h

    def submit_be(self, kernel, config=None, client=0, loop=False, end_of_step=False):
        self._keep.append(kernel)
        cfg = None
        if config is not None:
            cfg = C.byref(Config(config[0], config[1], config[2] if len(config) > 2 else 1, 0.0, 0.0))
        flags = (SUBMIT_LOOP if loop else 0) | (SUBMIT_END_OF_STEP if end_of_step else 0)
        _check(_lib.tally_sched_submit_be(self.h, client, C.byref(kernel.desc), cfg, flags),
               "tally_sched_submit_be")

    def submit_hi(self, kernels):
        arr = (KernelDesc * len(kernels))(*[k.desc for k in kernels])
        _check(_lib.tally_sched_submit_hi(self.h, arr, len(kernels)), "tally_sched_submit_hi")

    def poll(self, more_pending=False):
        """True while the high-priority request is still in flight."""
        f = C.c_int()
        _check(_lib.tally_sched_poll(self.h, 1 if more_pending else 0, C.byref(f)), "tally_sched_poll")
        return bool(f.value)

    def enable_be(self, on=True):
        _check(_lib.tally_sched_enable_be(self.h, 1 if on else 0), "tally_sched_enable_be")

    def stats(self):
        st = SchedStats()
        _check(_lib.tally_sched_stats(self.h, C.byref(st)), "tally_sched_stats")
        return {"hi_requests_done": st.hi_requests_done, "be_kernels_done": st.be_kernels_done,
                "be_steps_done": st.be_steps_done,
                "be_client_kernels_done": list(st.be_client_kernels_done),
                "n_preempts": st.n_preempts, "profile_samples": st.profile_samples,
                "configs_fixed": st.configs_fixed}

    def take_preempt_latencies(self, cap=4096):
        buf = (C.c_double * cap)()
        n = C.c_uint32()
        _check(_lib.tally_sched_take_preempt_latencies(self.h, buf, cap, C.byref(n)),
               "tally_sched_take_preempt_latencies")
        return np.array(buf[: n.value], dtype=np.float64)

    def close(self):
        if self.h is not None:
            h, self.h = self.h, None
            _check(_lib.tally_sched_destroy(h), "tally_sched_destroy")


def device_info():
    a, b, c = C.c_uint32(), C.c_uint32(), C.c_uint32()
    _check(_lib.tally_device_info(C.byref(a), C.byref(b), C.byref(c)), "tally_device_info")
    return {"num_cus": a.value, "lds_bytes_per_cu": b.value, "wave_size": c.value}


def ptb_turnaround_ms(latency_ms, workers, chunk, total):
    return _lib.tally_ptb_turnaround_ms(latency_ms, workers, chunk, total)


PARTS_UNEVEN = 0xFFFFFFFF


def parts_executions(pieces, which):
    """How often a block handed out in parts ran as a whole (coverage records)."""
    return _lib.tally_parts_executions(pieces, which)


def select_config(cands, threshold_ms=0.0316):
    """cands: list of dicts with kind, param, latency_ms, turnaround_ms (chunk optional)."""
    arr = (Config * len(cands))(*[Config(c["kind"], c["param"], c.get("chunk", 1),
                                         c["latency_ms"], c["turnaround_ms"]) for c in cands])
    return _lib.tally_select_config(arr, len(cands), threshold_ms)
