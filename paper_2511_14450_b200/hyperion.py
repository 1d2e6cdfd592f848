"""ctypes binding of libhyperion: the same names as the C ABI, argument marshalling only.

Every step of the path runs inside the library's CUDA kernels.  If the shared library has not been
built this module raises on first use; there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "lib", "libhyperion.so")

HYP_OK, HYP_EINVAL, HYP_ENOMEM, HYP_ECAPACITY, HYP_EINFEASIBLE, HYP_ECUDA, HYP_ESTATE = 0, -1, -2, -3, -4, -5, -6
HYP_ETIMEOUT = -7
(HYP_W_QKV, HYP_W_O, HYP_W_GATE_UP, HYP_W_DOWN, HYP_W_NORM1, HYP_W_NORM2, HYP_W_EMBED, HYP_W_FINAL_NORM,
 HYP_W_LM_HEAD) = range(9)
HYP_BATCH_ALL_LOGITS = 1
HYP_MAX_DECODE_BATCH = 128


class hyp_cfg(C.Structure):
    _fields_ = [("n_layers_total", C.c_int32), ("hidden", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("ffn", C.c_int32), ("vocab", C.c_int32),
                ("rms_eps", C.c_float), ("rope_theta", C.c_float), ("kv_block_size", C.c_int32),
                ("max_seqs", C.c_int32), ("max_ctx", C.c_int32), ("max_tokens", C.c_int32),
                ("kv_pages", C.c_int32)]


class hyp_batch(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("seq_ids", C.POINTER(C.c_int32)), ("q_lens", C.POINTER(C.c_int32)),
                ("ctx_lens", C.POINTER(C.c_int32)), ("flags", C.c_int32)]


class hyp_node_state(C.Structure):
    _fields_ = [("C", C.c_double), ("M_avail", C.c_double), ("F_rem", C.c_double), ("F_wait", C.c_double),
                ("available", C.c_int32)]


class hyp_attn_shape(C.Structure):
    _fields_ = [("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32)]


class hyp_attn_mod(C.Structure):
    _fields_ = [("softcap", C.c_float), ("window", C.c_int32), ("slopes", C.c_void_p), ("prefix_lens", C.c_void_p)]


class HyperionError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().hyp_strerror(code).decode()
        if code == HYP_ECUDA:
            msg += f" [cudaError {lib().hyp_last_cuda_error()}]"
        super().__init__(f"{where}: {msg} ({code})")


_LIB: Optional[C.CDLL] = None

# every exported symbol with (restype, argtypes); the export test walks this table
SIGNATURES = {
    "hyp_stage_create": (C.c_int, [C.c_int32, C.c_int32, C.POINTER(hyp_cfg), C.POINTER(C.c_void_p)]),
    "hyp_stage_load": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hyp_stage_prefill": (C.c_int, [C.c_void_p, C.POINTER(hyp_batch), C.c_void_p, C.c_void_p, C.c_void_p]),
    "hyp_stage_decode": (C.c_int, [C.c_void_p, C.POINTER(hyp_batch), C.c_void_p, C.c_void_p, C.c_void_p]),
    "hyp_stage_prefill_host": (C.c_int, [C.c_void_p, C.POINTER(hyp_batch), C.c_void_p, C.c_void_p, C.c_void_p]),
    "hyp_stage_decode_host": (C.c_int, [C.c_void_p, C.POINTER(hyp_batch), C.c_void_p, C.c_void_p, C.c_void_p]),
    "hyp_stage_profile": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_float),
                                    C.POINTER(C.c_size_t), C.c_void_p]),
    "hyp_stage_kernel_timing": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32]),
    "hyp_stage_kernel_timing_read": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_double)]),
    "hyp_stage_free_seq": (C.c_int, [C.c_void_p, C.c_int32]),
    "hyp_stage_seq_len": (C.c_int, [C.c_void_p, C.c_int32]),
    "hyp_stage_free_pages": (C.c_int, [C.c_void_p]),
    "hyp_stage_launch_count": (C.c_int64, [C.c_void_p]),
    "hyp_stage_destroy": (None, [C.c_void_p]),
    "hyp_split_dp": (C.c_int, [C.c_int32, C.c_int32, C.POINTER(C.c_double), C.POINTER(C.c_double),
                               C.POINTER(C.c_double), C.POINTER(C.c_double), C.c_double, C.POINTER(C.c_int32),
                               C.POINTER(C.c_double)]),
    "hyp_split_even": (C.c_int, [C.c_int32, C.c_int32, C.POINTER(C.c_double), C.POINTER(C.c_double),
                                 C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(C.c_int32),
                                 C.POINTER(C.c_double)]),
    "hyp_split_greedy": (C.c_int, [C.c_int32, C.c_int32, C.POINTER(C.c_double), C.POINTER(C.c_double),
                                   C.POINTER(C.c_double), C.POINTER(C.c_double), C.POINTER(C.c_int32),
                                   C.POINTER(C.c_double)]),
    "hyp_sched_rt": (C.c_int, [C.c_double, C.c_double, C.POINTER(hyp_node_state), C.c_int32, C.POINTER(C.c_int32)]),
    "hyp_op_rmsnorm": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float, C.c_void_p]),
    "hyp_op_weight_packed_bytes": (C.c_size_t, [C.c_int32, C.c_int32, C.c_int32]),
    "hyp_op_pack_weight": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hyp_tune": (C.c_int, [C.c_int32, C.c_int32]),
    "hyp_op_gemm": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                              C.c_int32, C.c_void_p]),
    "hyp_op_pack_weight_f16": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hyp_op_gemm_f16": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                  C.c_int32, C.c_void_p]),
    "hyp_device_wait_status": (C.c_int, [C.POINTER(C.c_int32), C.c_int32]),
    "hyp_op_attn_decode_splits": (C.c_int, [C.c_int32, C.c_int32, C.c_int32]),
    "hyp_op_attn_decode_scratch_bytes": (C.c_size_t, [C.c_int32, C.c_int32, C.c_int32, C.c_int32]),
    "hyp_op_attn_decode": (C.c_int, [C.POINTER(hyp_attn_shape), C.c_int32, C.c_void_p, C.c_int32, C.c_void_p,
                                     C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_size_t,
                                     C.c_void_p, C.c_void_p]),
    "hyp_op_attn_decode_static": (C.c_int, [C.POINTER(hyp_attn_shape), C.c_int32, C.c_void_p, C.c_int32, C.c_void_p,
                                            C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]),
    "hyp_op_attn_decode_step": (C.c_int, [C.POINTER(hyp_attn_shape), C.c_int32, C.c_void_p, C.c_int32, C.c_void_p,
                                          C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                          C.c_void_p]),
    "hyp_op_attn_prefill": (C.c_int, [C.POINTER(hyp_attn_shape), C.c_int32, C.c_int32, C.c_void_p, C.c_int32,
                                      C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.c_void_p]),
    "hyp_op_mx4_quantize": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]),
    "hyp_op_mx4_dequantize": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p]),
    "hyp_op_mx4_packed_bytes": (C.c_size_t, [C.c_int32, C.c_int32, C.c_int32]),
    "hyp_op_mx4_pack": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hyp_op_gemm_mx4_scratch_bytes": (C.c_size_t, [C.c_int32, C.c_int32, C.c_int32]),
    "hyp_op_gemm_mx4_plan": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_int32)]),
    "hyp_op_gemm_mx4": (C.c_int, [C.c_void_p, C.c_int32, C.c_int64, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                  C.c_void_p, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]),
    "hyp_op_kv8_write": (C.c_int, [C.POINTER(hyp_attn_shape), C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int32, C.c_int64,
                                   C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                   C.c_void_p]),
    "hyp_op_kv8_read": (C.c_int, [C.POINTER(hyp_attn_shape), C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                  C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]),
    "hyp_op_attn_kv8_scratch_bytes": (C.c_size_t, [C.POINTER(hyp_attn_shape), C.c_int32, C.c_int32]),
    "hyp_op_attn_decode_kv8": (C.c_int, [C.POINTER(hyp_attn_shape), C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                         C.c_int32, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]),
    "hyp_op_attn_mod_scratch_bytes": (C.c_size_t, [C.POINTER(hyp_attn_shape), C.c_int32, C.c_int32]),
    "hyp_op_attn_decode_mod": (C.c_int, [C.POINTER(hyp_attn_shape), C.POINTER(hyp_attn_mod), C.c_int32, C.c_void_p, C.c_int64,
                                         C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p,
                                         C.c_void_p]),
    "hyp_op_attn_prefill_mod": (C.c_int, [C.POINTER(hyp_attn_shape), C.POINTER(hyp_attn_mod), C.c_int32, C.c_int32, C.c_void_p,
                                          C.c_int64, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                          C.c_void_p]),
    "hyp_op_attn_scored_scratch_bytes": (C.c_size_t, [C.POINTER(hyp_attn_shape), C.c_int32, C.c_int32]),
    "hyp_op_attn_decode_scored": (C.c_int, [C.POINTER(hyp_attn_shape), C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                            C.c_int32, C.c_void_p, C.c_float, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p,
                                            C.c_size_t, C.c_void_p, C.c_void_p]),
    "hyp_op_kv_evict": (C.c_int, [C.POINTER(hyp_attn_shape), C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                  C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32,
                                  C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]),
    "hyp_op_attn_shared_scratch_bytes": (C.c_size_t, [C.POINTER(hyp_attn_shape), C.c_int32, C.c_int32, C.c_int32, C.c_int32]),
    "hyp_op_attn_decode_shared": (C.c_int, [C.POINTER(hyp_attn_shape), C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int32,
                                            C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                            C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]),
    "hyp_strerror": (C.c_char_p, [C.c_int]),
    "hyp_last_cuda_error": (C.c_int, []),
}


def lib() -> C.CDLL:
    """Load libhyperion.so (built in-tree by `paper_2511_14450_b200.build`)."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2511_14450_b200.build` "
                               "(there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _LIB = L
    return _LIB


def _check(code: int, where: str):
    if code != HYP_OK:
        raise HyperionError(code, where)


def _i32(seq: Sequence[int]):
    return (C.c_int32 * len(seq))(*[int(v) for v in seq])


def _f64(seq):
    return (C.c_double * len(seq))(*[float(v) for v in seq])


def _ptr(t) -> int:
    """Address of a torch tensor / numpy array / raw int."""
    if isinstance(t, int):
        return t
    if hasattr(t, "data_ptr"):
        return t.data_ptr()
    return t.ctypes.data


def _stream_handle(stream) -> int:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_cfg(shape, max_seqs: int, max_ctx: int, max_tokens: int, kv_pages: int = 0) -> hyp_cfg:
    return hyp_cfg(shape.n_layers_total, shape.hidden, shape.n_q_heads, shape.n_kv_heads, shape.head_dim,
                   shape.ffn, shape.vocab, shape.rms_eps, shape.rope_theta, shape.kv_block_size,
                   max_seqs, max_ctx, max_tokens, kv_pages)


def make_batch(seq_ids, q_lens, ctx_lens, flags: int = 0):
    """Returns (hyp_batch, keepalive) - keep `keepalive` referenced until the call returns."""
    a, b, c = _i32(seq_ids), _i32(q_lens), _i32(ctx_lens)
    hb = hyp_batch(len(seq_ids), a, b, c, flags)
    return hb, (a, b, c)


# --------------------------------------------------------------------------------------------
# same names as the C ABI
# --------------------------------------------------------------------------------------------
def hyp_stage_create(layer_lo: int, layer_hi: int, cfg: hyp_cfg) -> int:
    h = C.c_void_p()
    _check(lib().hyp_stage_create(layer_lo, layer_hi, C.byref(cfg), C.byref(h)), "hyp_stage_create")
    return h.value


def hyp_stage_load(stage: int, layer: int, tensor_id: int, src, stream=None):
    nbytes = src.numel() * src.element_size()
    _check(lib().hyp_stage_load(stage, layer, tensor_id, _ptr(src), nbytes, _stream_handle(stream)),
           "hyp_stage_load")


def _run(fn_name, stage, seq_ids, q_lens, ctx_lens, inp, out, stream, flags):
    hb, keep = make_batch(seq_ids, q_lens, ctx_lens, flags)
    _check(getattr(lib(), fn_name)(stage, C.byref(hb), _ptr(inp), _ptr(out), _stream_handle(stream)), fn_name)
    del keep


def hyp_stage_prefill(stage, seq_ids, q_lens, ctx_lens, inp, out, stream=None, flags=0):
    _run("hyp_stage_prefill", stage, seq_ids, q_lens, ctx_lens, inp, out, stream, flags)


def hyp_stage_decode(stage, seq_ids, ctx_lens, inp, out, stream=None):
    _run("hyp_stage_decode", stage, seq_ids, [1] * len(seq_ids), ctx_lens, inp, out, stream, 0)


def hyp_stage_prefill_host(stage, seq_ids, q_lens, ctx_lens, inp, out, stream=None, flags=0):
    _run("hyp_stage_prefill_host", stage, seq_ids, q_lens, ctx_lens, inp, out, stream, flags)


def hyp_stage_decode_host(stage, seq_ids, ctx_lens, inp, out, stream=None):
    _run("hyp_stage_decode_host", stage, seq_ids, [1] * len(seq_ids), ctx_lens, inp, out, stream, 0)


def hyp_stage_profile(stage, n_layers: int, mode: int, batch: int, ctx: int, iters: int = 5, stream=None):
    ms = (C.c_float * n_layers)()
    by = (C.c_size_t * n_layers)()
    _check(lib().hyp_stage_profile(stage, mode, batch, ctx, iters, ms, by, _stream_handle(stream)),
           "hyp_stage_profile")
    return list(ms), list(by)


(HYP_K_GEMM_QKV, HYP_K_GEMM_O, HYP_K_GEMM_GATE_UP, HYP_K_GEMM_DOWN, HYP_K_ATTN, HYP_K_NORM, HYP_K_ROPE,
 HYP_K_LM_HEAD) = range(8)


def hyp_stage_kernel_timing(stage, kernel_class: int, max_samples: int):
    _check(lib().hyp_stage_kernel_timing(stage, kernel_class, max_samples), "hyp_stage_kernel_timing")


def hyp_stage_kernel_timing_read(stage):
    """Returns (launches recorded, their summed milliseconds)."""
    n, ms = C.c_int32(), C.c_double()
    _check(lib().hyp_stage_kernel_timing_read(stage, C.byref(n), C.byref(ms)), "hyp_stage_kernel_timing_read")
    return n.value, ms.value


def hyp_stage_free_seq(stage, seq_id: int):
    _check(lib().hyp_stage_free_seq(stage, seq_id), "hyp_stage_free_seq")


def hyp_stage_seq_len(stage, seq_id: int) -> int:
    r = lib().hyp_stage_seq_len(stage, seq_id)
    if r < 0:
        raise HyperionError(r, "hyp_stage_seq_len")
    return r


def hyp_stage_free_pages(stage) -> int:
    r = lib().hyp_stage_free_pages(stage)
    if r < 0:
        raise HyperionError(r, "hyp_stage_free_pages")
    return r


def hyp_stage_launch_count(stage) -> int:
    return lib().hyp_stage_launch_count(stage)


def hyp_stage_destroy(stage):
    lib().hyp_stage_destroy(stage)


def hyp_split_dp(f, m, Cap, Mcap, eps: float = 0.0):
    """Returns (p, tau): p = tuple of 1-based last-block indices of tiers 1..T-1."""
    N, T = len(f), len(Cap)
    p = (C.c_int32 * max(T - 1, 1))()
    tau = C.c_double()
    _check(lib().hyp_split_dp(N, T, _f64(f), _f64(m), _f64(Cap), _f64(Mcap), eps, p, C.byref(tau)), "hyp_split_dp")
    return tuple(p[j] for j in range(T - 1)), tau.value


def _split_baseline(name, f, m, Cap, Mcap, tolerate_infeasible):
    N, T = len(f), len(Cap)
    p = (C.c_int32 * max(T - 1, 1))()
    tau = C.c_double()
    code = getattr(lib(), name)(N, T, _f64(f), _f64(m), _f64(Cap), _f64(Mcap), p, C.byref(tau))
    if not (tolerate_infeasible and code == HYP_EINFEASIBLE and N >= T):
        _check(code, name)
    return tuple(p[j] for j in range(T - 1)), tau.value, code == HYP_OK


def hyp_split_even(f, m, Cap, Mcap):
    """Equal-count contiguous partition.  Returns (p, tau, fits): fits is False if a memory limit is exceeded."""
    return _split_baseline("hyp_split_even", f, m, Cap, Mcap, True)


def hyp_split_greedy(f, m, Cap, Mcap):
    """Memory-aware greedy contiguous partition.  Returns (p, tau); raises HYP_EINFEASIBLE if it finds none."""
    p, tau, _ = _split_baseline("hyp_split_greedy", f, m, Cap, Mcap, False)
    return p, tau


def hyp_sched_rt(F_new: float, m_act: float, nodes) -> int:
    """nodes: sequence of (C, M_avail, F_rem, F_wait_total, available).  Returns the 0-based node."""
    arr = (hyp_node_state * len(nodes))(*[hyp_node_state(*n) for n in nodes])
    k = C.c_int32(-1)
    _check(lib().hyp_sched_rt(F_new, m_act, arr, len(nodes), C.byref(k)), "hyp_sched_rt")
    return k.value


# --------------------------------------------------------------------------------------------
# single-kernel entry points (hyperion_ops.h)
# --------------------------------------------------------------------------------------------
HYP_EPI_STORE_BF16, HYP_EPI_RESID_F32, HYP_EPI_SWIGLU_BF16, HYP_EPI_STORE_F32 = range(4)


def hyp_op_rmsnorm(x, g, out, eps: float, stream=None):
    M, H = x.shape
    _check(lib().hyp_op_rmsnorm(_ptr(x), _ptr(g), _ptr(out), M, H, eps, _stream_handle(stream)), "hyp_op_rmsnorm")


(HYP_TUNE_PDL, HYP_TUNE_STREAM_SLOTS, HYP_TUNE_ATTN_SPLITS, HYP_TUNE_ATTN_SLOTS, HYP_TUNE_STREAM_ROTATION,
 HYP_TUNE_SWAP_MIN_ROWS, HYP_TUNE_SWAP_MAX_ROWS, HYP_TUNE_SWAP_EPILOGUES, HYP_TUNE_PREFILL_ATTN_TC,
 HYP_TUNE_FIRST_BLOCK_SPLIT, HYP_TUNE_TILE_224, HYP_TUNE_WAIT_LIMIT_US, HYP_TUNE_STREAM_WITHHOLD_COPY,
 HYP_TUNE_STREAM_ACT_DEPTH, HYP_TUNE_STREAM_ACT_TMA, HYP_TUNE_ATTN_GLOBAL_MERGE) = range(16)


def hyp_tune(key: int, value: int):
    _check(lib().hyp_tune(key, value), "hyp_tune")


def _packed_buffer(nbytes: int, device, stream):
    """Bytes that a kernel on `stream` fills, from that stream's own memory: what another stream has freed it may still be using."""
    import torch
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def hyp_op_pack_weight(w, N: int, swiglu: bool, stream=None, f16: bool = False):
    """Packed copy of a bf16 [N (2N for SwiGLU), K] weight matrix, as hyp_op_gemm reads it (a uint8 tensor);
    f16: the values converted to fp16 on the way (hyp_op_pack_weight_f16, for hyp_op_gemm_f16).  The copy is memory of `stream`:
    for use on another stream, as with any tensor, wait for it and tell the allocator (record_stream)."""
    K = w.shape[1]
    nbytes = lib().hyp_op_weight_packed_bytes(N, K, int(swiglu))
    if nbytes == 0:
        raise HyperionError(HYP_EINVAL, "hyp_op_weight_packed_bytes")
    packed = _packed_buffer(nbytes, w.device, stream)
    name = "hyp_op_pack_weight_f16" if f16 else "hyp_op_pack_weight"
    _check(getattr(lib(), name)(_ptr(w), N, K, int(swiglu), _ptr(packed), nbytes, _stream_handle(stream)), name)
    return packed


def hyp_op_gemm(a, w_packed, N: int, epilogue: int, out, stream=None):
    M, K = a.shape
    _check(lib().hyp_op_gemm(_ptr(a), _ptr(w_packed), M, N, K, epilogue, _ptr(out), out.stride(0),
                             _stream_handle(stream)), "hyp_op_gemm")


def hyp_op_gemm_f16(a, w_packed, N: int, epilogue: int, out, stream=None):
    M, K = a.shape
    _check(lib().hyp_op_gemm_f16(_ptr(a), _ptr(w_packed), M, N, K, epilogue, _ptr(out), out.stride(0),
                                 _stream_handle(stream)), "hyp_op_gemm_f16")


def hyp_device_wait_status(clear: bool = False) -> int:
    """Code recorded by a kernel whose bounded wait ran out (0 = none); synchronises the device."""
    code = C.c_int32(0)
    _check(lib().hyp_device_wait_status(C.byref(code), int(clear)), "hyp_device_wait_status")
    return code.value


def hyp_op_attn_decode_splits(n_seqs: int, n_kv_heads: int, max_ctx: int) -> int:
    return lib().hyp_op_attn_decode_splits(n_seqs, n_kv_heads, max_ctx)


def hyp_op_attn_decode_scratch_bytes(n_seqs: int, n_q_heads: int, head_dim: int, n_splits: int) -> int:
    return lib().hyp_op_attn_decode_scratch_bytes(n_seqs, n_q_heads, head_dim, n_splits)


def hyp_op_attn_decode(shape3, q, kv_pages, block_table, ctx_lens, n_splits, scratch, out, stream=None):
    """shape3 = (n_q_heads, n_kv_heads, head_dim); tensors are CUDA tensors laid out as the header says."""
    sh = hyp_attn_shape(*shape3)
    _check(lib().hyp_op_attn_decode(C.byref(sh), q.shape[0], _ptr(q), q.stride(0), _ptr(kv_pages), _ptr(block_table),
                                    block_table.stride(0), _ptr(ctx_lens), n_splits, _ptr(scratch),
                                    scratch.numel() * scratch.element_size(), _ptr(out), _stream_handle(stream)),
           "hyp_op_attn_decode")


HYP_STATIC_SCRATCH_BYTES = 4 << 20


def hyp_op_attn_decode_static(shape3, q, kv_pages, block_table, ctx_lens, n_splits, out, stream=None):
    """Decode attention that allocates nothing: split partials go to the library's built-in 4 MiB
    device array (shared by all calls on the device; calls that may overlap on the GPU race on it).
    Raises HYP_ECAPACITY if this batch's partials would not fit."""
    sh = hyp_attn_shape(*shape3)
    _check(lib().hyp_op_attn_decode_static(C.byref(sh), q.shape[0], _ptr(q), q.stride(0), _ptr(kv_pages),
                                           _ptr(block_table), block_table.stride(0), _ptr(ctx_lens), n_splits,
                                           _ptr(out), _stream_handle(stream)), "hyp_op_attn_decode_static")


def hyp_op_attn_decode_step(shape3, qkv, kv_pages, block_table, ctx_lens, rope_table, n_splits, out, stream=None):
    sh = hyp_attn_shape(*shape3)
    _check(lib().hyp_op_attn_decode_step(C.byref(sh), qkv.shape[0], _ptr(qkv), qkv.stride(0), _ptr(kv_pages),
                                         _ptr(block_table), block_table.stride(0), _ptr(ctx_lens), _ptr(rope_table),
                                         n_splits, _ptr(out), _stream_handle(stream)), "hyp_op_attn_decode_step")


def hyp_op_attn_prefill(shape3, q, kv_pages, block_table, cu_q, ctx_lens, out, stream=None):
    sh = hyp_attn_shape(*shape3)
    _check(lib().hyp_op_attn_prefill(C.byref(sh), ctx_lens.shape[0], q.shape[0], _ptr(q), q.stride(0), _ptr(kv_pages),
                                     _ptr(block_table), block_table.stride(0), _ptr(cu_q), _ptr(ctx_lens), _ptr(out),
                                     _stream_handle(stream)), "hyp_op_attn_prefill")


# --------------------------------------------------------------------------------------------
# operators over the paged cache (hyperion_ops.h).  These check their tensors: type, device, shape, strides; a call that
# does not fit raises HYP_EINVAL before anything is launched, and a call on tensors of another device than the current one
# runs there (on that device's current stream unless one is given).
# A small call runs for a few microseconds on the device, so the checks are written to cost little: one comparison a
# property, the message is only formed where one fails, and the ctypes shape of a head layout is made once.
# --------------------------------------------------------------------------------------------
_F16 = _F32 = _I32 = _raw_stream = _current_device = None
_SHAPES = {}


def _bind_torch():
    global _F16, _F32, _I32, _raw_stream, _current_device
    import torch
    _F16, _F32, _I32, _current_device = torch.float16, torch.float32, torch.int32, torch.cuda.current_device
    # the stream's address without making a Stream object of it, where this torch has the call
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)


def _refuse(where: str, why: str):
    err = HyperionError(HYP_EINVAL, where)
    err.args = (f"{where}: {why} ({HYP_EINVAL})",)
    raise err


def _shape(shape3):
    s = _SHAPES.get(shape3 if type(shape3) is tuple else tuple(shape3))
    if s is None:
        if _F16 is None:
            _bind_torch()
        s = _SHAPES[tuple(shape3)] = C.byref(hyp_attn_shape(*shape3))
    return s


def _dense(where, name, t, dtype, dev, shape):
    """The address of a contiguous tensor of this type and shape on device `dev`."""
    if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous() or t.shape != shape:
        _refuse(where, f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on device {dev}, not {t.dtype} "
                       f"{tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _rows(where, name, t, dtype, dev, lead):
    """(address, size of the last dimension) of a contiguous tensor whose other dimensions are `lead`."""
    s = t.shape
    if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous() or not s or s[:-1] != lead:
        _refuse(where, f"{name} must be a contiguous {dtype} tensor of shape {(*lead, '*')} on device {dev}, not {t.dtype} "
                       f"{tuple(s)} on {t.device}")
    return t.data_ptr(), s[-1]


def _pool(where, name, t, dev, shape3):
    s = t.shape
    if t.dtype is not _F16 or t.get_device() != dev or not t.is_contiguous() or s[1:] != (2, shape3[1], 16, shape3[2]):
        _refuse(where, f"{name} must be a contiguous fp16 page pool [pages, 2, {shape3[1]}, 16, {shape3[2]}] on device {dev}, not {t.dtype} "
                       f"{tuple(s)} on {t.device}")
    return t.data_ptr()


def _query(where, q, shape3):
    """(device, rows, address, row stride) of the query matrix: dense rows, which may lie in a wider buffer."""
    width = shape3[0] * shape3[2]
    dev, s = q.get_device(), q.shape
    if q.dtype is not _F16 or dev < 0 or len(s) != 2 or s[1] < width:
        _refuse(where, f"q must be a CUDA fp16 matrix [rows, >= {width}], not {q.dtype} {tuple(s)} on {q.device}")
    stride, one = q.stride()
    if one != 1 or (stride < s[1] and s[0] > 1):
        _refuse(where, f"q must have dense rows that do not overlap, not strides {q.stride()}")
    return dev, s[0], q.data_ptr(), stride if s[0] > 1 else (width + 7) // 8 * 8


def _scratch(where, t, dev):
    if t.get_device() != dev or not t.is_contiguous():
        _refuse(where, f"scratch must be a contiguous tensor on device {dev}")
    return t.data_ptr(), t.nbytes


def _launch(where, fn, dev, stream, *args):
    if stream is None:
        st = _raw_stream(dev)
    else:
        st = stream if isinstance(stream, int) else stream.cuda_stream
    if dev == _current_device():
        code = fn(*args, st)
    else:
        import torch
        with torch.cuda.device(dev):
            code = fn(*args, st)
    if code != HYP_OK:
        raise HyperionError(code, where)


class AttnMod:
    """hyp_attn_mod with its device tensors: softcap (0 = none, else 2^-10 .. 2^20), window (0 = none), slopes fp32 [n_q_heads] or None,
    prefix_lens int32 [n_seqs] or None.  Keeps the tensors alive; make it once and use it in every call."""

    def __init__(self, softcap: float = 0.0, window: int = 0, slopes=None, prefix_lens=None):
        self.slopes, self.prefix_lens = slopes, prefix_lens
        self.struct = hyp_attn_mod(softcap, window, None if slopes is None else slopes.data_ptr(),
                                   None if prefix_lens is None else prefix_lens.data_ptr())
        self.ref = C.byref(self.struct)

    def check(self, where, shape3, n_seqs, dev):
        """The struct for a call with this head layout and batch; the tensors still have to be where they were."""
        self.struct.slopes = None if self.slopes is None else _dense(where, "slopes", self.slopes, _F32, dev, (shape3[0],))
        self.struct.prefix_lens = None if self.prefix_lens is None else _dense(where, "prefix_lens", self.prefix_lens, _I32, dev, (n_seqs,))
        return self.ref


def hyp_op_attn_mod_scratch_bytes(shape3, n_seqs: int, max_pages_per_seq: int) -> int:
    return lib().hyp_op_attn_mod_scratch_bytes(_shape(shape3), n_seqs, max_pages_per_seq)


def hyp_op_attn_decode_mod(shape3, mod: AttnMod, q, kv_pages, block_table, ctx_lens, scratch, out, stream=None):
    """q fp16 [n_seqs, >= n_q_heads * head_dim], kv_pages fp16 [pages, 2, n_kv_heads, 16, head_dim], block_table int32
    [n_seqs, pages per sequence], ctx_lens int32 [n_seqs], out fp16 [n_seqs, n_q_heads * head_dim]."""
    where, sh = "hyp_op_attn_decode_mod", _shape(shape3)
    dev, n, qp, qs = _query(where, q, shape3)
    pool = _pool(where, "kv_pages", kv_pages, dev, shape3)
    table, width = _rows(where, "block_table", block_table, _I32, dev, (n,))
    ctx = _dense(where, "ctx_lens", ctx_lens, _I32, dev, (n,))
    op = _dense(where, "out", out, _F16, dev, (n, shape3[0] * shape3[2]))
    sp, sb = _scratch(where, scratch, dev)
    _launch(where, lib().hyp_op_attn_decode_mod, dev, stream, sh, mod.check(where, shape3, n, dev), n, qp, qs, pool, table, width, ctx,
            sp, sb, op)


def hyp_op_attn_prefill_mod(shape3, mod: AttnMod, q, kv_pages, block_table, cu_q, ctx_lens, out, stream=None):
    """q fp16 [rows, >= n_q_heads * head_dim], cu_q int32 [n_seqs + 1], the rest as hyp_op_attn_decode_mod."""
    where, sh = "hyp_op_attn_prefill_mod", _shape(shape3)
    dev, m, qp, qs = _query(where, q, shape3)
    pool = _pool(where, "kv_pages", kv_pages, dev, shape3)
    ctx, n = _rows(where, "ctx_lens", ctx_lens, _I32, dev, ())
    table, width = _rows(where, "block_table", block_table, _I32, dev, (n,))
    cu = _dense(where, "cu_q", cu_q, _I32, dev, (n + 1,))
    op = _dense(where, "out", out, _F16, dev, (m, shape3[0] * shape3[2]))
    _launch(where, lib().hyp_op_attn_prefill_mod, dev, stream, sh, mod.check(where, shape3, n, dev), n, m, qp, qs, pool, table, width,
            cu, ctx, op)


def hyp_op_attn_scored_scratch_bytes(shape3, n_seqs: int, max_pages_per_seq: int) -> int:
    return lib().hyp_op_attn_scored_scratch_bytes(_shape(shape3), n_seqs, max_pages_per_seq)


def hyp_op_attn_decode_scored(shape3, q, kv_pages, block_table, ctx_lens, decay: float, weights_in, weights_out, scratch, out,
                              stream=None):
    """weights_in: fp32 [n_seqs, n_kv_heads, width] or None; weights_out the same shape, may be weights_in."""
    where, sh = "hyp_op_attn_decode_scored", _shape(shape3)
    dev, n, qp, qs = _query(where, q, shape3)
    pool = _pool(where, "kv_pages", kv_pages, dev, shape3)
    table, width = _rows(where, "block_table", block_table, _I32, dev, (n,))
    ctx = _dense(where, "ctx_lens", ctx_lens, _I32, dev, (n,))
    wo, ws = _rows(where, "weights_out", weights_out, _F32, dev, (n, shape3[1]))
    wi = None if weights_in is None else _dense(where, "weights_in", weights_in, _F32, dev, (n, shape3[1], ws))
    op = _dense(where, "out", out, _F16, dev, (n, shape3[0] * shape3[2]))
    sp, sb = _scratch(where, scratch, dev)
    _launch(where, lib().hyp_op_attn_decode_scored, dev, stream, sh, n, qp, qs, pool, table, width, ctx, decay, wi, wo, ws, sp, sb, op)


def hyp_op_kv_evict(shape3, kv_pages, block_table, n_cached, weights_in, n_keep: int, n_sink: int, n_recent: int, dst_pages,
                    dst_table, kept, new_lens, weights_out, stream=None):
    """dst_pages, dst_table: kv_pages and block_table themselves (in place), or pages that are not among the source's.
    kept int32 [n_seqs, n_kv_heads, n_keep], new_lens int32 [n_seqs], weights_* fp32 [n_seqs, n_kv_heads, *]."""
    where, sh, hkv = "hyp_op_kv_evict", _shape(shape3), shape3[1]
    dev = kv_pages.get_device()
    if dev < 0:
        _refuse(where, "kv_pages must be a CUDA tensor")
    src, dst = _pool(where, "kv_pages", kv_pages, dev, shape3), _pool(where, "dst_pages", dst_pages, dev, shape3)
    cached, n = _rows(where, "n_cached", n_cached, _I32, dev, ())
    table, width = _rows(where, "block_table", block_table, _I32, dev, (n,))
    dtable, dwidth = _rows(where, "dst_table", dst_table, _I32, dev, (n,))
    new = _dense(where, "new_lens", new_lens, _I32, dev, (n,))
    kp = _dense(where, "kept", kept, _I32, dev, (n, hkv, n_keep))
    wi, ws = _rows(where, "weights_in", weights_in, _F32, dev, (n, hkv))
    wo, wos = _rows(where, "weights_out", weights_out, _F32, dev, (n, hkv))
    _launch(where, lib().hyp_op_kv_evict, dev, stream, sh, n, src, table, width, cached, wi, ws, n_keep, n_sink, n_recent, dst, dtable,
            dwidth, kp, new, wo, wos)


def hyp_op_attn_shared_scratch_bytes(shape3, n_seqs: int, n_groups: int, max_prefix_pages: int, max_pages_per_seq: int) -> int:
    return lib().hyp_op_attn_shared_scratch_bytes(_shape(shape3), n_seqs, n_groups, max_prefix_pages, max_pages_per_seq)


def hyp_op_attn_decode_shared(shape3, q, kv_pages, cu_group, prefix_table, prefix_lens, block_table, ctx_lens, scratch, out,
                              stream=None):
    """cu_group int32 [n_groups + 1], prefix_table int32 [n_groups, pages], prefix_lens int32 [n_groups]; block_table and
    ctx_lens: what every sequence has behind its group's prefix."""
    where, sh = "hyp_op_attn_decode_shared", _shape(shape3)
    dev, n, qp, qs = _query(where, q, shape3)
    pool = _pool(where, "kv_pages", kv_pages, dev, shape3)
    pl, ng = _rows(where, "prefix_lens", prefix_lens, _I32, dev, ())
    cu = _dense(where, "cu_group", cu_group, _I32, dev, (ng + 1,))
    pt, pw = _rows(where, "prefix_table", prefix_table, _I32, dev, (ng,))
    table, width = _rows(where, "block_table", block_table, _I32, dev, (n,))
    ctx = _dense(where, "ctx_lens", ctx_lens, _I32, dev, (n,))
    op = _dense(where, "out", out, _F16, dev, (n, shape3[0] * shape3[2]))
    sp, sb = _scratch(where, scratch, dev)
    _launch(where, lib().hyp_op_attn_decode_shared, dev, stream, sh, n, qp, qs, pool, ng, cu, pt, pw, pl, table, width, ctx, sp, sb, op)


# --------------------------------------------------------------------------------------------
# operators in few bits (hyperion_ops.h): 4-bit weights, the 8-bit cache.  Tensors are checked as those of the operators over the paged cache.
# --------------------------------------------------------------------------------------------
HYP_TYPE_F32, HYP_TYPE_F16, HYP_TYPE_BF16 = range(3)
_U8 = None
_INT_MAX = 2 ** 31 - 1
_TYPES = {}


def _types():
    """torch dtype -> HYP_TYPE_*"""
    global _U8
    if not _TYPES:
        import torch
        if _F16 is None:
            _bind_torch()
        _U8 = torch.uint8
        _TYPES.update({torch.float32: HYP_TYPE_F32, torch.float16: HYP_TYPE_F16, torch.bfloat16: HYP_TYPE_BF16})
    return _TYPES


def _matrix(where, name, t):
    """(device, type, rows, columns, address, row stride) of a matrix with dense rows, which may lie in a wider buffer."""
    code = (_TYPES or _types()).get(t.dtype)
    dev, s = t.get_device(), t.shape
    if code is None or dev < 0 or len(s) != 2:
        _refuse(where, f"{name} must be a CUDA matrix of fp32, fp16 or bf16, not {t.dtype} {tuple(s)} on {t.device}")
    rows, cols = s
    stride, one = t.stride()
    if (one != 1 and cols > 1) or (stride < cols and rows > 1):
        _refuse(where, f"{name} must have dense rows that do not overlap, not strides {t.stride()}")
    if rows > _INT_MAX or cols > _INT_MAX:
        _refuse(where, f"{name} {tuple(s)} has more rows or columns than an int32 counts")
    return dev, code, rows, cols, t.data_ptr(), stride if rows > 1 else (cols + 7) // 8 * 8


def hyp_op_mx4_quantize(x, codes, scales, stream=None):
    """x [N, K] fp32, fp16 or bf16 -> codes uint8 [N, K / 2], scales uint8 [N, ceil(K / 32)]."""
    where = "hyp_op_mx4_quantize"
    dev, code, n, k, xp, xs = _matrix(where, "x", x)
    cp = _dense(where, "codes", codes, _U8, dev, (n, k // 2))
    sp = _dense(where, "scales", scales, _U8, dev, (n, (k + 31) // 32))
    _launch(where, lib().hyp_op_mx4_quantize, dev, stream, xp, code, n, k, xs, cp, sp)


def hyp_op_mx4_dequantize(codes, scales, out, stream=None):
    """codes uint8 [N, K / 2], scales uint8 [N, ceil(K / 32)] -> out [N, K] fp32, fp16 or bf16."""
    where = "hyp_op_mx4_dequantize"
    dev, code, n, k, op, os_ = _matrix(where, "out", out)
    cp = _dense(where, "codes", codes, _U8, dev, (n, k // 2))
    sp = _dense(where, "scales", scales, _U8, dev, (n, (k + 31) // 32))
    _launch(where, lib().hyp_op_mx4_dequantize, dev, stream, cp, sp, n, k, code, op, os_)


_PACKED_BYTES = {}


def hyp_op_mx4_packed_bytes(N: int, K: int, swiglu: bool) -> int:
    key = (N, K, swiglu)
    n = _PACKED_BYTES.get(key)
    if n is None:
        n = _PACKED_BYTES[key] = lib().hyp_op_mx4_packed_bytes(N, K, int(swiglu))
    return n


def hyp_op_mx4_pack(codes, scales, swiglu: bool = False, stream=None):
    """The packed copy (a uint8 tensor) of codes [N, K / 2] and scales [N, ceil(K / 32)], for hyp_op_gemm_mx4; SwiGLU: 2N rows of
    each, gate rows then up rows.  Memory of `stream`, as hyp_op_pack_weight's."""
    where = "hyp_op_mx4_pack"
    _types()
    dev, s = codes.get_device(), codes.shape
    if dev < 0 or len(s) != 2 or (swiglu and s[0] % 2):
        _refuse(where, f"codes must be a CUDA matrix{' of an even number of rows' if swiglu else ''}, not {tuple(s)} on {codes.device}")
    n, k = s[0] // 2 if swiglu else s[0], 2 * s[1]
    cp = _dense(where, "codes", codes, _U8, dev, s)
    sp = _dense(where, "scales", scales, _U8, dev, (s[0], (k + 31) // 32))
    nbytes = hyp_op_mx4_packed_bytes(n, k, swiglu)
    if not nbytes:
        _refuse(where, f"no matrix of {n} rows and {k} columns")
    packed = _packed_buffer(nbytes, codes.device, stream)
    _launch(where, lib().hyp_op_mx4_pack, dev, stream, cp, sp, n, k, int(swiglu), packed.data_ptr(), nbytes)
    return packed


def hyp_op_gemm_mx4_scratch_bytes(M: int, K: int, terms: int) -> int:
    return lib().hyp_op_gemm_mx4_scratch_bytes(M, K, terms)


_PLAN = ("row_tiles", "token_tiles", "shares", "ctas", "stages", "per_sm", "own_terms", "chunks")


def hyp_op_gemm_mx4_plan(M: int, N: int, K: int, terms: int, epilogue: int) -> dict:
    """How hyp_op_gemm_mx4 cuts a product on the current device."""
    plan = (C.c_int32 * 8)()
    _check(lib().hyp_op_gemm_mx4_plan(M, N, K, terms, epilogue, plan), "hyp_op_gemm_mx4_plan")
    return dict(zip(_PLAN, plan))


def hyp_op_gemm_mx4(a, w_packed, N: int, terms: int, epilogue: int, out, scratch, stream=None):
    """a [M, K] fp16 or bf16, w_packed from hyp_op_mx4_pack, out [M, >= N] (fp32, or a's type for the 16-bit epilogues)."""
    where = "hyp_op_gemm_mx4"
    dev, code, m, k, ap, as_ = _matrix(where, "a", a)
    odev, ocode, om, on, op, os_ = _matrix(where, "out", out)
    swiglu = epilogue == HYP_EPI_SWIGLU_BF16
    if odev != dev or om != m or on < N or os_ > _INT_MAX or ocode != (code if swiglu or epilogue == HYP_EPI_STORE_BF16 else HYP_TYPE_F32):
        _refuse(where, f"out {out.dtype} {tuple(out.shape)} on {out.device} does not fit {m} rows of {N} results of epilogue {epilogue}")
    nbytes = hyp_op_mx4_packed_bytes(N, k, swiglu)
    if w_packed.dtype is not _U8 or w_packed.get_device() != dev or not w_packed.is_contiguous() or w_packed.nbytes < max(nbytes, 1):
        _refuse(where, f"w_packed must be the uint8 tensor that hyp_op_mx4_pack gives for {N} x {k} on device {dev}")
    sp, sb = _scratch(where, scratch, dev)
    _launch(where, lib().hyp_op_gemm_mx4, dev, stream, ap, code, as_, w_packed.data_ptr(), m, N, k, terms, epilogue, op, max(os_, on), sp, sb)


HYP_KV8_INT8, HYP_KV8_E4M3 = range(2)


def hyp_kv8_half_page_bytes(head_dim: int) -> int:
    """Bytes of 16 tokens' codes and scales of one head (keys, or values)."""
    return 16 * head_dim + 64


def _pool8(where, t, dev, shape3):
    if _U8 is None:
        _types()
    s = t.shape
    if t.dtype is not _U8 or t.get_device() != dev or not t.is_contiguous() or s[1:] != (2, shape3[1], 16 * shape3[2] + 64):
        _refuse(where, f"kv8_pages must be a contiguous uint8 page pool [pages, 2, {shape3[1]}, {16 * shape3[2] + 64}] on device {dev}, not "
                       f"{t.dtype} {tuple(s)} on {t.device}")
    return t.data_ptr()


def hyp_op_kv8_write(shape3, fmt: int, qkv, kv8_pages, block_table, cu_q, ctx_lens, rope_table=None, q_out=None, stream=None):
    """qkv [rows, >= (n_q_heads + 2 n_kv_heads) * head_dim] fp32, fp16 or bf16; kv8_pages uint8 [pages, 2, n_kv_heads, 16 * head_dim + 64];
    block_table int32 [n_seqs, pages per sequence]; cu_q int32 [n_seqs + 1]; ctx_lens int32 [n_seqs]; rope_table fp32
    [positions, head_dim / 2, 2] or None; q_out fp16 [rows, n_q_heads * head_dim] or None."""
    where, sh = "hyp_op_kv8_write", _shape(shape3)
    dev, code, m, width, qp, qs = _matrix(where, "qkv", qkv)
    if width < (shape3[0] + 2 * shape3[1]) * shape3[2]:
        _refuse(where, f"qkv has {width} columns, the heads need {(shape3[0] + 2 * shape3[1]) * shape3[2]}")
    pool = _pool8(where, kv8_pages, dev, shape3)
    ctx, n = _rows(where, "ctx_lens", ctx_lens, _I32, dev, ())
    table, pages = _rows(where, "block_table", block_table, _I32, dev, (n,))
    cu = _dense(where, "cu_q", cu_q, _I32, dev, (n + 1,))
    rope, rp = 0, None
    if rope_table is not None:
        rope = rope_table.shape[0] if rope_table.dim() else 0
        rp = _dense(where, "rope_table", rope_table, _F32, dev, (rope, shape3[2] // 2, 2))
        if rope < 1:                                            # its address is that of no table at all
            _refuse(where, "rope_table holds no position")
    op = None if q_out is None else _dense(where, "q_out", q_out, _F16, dev, (m, shape3[0] * shape3[2]))
    _launch(where, lib().hyp_op_kv8_write, dev, stream, sh, fmt, n, m, qp, code, qs, rp, rope, pool, table, pages, cu, ctx, op)


def hyp_op_kv8_read(shape3, fmt: int, kv8_pages, block_table, first, lens, dst_pages, dst_table, stream=None):
    """first int32 [n_seqs] or None, lens int32 [n_seqs]; dst_pages fp16 [pages, 2, n_kv_heads, 16, head_dim], dst_table int32
    [n_seqs, pages per sequence]."""
    where, sh = "hyp_op_kv8_read", _shape(shape3)
    dev = kv8_pages.get_device()
    if dev < 0:
        _refuse(where, "kv8_pages must be a CUDA tensor")
    pool = _pool8(where, kv8_pages, dev, shape3)
    lp, n = _rows(where, "lens", lens, _I32, dev, ())
    fp = None if first is None else _dense(where, "first", first, _I32, dev, (n,))
    table, pages = _rows(where, "block_table", block_table, _I32, dev, (n,))
    dst = _pool(where, "dst_pages", dst_pages, dev, shape3)
    dtable, dpages = _rows(where, "dst_table", dst_table, _I32, dev, (n,))
    _launch(where, lib().hyp_op_kv8_read, dev, stream, sh, fmt, n, pool, table, pages, fp, lp, dst, dtable, dpages)


def hyp_op_attn_kv8_scratch_bytes(shape3, n_seqs: int, max_pages_per_seq: int) -> int:
    return lib().hyp_op_attn_kv8_scratch_bytes(_shape(shape3), n_seqs, max_pages_per_seq)


def hyp_op_attn_decode_kv8(shape3, fmt: int, q, kv8_pages, block_table, ctx_lens, scratch, out, stream=None):
    """hyp_op_attn_decode_mod without a modification, over the 8-bit cache."""
    where, sh = "hyp_op_attn_decode_kv8", _shape(shape3)
    dev, n, qp, qs = _query(where, q, shape3)
    pool = _pool8(where, kv8_pages, dev, shape3)
    table, width = _rows(where, "block_table", block_table, _I32, dev, (n,))
    ctx = _dense(where, "ctx_lens", ctx_lens, _I32, dev, (n,))
    op = _dense(where, "out", out, _F16, dev, (n, shape3[0] * shape3[2]))
    sp, sb = _scratch(where, scratch, dev)
    _launch(where, lib().hyp_op_attn_decode_kv8, dev, stream, sh, fmt, n, qp, qs, pool, table, width, ctx, sp, sb, op)


# --------------------------------------------------------------------------------------------
# convenience: a stage with its weights loaded from the seeded generator
# --------------------------------------------------------------------------------------------
class Stage:
    """Owns one hyp_stage handle.  Thin: holds the handle and the shape, forwards calls."""

    def __init__(self, shape, layer_lo: int, layer_hi: int, max_seqs: int, max_ctx: int, max_tokens: int,
                 kv_pages: int = 0):
        self.shape, self.lo, self.hi = shape, layer_lo, layer_hi
        self.cfg = make_cfg(shape, max_seqs, max_ctx, max_tokens, kv_pages)
        self.handle = hyp_stage_create(layer_lo, layer_hi, self.cfg)
        self.first, self.last = layer_lo == 0, layer_hi == shape.n_layers_total

    def load_layer(self, layer: int, w: dict, stream=None):
        for key, tid in (("wqkv", HYP_W_QKV), ("wo", HYP_W_O), ("wgu", HYP_W_GATE_UP), ("wd", HYP_W_DOWN),
                         ("g1", HYP_W_NORM1), ("g2", HYP_W_NORM2)):
            hyp_stage_load(self.handle, layer, tid, w[key].contiguous(), stream)

    def load_embed(self, E, stream=None):
        hyp_stage_load(self.handle, -1, HYP_W_EMBED, E.contiguous(), stream)

    def load_head(self, gf, wlm, stream=None):
        n = self.shape.n_layers_total
        hyp_stage_load(self.handle, n, HYP_W_FINAL_NORM, gf.contiguous(), stream)
        hyp_stage_load(self.handle, n, HYP_W_LM_HEAD, wlm.contiguous(), stream)

    def prefill(self, seq_ids, q_lens, ctx_lens, inp, out, stream=None, flags=0):
        hyp_stage_prefill(self.handle, seq_ids, q_lens, ctx_lens, inp, out, stream, flags)

    def decode(self, seq_ids, ctx_lens, inp, out, stream=None):
        hyp_stage_decode(self.handle, seq_ids, ctx_lens, inp, out, stream)

    def profile(self, mode, batch, ctx, iters=5, stream=None):
        return hyp_stage_profile(self.handle, self.hi - self.lo, mode, batch, ctx, iters, stream)

    def free_seq(self, seq_id):
        hyp_stage_free_seq(self.handle, seq_id)

    def close(self):
        if self.handle:
            hyp_stage_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
