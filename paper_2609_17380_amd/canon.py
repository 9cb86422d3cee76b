"""ctypes binding of libcanon (include/canon.h): argument marshalling only.

Every computation runs in the HIP library; this module passes device pointers, sizes and the current
HIP stream, and raises on a non-OK status.  There is no fallback: if the library is not built, loading
fails with an error.
"""
from __future__ import annotations

import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libcanon.so")

OK, EINVAL, EUNSUPPORTED, EDEVICE, EWORKSPACE = 0, -1, -2, -3, -4
FWD, BWD, FWD_F32 = 0, 1, 2
SOFTMAX_CAUSAL, XENT = 0, 1


class CanonError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {_lib().canon_status_str(status).decode()} ({status})")


class Order(ctypes.Structure):
    _fields_ = [("version", ctypes.c_int32), ("chunk", ctypes.c_int32), ("tree", ctypes.c_int32),
                ("ftz", ctypes.c_int32)]


class DPPlan(ctypes.Structure):
    _fields_ = [("accum", ctypes.c_int32), ("dp_shard", ctypes.c_int32), ("dp_replicate", ctypes.c_int32)]


PLAN_MAX_DEPTH = 31


class PlanCursor(ctypes.Structure):
    """The gradient plan's position and Algorithm 2 stack (plain data: bytes(cursor) persists it)."""
    _fields_ = [("plan", DPPlan), ("next", ctypes.c_int32), ("n", ctypes.c_int64), ("inner", ctypes.c_int32),
                ("depth", ctypes.c_int32), ("level", ctypes.c_int32 * PLAN_MAX_DEPTH),
                ("slot", ctypes.c_int32 * PLAN_MAX_DEPTH)]


class ModelCfg(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("d_ffn", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("seq", ctypes.c_int32), ("micro_seqs", ctypes.c_int32), ("rms_eps", ctypes.c_float),
                ("n_kv_heads", ctypes.c_int32), ("qk_norm", ctypes.c_int32), ("embed_norm", ctypes.c_int32),
                ("swa_window", ctypes.c_int32), ("swa_full_every", ctypes.c_int32), ("z_loss", ctypes.c_float),
                ("pv_int8", ctypes.c_int32), ("dq_fixed_bits", ctypes.c_int32), ("int8_linear", ctypes.c_int32)]


class AdamWConsts(ctypes.Structure):
    _fields_ = [(n, ctypes.c_float) for n in ("lr", "beta1", "one_minus_beta1", "beta2", "one_minus_beta2",
                                              "inv_bc1", "inv_bc2", "eps", "decay_factor")]


class Clip(ctypes.Structure):
    """R15 settings and device outputs (pointers are device addresses, 0 for none)."""
    _fields_ = [("max_norm", ctypes.c_float), ("spike_norm", ctypes.c_float), ("skip_steps", ctypes.c_int32),
                ("norm_out", ctypes.c_void_p), ("skip_state", ctypes.c_void_p), ("skipped_out", ctypes.c_void_p)]


def make_clip(max_norm, spike_norm, skip_steps, norm_out=None, skip_state=None, skipped_out=None) -> Clip:
    return Clip(max_norm, spike_norm, skip_steps, _ptr(norm_out), _ptr(skip_state), _ptr(skipped_out))


ORDER_V1 = Order(1, 32, 0, 1)
_L = None


def _lib():
    global _L
    if _L is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        lib = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        sigs = {
            "canon_gemm": (i32, [vp, i32, i32, i64, i64, i64, vp, i64, vp, i64, vp, i64, vp, vp]),
            "canon_gemm_strided_batched": (i32, [vp, i32, i32, i64, i64, i64, vp, i64, i64, vp, i64, i64, vp, i64,
                                                 i64, i64, vp]),
            "canon_rownorm": (i32, [vp, i32, i64, i64, vp, vp, f32, vp, vp, vp, vp, vp, vp]),
            "canon_softmax_xent": (i32, [vp, i32, i64, i64, vp, f32, i64, vp, f32, f32, vp, vp, vp, vp]),
            "canon_grad_accum": (i32, [vp, vp, i64, vp, vp, vp]),
            "canon_plan_state_bytes": (sz, [vp, i64]),
            "canon_plan_begin": (i32, [vp, i64, vp]),
            "canon_plan_push": (i32, [vp, vp, vp, vp, sz, vp]),
            "canon_plan_finish": (i32, [vp, vp, vp, sz, vp, vp]),
            "canon_adamw": (i32, [i64, vp, vp, vp, vp, vp, vp, vp, vp]),
            "canon_block_fwd_bwd": (i32, [vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
            "canon_block_workspace_bytes": (sz, [vp, i32]),
            "canon_step": (i32, [vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp, vp, vp, vp]),
            "canon_clip_grad_norm": (i32, [vp, i64, vp, vp, vp, vp, sz, vp]),
            "canon_clip_grad_norm_workspace_bytes": (sz, [i64, vp]),
            "canon_step_workspace_bytes": (sz, [vp, vp]),
            "canon_devmath": (i32, [i32, i64, vp, vp, vp, vp, vp]),
            "canon_quant_scales": (i32, [vp, i64, i64, vp, vp, vp]),
            "canon_quantize": (i32, [i64, i64, i32, vp, vp, i32, vp, vp]),
            "canon_gemm_i8": (i32, [i64, i64, i64, vp, i64, vp, i64, vp, vp, i64, vp, vp, vp]),
            "canon_qlinear_bwd": (i32, [vp, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
            "canon_qlinear_bwd_workspace_bytes": (sz, [i64, i64, i64]),
            "canon_state_hash": (i32, [i64, vp, vp, vp, vp, sz, vp]),
            "canon_state_hash_workspace_bytes": (sz, [i64, vp]),
            "canon_attn_pv_i8": (i32, [i64, i64, i64, i64, i64, i64, vp, vp, vp, vp, vp, sz, vp]),
            "canon_attn_pv_i8_workspace_bytes": (sz, [i64, i64, i64, i64]),
            "canon_attn_dq_fixed": (i32, [i64, i64, i64, i64, i64, i64, i32, vp, vp, vp, vp]),
            "canon_lsq_step_grad": (i32, [vp, i64, i64, vp, vp, vp, vp, vp, sz, vp]),
            "canon_lsq_step_grad_workspace_bytes": (sz, [i64, i64]),
            "canon_lsq_step_grad_noalloc": (i32, [vp, i64, i64, vp, vp, vp, vp, vp]),
            "canon_embed_bwd": (i32, [vp, i64, i64, i64, vp, vp, vp, vp, sz, vp]),
            "canon_embed_bwd_workspace_bytes": (sz, [i64, i64]),
            "canon_lsq_step_grad_noalloc_max_terms": (i64, []),
            "canon_act8_groups": (i64, [i64, i32]),
            "canon_act8_pack": (i32, [i64, i64, i32, vp, vp, vp]),
            "canon_act8_unpack": (i32, [i64, i64, vp, i32, vp, vp]),
            "canon_swiglu": (i32, [i64, i64, i32, vp, vp, vp, vp]),
            "canon_swiglu_bwd": (i32, [i64, i64, i32, vp, vp, vp, vp, vp, vp]),
            "canon_layernorm": (i32, [vp, i64, i64, i32, vp, vp, vp, f32, i32, vp, vp, vp, vp, vp]),
            "canon_layernorm_bwd": (i32, [vp, i64, i64, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
            "canon_layernorm_bwd_workspace_bytes": (sz, [i64, i64]),
            "canon_relbias_log": (i32, [i32, i32, i32, vp]),
            "canon_softmax_relbias": (i32, [vp, vp, vp, vp, vp, vp, vp]),
            "canon_softmax_relbias_bwd": (i32, [vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
            "canon_softmax_relbias_bwd_workspace_bytes": (sz, [vp, vp]),
            "canon_quant_tokens": (i32, [i64, i64, i32, vp, vp, vp, vp]),
            "canon_gemm_i8_tokens": (i32, [i64, i64, i64, vp, i64, vp, vp, i64, vp, i32, vp, i64, vp]),
            "canon_rope_tables": (i32, [i32, ctypes.c_double, vp, i64, i64, vp, vp]),
            "canon_rope": (i32, [i32, i64, i64, i64, vp, vp, i32, vp, i64, i32, vp, i64, vp]),
            "canon_cache_append": (i32, [vp, vp, i32, vp, i64, vp, i64, vp, vp]),
            "canon_cache_read": (i32, [vp, vp, i32, vp, vp, vp]),
            "canon_cache_attention": (i32, [vp, vp, vp, i32, vp, i64, vp, vp, sz, vp]),
            "canon_cache_attention_workspace_bytes": (sz, [vp, vp]),
            "canon_status_str": (ctypes.c_char_p, [i32]),
            "canon_version": (i32, []),
        }
        for name, (res, args) in sigs.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _L = lib
    return _L


def lib():
    return _lib()


def _check(st: int, where: str):
    if st != OK:
        raise CanonError(st, where)


def _ptr(t) -> int:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA/HIP tensors"
    return t.data_ptr()


def _ptrs(ts):
    return (ctypes.c_void_p * len(ts))(*[_ptr(t) for t in ts])


def _stream(stream=None) -> int:
    if isinstance(stream, int):  # a raw hipStream_t (0: the null stream)
        return stream
    if stream is None:  # the current stream's handle, without a Stream object around it
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


# ---- entry points (same names as the C ABI, without the prefix) -------------------------------------

EPI_NONE, EPI_ACCUM_PLAN = 0, 1


class GemmEpilogue(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("scale", ctypes.c_float)]


def gemm(m, n, k, a, lda, b, ldb, c, ldc, trans_a=0, trans_b=0, order=ORDER_V1, stream=None, accum_scale=None):
    """C = A B, or with accum_scale the plan's accumulation C = RN(C + RN(A B * accum_scale))."""
    epi = None if accum_scale is None else ctypes.byref(GemmEpilogue(EPI_ACCUM_PLAN, accum_scale))
    _check(_lib().canon_gemm(ctypes.byref(order), int(trans_a), int(trans_b), m, n, k, _ptr(a), lda, _ptr(b), ldb,
                             _ptr(c), ldc, epi, _stream(stream)), "canon_gemm")


def gemm_strided_batched(m, n, k, a, lda, stride_a, b, ldb, stride_b, c, ldc, stride_c, batch, trans_a=0, trans_b=0,
                         order=ORDER_V1, stream=None):
    _check(_lib().canon_gemm_strided_batched(ctypes.byref(order), int(trans_a), int(trans_b), m, n, k, _ptr(a), lda,
                                             stride_a, _ptr(b), ldb, stride_b, _ptr(c), ldc, stride_c, batch,
                                             _stream(stream)), "canon_gemm_strided_batched")


def rownorm(direction, rows, cols, x, gain, eps, y=None, rstd=None, dy=None, dx=None, dgain=None, order=ORDER_V1,
            stream=None):
    _check(_lib().canon_rownorm(ctypes.byref(order), direction, rows, cols, _ptr(x), _ptr(gain), eps, _ptr(y),
                                _ptr(rstd), _ptr(dy), _ptr(dx), _ptr(dgain), _stream(stream)), "canon_rownorm")


def softmax_xent(mode, rows, cols, x, out, scale=1.0, targets=None, inv_tokens=1.0, row_loss=None, mean_loss=None,
                 order=ORDER_V1, stream=None, window=0, z_loss=0.0):
    _check(_lib().canon_softmax_xent(ctypes.byref(order), mode, rows, cols, _ptr(x), scale, window, _ptr(targets),
                                     inv_tokens, z_loss, _ptr(out), _ptr(row_loss), _ptr(mean_loss),
                                     _stream(stream)), "canon_softmax_xent")


def grad_accum(plan: DPPlan, n, grads, out, order=ORDER_V1, stream=None):
    _check(_lib().canon_grad_accum(ctypes.byref(order), ctypes.byref(plan), n, _ptrs(grads), _ptr(out),
                                   _stream(stream)), "canon_grad_accum")


def plan_state_bytes(plan: DPPlan, n: int) -> int:
    return int(_lib().canon_plan_state_bytes(ctypes.byref(plan), n))


def plan_begin(plan: DPPlan, n: int) -> PlanCursor:
    cur = PlanCursor()
    _check(_lib().canon_plan_begin(ctypes.byref(plan), n, ctypes.byref(cur)), "canon_plan_begin")
    return cur


def _state_bytes(state, state_bytes):
    if state_bytes is not None:
        return state_bytes
    return 0 if state is None or isinstance(state, int) else state.numel() * state.element_size()


def plan_push(cursor: PlanCursor, grad, state, order=ORDER_V1, stream=None, state_bytes=None):
    """Feed the next microbatch's gradient (Algorithm 1's order); updates cursor in place."""
    _check(_lib().canon_plan_push(ctypes.byref(order), ctypes.byref(cursor), _ptr(grad), _ptr(state),
                                  _state_bytes(state, state_bytes), _stream(stream)), "canon_plan_push")


def plan_finish(cursor: PlanCursor, state, out, order=ORDER_V1, stream=None, state_bytes=None):
    _check(_lib().canon_plan_finish(ctypes.byref(order), ctypes.byref(cursor), _ptr(state),
                                    _state_bytes(state, state_bytes), _ptr(out), _stream(stream)),
           "canon_plan_finish")


def adamw(params, m, v, grads, decay_mask, consts: AdamWConsts, stream=None):
    n = len(params)
    sizes = (ctypes.c_int64 * n)(*[p.numel() for p in params])
    mask = (ctypes.c_uint8 * n)(*[int(x) for x in decay_mask])
    _check(_lib().canon_adamw(n, sizes, _ptrs(params), _ptrs(m), _ptrs(v), _ptrs(grads), mask, ctypes.byref(consts),
                              _stream(stream)), "canon_adamw")


def attn_pv_i8_workspace_bytes(batch, n_kv_heads, seq, head_dim) -> int:
    return int(_lib().canon_attn_pv_i8_workspace_bytes(batch, n_kv_heads, seq, head_dim))


def attn_pv_i8(batch, n_heads, n_kv_heads, seq, head_dim, window, P, V, workspace, o_f32=None, o_bf16=None,
               stream=None):
    _check(_lib().canon_attn_pv_i8(batch, n_heads, n_kv_heads, seq, head_dim, window, _ptr(P), _ptr(V), _ptr(o_f32),
                                   _ptr(o_bf16), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                   _stream(stream)), "canon_attn_pv_i8")


def attn_dq_fixed(batch, n_heads, n_kv_heads, seq, head_dim, window, frac_bits, dS, K, dQ, stream=None):
    _check(_lib().canon_attn_dq_fixed(batch, n_heads, n_kv_heads, seq, head_dim, window, frac_bits, _ptr(dS), _ptr(K),
                                      _ptr(dQ), _stream(stream)), "canon_attn_dq_fixed")


def lsq_step_grad_workspace_bytes(T, K) -> int:
    return int(_lib().canon_lsq_step_grad_workspace_bytes(T, K))


def lsq_step_grad(T, K, x, s, dx, grad, workspace, order=ORDER_V1, stream=None):
    _check(_lib().canon_lsq_step_grad(ctypes.byref(order), T, K, _ptr(x), _ptr(s), _ptr(dx), _ptr(grad),
                                      _ptr(workspace), workspace.numel() * workspace.element_size(),
                                      _stream(stream)), "canon_lsq_step_grad")


def embed_bwd_workspace_bytes(T, d) -> int:
    return int(_lib().canon_embed_bwd_workspace_bytes(T, d))


def embed_bwd(T, V, d, tokens, dx, dE, workspace, order=ORDER_V1, stream=None):
    """R11: dE [V, d] from the int32 tokens [T] and dx [T, d] (device tensors)."""
    _check(_lib().canon_embed_bwd(ctypes.byref(order), T, V, d, _ptr(tokens), _ptr(dx), _ptr(dE), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(), _stream(stream)), "canon_embed_bwd")


def lsq_step_grad_noalloc(T, K, x, s, dx, grad, order=ORDER_V1, stream=None):
    """canon_lsq_step_grad with the block sums in the library's own device array (no workspace)."""
    _check(_lib().canon_lsq_step_grad_noalloc(ctypes.byref(order), T, K, _ptr(x), _ptr(s), _ptr(dx), _ptr(grad),
                                              _stream(stream)), "canon_lsq_step_grad_noalloc")


def lsq_step_grad_noalloc_max_terms() -> int:
    return int(_lib().canon_lsq_step_grad_noalloc_max_terms())


def block_workspace_bytes(cfg: ModelCfg, batch: int) -> int:
    return int(_lib().canon_block_workspace_bytes(ctypes.byref(cfg), batch))


def block_fwd_bwd(cfg: ModelCfg, batch, x, dy, w, rope_cos, rope_sin, y, dx, dw, workspace, order=ORDER_V1,
                  stream=None):
    _check(_lib().canon_block_fwd_bwd(ctypes.byref(order), ctypes.byref(cfg), batch, _ptr(x), _ptr(dy), _ptrs(w),
                                      _ptr(rope_cos), _ptr(rope_sin), _ptr(y), _ptr(dx), _ptrs(dw), _ptr(workspace),
                                      workspace.numel() * workspace.element_size(), _stream(stream)),
           "canon_block_fwd_bwd")


def step_workspace_bytes(cfg: ModelCfg, plan: DPPlan) -> int:
    return int(_lib().canon_step_workspace_bytes(ctypes.byref(cfg), ctypes.byref(plan)))


def step(cfg: ModelCfg, plan: DPPlan, params, m, v, windows, rope_cos, rope_sin, consts: AdamWConsts, workspace,
         loss_out, grads_out=None, step_t=1, order=ORDER_V1, stream=None, clip: Clip | None = None,
         state_digest=None):
    """state_digest: None, or a 32-byte device tensor for the per-step audit hash (H1 of the windows, the
    parameters, m and v after the step, and the reduced gradient)."""
    _check(_lib().canon_step(ctypes.byref(order), ctypes.byref(cfg), ctypes.byref(plan), _ptrs(params), _ptrs(m),
                             _ptrs(v), step_t, _ptr(windows), _ptr(rope_cos), _ptr(rope_sin), ctypes.byref(consts),
                             ctypes.byref(clip) if clip is not None else None,
                             _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(loss_out),
                             _ptrs(grads_out) if grads_out is not None else None, _ptr(state_digest),
                             _stream(stream)), "canon_step")


def _sizes(tensors):
    return (ctypes.c_int64 * len(tensors))(*[t.numel() for t in tensors])


def clip_grad_norm_workspace_bytes(grads) -> int:
    return int(_lib().canon_clip_grad_norm_workspace_bytes(len(grads), _sizes(grads)))


def clip_grad_norm(grads, clip: Clip, workspace, order=ORDER_V1, stream=None):
    """R15 norm, spike decision and in-place clip of fp32 device tensors taken end to end in list order."""
    _check(_lib().canon_clip_grad_norm(ctypes.byref(order), len(grads), _sizes(grads), _ptrs(grads),
                                       ctypes.byref(clip), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream)),
           "canon_clip_grad_norm")


DEVMATH_OPS = {"add": 0, "sub": 1, "mul": 2, "fma": 3, "div": 4, "sqrt": 5, "exp": 6, "log": 7, "sigmoid": 8,
               "silu": 9, "bf16": 10}


F32, BF16 = 0, 1


def quant_scales(rows, cols, w, scale, order=ORDER_V1, stream=None):
    _check(_lib().canon_quant_scales(ctypes.byref(order), rows, cols, _ptr(w), _ptr(scale), _stream(stream)),
           "canon_quant_scales")


def quantize(rows, cols, x, scale, per_row, q, stream=None):
    dtype = F32 if x.dtype == torch.float32 else BF16
    _check(_lib().canon_quantize(rows, cols, dtype, _ptr(x), _ptr(scale), int(per_row), _ptr(q), _stream(stream)),
           "canon_quantize")


def gemm_i8(m, n, k, a, lda, b, ldb, acc=None, y=None, ldc=None, sa=None, sb=None, stream=None):
    _check(_lib().canon_gemm_i8(m, n, k, _ptr(a), lda, _ptr(b), ldb, _ptr(acc), _ptr(y), n if ldc is None else ldc,
                                _ptr(sa), _ptr(sb), _stream(stream)), "canon_gemm_i8")


def qlinear_bwd_workspace_bytes(T, N, K) -> int:
    return int(_lib().canon_qlinear_bwd_workspace_bytes(T, N, K))


def qlinear_bwd(T, N, K, dy, qx, sx, qw, sw, dx, dw, workspace, order=ORDER_V1, stream=None):
    _check(_lib().canon_qlinear_bwd(ctypes.byref(order), T, N, K, _ptr(dy), _ptr(qx), _ptr(sx), _ptr(qw), _ptr(sw),
                                    _ptr(dx), _ptr(dw), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                    _stream(stream)), "canon_qlinear_bwd")


def _nbytes(tensors):
    return (ctypes.c_int64 * len(tensors))(*[t.numel() * t.element_size() for t in tensors])


def state_hash_workspace_bytes(tensors) -> int:
    return int(_lib().canon_state_hash_workspace_bytes(len(tensors), _nbytes(tensors)))


def state_hash(tensors, digest, workspace, stream=None):
    """Canonical state hash H1 of the tensors (declared order) into digest (device uint8 [32])."""
    _check(_lib().canon_state_hash(len(tensors), _ptrs(tensors), _nbytes(tensors), _ptr(digest), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream)),
           "canon_state_hash")


def devmath(op: str, n, a, b=None, c=None, out=None, stream=None):
    _check(_lib().canon_devmath(DEVMATH_OPS[op], n, _ptr(a), _ptr(b), _ptr(c), _ptr(out), _stream(stream)),
           "canon_devmath")


# ---- activations kept in 8 bits, SwiGLU, layer norm, attention rows with a relative position bias ----------------
#
# These calls take sizes and element types from their arguments, so they check them: a tensor of another type, size or
# device than the call needs raises ValueError and enqueues nothing.

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}
_T32, _T16, _TF, _TI8, _TI32 = (torch.float32,), (torch.bfloat16,), (torch.float32, torch.bfloat16), (torch.int8,), (torch.int32,)


def _device() -> int:
    """The current device; without one, a number that no tensor's is."""
    try:
        return torch._C._cuda_getDevice()
    except RuntimeError:
        return -2


def _arg(t, what, numel, dtypes, dev):
    """The device address of an argument of `numel` elements (None: no pointer)."""
    if t is None and dtypes is not _TF:  # where two types may stand the call needs one
        return None
    if isinstance(t, torch.Tensor) and t.dtype in dtypes and t.get_device() == dev and t.numel() == numel and t.is_contiguous():
        return t.data_ptr()
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes:
        raise ValueError(f"{what}: a tensor of {' or '.join(map(str, dtypes))} is needed")
    if t.get_device() != dev:
        raise ValueError(f"{what}: a tensor on the current device is needed, not on {t.device}")
    raise ValueError(f"{what}: {numel} elements are needed, contiguous, not {tuple(t.shape)} of strides {t.stride()}")


def _scratch(ws, dev):
    """(address, bytes) of a workspace; without one, none."""
    if ws is None:
        return None, 0
    if not isinstance(ws, torch.Tensor):
        raise ValueError("workspace: a tensor is needed")
    return _arg(ws, "workspace", ws.numel(), (ws.dtype,), dev), ws.numel() * ws.element_size()


def _stream_on(stream, dev):
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream(stream)


class Act8(ctypes.Structure):
    """A matrix [rows][cols] kept in 8 bits: codes int8 [rows, cols] and steps fp32 [rows, act8_groups(cols, group)]."""
    _fields_ = [("group", ctypes.c_int32), ("codes", ctypes.c_void_p), ("steps", ctypes.c_void_p)]

    def __init__(self, group, codes, steps):
        if not isinstance(codes, torch.Tensor) or not isinstance(steps, torch.Tensor):
            raise ValueError("codes and steps: tensors are needed")
        self.tensors = codes, steps
        super().__init__(group, codes.data_ptr(), steps.data_ptr())

    def _of(self, rows, cols, dev):
        """The record's address, once its tensors are those of [rows][cols] on the current device."""
        groups = act8_groups(cols, self.group)
        if not groups and cols:
            raise ValueError("group: 32, 64, 128 or 256 is needed")
        self.codes = _arg(self.tensors[0], "codes", rows * cols, _TI8, dev)
        self.steps = _arg(self.tensors[1], "steps", rows * groups, _T32, dev)
        return ctypes.byref(self)


def act8_groups(cols, group) -> int:
    return int(_lib().canon_act8_groups(cols, group))


def act8_pack(rows, cols, x, kept: Act8, stream=None):
    dev = _device()
    px = _arg(x, "x", rows * cols, _TF, dev)
    _check(_lib().canon_act8_pack(rows, cols, _DTYPES[x.dtype], px, kept._of(rows, cols, dev), _stream_on(stream, dev)),
           "canon_act8_pack")


def act8_unpack(rows, cols, kept: Act8, out, stream=None):
    dev = _device()
    po = _arg(out, "out", rows * cols, _TF, dev)
    _check(_lib().canon_act8_unpack(rows, cols, kept._of(rows, cols, dev), _DTYPES[out.dtype], po, _stream_on(stream, dev)),
           "canon_act8_unpack")


def swiglu(T, F, gu, a, keep: Act8 | None = None, stream=None):
    """a = silu(gate) up from gu [T, 2F]; keep: also keeps gu in 8 bits, as the matrix [2T][F]."""
    dev = _device()
    pg = _arg(gu, "gu", 2 * T * F, _TF, dev)
    _check(_lib().canon_swiglu(T, F, _DTYPES[gu.dtype], pg, _arg(a, "a", T * F, _T16, dev),
                               None if keep is None else keep._of(2 * T, F, dev), _stream_on(stream, dev)), "canon_swiglu")


def swiglu_bwd(T, F, gu, da, dgu, a=None, stream=None):
    """gu: the forward's input, or the Act8 that it was kept as."""
    dev = _device()
    kept = gu._of(2 * T, F, dev) if isinstance(gu, Act8) else None
    pg = None if kept else _arg(gu, "gu", 2 * T * F, _TF, dev)
    _check(_lib().canon_swiglu_bwd(T, F, F32 if kept else _DTYPES[gu.dtype], pg, kept,
                                   _arg(da, "da", T * F, _T32, dev), _arg(dgu, "dgu", 2 * T * F, _T16, dev),
                                   _arg(a, "a", T * F, _T16, dev), _stream_on(stream, dev)), "canon_swiglu_bwd")


def layernorm(rows, cols, x, gain, bias, eps, y, mean, rstd, keep: Act8 | None = None, order=ORDER_V1, stream=None):
    dev = _device()
    px = _arg(x, "x", rows * cols, _TF, dev)
    py = _arg(y, "y", rows * cols, _TF, dev)
    _check(_lib().canon_layernorm(ctypes.byref(order), rows, cols, _DTYPES[x.dtype], px,
                                  _arg(gain, "gain", cols, _T16, dev), _arg(bias, "bias", cols, _T16, dev), eps,
                                  _DTYPES[y.dtype], py, _arg(mean, "mean", rows, _T32, dev),
                                  _arg(rstd, "rstd", rows, _T32, dev),
                                  None if keep is None else keep._of(rows, cols, dev), _stream_on(stream, dev)), "canon_layernorm")


def layernorm_bwd_workspace_bytes(rows, cols) -> int:
    return int(_lib().canon_layernorm_bwd_workspace_bytes(rows, cols))


def layernorm_bwd(rows, cols, x, gain, mean, rstd, dy, dx, workspace=None, dgain=None, dbias=None, order=ORDER_V1,
                  stream=None):
    """x: the forward's input, or the Act8 that it was kept as.  workspace: needed for dgain and dbias."""
    dev = _device()
    kept = x._of(rows, cols, dev) if isinstance(x, Act8) else None
    px = None if kept else _arg(x, "x", rows * cols, _TF, dev)
    ws, ws_bytes = _scratch(workspace, dev)
    _check(_lib().canon_layernorm_bwd(ctypes.byref(order), rows, cols, F32 if kept else _DTYPES[x.dtype], px, kept,
                                      _arg(gain, "gain", cols, _T16, dev), _arg(mean, "mean", rows, _T32, dev),
                                      _arg(rstd, "rstd", rows, _T32, dev),
                                      _arg(dy, "dy", rows * cols, _T32, dev),
                                      _arg(dx, "dx", rows * cols, _T32, dev),
                                      _arg(dgain, "dgain", cols, _T32, dev),
                                      _arg(dbias, "dbias", cols, _T32, dev), ws, ws_bytes, _stream_on(stream, dev)),
           "canon_layernorm_bwd")


RELBIAS_MAX_STARTS = 128


class RelBias(ctypes.Structure):
    """The buckets of a relative position bias: the distances at which those of one side begin."""
    _fields_ = [("n_starts", ctypes.c_int32), ("bidirectional", ctypes.c_int32),
                ("start", ctypes.c_int32 * RELBIAS_MAX_STARTS)]

    def __init__(self, starts=(), bidirectional=False):
        if len(starts) > RELBIAS_MAX_STARTS:
            raise ValueError(f"starts: at most {RELBIAS_MAX_STARTS}")
        super().__init__(len(starts), int(bidirectional), (ctypes.c_int32 * RELBIAS_MAX_STARTS)(*starts))

    @property
    def buckets(self) -> int:
        return self.n_starts * (2 if self.bidirectional else 1)


def relbias_log(n_buckets, max_distance, bidirectional=False) -> RelBias:
    """Buckets that widen with the distance: n_buckets in all, the last of a side from about max_distance on."""
    r = RelBias()
    _check(_lib().canon_relbias_log(n_buckets, int(bidirectional), max_distance, ctypes.byref(r)), "canon_relbias_log")
    return r


class AttnRows(ctypes.Structure):
    """The rows of attention [batch][n_heads][q_len][ld >= k_len] and the keys that each sees; q_starts, q_lens and k_lens
    are int32 device tensors [batch] or None.  A matrix of such rows may end with the last one's k_len keys."""
    _fields_ = [(n, ctypes.c_int64) for n in ("batch", "n_heads", "q_len", "k_len", "ld", "q_start", "window")] + \
               [("causal", ctypes.c_int32), ("scale", ctypes.c_float)] + \
               [(n, ctypes.c_void_p) for n in ("q_starts", "q_lens", "k_lens")]

    def __init__(self, batch, n_heads, q_len, k_len, causal=True, window=0, scale=1.0, ld=0, q_start=0, q_starts=None,
                 q_lens=None, k_lens=None):
        self.tensors = q_starts, q_lens, k_lens
        super().__init__(batch, n_heads, q_len, k_len, ld, q_start, window, int(causal), scale)
        self._of(_device())

    def _of(self, dev):
        """The record's address, once its tensors are a batch's on the current device."""
        starts, queries, keys = self.tensors
        if starts is not None or queries is not None or keys is not None:
            self.q_starts = _arg(starts, "q_starts", self.batch, _TI32, dev)
            self.q_lens = _arg(queries, "q_lens", self.batch, _TI32, dev)
            self.k_lens = _arg(keys, "k_lens", self.batch, _TI32, dev)
        return ctypes.byref(self)

    def _matrix(self, t, what, dtypes, dev):
        """A matrix of these rows: all of them, `ld` apart; what would follow the last one's keys may be absent."""
        rows, ld = self.batch * self.n_heads * self.q_len, self.ld or self.k_len
        least = (rows - 1) * ld + self.k_len if rows > 0 else 0
        short = isinstance(t, torch.Tensor) and t.numel() == least
        return _arg(t, what, least if short else rows * ld, dtypes, dev)


def softmax_relbias(rows: AttnRows, bias: RelBias, table, scores, probs, order=ORDER_V1, stream=None):
    """probs (bf16) of the raw scores (fp32), with table (bf16 [buckets, n_heads]) added by distance."""
    dev = _device()
    _check(_lib().canon_softmax_relbias(ctypes.byref(order), rows._of(dev), ctypes.byref(bias),
                                        _arg(table, "table", bias.buckets * rows.n_heads, _T16, dev),
                                        rows._matrix(scores, "scores", _T32, dev),
                                        rows._matrix(probs, "probs", _T16, dev), _stream_on(stream, dev)),
           "canon_softmax_relbias")


def softmax_relbias_bwd_workspace_bytes(rows: AttnRows, bias: RelBias) -> int:
    return int(_lib().canon_softmax_relbias_bwd_workspace_bytes(ctypes.byref(rows), ctypes.byref(bias)))


def softmax_relbias_bwd(rows: AttnRows, bias: RelBias, probs, dprobs, dscores, workspace=None, dtable=None,
                        order=ORDER_V1, stream=None):
    """dscores (bf16) and dtable (fp32 [buckets, n_heads]); workspace: needed for dtable."""
    dev = _device()
    ws, ws_bytes = _scratch(workspace, dev)
    _check(_lib().canon_softmax_relbias_bwd(ctypes.byref(order), rows._of(dev), ctypes.byref(bias),
                                            rows._matrix(probs, "probs", _T16, dev),
                                            rows._matrix(dprobs, "dprobs", _T32, dev),
                                            rows._matrix(dscores, "dscores", _T16, dev),
                                            _arg(dtable, "dtable", bias.buckets * rows.n_heads, _T32, dev), ws, ws_bytes,
                                            _stream_on(stream, dev)), "canon_softmax_relbias_bwd")


# ---- products in int8 with a step per token, rotary positions, a paged cache in 8 bits and attention over it ------
#
# As above, these calls check their arguments.  Tokens' heads may be part of wider rows: a tensor [tokens, heads * dim] (or
# [tokens, heads, dim]) whose rows are apart, each row's elements together.


def _rows(t, what, rows, width, dtypes, dev):
    """(address, elements from a row to the next) of `rows` rows of `width` elements."""
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes:
        raise ValueError(f"{what}: a tensor of {' or '.join(map(str, dtypes))} is needed")
    if t.get_device() != dev:
        raise ValueError(f"{what}: a tensor on the current device is needed, not on {t.device}")
    if t.is_contiguous() and t.numel() == rows * width:
        return t.data_ptr(), width
    if t.dim() >= 2 and t.shape[0] == rows and t.numel() == rows * width and (rows == 0 or t[0].is_contiguous()):
        return t.data_ptr(), t.stride(0) if rows > 1 else width
    raise ValueError(f"{what}: {rows} rows of {width} elements are needed, each contiguous, not {tuple(t.shape)} of strides "
                     f"{t.stride()}")


def _lead(ld, least, rows, t, what, dtypes, dev):
    """The address of a matrix of `rows` rows, `ld` (at least `least`) elements apart; the last may end with its elements."""
    if ld < least:
        raise ValueError(f"{what}: rows of {least} elements do not fit a leading dimension of {ld}")
    full = rows * ld
    short = full - ld + least if rows > 0 else 0
    return _arg(t, what, short if short != full and isinstance(t, torch.Tensor) and t.numel() == short else full, dtypes, dev)


def quant_tokens(rows, cols, x, codes, steps, stream=None):
    """codes (int8 [rows, cols]) and steps (fp32 [rows]) of x: a step of its own for every row."""
    dev = _device()
    px = _arg(x, "x", rows * cols, _TF, dev)
    _check(_lib().canon_quant_tokens(rows, cols, _DTYPES[x.dtype], px, _arg(codes, "codes", rows * cols, _TI8, dev),
                                     _arg(steps, "steps", rows, _T32, dev), _stream_on(stream, dev)), "canon_quant_tokens")


def gemm_i8_tokens(m, n, k, a, lda, sa, b, ldb, sb, y, ldc=None, stream=None):
    """y = (a . b) sa sb: a int8 [m, k] with steps sa [m], b int8 [n, k] with steps sb [n], y fp32 or bf16 [m, n]."""
    dev = _device()
    ldc = n if ldc is None else ldc
    if not isinstance(y, torch.Tensor) or y.dtype not in _TF:
        raise ValueError("y: a tensor of torch.float32 or torch.bfloat16 is needed")
    _check(_lib().canon_gemm_i8_tokens(m, n, k, _lead(lda, k, m, a, "a", _TI8, dev), lda, _arg(sa, "sa", m, _T32, dev),
                                       _lead(ldb, k, n, b, "b", _TI8, dev), ldb, _arg(sb, "sb", n, _T32, dev), _DTYPES[y.dtype],
                                       _lead(ldc, n, m, y, "y", _TF, dev), ldc, _stream_on(stream, dev)), "canon_gemm_i8_tokens")


ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_BANDS = 0, 1, 2, 3


class RopeScaling(ctypes.Structure):
    """How a rotation's frequencies are scaled for contexts longer than those trained on (canon_rope_tables)."""
    _fields_ = [("kind", ctypes.c_int32)] + [(n, ctypes.c_double) for n in ("factor", "low", "high", "context", "amplitude")]

    def __init__(self, kind=ROPE_PLAIN, factor=1.0, low=0.0, high=1.0, context=1.0, amplitude=1.0):
        super().__init__(kind, factor, low, high, context, amplitude)


def rope_tables(rot_dim, positions, theta=5e5, scaling: RopeScaling | None = None, first=0):
    """(cos, sin) on the host, fp32 [positions, rot_dim / 2]."""
    cos, sin = (torch.empty(max(positions, 0), max(rot_dim, 0) // 2, dtype=torch.float32) for _ in range(2))
    _check(_lib().canon_rope_tables(rot_dim, theta, None if scaling is None else ctypes.byref(scaling), first, positions,
                                    cos.data_ptr(), sin.data_ptr()), "canon_rope_tables")
    return cos, sin


class _Kept(ctypes.Structure):
    """A record that is kept from call to call.  Its tensors may be resized or given other memory in between: every call looks
    whether they are as they were last taken (`kept`: tensor, address, elements, type), and takes them again if not."""

    def _of(self, dev):
        """The record's address, once its tensors are what they were when it was made, wherever they are now."""
        if self.kept is None or dev != self.device:
            self._take(dev)
        for t, address, numel, dtype in self.kept:
            if t.data_ptr() != address or t.numel() != numel or t.dtype is not dtype or not t.is_contiguous():
                self._take(dev)
                break
        return ctypes.byref(self)

    def _take(self, dev):
        self.kept, kept = None, ()  # None: the next call takes them, if one is refused here
        for name, t, numel, dtypes in self._tensors():
            address = _arg(t, name, numel, dtypes, dev)
            setattr(self, name, address)
            kept += ((t, address, numel, dtypes[0]),)
        self.kept, self.device = kept, dev


class Rotation(_Kept):
    """The turns of the first rot_dim elements of a head: cos and sin fp32 [positions, rot_dim / 2] on the device; halves of
    those elements together, or (interleaved) neighbours."""
    _fields_ = [("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("positions", ctypes.c_int64),
                ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p)]

    def __init__(self, cos, sin, rot_dim, interleaved=False):
        if not isinstance(cos, torch.Tensor) or not isinstance(sin, torch.Tensor):
            raise ValueError("cos and sin: tensors are needed")
        half, n = max(rot_dim // 2, 1), cos.numel()
        if n % half or n != sin.numel():
            raise ValueError(f"cos and sin: [positions, {rot_dim // 2}] are needed, not {tuple(cos.shape)} and {tuple(sin.shape)}")
        dev = cos.get_device()
        c, s = _arg(cos, "cos", n, _T32, dev), _arg(sin, "sin", n, _T32, dev)
        super().__init__(rot_dim, int(interleaved), n // half if rot_dim > 0 else 0, c, s)
        self.tensors, self.numel, self.device = (cos, sin), n, dev
        self.kept = (cos, c, n, torch.float32), (sin, s, n, torch.float32)

    def _tensors(self):
        return [(name, t, self.numel, _T32) for name, t in zip(("cos", "sin"), self.tensors)]


def rope(tokens, heads, dim, rotation: Rotation, x, y, positions=None, backward=False, stream=None):
    """y = the heads of x [tokens, heads * dim] turned at their tokens' positions (int32 [tokens]; None: token t at t), or,
    backward, the gradient of x from that of y.  y may be x."""
    dev = _device()
    px, xs = _rows(x, "x", tokens, heads * dim, _TF, dev)
    py, ys = _rows(y, "y", tokens, heads * dim, _TF, dev)
    _check(_lib().canon_rope(int(backward), tokens, heads, dim, rotation._of(dev), _arg(positions, "positions", tokens, _TI32, dev),
                             _DTYPES[x.dtype], px, xs, _DTYPES[y.dtype], py, ys, _stream_on(stream, dev)), "canon_rope")


class KVCache(_Kept):
    """A paged cache of keys and values in 8 bits: k_codes int8 [pages, kv_heads, page, dim], v_codes int8 [pages, kv_heads,
    page / 16, dim, 16], k_steps and v_steps fp32 [pages, kv_heads, page], table int32 [batch, table_len]."""
    _fields_ = [(n, ctypes.c_int64) for n in ("n_pages", "page", "n_kv_heads", "head_dim")] + \
               [(n, ctypes.c_void_p) for n in ("k_codes", "v_codes", "k_steps", "v_steps")] + \
               [("batch", ctypes.c_int64), ("table_len", ctypes.c_int64), ("table", ctypes.c_void_p)]

    def __init__(self, page, kv_heads, dim, k_codes, v_codes, k_steps, v_steps, table):
        one = page * kv_heads * dim
        if not isinstance(k_codes, torch.Tensor) or page < 1 or kv_heads < 1 or dim < 1 or k_codes.numel() % one:
            raise ValueError(f"k_codes: a tensor of pages of {one} codes is needed")
        if not all(isinstance(t, torch.Tensor) for t in (v_codes, k_steps, v_steps)):
            raise ValueError("codes and steps: tensors are needed")
        codes, dev = k_codes.numel(), k_codes.get_device()
        steps = codes // dim
        k, v = _arg(k_codes, "k_codes", codes, _TI8, dev), _arg(v_codes, "v_codes", codes, _TI8, dev)
        ks, vs = _arg(k_steps, "k_steps", steps, _T32, dev), _arg(v_steps, "v_steps", steps, _T32, dev)
        super().__init__(codes // one, page, kv_heads, dim, k, v, ks, vs)
        self.tensors, self.numel, self.device = (k_codes, v_codes, k_steps, v_steps), codes, dev
        self.kept = ((k_codes, k, codes, torch.int8), (v_codes, v, codes, torch.int8), (k_steps, ks, steps, torch.float32),
                     (v_steps, vs, steps, torch.float32))
        self.set_table(table)

    def set_table(self, table):
        """The pages of other sequences, or more of the same ones'."""
        if not isinstance(table, torch.Tensor) or table.dim() != 2:
            raise ValueError("table: a tensor [batch, table_len] is needed")
        batch, table_len = table.shape
        address = _arg(table, "table", batch * table_len, _TI32, self.device)
        self.table, self.pages, self.batch, self.table_len = address, table, batch, table_len
        if self.kept is not None:
            self.kept = self.kept[:4] + ((table, address, batch * table_len, torch.int32),)

    def _tensors(self):
        k, v, ks, vs = self.tensors
        steps = self.numel // self.head_dim
        return (("k_codes", k, self.numel, _TI8), ("v_codes", v, self.numel, _TI8), ("k_steps", ks, steps, _T32),
                ("v_steps", vs, steps, _T32), ("table", self.pages, self.batch * self.table_len, _TI32))


class CacheRows(ctypes.Structure):
    """New tokens [batch][q_len] of a cache's sequences: token i at position q_start + i or q_starts[b] + i, the first q_lens[b]
    of them real (int32 device tensors [batch] or None)."""
    _fields_ = [("q_len", ctypes.c_int64), ("q_start", ctypes.c_int64), ("q_starts", ctypes.c_void_p), ("q_lens", ctypes.c_void_p)]

    def __init__(self, batch, q_len, q_start=0, q_starts=None, q_lens=None):
        self.batch = batch
        self.tensors = q_starts, q_lens
        super().__init__(q_len, q_start)

    def _of(self, cache, dev):
        """The record's address, once its tensors are those of the cache's sequences on the current device."""
        if self.batch != cache.batch:
            raise ValueError(f"rows of {self.batch} sequences, a cache's table of {cache.batch}")
        self.q_starts = _arg(self.tensors[0], "q_starts", self.batch, _TI32, dev)
        self.q_lens = _arg(self.tensors[1], "q_lens", self.batch, _TI32, dev)
        return ctypes.byref(self)


def cache_append(cache: KVCache, rows: CacheRows, k, v, rotation: Rotation | None = None, stream=None):
    """Keys (turned first by `rotation`, if given) and values [batch * q_len, kv_heads * dim] of new tokens into their pages: no
    two of them into one slot, whose contents would not be defined."""
    dev = _device()
    n, width = cache.batch * rows.q_len, cache.n_kv_heads * cache.head_dim
    pk, ks = _rows(k, "k", n, width, _TF, dev)
    pv, vs = _rows(v, "v", n, width, (k.dtype,), dev)
    _check(_lib().canon_cache_append(cache._of(dev), rows._of(cache, dev), _DTYPES[k.dtype], pk, ks, pv, vs,
                                     None if rotation is None else rotation._of(dev), _stream_on(stream, dev)),
           "canon_cache_append")


def cache_read(cache: KVCache, rows: CacheRows, k=None, v=None, stream=None):
    """What is kept of the tokens of `rows`, into k and v [batch * q_len, kv_heads * dim] (fp32 or bf16, both alike)."""
    dev = _device()
    n = cache.batch * rows.q_len * cache.n_kv_heads * cache.head_dim
    some = k if k is not None else v
    if not isinstance(some, torch.Tensor) or some.dtype not in _TF:
        raise ValueError("k, v: a tensor of torch.float32 or torch.bfloat16 is needed")
    one = (some.dtype,)
    _check(_lib().canon_cache_read(cache._of(dev), rows._of(cache, dev), _DTYPES[some.dtype], _arg(k, "k", n, one, dev),
                                   _arg(v, "v", n, one, dev), _stream_on(stream, dev)), "canon_cache_read")


def cache_attention_workspace_bytes(cache: KVCache, rows: AttnRows) -> int:
    return int(_lib().canon_cache_attention_workspace_bytes(ctypes.byref(cache), ctypes.byref(rows)))


def cache_attention(cache: KVCache, rows: AttnRows, q, out, workspace=None, order=ORDER_V1, stream=None):
    """out (bf16 [batch * q_len, heads * dim]) = attention of the queries q [batch * q_len, heads * dim] over the cache."""
    dev = _device()
    n, width = rows.batch * rows.q_len, rows.n_heads * cache.head_dim
    pq, qs = _rows(q, "q", n, width, _TF, dev)
    ws, ws_bytes = _scratch(workspace, dev)
    _check(_lib().canon_cache_attention(ctypes.byref(order), cache._of(dev), rows._of(dev), _DTYPES[q.dtype], pq, qs,
                                        _arg(out, "out", n * width, _T16, dev), ws, ws_bytes, _stream_on(stream, dev)),
           "canon_cache_attention")


def version() -> int:
    return int(_lib().canon_version())
