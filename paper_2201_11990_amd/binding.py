"""Thin ctypes binding of libmtnlg.so (same names as include/mtnlg.h).

Argument marshalling only: torch tensors give device pointers and the current
stream; every step of the layer runs in the library's HIP kernels.  If the
library is not built this module raises -- there is no fallback.
"""
import ctypes
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmtnlg.so")

PARAM_NAMES = ("ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o",
               "ln2_g", "ln2_b", "w_fc1", "b_fc1", "w_fc2", "b_fc2")

F32, BF16 = 0, 1
GELU_TANH, GELU_ERF = 0, 1
RECOMPUTE, ACCUMULATE_WGRAD, WGRAD_FP32 = 1, 2, 4
GEMM_NT, GEMM_NN, GEMM_TN = 0, 1, 2
EPI_BIAS, EPI_GELU, EPI_RESIDUAL, EPI_ACCUMULATE, EPI_OUT_F32, EPI_GELU_ERF, EPI_GELU_GRAD = 1, 2, 4, 8, 16, 32, 64
ROTARY_HALF, ROTARY_INTERLEAVED = 0, 1
ROTARY_UNSCALED, ROTARY_LINEAR, ROTARY_BASE, ROTARY_PARTS = 0, 1, 2, 3
KERNEL_CLASSES = ("gemm_nt", "gemm_nn", "gemm_tn", "attn_fwd", "attn_bwd", "ln_fwd", "ln_bwd",
                  "gelu", "colsum", "elementwise")


class MtnlgError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class LayerDesc(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int32), ("heads_local", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("ffn_local", ctypes.c_int32),
                ("seq", ctypes.c_int32), ("micro_batch", ctypes.c_int32),
                ("tp_size", ctypes.c_int32), ("tp_rank", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("gelu", ctypes.c_int32),
                ("ln_eps", ctypes.c_float), ("softmax_scale", ctypes.c_float),
                ("flags", ctypes.c_uint32)]


class AdamDesc(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float), ("eps", ctypes.c_float),
                ("weight_decay", ctypes.c_float), ("max_grad_norm", ctypes.c_float), ("step", ctypes.c_int32)]


class HeadDesc(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int32), ("vocab_local", ctypes.c_int32), ("vocab_start", ctypes.c_int32),
                ("seq", ctypes.c_int32), ("micro_batch", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("ln_eps", ctypes.c_float)]


class Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token", ctypes.c_int64), ("group", ctypes.c_int64), ("head", ctypes.c_int64)]


class RotaryDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("scaling", ctypes.c_int32),
                ("original_positions", ctypes.c_int32), ("tokens", ctypes.c_int64), ("base", ctypes.c_double),
                ("factor", ctypes.c_double), ("slow", ctypes.c_double), ("fast", ctypes.c_double), ("amplitude", ctypes.c_double)]


class PackedDesc(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("sequences", ctypes.c_int32), ("max_q", ctypes.c_int32), ("max_k", ctypes.c_int32),
                ("q_tokens", ctypes.c_int64), ("k_tokens", ctypes.c_int64), ("scale", ctypes.c_float)]


class PackedSequences(ctypes.Structure):
    _fields_ = [("q_offsets", ctypes.c_void_p), ("k_offsets", ctypes.c_void_p), ("q_lengths", ctypes.c_void_p),
                ("k_lengths", ctypes.c_void_p)]


REDUCE_OP_FN = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int,
                                ctypes.c_void_p, ctypes.c_void_p)
REDUCE_SUM, REDUCE_MAX = 0, 1


class _Ptrs12(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in PARAM_NAMES]


class SavedLayout(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in
                ("u1", "qkv", "a", "x1", "u2", "z", "g", "mu1", "rs1", "mu2", "rs2", "lse", "total")]


REDUCE_FN = ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int,
                             ctypes.c_void_p, ctypes.c_void_p)

_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2201_11990_amd.build` "
                               "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, sz, i32, i64, u32, f32 = (ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64,
                                      ctypes.c_uint32, ctypes.c_float)
        dp = ctypes.POINTER(LayerDesc)
        pp = ctypes.POINTER(_Ptrs12)
        sigs = {
            "mtnlg_version": (ctypes.c_int, []),
            "mtnlg_status_string": (ctypes.c_char_p, [ctypes.c_int]),
            "mtnlg_layer_desc_check": (ctypes.c_int, [dp]),
            "mtnlg_saved_layout_get": (ctypes.c_int, [dp, ctypes.POINTER(SavedLayout)]),
            "mtnlg_saved_bytes": (sz, [dp]),
            "mtnlg_stage_saved_bytes": (sz, [dp, ctypes.c_int]),
            "mtnlg_workspace_bytes": (sz, [dp]),
            "mtnlg_layer_fwd": (ctypes.c_int, [dp, pp, vp, vp, vp, vp, sz, REDUCE_FN, vp, vp]),
            "mtnlg_layer_bwd": (ctypes.c_int, [dp, pp, vp, vp, vp, vp, pp, vp, sz, REDUCE_FN, vp, vp]),
            "mtnlg_stage_step": (ctypes.c_int, [dp, ctypes.c_int, pp, vp, vp, vp, vp, pp, vp, sz, vp, sz,
                                                REDUCE_FN, vp, vp]),
            "mtnlg_stage_step_accumulate": (ctypes.c_int, [dp, ctypes.c_int, pp, ctypes.c_int, vp, vp, vp, vp, pp, vp,
                                                           sz, vp, sz, REDUCE_FN, vp, vp]),
            "mtnlg_lm_head_workspace": (sz, [ctypes.POINTER(HeadDesc)]),
            "mtnlg_embedding_fwd": (ctypes.c_int, [ctypes.POINTER(HeadDesc), vp, vp, vp, vp, REDUCE_OP_FN, vp, vp]),
            "mtnlg_embedding_bwd": (ctypes.c_int, [ctypes.POINTER(HeadDesc), vp, vp, vp, vp, vp]),
            "mtnlg_lm_head_step": (ctypes.c_int, [ctypes.POINTER(HeadDesc), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                                  vp, sz, REDUCE_OP_FN, vp, vp]),
            "mtnlg_grad_sqnorm_workspace": (sz, []),
            "mtnlg_grad_sqnorm": (ctypes.c_int, [i64, vp, vp, vp, ctypes.c_int, vp]),
            "mtnlg_adam_step": (ctypes.c_int, [ctypes.POINTER(AdamDesc), i64, vp, vp, vp, vp, vp, vp, vp]),
            "mtnlg_gemm_workspace": (sz, [ctypes.c_int, ctypes.c_int, i64, i64, i64]),
            "mtnlg_gemm": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, i64, i64, i64, vp, vp, vp, vp, vp, u32, vp, sz, vp]),
            "mtnlg_layernorm_fwd": (ctypes.c_int, [ctypes.c_int, i64, i64, vp, vp, vp, vp, vp, f32, vp, vp, vp, vp, vp]),
            "mtnlg_layernorm_bwd_workspace": (sz, [i64, i64]),
            "mtnlg_layernorm_bwd": (ctypes.c_int, [ctypes.c_int, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                                   ctypes.c_int, ctypes.c_int, vp, vp]),
            "mtnlg_attention_fwd": (ctypes.c_int, [ctypes.c_int, i32, i32, i32, i32, f32, vp, vp, vp, vp]),
            "mtnlg_attention_bwd_workspace": (sz, [i32, i32, i32, i32]),
            "mtnlg_attention_bwd": (ctypes.c_int, [ctypes.c_int, i32, i32, i32, i32, f32, vp, vp, vp, vp, vp, vp, vp]),
            "mtnlg_gelu_fwd": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, i64, vp, vp, vp]),
            "mtnlg_gelu_bwd": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, i64, vp, vp, vp, vp]),
            "mtnlg_colsum_workspace": (sz, [i64, i64]),
            "mtnlg_colsum": (ctypes.c_int, [ctypes.c_int, i64, i64, vp, vp, ctypes.c_int, ctypes.c_int, vp, vp]),
            "mtnlg_colsum_static_max_columns": (i64, []),
            "mtnlg_colsum_static": (ctypes.c_int, [ctypes.c_int, i64, i64, vp, vp, ctypes.c_int, ctypes.c_int, vp]),
            "mtnlg_bias_residual": (ctypes.c_int, [ctypes.c_int, i64, i64, vp, vp, vp, vp, vp]),
            "mtnlg_rmsnorm_fwd": (ctypes.c_int, [ctypes.c_int, i64, i64, vp, vp, vp, f32, vp, vp, vp, vp]),
            "mtnlg_rmsnorm_fwd_e4m3": (ctypes.c_int, [ctypes.c_int, i64, i64, vp, vp, vp, f32, i32, vp, vp, vp, vp, vp]),
            "mtnlg_rmsnorm_bwd_workspace": (sz, [i64, i64]),
            "mtnlg_rmsnorm_bwd": (ctypes.c_int, [ctypes.c_int, i64, i64, vp, vp, vp, vp, vp, vp, vp, ctypes.c_int, ctypes.c_int,
                                                 vp, sz, vp]),
            "mtnlg_rotary_fwd": (ctypes.c_int, [vp, vp, vp, vp, vp, vp, vp]),
            "mtnlg_rotary_bwd": (ctypes.c_int, [vp, vp, vp, vp, vp, vp, vp]),
            "mtnlg_packed_attention_fwd_workspace": (sz, [ctypes.POINTER(PackedDesc)]),
            "mtnlg_packed_attention_fwd": (ctypes.c_int, [vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
            "mtnlg_packed_attention_bwd_workspace": (sz, [ctypes.POINTER(PackedDesc)]),
            "mtnlg_packed_attention_bwd": (ctypes.c_int, [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
            "mtnlg_calibrate_mfma_operand_bytes": (sz, [ctypes.c_int]),
            "mtnlg_calibrate_mfma_flops": (i64, [ctypes.c_int, ctypes.c_int]),
            "mtnlg_calibrate_mfma": (ctypes.c_int, [ctypes.c_int, ctypes.c_int, vp, vp, vp]),
            "mtnlg_calibrate_copy": (ctypes.c_int, [vp, vp, i64, vp]),
            "mtnlg_profile_enable": (ctypes.c_int, [ctypes.c_int]),
            "mtnlg_profile_pause": (ctypes.c_int, [ctypes.c_int]),
            "mtnlg_profile_read": (ctypes.c_int, [ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_float)]),
        }
        for name, (res, args) in sigs.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


EXPORTED = ("mtnlg_version", "mtnlg_status_string", "mtnlg_layer_desc_check", "mtnlg_saved_layout_get",
            "mtnlg_saved_bytes", "mtnlg_stage_saved_bytes", "mtnlg_workspace_bytes", "mtnlg_layer_fwd",
            "mtnlg_layer_bwd", "mtnlg_stage_step", "mtnlg_stage_step_accumulate", "mtnlg_gemm_workspace", "mtnlg_gemm", "mtnlg_layernorm_fwd",
            "mtnlg_layernorm_bwd_workspace", "mtnlg_layernorm_bwd", "mtnlg_attention_fwd",
            "mtnlg_attention_bwd_workspace", "mtnlg_attention_bwd", "mtnlg_gelu_fwd", "mtnlg_gelu_bwd",
            "mtnlg_colsum_workspace", "mtnlg_colsum", "mtnlg_colsum_static_max_columns", "mtnlg_colsum_static",
            "mtnlg_bias_residual", "mtnlg_grad_sqnorm_workspace", "mtnlg_grad_sqnorm", "mtnlg_adam_step",
            "mtnlg_lm_head_workspace", "mtnlg_embedding_fwd", "mtnlg_embedding_bwd", "mtnlg_lm_head_step",
            "mtnlg_rmsnorm_fwd", "mtnlg_rmsnorm_fwd_e4m3", "mtnlg_rmsnorm_bwd_workspace", "mtnlg_rmsnorm_bwd",
            "mtnlg_rotary_fwd", "mtnlg_rotary_bwd", "mtnlg_packed_attention_fwd_workspace", "mtnlg_packed_attention_fwd",
            "mtnlg_packed_attention_bwd_workspace", "mtnlg_packed_attention_bwd",
            "mtnlg_calibrate_mfma_operand_bytes", "mtnlg_calibrate_mfma_flops", "mtnlg_calibrate_mfma",
            "mtnlg_calibrate_copy", "mtnlg_profile_enable", "mtnlg_profile_pause", "mtnlg_profile_read")


def status_string(status):
    return lib().mtnlg_status_string(int(status)).decode()


def _check(status, where):
    if status != 0:
        raise MtnlgError(status, where)


def _dtype_code(t):
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _p(t):
    """Device pointer of a contiguous CUDA tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors handed to the library must be contiguous device tensors")
    return ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def make_desc(hidden, heads_local, head_dim, ffn_local, seq, micro_batch, dtype, tp_size=1, tp_rank=0,
              gelu=GELU_TANH, ln_eps=0.0, softmax_scale=0.0, flags=0):
    code = dtype if isinstance(dtype, int) else {"fp32": F32, "bf16": BF16,
                                                 torch.float32: F32, torch.bfloat16: BF16}[dtype]
    return LayerDesc(hidden, heads_local, head_dim, ffn_local, seq, micro_batch, tp_size, tp_rank, code,
                     gelu, ln_eps, softmax_scale, flags)


def desc_from_workload(wl, flags=0, **kw):
    return make_desc(wl.hidden, wl.heads, wl.head_dim, wl.ffn, wl.seq, wl.micro_batch, wl.dtype,
                     tp_size=wl.tp_size, flags=flags | (RECOMPUTE if wl.recompute else 0), **kw)


def mtnlg_version():
    return lib().mtnlg_version()


def mtnlg_layer_desc_check(desc):
    return lib().mtnlg_layer_desc_check(ctypes.byref(desc))


def mtnlg_saved_layout_get(desc):
    out = SavedLayout()
    _check(lib().mtnlg_saved_layout_get(ctypes.byref(desc), ctypes.byref(out)), "mtnlg_saved_layout_get")
    return out


def mtnlg_saved_bytes(desc):
    return lib().mtnlg_saved_bytes(ctypes.byref(desc))


def mtnlg_stage_saved_bytes(desc, n_layers):
    return lib().mtnlg_stage_saved_bytes(ctypes.byref(desc), n_layers)


def mtnlg_workspace_bytes(desc):
    return lib().mtnlg_workspace_bytes(ctypes.byref(desc))


def _table(tensors):
    st = _Ptrs12()
    for n in PARAM_NAMES:
        setattr(st, n, _p(tensors[n]))
    return st


def _tables(list_of_dicts):
    arr = (_Ptrs12 * len(list_of_dicts))()
    for i, d in enumerate(list_of_dicts):
        for n in PARAM_NAMES:
            setattr(arr[i], n, _p(d[n]))
    return arr


def _hook(reduce):
    """reduce(ptr:int, count:int, dtype:int, stream:int) -> None, or None."""
    if reduce is None:
        return ctypes.cast(None, REDUCE_FN)

    def cb(buf, count, dtype, stream, _user):
        try:
            reduce(buf, count, dtype, stream)
            return 0
        except Exception:  # noqa: BLE001 - must not unwind through C
            return 1

    return REDUCE_FN(cb)


def _nbytes(t):
    return t.numel() * t.element_size()


def mtnlg_layer_fwd(desc, weights, x, y, saved, workspace, reduce=None):
    hook = _hook(reduce)
    _check(lib().mtnlg_layer_fwd(ctypes.byref(desc), ctypes.byref(_table(weights)), _p(x), _p(y), _p(saved),
                                 _p(workspace), _nbytes(workspace), hook, None, _stream()), "mtnlg_layer_fwd")


def mtnlg_layer_bwd(desc, weights, x, saved, dy, dx, grads, workspace, reduce=None):
    hook = _hook(reduce)
    _check(lib().mtnlg_layer_bwd(ctypes.byref(desc), ctypes.byref(_table(weights)), _p(x), _p(saved), _p(dy),
                                 _p(dx), ctypes.byref(_table(grads)), _p(workspace), _nbytes(workspace), hook,
                                 None, _stream()), "mtnlg_layer_bwd")


class StageArgs:
    """Marshalled argument tables of mtnlg_stage_step, built once and reused per call."""

    def __init__(self, desc, weights, grads):
        self.desc, self.n_layers = desc, len(weights)
        self.w, self.g = _tables(weights), _tables(grads)
        self._keep = (weights, grads)


def mtnlg_stage_step(desc, weights, x_in, dy_out, y_out, dx_in, grads, saved, workspace, reduce=None,
                     args=None):
    a = args if args is not None else StageArgs(desc, weights, grads)
    hook = _hook(reduce)
    _check(lib().mtnlg_stage_step(ctypes.byref(a.desc), a.n_layers, a.w, _p(x_in), _p(dy_out), _p(y_out),
                                  _p(dx_in), a.g, _p(saved), _nbytes(saved), _p(workspace),
                                  _nbytes(workspace), hook, None, _stream()), "mtnlg_stage_step")


def mtnlg_stage_step_accumulate(desc, weights, x_in, dy_out, y_out, dx_in, grads, saved, workspace, reduce=None,
                                args=None):
    """x_in, dy_out, y_out, dx_in: [n_micro, b, s, h] contiguous."""
    a = args if args is not None else StageArgs(desc, weights, grads)
    hook = _hook(reduce)
    n_micro = x_in.shape[0]
    assert x_in.is_contiguous() and dy_out.is_contiguous() and y_out.is_contiguous() and dx_in.is_contiguous()
    assert dy_out.shape[0] == n_micro and y_out.shape[0] == n_micro and dx_in.shape[0] == n_micro
    _check(lib().mtnlg_stage_step_accumulate(ctypes.byref(a.desc), a.n_layers, a.w, n_micro, _p(x_in), _p(dy_out),
                                             _p(y_out), _p(dx_in), a.g, _p(saved), _nbytes(saved), _p(workspace),
                                             _nbytes(workspace), hook, None, _stream()),
           "mtnlg_stage_step_accumulate")


def mtnlg_gemm_workspace(dtype, layout, M, N, K):
    return lib().mtnlg_gemm_workspace(dtype, layout, M, N, K)


def mtnlg_gemm(layout, A, B, C, bias=None, aux=None, epilogue=0, workspace=None):
    if layout == GEMM_NT:
        (M, K), N = A.shape, B.shape[0]
        assert B.shape == (N, K)
    elif layout == GEMM_NN:
        (M, K), N = A.shape, B.shape[1]
        assert B.shape == (K, N)
    else:
        (K, M), N = A.shape, B.shape[1]
        assert B.shape == (K, N)
    assert C.shape == (M, N)
    _check(lib().mtnlg_gemm(_dtype_code(A), layout, M, N, K, _p(A), _p(B), _p(C), _p(bias), _p(aux), epilogue,
                            _p(workspace), _nbytes(workspace) if workspace is not None else 0, _stream()),
           "mtnlg_gemm")


def mtnlg_layernorm_fwd(x, gamma, beta, eps, out, mean, rstd, partial=None, bias=None, xsum=None):
    T, h = x.shape
    _check(lib().mtnlg_layernorm_fwd(_dtype_code(x), T, h, _p(x), _p(partial), _p(bias), _p(gamma), _p(beta),
                                     eps, _p(xsum), _p(out), _p(mean), _p(rstd), _stream()),
           "mtnlg_layernorm_fwd")


def mtnlg_layernorm_bwd_workspace(T, h):
    return lib().mtnlg_layernorm_bwd_workspace(T, h)


def mtnlg_layernorm_bwd(x, gamma, mean, rstd, dout, dx, dgamma, dbeta, workspace, dres=None, colsum_dx=None,
                        grad_f32=False, accumulate=False):
    T, h = x.shape
    _check(lib().mtnlg_layernorm_bwd(_dtype_code(x), T, h, _p(x), _p(gamma), _p(mean), _p(rstd), _p(dout),
                                     _p(dres), _p(dx), _p(dgamma), _p(dbeta), _p(colsum_dx), int(grad_f32),
                                     int(accumulate), _p(workspace), _stream()), "mtnlg_layernorm_bwd")


def mtnlg_attention_fwd(b, s, n, d, scale, qkv, a, lse):
    _check(lib().mtnlg_attention_fwd(_dtype_code(qkv), b, s, n, d, scale, _p(qkv), _p(a), _p(lse), _stream()),
           "mtnlg_attention_fwd")


def mtnlg_attention_bwd_workspace(b, s, n, d):
    return lib().mtnlg_attention_bwd_workspace(b, s, n, d)


def mtnlg_attention_bwd(b, s, n, d, scale, qkv, a, lse, da, dqkv, workspace):
    _check(lib().mtnlg_attention_bwd(_dtype_code(qkv), b, s, n, d, scale, _p(qkv), _p(a), _p(lse), _p(da),
                                     _p(dqkv), _p(workspace), _stream()), "mtnlg_attention_bwd")


def mtnlg_gelu_fwd(z, g, gelu=GELU_TANH):
    _check(lib().mtnlg_gelu_fwd(_dtype_code(z), gelu, z.numel(), _p(z), _p(g), _stream()), "mtnlg_gelu_fwd")


def mtnlg_gelu_bwd(z, dg, dz, gelu=GELU_TANH):
    _check(lib().mtnlg_gelu_bwd(_dtype_code(z), gelu, z.numel(), _p(z), _p(dg), _p(dz), _stream()),
           "mtnlg_gelu_bwd")


def mtnlg_colsum_workspace(T, C):
    return lib().mtnlg_colsum_workspace(T, C)


def mtnlg_colsum(x, out, workspace, accumulate=False):
    T, C = x.shape
    _check(lib().mtnlg_colsum(_dtype_code(x), T, C, _p(x), _p(out), int(out.dtype == torch.float32),
                              int(accumulate), _p(workspace), _stream()), "mtnlg_colsum")


def mtnlg_colsum_static_max_columns():
    return lib().mtnlg_colsum_static_max_columns()


def mtnlg_colsum_static(x, out, accumulate=False):
    T, C = x.shape
    _check(lib().mtnlg_colsum_static(_dtype_code(x), T, C, _p(x), _p(out), int(out.dtype == torch.float32),
                                     int(accumulate), _stream()), "mtnlg_colsum_static")


def mtnlg_bias_residual(res, partial, bias, out):
    T, h = res.shape
    _check(lib().mtnlg_bias_residual(_dtype_code(res), T, h, _p(res), _p(partial), _p(bias), _p(out), _stream()),
           "mtnlg_bias_residual")


def head_desc(hidden, vocab_local, vocab_start, seq, micro_batch, dtype, ln_eps=1e-5):
    return HeadDesc(hidden, vocab_local, vocab_start, seq, micro_batch, {"fp32": F32, "bf16": BF16}[dtype], ln_eps)


def _op_hook(reduce):
    """reduce(ptr:int, count:int, dtype:int, op:int, stream:int) -> None, or None."""
    if reduce is None:
        return ctypes.cast(None, REDUCE_OP_FN)

    def cb(buf, count, dtype, op, stream, _user):
        try:
            reduce(buf, count, dtype, op, stream)
            return 0
        except Exception:  # noqa: BLE001 - must not unwind through C
            return 1

    return REDUCE_OP_FN(cb)


def mtnlg_lm_head_workspace(desc):
    return lib().mtnlg_lm_head_workspace(ctypes.byref(desc))


def mtnlg_embedding_fwd(desc, tokens, emb, pos, x, reduce=None):
    assert tokens.dtype == torch.int32
    _check(lib().mtnlg_embedding_fwd(ctypes.byref(desc), _p(tokens), _p(emb), _p(pos), _p(x), _op_hook(reduce), None,
                                     _stream()), "mtnlg_embedding_fwd")


def mtnlg_embedding_bwd(desc, tokens, dx, demb, dpos):
    assert tokens.dtype == torch.int32
    _check(lib().mtnlg_embedding_bwd(ctypes.byref(desc), _p(tokens), _p(dx), _p(demb), _p(dpos), _stream()),
           "mtnlg_embedding_bwd")


def mtnlg_lm_head_step(desc, x, ln_g, ln_b, emb, targets, dloss, loss, dx, d_ln_g, d_ln_b, demb, workspace, reduce=None):
    assert targets.dtype == torch.int32 and loss.dtype == torch.float32
    assert dloss is None or dloss.dtype == torch.float32
    _check(lib().mtnlg_lm_head_step(ctypes.byref(desc), _p(x), _p(ln_g), _p(ln_b), _p(emb), _p(targets), _p(dloss),
                                    _p(loss), _p(dx), _p(d_ln_g), _p(d_ln_b), _p(demb), _p(workspace),
                                    _nbytes(workspace), _op_hook(reduce), None, _stream()), "mtnlg_lm_head_step")


def _device_stream(*tensors):
    """The current stream, of the current device, on which all the tensors (None aside) have to be."""
    device = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("tensors handed to the library must be on the current device")
    return torch._C._cuda_getCurrentRawStream(device)


def _like(t, dtype, shape, what):
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{what}: expected {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")


def _dense(t):
    """Address of a contiguous tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors handed to the library must be contiguous device tensors")
    return t.data_ptr()


def _strides(t, kv_heads):
    """Address and strides (token, group, head of the group) of a matrix of heads: [tokens, heads, head_dim] or [tokens, kv_heads, heads of a
    group, head_dim], any strides but the last's."""
    st, shape = t.stride(), t.shape
    if len(st) not in (3, 4) or shape[-1] == 0 or (shape[-1] > 1 and st[-1] != 1):
        raise ValueError("heads: [tokens, heads, head_dim] or [tokens, kv_heads, group, head_dim] with dense rows")
    if len(st) == 4:
        return t.data_ptr(), st[0], st[1], st[2]
    return t.data_ptr(), st[0], st[1] * (shape[1] // kv_heads), st[1]


def _heads(t, kv_heads):
    return None if t is None else Heads(*_strides(t, kv_heads))


def _counts(q, k):
    """heads, kv_heads, head_dim of a matrix of query heads beside one of key heads."""
    if q.dim() not in (3, 4):
        raise ValueError("heads: [tokens, heads, head_dim] or [tokens, kv_heads, group, head_dim]")
    shape = q.shape
    heads = shape[1] if len(shape) == 3 else shape[1] * shape[2]
    kv_heads = shape[1]
    if k is not None:
        if k.dim() != 3 or k.shape[2] != shape[-1] or k.dtype != q.dtype:
            raise ValueError("keys and values: [tokens, kv_heads, head_dim] of the queries' type and head size")
        kv_heads = k.shape[1]
    if kv_heads == 0 or heads % kv_heads or (len(shape) == 4 and shape[1] != kv_heads):
        raise ValueError("the number of query heads is a multiple of that of key heads")
    return heads, kv_heads, shape[-1]


class _Structs:
    """The structs of a call side by side in one buffer: one packing for all their fields, and an address for each."""

    def __init__(self, layout, *fields):
        self.bytes = bytearray(layout.pack(*fields))
        self.at = ctypes.addressof(ctypes.c_char.from_buffer(self.bytes))


def mtnlg_rmsnorm_fwd(x, gamma, eps, out, rstd, residual=None, xsum=None):
    """x, residual, xsum, out: [T, h] (contiguous); rstd: fp32 [T]."""
    T, h = shape = x.shape
    dtype = x.dtype
    stream = _device_stream(x, gamma, out, rstd, residual, xsum)
    _like(out, dtype, shape, "out")
    _like(gamma, dtype, (h,), "gamma")
    _like(rstd, torch.float32, (T,), "rstd")
    if residual is not None:
        _like(residual, dtype, shape, "residual")
    if xsum is not None:
        _like(xsum, dtype, shape, "xsum")
    _check(lib().mtnlg_rmsnorm_fwd(_dtype_code(x), T, h, _dense(x), _dense(residual), _dense(gamma), eps, _dense(xsum), _dense(out),
                                   _dense(rstd), stream), "mtnlg_rmsnorm_fwd")


def mtnlg_rmsnorm_fwd_e4m3(x, gamma, eps, out, scale, rstd, columns=0, residual=None, xsum=None):
    """out: e4m3 [T, h]; scale: fp32 [T, number of groups of `columns` columns] (columns 0: one to a row)."""
    T, h = shape = x.shape
    dtype = x.dtype
    stream = _device_stream(x, gamma, out, scale, rstd, residual, xsum)
    _like(out, torch.float8_e4m3fn, shape, "out")
    _like(gamma, dtype, (h,), "gamma")
    _like(scale, torch.float32, (T, -(-h // columns) if columns > 0 else 1), "scale")
    _like(rstd, torch.float32, (T,), "rstd")
    if residual is not None:
        _like(residual, dtype, shape, "residual")
    if xsum is not None:
        _like(xsum, dtype, shape, "xsum")
    _check(lib().mtnlg_rmsnorm_fwd_e4m3(_dtype_code(x), T, h, _dense(x), _dense(residual), _dense(gamma), eps, columns, _dense(xsum),
                                        _dense(out), _dense(scale), _dense(rstd), stream), "mtnlg_rmsnorm_fwd_e4m3")


def mtnlg_rmsnorm_bwd_workspace(T, h):
    return lib().mtnlg_rmsnorm_bwd_workspace(T, h)


def mtnlg_rmsnorm_bwd(x, gamma, rstd, dout, dx, dgamma, workspace, dres=None, accumulate=False):
    """x: what was normalised; dgamma: [h], fp32 or x's type."""
    T, h = shape = x.shape
    dtype = x.dtype
    stream = _device_stream(x, gamma, rstd, dout, dx, dgamma, workspace, dres)
    _like(dout, dtype, shape, "dout")
    _like(dx, dtype, shape, "dx")
    if dres is not None:
        _like(dres, dtype, shape, "dres")
    _like(gamma, dtype, (h,), "gamma")
    _like(rstd, torch.float32, (T,), "rstd")
    grad_f32 = dgamma.dtype == torch.float32
    _like(dgamma, torch.float32 if grad_f32 else dtype, (h,), "dgamma")
    _check(lib().mtnlg_rmsnorm_bwd(_dtype_code(x), T, h, _dense(x), _dense(gamma), _dense(rstd), _dense(dout), _dense(dres), _dense(dx),
                                   _dense(dgamma), int(grad_f32), int(accumulate), _dense(workspace), _nbytes(workspace), stream),
           "mtnlg_rmsnorm_bwd")


def rotary_desc(rotary_dim, layout=ROTARY_HALF, base=10000.0, scaling=ROTARY_UNSCALED, factor=1.0, original_positions=0, slow=1.0,
                fast=32.0, amplitude=0.0):
    """How heads turn; their number, size and type come from the tensors of the call."""
    return RotaryDesc(0, 0, 0, 0, rotary_dim, layout, scaling, original_positions, 0, base, factor, slow, fast, amplitude)


# a RotaryDesc, then four Heads
_ROTARY = struct.Struct("8i q5d 16q")


def _rotary(name, desc, q, k, q_out, k_out, positions):
    heads, n, d = _counts(q, k)
    stream = _device_stream(q, k, q_out, k_out, positions)
    if (k is None) != (k_out is None):
        raise ValueError("keys go with an output of theirs")
    _like(q_out, q.dtype, q.shape, "the output of the queries")
    tokens = q.shape[0]
    none = (0, 0, 0, 0)
    if k is not None:
        if k.shape[0] != tokens:
            raise ValueError("queries and keys of the same tokens")
        _like(k_out, k.dtype, k.shape, "the output of the keys")
    if positions is not None:
        _like(positions, torch.int32, (tokens,), "positions")
    s = _Structs(_ROTARY, _dtype_code(q), heads, n, d, desc.rotary_dim, desc.layout, desc.scaling, desc.original_positions, tokens,
                 desc.base, desc.factor, desc.slow, desc.fast, desc.amplitude, *_strides(q, n), *(_strides(k, n) if k is not None else none),
                 *_strides(q_out, n), *(_strides(k_out, n) if k is not None else none))
    first = s.at + ctypes.sizeof(RotaryDesc)
    _check(getattr(lib(), name)(s.at, first, first + 32 if k is not None else None, first + 64, first + 96 if k is not None else None,
                                _dense(positions), stream), name)


def mtnlg_rotary_fwd(desc, q, k, q_out, k_out, positions=None):
    """q: [tokens, heads, head_dim] or [tokens, kv_heads, group, head_dim], k (nullable): [tokens, kv_heads, head_dim]; positions: int32 [tokens]."""
    _rotary("mtnlg_rotary_fwd", desc, q, k, q_out, k_out, positions)


def mtnlg_rotary_bwd(desc, dq_out, dk_out, dq, dk, positions=None):
    _rotary("mtnlg_rotary_bwd", desc, dq_out, dk_out, dq, dk, positions)


def packed_desc(q, k, sequences, max_q, max_k, scale=0.0):
    """Sizes of calls of attention over packed sequences: q [tokens, heads, head_dim] or [tokens, kv_heads, group, head_dim], k [tokens, kv_heads, head_dim]."""
    heads, kv_heads, d = _counts(q, k)
    return PackedDesc(_dtype_code(q), heads, kv_heads, d, sequences, max_q, max_k, q.shape[0], k.shape[0], scale)


def mtnlg_packed_attention_fwd_workspace(desc):
    return lib().mtnlg_packed_attention_fwd_workspace(ctypes.byref(desc))


def mtnlg_packed_attention_bwd_workspace(desc):
    return lib().mtnlg_packed_attention_bwd_workspace(ctypes.byref(desc))


# a PackedDesc, a PackedSequences, then Heads
_PACKED = "7i4x2qf4x 4P"
_PACKED_FWD, _PACKED_BWD = struct.Struct(_PACKED + "16q"), struct.Struct(_PACKED + "32q")
_PACKED_HEADS = ctypes.sizeof(PackedDesc) + ctypes.sizeof(PackedSequences)


def _packed(q, k, v, a, lse, q_offsets, k_offsets, max_q, max_k, scale, q_lengths, k_lengths):
    """Fields of the descriptor, the sequences and the heads of q, k, v, a; the number of key heads."""
    heads, n, d = _counts(q, k)
    sequences = q_offsets.shape[0] - 1
    _like(v, k.dtype, k.shape, "v")
    _like(a, q.dtype, q.shape, "a")
    _like(lse, torch.float32, (heads, q.shape[0]), "lse")
    _like(q_offsets, torch.int32, (sequences + 1,), "q_offsets")
    _like(k_offsets, torch.int32, (sequences + 1,), "k_offsets")
    if q_lengths is not None:
        _like(q_lengths, torch.int32, (sequences,), "q_lengths")
    if k_lengths is not None:
        _like(k_lengths, torch.int32, (sequences,), "k_lengths")
    return (_dtype_code(q), heads, n, d, sequences, max_q, max_k, q.shape[0], k.shape[0], scale, _dense(q_offsets), _dense(k_offsets),
            _dense(q_lengths) or 0, _dense(k_lengths) or 0, *_strides(q, n), *_strides(k, n), *_strides(v, n), *_strides(a, n)), n


def mtnlg_packed_attention_fwd(q, k, v, a, lse, q_offsets, k_offsets, max_q, max_k, scale=0.0, q_lengths=None, k_lengths=None,
                               workspace=None):
    """q, a: [tokens, heads, head_dim] or [tokens, kv_heads, group, head_dim]; k, v: [tokens, kv_heads, head_dim]; lse: fp32 [heads, tokens];
    offsets: int32 [sequences + 1] on the device, lengths (nullable) [sequences]; max_q, max_k: no sequence is longer."""
    stream = _device_stream(q, k, v, a, lse, q_offsets, k_offsets, q_lengths, k_lengths, workspace)
    fields, _ = _packed(q, k, v, a, lse, q_offsets, k_offsets, max_q, max_k, scale, q_lengths, k_lengths)
    s = _Structs(_PACKED_FWD, *fields)
    h = s.at + _PACKED_HEADS
    _check(lib().mtnlg_packed_attention_fwd(s.at, s.at + ctypes.sizeof(PackedDesc), h, h + 32, h + 64, h + 96, _dense(lse), _dense(workspace),
                                            _nbytes(workspace) if workspace is not None else 0, stream), "mtnlg_packed_attention_fwd")


def mtnlg_packed_attention_bwd(q, k, v, a, lse, da, dq, dk, dv, q_offsets, k_offsets, max_q, max_k, workspace, scale=0.0, q_lengths=None,
                               k_lengths=None):
    stream = _device_stream(q, k, v, a, lse, da, dq, dk, dv, q_offsets, k_offsets, q_lengths, k_lengths, workspace)
    fields, n = _packed(q, k, v, a, lse, q_offsets, k_offsets, max_q, max_k, scale, q_lengths, k_lengths)
    _like(da, q.dtype, q.shape, "da")
    _like(dq, q.dtype, q.shape, "dq")
    _like(dk, k.dtype, k.shape, "dk")
    _like(dv, k.dtype, k.shape, "dv")
    s = _Structs(_PACKED_BWD, *fields, *_strides(da, n), *_strides(dq, n), *_strides(dk, n), *_strides(dv, n))
    h = s.at + _PACKED_HEADS
    _check(lib().mtnlg_packed_attention_bwd(s.at, s.at + ctypes.sizeof(PackedDesc), h, h + 32, h + 64, h + 96, _dense(lse), h + 128, h + 160,
                                            h + 192, h + 224, _dense(workspace), _nbytes(workspace), stream), "mtnlg_packed_attention_bwd")


def mtnlg_grad_sqnorm_workspace():
    return lib().mtnlg_grad_sqnorm_workspace()


def mtnlg_grad_sqnorm(grad, workspace, sqnorm, accumulate=False):
    """grad: fp32 tensor (any shape, contiguous); sqnorm: fp32 device tensor of one element."""
    assert grad.dtype == torch.float32 and grad.is_contiguous() and sqnorm.dtype == torch.float32
    _check(lib().mtnlg_grad_sqnorm(grad.numel(), _p(grad), _p(workspace), _p(sqnorm), int(bool(accumulate)), _stream()),
           "mtnlg_grad_sqnorm")


def mtnlg_adam_step(master, m, v, grad, weight_bf16=None, sqnorm=None, *, lr, step, beta1=0.9, beta2=0.95, eps=1e-8,
                    weight_decay=0.1, max_grad_norm=1.0):
    """In-place Adam update of fp32 tensors master, m, v from fp32 grad; weight_bf16 receives the rounded weight."""
    for t in (master, m, v, grad):
        assert t.dtype == torch.float32 and t.is_contiguous() and t.numel() == master.numel()
    if weight_bf16 is not None:
        assert weight_bf16.dtype == torch.bfloat16 and weight_bf16.is_contiguous() and weight_bf16.numel() == master.numel()
    d = AdamDesc(lr, beta1, beta2, eps, weight_decay, max_grad_norm, step)
    _check(lib().mtnlg_adam_step(ctypes.byref(d), master.numel(), _p(master), _p(m), _p(v), _p(grad), _p(weight_bf16),
                                 _p(sqnorm), _stream()), "mtnlg_adam_step")


def mtnlg_calibrate_mfma_operand_bytes(workgroups):
    return lib().mtnlg_calibrate_mfma_operand_bytes(workgroups)


def mtnlg_calibrate_mfma_flops(workgroups, iters):
    return lib().mtnlg_calibrate_mfma_flops(workgroups, iters)


def mtnlg_calibrate_mfma(workgroups, iters, operands, out):
    assert operands.dtype == torch.bfloat16 and _nbytes(operands) >= mtnlg_calibrate_mfma_operand_bytes(workgroups)
    assert out.dtype == torch.float32 and out.numel() >= workgroups * 512
    _check(lib().mtnlg_calibrate_mfma(workgroups, iters, _p(operands), _p(out), _stream()), "mtnlg_calibrate_mfma")


def mtnlg_calibrate_copy(dst, src):
    assert _nbytes(dst) == _nbytes(src)
    _check(lib().mtnlg_calibrate_copy(_p(dst), _p(src), _nbytes(src), _stream()), "mtnlg_calibrate_copy")


def mtnlg_profile_enable(on):
    _check(lib().mtnlg_profile_enable(int(bool(on))), "mtnlg_profile_enable")


def mtnlg_profile_pause(paused):
    _check(lib().mtnlg_profile_pause(int(bool(paused))), "mtnlg_profile_pause")


def mtnlg_profile_read():
    n = len(KERNEL_CLASSES)
    launches, ms = (ctypes.c_int32 * n)(), (ctypes.c_float * n)()
    _check(lib().mtnlg_profile_read(launches, ms), "mtnlg_profile_read")
    return {k: (launches[i], ms[i]) for i, k in enumerate(KERNEL_CLASSES)}
