"""ctypes binding of libtweo_hip.so: same names as include/tweo.h, argument marshalling only.

Tensors are torch tensors on the GPU (torch provides device memory and streams,
nothing else); bf16 tensors have dtype torch.bfloat16, E4M3 code tensors
torch.uint8, INT8 tensors torch.int8.  Every call is enqueued on torch's current
stream.  A non-zero status raises TweoError; a missing library raises at load
time - there is no fallback path.
"""
import ctypes
import functools
import os
import struct

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libtweo_hip.so")

TWEO_OK, TWEO_ERR_INVALID_ARG, TWEO_ERR_UNSUPPORTED, TWEO_ERR_WORKSPACE, TWEO_ERR_HIP = range(5)
(TWEO_OP_FP8_LINEAR_FWD, TWEO_OP_FP8_LINEAR_BWD, TWEO_OP_W8A8_LINEAR, TWEO_OP_FP8_LINEAR_FWD_BF16,
 TWEO_OP_FP8_LINEAR_BWD_BF16, TWEO_OP_LAYERNORM_QUANTIZE, TWEO_OP_LAYERNORM_BWD, TWEO_OP_GRAD_SUMSQ,
 TWEO_OP_HEAD_NORM_ROTARY_BWD, TWEO_OP_FP8_GATED_FWD_BF16, TWEO_OP_FP8_GATED_BWD_BF16) = range(11)

EXPORTS = ("tweo_workspace_bytes", "tweo_status_string", "tweo_amax", "tweo_quantize_e4m3",
           "tweo_fp8_linear_fwd", "tweo_fp8_linear_bwd", "tweo_quantize_i8", "tweo_w8a8_linear",
           "tweo_fp8_linear_fwd_bf16", "tweo_fp8_linear_bwd_bf16", "tweo_set_gemm_tile",
           "tweo_set_stream_k", "tweo_gemm_plan", "tweo_set_fused_cast", "tweo_fused_cast_timeouts", "tweo_amax_quantize_f8",
           "tweo_penalty_grad_inject", "tweo_delayed_state_bytes",
           "tweo_delayed_state_init", "tweo_quantize_e4m3_delayed", "tweo_profile_gemm_launches",
           "tweo_quantize_e5m2", "tweo_fp8_linear_bwd_hybrid", "tweo_fp8_linear_bwd_bf16_hybrid",
           "tweo_quantize_i8_rows", "tweo_w8a8_linear_scaled", "tweo_w8a8_linear_scaled_i8out",
           "tweo_quantize_e5m2_delayed", "tweo_fp8_linear_bwd_bf16_inject",
           "tweo_fp8_linear_fwd_static", "tweo_static_scratch_bytes",
           "tweo_layernorm_quantize_e4m3", "tweo_layernorm_quantize_e4m3_delayed",
           "tweo_fp8_linear_fwd_bf16_delayed", "tweo_fp8_linear_bwd_bf16_delayed",
           "tweo_layernorm_fwd", "tweo_layernorm_bwd", "tweo_optim_table_bytes", "tweo_optim_plan_init",
           "tweo_grad_sumsq", "tweo_adamw_step", "tweo_rotary", "tweo_rotary_freqs", "tweo_head_norm_rotary_fwd",
           "tweo_head_norm_rotary_bwd", "tweo_fp8_gated_fwd", "tweo_fp8_gated_fwd_bf16", "tweo_fp8_gated_bwd_bf16",
           "tweo_w8a8_gated", "tweo_w8a8_gated_i8out")


class TweoError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s: status %d (%s)" % (where, status, status_string(status)))


class PenaltyCfg(ctypes.Structure):
    _fields_ = [("tau", ctypes.c_float), ("eps", ctypes.c_float), ("p", ctypes.c_int)]


class GemmPlan(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int), ("runs", ctypes.c_int), ("shared", ctypes.c_int)]


class Fp8Saved(ctypes.Structure):
    _fields_ = [("xq", ctypes.c_void_p), ("xqT", ctypes.c_void_p), ("wq", ctypes.c_void_p),
                ("wqT", ctypes.c_void_p), ("scalars", ctypes.c_void_p)]


class OptimTensor(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_void_p) for k in ("param", "master", "grad", "m", "v", "m_step", "v_step")] +
                [("n", ctypes.c_int64), ("weight_decay", ctypes.c_float), ("param_f32", ctypes.c_int), ("grad_f32", ctypes.c_int)])


class OptimPlan(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("chunks", ctypes.c_int64), ("count", ctypes.c_int), ("state_bits", ctypes.c_int)]


class AdamwCfg(ctypes.Structure):
    _fields_ = [(k, ctypes.c_double) for k in ("lr", "beta1", "beta2", "eps", "max_norm")] + [("step", ctypes.c_int64)]


class Heads(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_void_p) for k in ("x", "y")] + [(k, ctypes.c_int64) for k in ("x_token", "x_head", "y_token", "y_head")] +
                [("gain", ctypes.c_void_p), ("heads", ctypes.c_int)])


class HeadsGrad(ctypes.Structure):
    _fields_ = ([(k, ctypes.c_void_p) for k in ("dy", "x", "dx")] +
                [(k, ctypes.c_int64) for k in ("dy_token", "dy_head", "x_token", "x_head", "dx_token", "dx_head")] +
                [(k, ctypes.c_void_p) for k in ("gain", "dgain")] + [("heads", ctypes.c_int)])


class RotaryCfg(ctypes.Structure):
    _fields_ = [("positions", ctypes.c_void_p), ("freqs", ctypes.c_void_p), ("rot_dim", ctypes.c_int), ("layout", ctypes.c_int),
                ("scale", ctypes.c_float)]


class RotaryFreqCfg(ctypes.Structure):
    _fields_ = [("base", ctypes.c_double), ("kind", ctypes.c_int)] + [(k, ctypes.c_double) for k in ("factor", "context", "low_turns", "high_turns")]


_lib = None


def load():
    """Loads the HIP library (after torch, so that both share one HIP runtime)."""
    global _lib
    if _lib is not None:
        return _lib
    import torch  # noqa: F401  (loads libamdhip64 first)
    if not os.path.exists(LIB_PATH):
        raise ImportError("%s is missing: run `python -m paper_2511_23225_amd.build` "
                          "(or __graft_entry__.build()) first" % LIB_PATH)
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, f32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    L.tweo_workspace_bytes.restype = sz
    L.tweo_workspace_bytes.argtypes = [ctypes.c_int, i64, i64, i64]
    L.tweo_status_string.restype = ctypes.c_char_p
    L.tweo_status_string.argtypes = [ctypes.c_int]
    L.tweo_amax.argtypes = [vp, i64, vp, vp]
    L.tweo_quantize_e4m3.argtypes = [vp, i64, i64, vp, vp, vp, vp, vp, vp]
    L.tweo_quantize_e5m2.argtypes = [vp, i64, i64, vp, vp, vp, vp, vp, vp]
    L.tweo_amax_quantize_f8.argtypes = [vp, i64, i64, ctypes.c_int, vp, vp, vp, vp, vp, vp, sz, vp]
    L.tweo_fp8_linear_fwd.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, vp,
                                      ctypes.POINTER(PenaltyCfg), vp, vp, sz, vp]
    L.tweo_fp8_linear_fwd_static.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, vp,
                                             ctypes.POINTER(PenaltyCfg), vp, vp]
    L.tweo_layernorm_quantize_e4m3.argtypes = [vp, vp, vp, vp, i64, i64, f32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.tweo_layernorm_quantize_e4m3_delayed.argtypes = [vp, vp, vp, vp, i64, i64, f32, vp, ctypes.c_int, vp, vp, vp,
                                                       vp, vp, sz, vp]
    L.tweo_fp8_linear_fwd_bf16_delayed.argtypes = [vp, vp, vp, i64, i64, i64, vp, ctypes.POINTER(PenaltyCfg), vp,
                                                   ctypes.POINTER(Fp8Saved), vp, vp, ctypes.c_int, vp, sz, vp]
    L.tweo_fp8_linear_bwd_bf16_delayed.argtypes = [vp, ctypes.POINTER(Fp8Saved), vp, ctypes.c_int, ctypes.c_int, i64,
                                                   i64, i64, vp, vp, vp, vp, vp, sz, vp]
    L.tweo_static_scratch_bytes.argtypes = []
    L.tweo_static_scratch_bytes.restype = ctypes.c_size_t
    L.tweo_fp8_linear_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, vp, vp, vp, sz, vp]
    L.tweo_fp8_linear_bwd_hybrid.argtypes = [vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, vp, vp, vp, sz, vp]
    L.tweo_quantize_i8.argtypes = [vp, i64, f32, vp, vp]
    L.tweo_w8a8_linear.argtypes = [vp, vp, i64, i64, i64, f32, vp, vp, sz, vp]
    L.tweo_quantize_i8_rows.argtypes = [vp, i64, i64, f32, vp, vp, vp]
    L.tweo_w8a8_linear_scaled.argtypes = [vp, vp, i64, i64, i64, vp, ctypes.c_int, vp, ctypes.c_int, vp, vp]
    L.tweo_w8a8_linear_scaled_i8out.argtypes = [vp, vp, i64, i64, i64, vp, ctypes.c_int, vp, ctypes.c_int, f32, vp, vp]
    L.tweo_fp8_linear_fwd_bf16.argtypes = [vp, vp, vp, i64, i64, i64, vp, ctypes.POINTER(PenaltyCfg),
                                           vp, ctypes.POINTER(Fp8Saved), vp, sz, vp]
    L.tweo_fp8_linear_bwd_bf16.argtypes = [vp, ctypes.POINTER(Fp8Saved), i64, i64, i64, vp, vp, vp,
                                           vp, vp, sz, vp]
    L.tweo_fp8_linear_bwd_bf16_hybrid.argtypes = L.tweo_fp8_linear_bwd_bf16.argtypes
    L.tweo_fp8_linear_bwd_bf16_inject.argtypes = [vp, vp, ctypes.POINTER(PenaltyCfg), f32, ctypes.c_int,
                                                  ctypes.POINTER(Fp8Saved), i64, i64, i64, vp, vp, vp, vp, vp, sz, vp]
    L.tweo_set_gemm_tile.argtypes = [ctypes.c_int]
    L.tweo_set_stream_k.argtypes = [ctypes.c_int]
    L.tweo_gemm_plan.argtypes = [ctypes.c_int, i64, i64, i64, ctypes.c_int, ctypes.c_int, sz, ctypes.POINTER(GemmPlan)]
    L.tweo_set_fused_cast.argtypes = [ctypes.c_int]
    L.tweo_fused_cast_timeouts.argtypes = [ctypes.POINTER(ctypes.c_uint)]
    L.tweo_profile_gemm_launches.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int]
    L.tweo_delayed_state_bytes.argtypes = []
    L.tweo_delayed_state_bytes.restype = ctypes.c_size_t
    L.tweo_delayed_state_init.argtypes = [vp, vp]
    L.tweo_quantize_e4m3_delayed.argtypes = [vp, i64, i64, vp, ctypes.c_int, vp, vp, vp]
    L.tweo_quantize_e5m2_delayed.argtypes = [vp, i64, i64, vp, ctypes.c_int, vp, vp, vp]
    L.tweo_penalty_grad_inject.argtypes = [vp, vp, i64, ctypes.POINTER(PenaltyCfg), ctypes.c_float, vp, vp]
    L.tweo_layernorm_fwd.argtypes = [vp, vp, vp, vp, i64, i64, f32, vp, vp, vp, vp]
    L.tweo_layernorm_bwd.argtypes = [vp, vp, vp, vp, vp, i64, i64, vp, vp, vp, vp, sz, vp]
    L.tweo_optim_table_bytes.argtypes = [ctypes.c_int]
    L.tweo_optim_table_bytes.restype = sz
    L.tweo_optim_plan_init.argtypes = [ctypes.POINTER(OptimTensor), ctypes.c_int, vp, sz, ctypes.POINTER(OptimPlan), vp]
    L.tweo_grad_sumsq.argtypes = [ctypes.POINTER(OptimPlan), vp, vp, sz, vp]
    L.tweo_adamw_step.argtypes = [ctypes.POINTER(OptimPlan), ctypes.POINTER(AdamwCfg), vp, vp, vp]
    L.tweo_rotary.argtypes = [vp, ctypes.c_int, i64, ctypes.c_int, vp, ctypes.c_int, vp]
    L.tweo_rotary_freqs.argtypes = [ctypes.POINTER(RotaryFreqCfg), ctypes.c_int, vp]
    L.tweo_head_norm_rotary_fwd.argtypes = [vp, ctypes.c_int, i64, ctypes.c_int, f32, vp, vp]
    L.tweo_head_norm_rotary_bwd.argtypes = [vp, ctypes.c_int, i64, ctypes.c_int, f32, vp, vp, sz, vp]
    c_int = ctypes.c_int
    L.tweo_fp8_gated_fwd.argtypes = [vp, vp, vp, vp, i64, i64, i64, c_int, vp, vp, vp]
    L.tweo_fp8_gated_fwd_bf16.argtypes = [vp, vp, i64, i64, i64, c_int, vp, vp, ctypes.POINTER(Fp8Saved), vp, vp, c_int, vp, sz, vp]
    L.tweo_fp8_gated_bwd_bf16.argtypes = [vp, vp, ctypes.POINTER(Fp8Saved), i64, i64, i64, c_int, c_int, vp, c_int, vp, vp, vp, vp, vp, sz, vp]
    L.tweo_w8a8_gated.argtypes = [vp, vp, i64, i64, i64, vp, c_int, vp, c_int, c_int, vp, vp]
    L.tweo_w8a8_gated_i8out.argtypes = [vp, vp, i64, i64, i64, vp, c_int, vp, c_int, c_int, f32, vp, vp]
    for name in EXPORTS:
        if name not in ("tweo_workspace_bytes", "tweo_status_string", "tweo_delayed_state_bytes",
                        "tweo_static_scratch_bytes", "tweo_optim_table_bytes"):
            getattr(L, name).restype = ctypes.c_int
    _lib = L
    return L


def status_string(status):
    return load().tweo_status_string(int(status)).decode()


def _ptr(t):
    # The functions' argtypes make a pointer of it.  An object per argument, and a struct per penalty, took 0.9 of the 20.8 us
    # that issuing a small layer's forward and backward took, 0.5 of 9.2 of quantise + W8A8 linear.
    return None if t is None else t.data_ptr()


_current = None  # (current device, raw stream handle of a device), once the GPU is initialised


def _forget_current():
    global _current
    _current = None


# a forked child cannot use its parent's GPU: it goes through torch.cuda.init() again, which refuses it
os.register_at_fork(after_in_child=_forget_current)


def _stream():
    """Handle of torch's current stream on the current device, looked up on every call.

    torch.cuda.current_stream() builds a Stream object on the way: 2.6 us, where the raw lookup takes 0.2.
    That was a third of a call of one launch (tweo_quantize_i8 7.2 us) and what bounded the small calls:
    quantise + linear at M = 1 takes the GPU less time than the host took to issue it.
    """
    global _current
    if _current is None:
        import torch
        torch.cuda.init()
        _current = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    return _current[1](_current[0]())


def _check(status, where):
    if status != TWEO_OK:
        raise TweoError(status, where)


@functools.lru_cache(maxsize=64)
def _pen_cfg(tau, eps, p):  # by value; the library only reads it
    return ctypes.byref(PenaltyCfg(tau, eps, p))


def _pen(pen):
    if pen is None:
        return None
    tau, eps, p = pen
    return _pen_cfg(float(tau), float(eps), int(p))


def _ws(workspace):
    if workspace is None:
        return None, 0
    return workspace.data_ptr(), workspace.nbytes


def tweo_workspace_bytes(op, M, N, K):
    return int(load().tweo_workspace_bytes(int(op), int(M), int(N), int(K)))


def tweo_set_gemm_tile(variant):
    _check(load().tweo_set_gemm_tile(int(variant)), "tweo_set_gemm_tile")


def tweo_set_stream_k(on):
    _check(load().tweo_set_stream_k(1 if on else 0), "tweo_set_stream_k")


def tweo_gemm_plan(op, M, N, K, p=0, residual=False, workspace_bytes=0):
    """(kernel variant, runs of the contraction, both gradients in one launch) of an FP8 call of these sizes.  The gated feed-forward's product:
    N = F, residual: both projections are kept."""
    plan = GemmPlan()
    _check(load().tweo_gemm_plan(op, M, N, K, p, 1 if residual else 0, workspace_bytes, ctypes.byref(plan)), "tweo_gemm_plan")
    return plan.kernel, plan.runs, bool(plan.shared)


def tweo_amax_quantize_f8(x_bf16, amax_out, q, qT, scale_out, scale_inv_out, workspace, e5m2=False):
    rows, cols = x_bf16.shape
    wp, wb = _ws(workspace)
    _check(load().tweo_amax_quantize_f8(_ptr(x_bf16), rows, cols, 1 if e5m2 else 0, _ptr(amax_out), _ptr(q), _ptr(qT),
                                        _ptr(scale_out), _ptr(scale_inv_out), wp, wb, _stream()),
           "tweo_amax_quantize_f8")


def tweo_set_fused_cast(on):
    _check(load().tweo_set_fused_cast(1 if on else 0), "tweo_set_fused_cast")


def tweo_fused_cast_timeouts():
    c = ctypes.c_uint(0)
    _check(load().tweo_fused_cast_timeouts(ctypes.byref(c)), "tweo_fused_cast_timeouts")
    return int(c.value)


def tweo_profile_gemm_launches(events):
    """events: flat list of hipEvent_t handles (ints), start/stop per upcoming GEMM kernel launch."""
    n = len(events)
    arr = (ctypes.c_void_p * max(n, 1))(*[ctypes.c_void_p(int(e)) for e in events])
    _check(load().tweo_profile_gemm_launches(arr, n // 2), "tweo_profile_gemm_launches")


def tweo_penalty_grad_inject(dy_bf16, a_bf16, pen, g, out_bf16):
    cfg = PenaltyCfg(float(pen[0]), float(pen[1]), int(pen[2]))
    _check(load().tweo_penalty_grad_inject(_ptr(dy_bf16), _ptr(a_bf16), dy_bf16.numel(), ctypes.byref(cfg),
                                           float(g), _ptr(out_bf16), _stream()), "tweo_penalty_grad_inject")


DELAYED_STATE_WORDS, DELAYED_NEXT_SCALE, DELAYED_USED_SCALE, DELAYED_USED_SCALE_INV = 32, 17, 21, 22


def tweo_delayed_state_bytes():
    return int(load().tweo_delayed_state_bytes())


def tweo_delayed_state_init(state):
    _check(load().tweo_delayed_state_init(_ptr(state), _stream()), "tweo_delayed_state_init")


def tweo_quantize_e4m3_delayed(x_bf16, state, q, qT=None, bootstrap=False):
    rows, cols = x_bf16.shape
    _check(load().tweo_quantize_e4m3_delayed(_ptr(x_bf16), rows, cols, _ptr(state), 1 if bootstrap else 0,
                                             _ptr(q), _ptr(qT), _stream()), "tweo_quantize_e4m3_delayed")


def tweo_quantize_e5m2_delayed(x_bf16, state, q, qT=None, bootstrap=False):
    rows, cols = x_bf16.shape
    _check(load().tweo_quantize_e5m2_delayed(_ptr(x_bf16), rows, cols, _ptr(state), 1 if bootstrap else 0,
                                             _ptr(q), _ptr(qT), _stream()), "tweo_quantize_e5m2_delayed")


def tweo_amax(x_bf16, amax_out):
    _check(load().tweo_amax(_ptr(x_bf16), x_bf16.numel(), _ptr(amax_out), _stream()), "tweo_amax")


def tweo_quantize_e4m3(x_bf16, amax, q, qT=None, scale_out=None, scale_inv_out=None):
    rows, cols = x_bf16.shape
    _check(load().tweo_quantize_e4m3(_ptr(x_bf16), rows, cols, _ptr(amax), _ptr(q), _ptr(qT),
                                     _ptr(scale_out), _ptr(scale_inv_out), _stream()),
           "tweo_quantize_e4m3")


def tweo_quantize_e5m2(x_bf16, amax, q, qT=None, scale_out=None, scale_inv_out=None):
    rows, cols = x_bf16.shape
    _check(load().tweo_quantize_e5m2(_ptr(x_bf16), rows, cols, _ptr(amax), _ptr(q), _ptr(qT),
                                     _ptr(scale_out), _ptr(scale_inv_out), _stream()),
           "tweo_quantize_e5m2")


def tweo_fp8_linear_fwd(xq, sx_inv, wq, sw_inv, y_bf16, residual_bf16=None, pen=None,
                        penalty_sum=None, workspace=None):
    M, K = xq.shape
    N = wq.shape[0]
    wp, wb = _ws(workspace)
    _check(load().tweo_fp8_linear_fwd(_ptr(xq), _ptr(sx_inv), _ptr(wq), _ptr(sw_inv),
                                      _ptr(residual_bf16), M, N, K, _ptr(y_bf16), _pen(pen),
                                      _ptr(penalty_sum), wp, wb, _stream()), "tweo_fp8_linear_fwd")


def tweo_layernorm_quantize_e4m3(x_bf16, gamma_bf16, q, workspace, beta_bf16=None, residual_bf16=None, eps=1e-5,
                                 h_out_bf16=None, y_out_bf16=None, amax_out=None, qT=None, scale_out=None,
                                 scale_inv_out=None):
    rows, cols = x_bf16.shape
    wp, wb = _ws(workspace)
    _check(load().tweo_layernorm_quantize_e4m3(_ptr(x_bf16), _ptr(residual_bf16), _ptr(gamma_bf16), _ptr(beta_bf16),
                                               rows, cols, float(eps), _ptr(h_out_bf16), _ptr(y_out_bf16),
                                               _ptr(amax_out), _ptr(q), _ptr(qT), _ptr(scale_out),
                                               _ptr(scale_inv_out), wp, wb, _stream()),
           "tweo_layernorm_quantize_e4m3")


def tweo_layernorm_quantize_e4m3_delayed(x_bf16, gamma_bf16, state, q, workspace, bootstrap=False, beta_bf16=None,
                                         residual_bf16=None, eps=1e-5, h_out_bf16=None, y_out_bf16=None, qT=None):
    rows, cols = x_bf16.shape
    wp, wb = _ws(workspace)
    _check(load().tweo_layernorm_quantize_e4m3_delayed(_ptr(x_bf16), _ptr(residual_bf16), _ptr(gamma_bf16),
                                                       _ptr(beta_bf16), rows, cols, float(eps), _ptr(state),
                                                       1 if bootstrap else 0, _ptr(h_out_bf16), _ptr(y_out_bf16),
                                                       _ptr(q), _ptr(qT), wp, wb, _stream()),
           "tweo_layernorm_quantize_e4m3_delayed")


def tweo_fp8_linear_fwd_bf16_delayed(x_bf16, w_bf16, y_bf16, saved, state_x, state_w, bootstrap=False,
                                     residual_bf16=None, pen=None, penalty_sum=None, workspace=None):
    M, K = x_bf16.shape
    N = w_bf16.shape[0]
    wp, wb = _ws(workspace)
    _check(load().tweo_fp8_linear_fwd_bf16_delayed(_ptr(x_bf16), _ptr(w_bf16), _ptr(residual_bf16), M, N, K,
                                                   _ptr(y_bf16), _pen(pen), _ptr(penalty_sum), ctypes.byref(saved),
                                                   _ptr(state_x), _ptr(state_w), 1 if bootstrap else 0, wp, wb,
                                                   _stream()), "tweo_fp8_linear_fwd_bf16_delayed")


def tweo_fp8_linear_bwd_bf16_delayed(dy_bf16, saved, state_dy, K, dyq, dyqT, dx_bf16=None, dw_bf16=None,
                                     workspace=None, bootstrap=False, dy_e5m2=False):
    M, N = dy_bf16.shape
    wp, wb = _ws(workspace)
    _check(load().tweo_fp8_linear_bwd_bf16_delayed(_ptr(dy_bf16), ctypes.byref(saved), _ptr(state_dy),
                                                   1 if bootstrap else 0, 1 if dy_e5m2 else 0, M, N, K, _ptr(dyq),
                                                   _ptr(dyqT), _ptr(dx_bf16), _ptr(dw_bf16), wp, wb, _stream()),
           "tweo_fp8_linear_bwd_bf16_delayed")


def tweo_static_scratch_bytes():
    return int(load().tweo_static_scratch_bytes())


def tweo_fp8_linear_fwd_static(xq, sx_inv, wq, sw_inv, y_bf16, residual_bf16=None, pen=None, penalty_sum=None):
    M, K = xq.shape
    N = wq.shape[0]
    _check(load().tweo_fp8_linear_fwd_static(_ptr(xq), _ptr(sx_inv), _ptr(wq), _ptr(sw_inv),
                                             _ptr(residual_bf16), M, N, K, _ptr(y_bf16), _pen(pen),
                                             _ptr(penalty_sum), _stream()), "tweo_fp8_linear_fwd_static")


def tweo_fp8_linear_bwd(dyq, dyqT, sdy_inv, wqT, sw_inv, xqT, sx_inv, M, N, K, dx_bf16=None,
                        dw_bf16=None, workspace=None):
    wp, wb = _ws(workspace)
    _check(load().tweo_fp8_linear_bwd(_ptr(dyq), _ptr(dyqT), _ptr(sdy_inv), _ptr(wqT), _ptr(sw_inv),
                                      _ptr(xqT), _ptr(sx_inv), M, N, K, _ptr(dx_bf16), _ptr(dw_bf16),
                                      wp, wb, _stream()), "tweo_fp8_linear_bwd")


def tweo_fp8_linear_bwd_hybrid(dyq, dyqT, sdy_inv, wqT, sw_inv, xqT, sx_inv, M, N, K, dx_bf16=None,
                               dw_bf16=None, workspace=None):
    wp, wb = _ws(workspace)
    _check(load().tweo_fp8_linear_bwd_hybrid(_ptr(dyq), _ptr(dyqT), _ptr(sdy_inv), _ptr(wqT), _ptr(sw_inv),
                                             _ptr(xqT), _ptr(sx_inv), M, N, K, _ptr(dx_bf16), _ptr(dw_bf16),
                                             wp, wb, _stream()), "tweo_fp8_linear_bwd_hybrid")


def tweo_quantize_i8(x_bf16, inv_step, out):
    _check(load().tweo_quantize_i8(_ptr(x_bf16), x_bf16.numel(), float(inv_step), _ptr(out),
                                   _stream()), "tweo_quantize_i8")


def tweo_w8a8_linear(xq, wq, alpha, y_bf16, workspace=None):
    M, K = xq.shape
    N = wq.shape[0]
    wp, wb = _ws(workspace)
    _check(load().tweo_w8a8_linear(_ptr(xq), _ptr(wq), M, N, K, float(alpha), _ptr(y_bf16), wp, wb,
                                   _stream()), "tweo_w8a8_linear")


def tweo_quantize_i8_rows(x_bf16, eps, q, step_out):
    rows, cols = x_bf16.shape
    _check(load().tweo_quantize_i8_rows(_ptr(x_bf16), rows, cols, float(eps), _ptr(q), _ptr(step_out),
                                        _stream()), "tweo_quantize_i8_rows")


def tweo_w8a8_linear_scaled(xq, wq, x_step, w_step, y_bf16):
    """x_step holds M steps (per token) or 1 (per tensor); w_step N (per channel) or 1."""
    M, K = xq.shape
    N = wq.shape[0]
    if x_step.numel() not in (1, M) or w_step.numel() not in (1, N):
        raise ValueError("step vectors must have 1 or M / N elements")
    _check(load().tweo_w8a8_linear_scaled(_ptr(xq), _ptr(wq), M, N, K, _ptr(x_step),
                                          1 if x_step.numel() > 1 else 0,
                                          _ptr(w_step), 1 if w_step.numel() > 1 else 0, _ptr(y_bf16),
                                          _stream()), "tweo_w8a8_linear_scaled")


def tweo_w8a8_linear_scaled_i8out(xq, wq, x_step, w_step, inv_step_out, yq):
    """INT8 result with the static step 1 / inv_step_out * 127 (quantised residual stream)."""
    M, K = xq.shape
    N = wq.shape[0]
    if x_step.numel() not in (1, M) or w_step.numel() not in (1, N):
        raise ValueError("step vectors must have 1 or M / N elements")
    _check(load().tweo_w8a8_linear_scaled_i8out(_ptr(xq), _ptr(wq), M, N, K, _ptr(x_step),
                                                1 if x_step.numel() > 1 else 0, _ptr(w_step),
                                                1 if w_step.numel() > 1 else 0, float(inv_step_out), _ptr(yq),
                                                _stream()), "tweo_w8a8_linear_scaled_i8out")


def make_saved(xq, xqT, wq, wqT, scalars):
    return Fp8Saved(xq.data_ptr(), xqT.data_ptr(), wq.data_ptr(), wqT.data_ptr(), scalars.data_ptr())


def tweo_fp8_linear_fwd_bf16(x_bf16, w_bf16, y_bf16, saved, residual_bf16=None, pen=None,
                             penalty_sum=None, workspace=None):
    M, K = x_bf16.shape
    N = w_bf16.shape[0]
    wp, wb = _ws(workspace)
    _check(load().tweo_fp8_linear_fwd_bf16(_ptr(x_bf16), _ptr(w_bf16), _ptr(residual_bf16), M, N, K,
                                           _ptr(y_bf16), _pen(pen), _ptr(penalty_sum),
                                           ctypes.byref(saved), wp, wb, _stream()),
           "tweo_fp8_linear_fwd_bf16")


def tweo_fp8_linear_bwd_bf16(dy_bf16, saved, K, dyq, dyqT, dx_bf16=None, dw_bf16=None,
                             workspace=None):
    M, N = dy_bf16.shape
    wp, wb = _ws(workspace)
    _check(load().tweo_fp8_linear_bwd_bf16(_ptr(dy_bf16), ctypes.byref(saved), M, N, K, _ptr(dyq),
                                           _ptr(dyqT), _ptr(dx_bf16), _ptr(dw_bf16), wp, wb,
                                           _stream()), "tweo_fp8_linear_bwd_bf16")


def tweo_fp8_linear_bwd_bf16_inject(dy_bf16, a_bf16, pen, g, saved, K, dyq, dyqT, dx_bf16=None, dw_bf16=None,
                                    workspace=None, dy_e5m2=False):
    M, N = dy_bf16.shape
    wp, wb = _ws(workspace)
    cfg = PenaltyCfg(float(pen[0]), float(pen[1]), int(pen[2]))
    _check(load().tweo_fp8_linear_bwd_bf16_inject(_ptr(dy_bf16), _ptr(a_bf16), ctypes.byref(cfg), float(g),
                                                  1 if dy_e5m2 else 0, ctypes.byref(saved), M, N, K, _ptr(dyq),
                                                  _ptr(dyqT), _ptr(dx_bf16), _ptr(dw_bf16), wp, wb, _stream()),
           "tweo_fp8_linear_bwd_bf16_inject")


def tweo_fp8_linear_bwd_bf16_hybrid(dy_bf16, saved, K, dyq, dyqT, dx_bf16=None, dw_bf16=None,
                                    workspace=None):
    M, N = dy_bf16.shape
    wp, wb = _ws(workspace)
    _check(load().tweo_fp8_linear_bwd_bf16_hybrid(_ptr(dy_bf16), ctypes.byref(saved), M, N, K, _ptr(dyq),
                                                  _ptr(dyqT), _ptr(dx_bf16), _ptr(dw_bf16), wp, wb,
                                                  _stream()), "tweo_fp8_linear_bwd_bf16_hybrid")


def _device():
    """The current device.  (As _stream: three looks at it and the stream by way of torch.cuda are what a small call takes.)"""
    if _current is None:
        _stream()
    return _current[0]()


def _same(device, shape, dtype, tensors, names):
    """Refuses what a kernel would read as something else: another shape or type, strides, another device than the current one.
    0.3 us a tensor."""
    for i, t in enumerate(tensors):
        if t is not None and (t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != device):
            raise ValueError("%s: a contiguous %s tensor of shape %s on cuda:%d, the current device, is needed, got %s of %s on %s" %
                             (names[i], dtype, tuple(shape), device, t.dtype, tuple(t.shape), t.device))


@functools.lru_cache(maxsize=1)
def _types():
    import torch
    return torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.uint32, torch.int64


def _scratch(device, t, name):
    """Address and bytes of a workspace or table, which has to lie in one piece on the current device."""
    if t is not None and (t.get_device() != device or not t.is_contiguous()):
        raise ValueError("%s: a contiguous tensor on cuda:%d, the current device, is needed, got strides %s on %s" % (name, device, t.stride(), t.device))
    return _ws(t)


_LN_FWD, _LN_FWD_PARAMS, _LN_STATS = ("x_bf16", "y_bf16", "residual_bf16", "h_out_bf16"), ("gamma_bf16", "beta_bf16"), ("stats",)
_LN_BWD, _LN_BWD_SUMS = ("dy_bf16", "h_bf16", "dx_bf16", "residual_grad_bf16"), ("dgamma", "dbeta")


def tweo_layernorm_fwd(x_bf16, gamma_bf16, y_bf16, beta_bf16=None, residual_bf16=None, eps=1e-5, h_out_bf16=None,
                       stats_out=None):
    shape = x_bf16.shape
    if len(shape) != 2:
        raise ValueError("x_bf16: two dimensions are needed")
    rows, cols = shape
    dev, (bf16, _, f64) = _device(), _types()[:3]
    if residual_bf16 is None:
        _same(dev, shape, bf16, (x_bf16, y_bf16), _LN_FWD)
    else:
        _same(dev, shape, bf16, (x_bf16, y_bf16, residual_bf16, h_out_bf16), _LN_FWD)
    _same(dev, shape[1:], bf16, (gamma_bf16, beta_bf16), _LN_FWD_PARAMS)
    if stats_out is not None:
        _same(dev, (rows, 2), f64, (stats_out,), _LN_STATS)
    _check(load().tweo_layernorm_fwd(_ptr(x_bf16), _ptr(residual_bf16), _ptr(gamma_bf16), _ptr(beta_bf16), rows, cols,
                                     float(eps), _ptr(h_out_bf16), _ptr(y_bf16), _ptr(stats_out), _stream()),
           "tweo_layernorm_fwd")


LAYERNORM_STATS_OFFSET = 2304  # TWEO_LAYERNORM_STATS_OFFSET


def layernorm_stats(workspace, rows):
    """The row statistics (mean, 1 / sqrt(var + eps)), fp64 [rows, 2], that a LayerNorm -> cast call left in its workspace, a contiguous
    tensor of any type."""
    import torch
    end = LAYERNORM_STATS_OFFSET + 16 * rows
    if rows < 1 or not workspace.is_contiguous() or workspace.nbytes < end:
        raise ValueError("the workspace of a LayerNorm -> cast of %d rows has at least %d contiguous bytes, got %d of strides %s" %
                         (rows, end, workspace.nbytes, workspace.stride()))
    return workspace.view(-1).view(torch.uint8)[LAYERNORM_STATS_OFFSET:end].view(torch.float64).view(rows, 2)


def tweo_layernorm_bwd(dy_bf16, h_bf16, gamma_bf16, stats, dx_bf16, dgamma, dbeta=None, residual_grad_bf16=None,
                       workspace=None):
    shape = dy_bf16.shape
    if len(shape) != 2:
        raise ValueError("dy_bf16: two dimensions are needed")
    rows, cols = shape
    dev, (bf16, f32, f64) = _device(), _types()[:3]
    _same(dev, shape, bf16, (dy_bf16, h_bf16, dx_bf16, residual_grad_bf16), _LN_BWD)
    _same(dev, shape[1:], bf16, (gamma_bf16,), _LN_FWD_PARAMS)
    _same(dev, shape[1:], f32, (dgamma, dbeta), _LN_BWD_SUMS)
    _same(dev, (rows, 2), f64, (stats,), _LN_STATS)
    wp, wb = _scratch(dev, workspace, "workspace")
    _check(load().tweo_layernorm_bwd(_ptr(dy_bf16), _ptr(h_bf16), _ptr(gamma_bf16), _ptr(stats), _ptr(residual_grad_bf16),
                                     rows, cols, _ptr(dx_bf16), _ptr(dgamma), _ptr(dbeta), wp, wb, _stream()),
           "tweo_layernorm_bwd")


def optim_tensor(grad, param=None, m=None, v=None, m_step=None, v_step=None, master=None, weight_decay=0.0):
    """One row of an optimizer's table, checked: grad (bf16 or fp32) alone for the norm, else with param, m and v of as many
    elements (uint8 codes with their steps, or fp32) and, for a bf16 param, its fp32 copy if there is one."""
    import torch
    floats, n, dev = (torch.bfloat16, torch.float32), grad.numel(), grad.get_device()
    eight = m_step is not None or v_step is not None
    state = torch.uint8 if eight else torch.float32
    for name, t, kinds, numel in (("grad", grad, floats, n), ("param", param, floats, n), ("master", master, floats[1:], n),
                                  ("m", m, (state,), n), ("v", v, (state,), n), ("m_step", m_step, floats[1:], -(-n // 256)),
                                  ("v_step", v_step, floats[1:], -(-n // 256))):
        if t is not None and (t.dtype not in kinds or t.numel() != numel or not t.is_contiguous() or t.get_device() != dev):
            raise ValueError("%s: a contiguous tensor of %d elements of %s on the gradient's device is needed, got %s of %s on %s" %
                             (name, numel, " or ".join(map(str, kinds)), t.dtype, tuple(t.shape), t.device))
    row = OptimTensor(_ptr(param), _ptr(master), _ptr(grad), _ptr(m), _ptr(v), _ptr(m_step), _ptr(v_step), n, float(weight_decay),
                      int(param is not None and param.dtype is torch.float32), int(grad.dtype is torch.float32))
    row.tensors = [t for t in (param, master, grad, m, v, m_step, v_step) if t is not None]
    return row


def tweo_optim_table_bytes(count):
    return int(load().tweo_optim_table_bytes(int(count)))


def make_optim_plan(rows, table):
    """The plan of tweo_grad_sumsq and tweo_adamw_step over `rows` (optim_tensor), whose table is written into `table`, a uint8
    tensor of tweo_optim_table_bytes(len(rows)), on the current stream.  Keeps the tensors alive."""
    dev = _device()
    for t in [table] + [t for r in rows for t in r.tensors]:
        if t.get_device() != dev:
            raise ValueError("a tensor on %s, but cuda:%d is current" % (t.device, dev))
    plan = OptimPlan()
    wp, wb = _scratch(dev, table, "table")
    _check(load().tweo_optim_plan_init((OptimTensor * len(rows))(*rows), len(rows), wp, wb, ctypes.byref(plan), _stream()),
           "tweo_optim_plan_init")
    plan.device, plan.tensors = dev, [table] + [t for r in rows for t in r.tensors]
    return plan


def _on_device(plan, sumsq):
    dev = _device()
    if dev != plan.device:
        raise ValueError("a plan of cuda:%d, but cuda:%d is current" % (plan.device, dev))
    if sumsq is not None and (sumsq.dtype is not _types()[2] or sumsq.numel() < 1 or sumsq.get_device() != dev):
        raise ValueError("the sum of squares: one torch.float64 on cuda:%d is needed, got %s on %s" % (dev, sumsq.dtype, sumsq.device))
    return dev


def tweo_grad_sumsq(plan, sumsq_out, workspace):
    wp, wb = _scratch(_on_device(plan, sumsq_out), workspace, "workspace")
    _check(load().tweo_grad_sumsq(ctypes.byref(plan), _ptr(sumsq_out), wp, wb, _stream()), "tweo_grad_sumsq")


def tweo_adamw_step(plan, lr=None, step=None, beta1=0.9, beta2=0.999, eps=1e-8, grad_sumsq=None, max_norm=1.0, schedule=None):
    """lr and step, or schedule: a torch.int32 (or uint32) tensor of two words on the device, the bits of lr as fp32 and step
    (schedule[:1].view(torch.float32).fill_(lr); schedule[1:].fill_(step))."""
    dev = _on_device(plan, grad_sumsq)
    if schedule is not None and (schedule.dtype not in _types()[3:5] or schedule.numel() < 2 or not schedule.is_contiguous() or schedule.get_device() != dev):
        raise ValueError("schedule: two contiguous 32-bit integers on cuda:%d are needed, got %d of %s, strides %s, on %s" %
                         (dev, schedule.numel(), schedule.dtype, schedule.stride(), schedule.device))
    if schedule is None:
        if lr is None or step is None:
            raise ValueError("lr and step are needed without a schedule")
        cfg = AdamwCfg(lr, beta1, beta2, eps, max_norm, step)
    else:
        cfg = AdamwCfg(0.0, beta1, beta2, eps, max_norm, 1)
    _check(load().tweo_adamw_step(ctypes.byref(plan), ctypes.byref(cfg), _ptr(grad_sumsq), _ptr(schedule), _stream()),
           "tweo_adamw_step")


ROTARY_LAYOUTS = {"halves": 0, "pairs": 1}  # TWEO_ROTARY_HALVES, TWEO_ROTARY_PAIRS
ROTARY_FREQS = {"plain": 0, "linear": 1, "base": 2, "turns": 3}  # TWEO_ROTARY_FREQS_*


def tweo_rotary_freqs(rot_dim, base=10000.0, kind="plain", factor=1.0, context=0.0, low_turns=0.0, high_turns=0.0):
    """The frequencies of rot_dim / 2 pairs, radians a position: a torch.float64 tensor on the CPU, to be moved to the GPU once."""
    import torch
    if kind not in ROTARY_FREQS:
        raise ValueError("kind: one of %s is needed, got %r" % (", ".join(ROTARY_FREQS), kind))
    freqs = torch.empty(max(1, rot_dim // 2), dtype=torch.float64)
    cfg = RotaryFreqCfg(base, ROTARY_FREQS[kind], factor, context, low_turns, high_turns)
    _check(load().tweo_rotary_freqs(ctypes.byref(cfg), rot_dim, freqs.data_ptr()), "tweo_rotary_freqs")
    return freqs


def _heads(device, shape, tensors, names):
    """Strides of heads, [tokens, heads, dim] of bf16 on the current device with a contiguous last index; refuses others."""
    bf16, strides = _types()[0], []
    for t in tensors:
        token, head, last = t.stride() if t.dim() == 3 else (0, 0, 0)
        if t.dtype is not bf16 or t.shape != shape or last != 1 and shape[2] != 1 or t.get_device() != device:
            i = [u is t for u in tensors].index(True)
            raise ValueError("%s: a %s tensor of shape %s on cuda:%d, the current device, with a contiguous last index is needed, got %s of %s, strides %s, on %s" %
                             (names[i], bf16, tuple(shape), device, t.dtype, tuple(t.shape), t.stride(), t.device))
        strides.append(token)
        strides.append(head)
    return strides


def _rotary(device, tokens, positions, freqs, layout, scale):
    """The rotation (a tweo_rotary_cfg), or None where there is none."""
    if positions is None and freqs is None:
        return None
    _, _, f64, _, _, i64 = _types()
    if (positions is None or freqs is None or positions.dtype is not i64 or positions.shape != (tokens,) or freqs.dtype is not f64 or
            positions.get_device() != device or freqs.get_device() != device or not positions.is_contiguous() or freqs.dim() != 1 or
            not freqs.is_contiguous()):
        raise ValueError("positions and freqs: contiguous vectors on cuda:%d, the current device, are needed, %d of %s and rot_dim / 2 of %s, got %s" %
                         (device, tokens, i64, f64, " and ".join("None" if t is None else "%s of %s on %s" % (tuple(t.shape), t.dtype, t.device)
                                                                 for t in (positions, freqs))))
    if layout not in ROTARY_LAYOUTS:
        raise ValueError("layout: halves or pairs is needed, got %r" % (layout,))
    return _ROTARY_CFG.pack(positions.data_ptr(), freqs.data_ptr(), 2 * freqs.numel(), ROTARY_LAYOUTS[layout], scale)


# tweo_rotary_cfg; one and two of tweo_heads and of tweo_heads_grad.  Packed bytes in the place of ctypes structures: two groups' fields, set one by
# one, took 5 of the 14 us that issuing a rotation took.
_ROTARY_CFG = struct.Struct("PPiif4x")
_ROWS, _GRAD_ROWS = ([struct.Struct(row * n) for n in range(3)] for row in ("PPqqqqPi4x", "PPPqqqqqqPPi4x"))


def _shape(groups, width):
    """Shapes of one or two groups' heads, of the same tokens and dim."""
    if len(groups) == 1 and len(groups[0]) == width:
        shapes = (groups[0][0].shape,)
        if len(shapes[0]) == 3:
            return shapes
    elif len(groups) == 2 and len(groups[0]) == len(groups[1]) == width:
        shapes = a, b = groups[0][0].shape, groups[1][0].shape
        if len(a) == len(b) == 3 and a[0] == b[0] and a[2] == b[2]:
            return shapes
    raise ValueError("one or two groups of %d tensors, the heads [tokens, heads, dim] of the same tokens and dim, are needed, got %s" %
                     (width, ", ".join("%d, %s" % (len(g), tuple(g[0].shape)) for g in groups) or "none"))


_HEADS, _HEADS_GRAD, _GAIN, _DGAIN = ("x", "y"), ("dy", "x", "dx"), ("gain",), ("dgain",)


def tweo_rotary(groups, positions, freqs, layout="halves", scale=1.0, transpose=False):
    """groups: one or two (x, y), bf16 [tokens, heads, dim] of any token and head stride; y may be x.  positions: int64 [tokens], negative:
    padding.  freqs: float64 [rot_dim / 2] (tweo_rotary_freqs)."""
    shapes, dev = _shape(groups, 2), _device()
    tokens, _, dim = shapes[0]
    cfg = _rotary(dev, tokens, positions, freqs, layout, scale)
    if cfg is None:
        raise ValueError("positions and freqs are needed")
    fields = []
    for shape, (x, y) in zip(shapes, groups):
        fields += (x.data_ptr(), y.data_ptr(), *_heads(dev, shape, (x, y), _HEADS), 0, shape[1])
    _check(load().tweo_rotary(_ROWS[len(groups)].pack(*fields), len(groups), tokens, dim, cfg, 1 if transpose else 0, _stream()), "tweo_rotary")


def tweo_head_norm_rotary_fwd(groups, positions=None, freqs=None, layout="halves", scale=1.0, eps=1e-6):
    """groups: one or two (x, gain, y); x and y as in tweo_rotary, gain bf16 [dim] or None.  Without positions and freqs the norm alone."""
    shapes, dev, bf16 = _shape(groups, 3), _device(), _types()[0]
    tokens, _, dim = shapes[0]
    cfg = _rotary(dev, tokens, positions, freqs, layout, scale)
    fields = []
    for shape, (x, gain, y) in zip(shapes, groups):
        if gain is not None:
            _same(dev, (dim,), bf16, (gain,), _GAIN)
        fields += (x.data_ptr(), y.data_ptr(), *_heads(dev, shape, (x, y), _HEADS), 0 if gain is None else gain.data_ptr(), shape[1])
    _check(load().tweo_head_norm_rotary_fwd(_ROWS[len(groups)].pack(*fields), len(groups), tokens, dim, eps, cfg, _stream()), "tweo_head_norm_rotary_fwd")


def tweo_head_norm_rotary_bwd(groups, positions=None, freqs=None, layout="halves", scale=1.0, eps=1e-6, workspace=None):
    """groups: one or two (dy, x, gain, dx, dgain): the gradient of the forward's y, its x and gain, where the gradient of x goes (dy or x
    itself, or another) and that of gain (float32 [dim], or None)."""
    shapes, dev, (bf16, f32) = _shape(groups, 5), _device(), _types()[:2]
    tokens, _, dim = shapes[0]
    cfg = _rotary(dev, tokens, positions, freqs, layout, scale)
    fields = []
    for shape, (dy, x, gain, dx, dgain) in zip(shapes, groups):
        if gain is not None:
            _same(dev, (dim,), bf16, (gain,), _GAIN)
        if dgain is not None:
            _same(dev, (dim,), f32, (dgain,), _DGAIN)
        fields += (dy.data_ptr(), x.data_ptr(), dx.data_ptr(), *_heads(dev, shape, (dy, x, dx), _HEADS_GRAD), 0 if gain is None else gain.data_ptr(),
                   0 if dgain is None else dgain.data_ptr(), shape[1])
    wp, wb = _scratch(dev, workspace, "workspace")
    _check(load().tweo_head_norm_rotary_bwd(_GRAD_ROWS[len(groups)].pack(*fields), len(groups), tokens, dim, eps, cfg, wp, wb, _stream()),
           "tweo_head_norm_rotary_bwd")


ACTS = {"silu": 0, "gelu": 1}  # TWEO_ACT_SILU, TWEO_ACT_GELU


def _act(act):
    if act not in ACTS:
        raise ValueError("act: silu or gelu is needed, got %r" % (act,))
    return ACTS[act]


def _gated_shape(x, w, names):
    """M, F, K of [M, K] and [2F, K]."""
    a, b = x.shape, w.shape
    if len(a) != 2 or len(b) != 2 or a[1] != b[1] or b[0] % 2 != 0:
        raise ValueError("%s, %s: [M, K] and [2F, K] are needed, got %s and %s" % (names + (tuple(a), tuple(b))))
    return a[0], b[0] // 2, a[1]


@functools.lru_cache(maxsize=1)
def _bytes_types():
    import torch
    return torch.uint8, torch.int8


def _scalar(device, t, name):
    if t.dtype is not _types()[1] or t.numel() < 1 or t.get_device() != device:
        raise ValueError("%s: one torch.float32 on cuda:%d, the current device, is needed, got %s on %s" % (name, device, t.dtype, t.device))


def _state(device, t, name):
    """A delayed-scaling state."""
    if t is not None and (t.nbytes < 4 * DELAYED_STATE_WORDS or not t.is_contiguous() or t.get_device() != device):
        raise ValueError("%s: %d contiguous bytes on cuda:%d, the current device, are needed, got %d on %s" %
                         (name, 4 * DELAYED_STATE_WORDS, device, t.nbytes, t.device))


_XQ, _WQ, _HB, _GU, _XB, _WB, _DGUQ, _DGUQT, _HQ = (("xq",), ("wq",), ("h_bf16",), ("gu_bf16",), ("x_bf16",), ("w_bf16",), ("dguq",), ("dguqT",), ("hq",))


def tweo_fp8_gated_fwd(xq, sx_inv, wq, sw_inv, h_bf16, gu_bf16=None, act="silu"):
    """wq [2F, K]: the gate's rows, then the up projection's.  gu_bf16 [M, 2F]: both projections, for the backward pass."""
    M, F, K = _gated_shape(xq, wq, ("xq", "wq"))
    dev, u8, bf16 = _device(), _bytes_types()[0], _types()[0]
    _same(dev, (M, K), u8, (xq,), _XQ)
    _same(dev, (2 * F, K), u8, (wq,), _WQ)
    _same(dev, (M, F), bf16, (h_bf16,), _HB)
    if gu_bf16 is not None:
        _same(dev, (M, 2 * F), bf16, (gu_bf16,), _GU)
    _scalar(dev, sx_inv, "sx_inv")
    _scalar(dev, sw_inv, "sw_inv")
    _check(load().tweo_fp8_gated_fwd(_ptr(xq), _ptr(sx_inv), _ptr(wq), _ptr(sw_inv), M, F, K, _act(act), _ptr(h_bf16), _ptr(gu_bf16), _stream()),
           "tweo_fp8_gated_fwd")


def tweo_fp8_gated_fwd_bf16(x_bf16, w_bf16, h_bf16, gu_bf16, saved, act="silu", state_x=None, state_w=None, bootstrap=False, workspace=None):
    """saved: make_saved of xq [M, K], wq [2F, K] and their transposes.  gu_bf16 may be None.  state_x and state_w: delayed scaling."""
    M, F, K = _gated_shape(x_bf16, w_bf16, ("x_bf16", "w_bf16"))
    dev, bf16 = _device(), _types()[0]
    _same(dev, (M, K), bf16, (x_bf16,), _XB)
    _same(dev, (2 * F, K), bf16, (w_bf16,), _WB)
    _same(dev, (M, F), bf16, (h_bf16,), _HB)
    _same(dev, (M, 2 * F), bf16, (gu_bf16,), _GU)
    _state(dev, state_x, "state_x")
    _state(dev, state_w, "state_w")
    wp, wb = _scratch(dev, workspace, "workspace")
    _check(load().tweo_fp8_gated_fwd_bf16(_ptr(x_bf16), _ptr(w_bf16), M, F, K, _act(act), _ptr(h_bf16), _ptr(gu_bf16), ctypes.byref(saved),
                                          _ptr(state_x), _ptr(state_w), 1 if bootstrap else 0, wp, wb, _stream()), "tweo_fp8_gated_fwd_bf16")


def tweo_fp8_gated_bwd_bf16(dh_bf16, gu_bf16, saved, K, dguq, dguqT, dx_bf16=None, dw_bf16=None, act="silu", dy_e5m2=False, state_dgu=None,
                            bootstrap=False, workspace=None):
    """dguq [M, 2F], dguqT [2F, M]: the codes of both projections' gradients.  dx_bf16 [M, K], dw_bf16 [2F, K] or None."""
    if dh_bf16.dim() != 2:
        raise ValueError("dh_bf16: two dimensions are needed")
    M, F = dh_bf16.shape
    dev, u8, bf16 = _device(), _bytes_types()[0], _types()[0]
    _same(dev, (M, F), bf16, (dh_bf16,), ("dh_bf16",))
    _same(dev, (M, 2 * F), bf16, (gu_bf16,), _GU)
    _same(dev, (M, 2 * F), u8, (dguq,), _DGUQ)
    _same(dev, (2 * F, M), u8, (dguqT,), _DGUQT)
    _same(dev, (M, K), bf16, (dx_bf16,), ("dx_bf16",))
    _same(dev, (2 * F, K), bf16, (dw_bf16,), ("dw_bf16",))
    _state(dev, state_dgu, "state_dgu")
    wp, wb = _scratch(dev, workspace, "workspace")
    _check(load().tweo_fp8_gated_bwd_bf16(_ptr(dh_bf16), _ptr(gu_bf16), ctypes.byref(saved), M, F, K, _act(act), 1 if dy_e5m2 else 0, _ptr(state_dgu),
                                          1 if bootstrap else 0, _ptr(dguq), _ptr(dguqT), _ptr(dx_bf16), _ptr(dw_bf16), wp, wb, _stream()),
           "tweo_fp8_gated_bwd_bf16")


def _w8a8_gated(xq, wq, x_step, w_step, out, dtype, name):
    M, F, K = _gated_shape(xq, wq, ("xq", "wq"))
    dev, i8, f32 = _device(), _bytes_types()[1], _types()[1]
    _same(dev, (M, K), i8, (xq,), _XQ)
    _same(dev, (2 * F, K), i8, (wq,), _WQ)
    _same(dev, (M, F), dtype, (out,), name)
    for t, n, what in ((x_step, M, "x_step"), (w_step, 2 * F, "w_step")):
        if t.numel() not in (1, n) or t.dtype is not f32 or not t.is_contiguous() or t.get_device() != dev:
            raise ValueError("%s: 1 or %d contiguous torch.float32 on cuda:%d, the current device, are needed, got %d of %s on %s" %
                             (what, n, dev, t.numel(), t.dtype, t.device))
    return M, F, K


def tweo_w8a8_gated(xq, wq, x_step, w_step, h_bf16, act="silu"):
    """wq [2F, K]: the gate's rows, then the up projection's.  x_step holds M steps (per token) or 1; w_step 2F (per channel) or 1."""
    M, F, K = _w8a8_gated(xq, wq, x_step, w_step, h_bf16, _types()[0], _HB)
    _check(load().tweo_w8a8_gated(_ptr(xq), _ptr(wq), M, F, K, _ptr(x_step), 1 if x_step.numel() > 1 else 0, _ptr(w_step),
                                  1 if w_step.numel() > 1 else 0, _act(act), _ptr(h_bf16), _stream()), "tweo_w8a8_gated")


def tweo_w8a8_gated_i8out(xq, wq, x_step, w_step, inv_step_h, hq, act="silu"):
    """The same with an INT8 result under the static step 127 / inv_step_h, the input of the down projection."""
    M, F, K = _w8a8_gated(xq, wq, x_step, w_step, hq, _bytes_types()[1], _HQ)
    _check(load().tweo_w8a8_gated_i8out(_ptr(xq), _ptr(wq), M, F, K, _ptr(x_step), 1 if x_step.numel() > 1 else 0, _ptr(w_step),
                                        1 if w_step.numel() > 1 else 0, _act(act), float(inv_step_h), _ptr(hq), _stream()), "tweo_w8a8_gated_i8out")
