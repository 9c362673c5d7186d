"""ctypes binding with the same names as the C ABI (include/hts.h).  Argument marshalling only."""
from __future__ import annotations

import ctypes as C
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhts.so")

PRECISION_FP32, PRECISION_BF16 = 0, 1
ALGO_A2C, ALGO_PPO, ALGO_A2C_TIS = 0, 1, 2
OPT_ADAM, OPT_RMSPROP = 0, 1
ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU = 0, 1, 2, 3

EXPORTS = ["hts_param_count", "hts_create", "hts_destroy", "hts_act", "hts_sync_params", "hts_sample_from_logits", "hts_returns_gae",
           "hts_normalize_advantages", "hts_learner_step", "hts_learner_step_delayed", "hts_loss_and_grads", "hts_adam_apply", "hts_test_gemm",
           "hts_last_hip_error", "hts_strerror", "hts_profile_site_count", "hts_profile_site_name", "hts_profile_begin",
           "hts_profile_end", "hts_profile_overhead", "hts_profile_begin_sampled", "hts_adam_apply_static", "hts_track_params",
           "hts_stream_create_cu_range", "hts_stream_destroy", "hts_seq_create", "hts_seq_destroy", "hts_linear_workspace", "hts_linear",
           "hts_linear_backward", "hts_short_conv_workspace", "hts_short_conv", "hts_short_conv_backward", "hts_selective_scan_workspace",
           "hts_selective_scan_states", "hts_selective_scan", "hts_selective_scan_backward", "hts_layer_norm_workspace", "hts_layer_norm",
           "hts_layer_norm_backward", "hts_delta_rule_workspace", "hts_delta_rule_states", "hts_delta_rule", "hts_delta_rule_backward", "hts_adamw_create",
           "hts_adamw_destroy", "hts_adamw_step"]


class HtsError(RuntimeError):
    pass


class NetDesc(C.Structure):
    _fields_ = [("C", C.c_int32), ("H", C.c_int32), ("W", C.c_int32), ("A", C.c_int32), ("precision", C.c_int32)]


class Buffer(C.Structure):
    _fields_ = [("obs", C.c_void_p), ("actions", C.c_void_p), ("old_logp", C.c_void_p), ("old_values", C.c_void_p),
                ("advantages", C.c_void_p), ("returns", C.c_void_p), ("count", C.c_int32), ("index", C.c_void_p),
                ("B", C.c_int32)]


class HParams(C.Structure):
    _fields_ = [("algo", C.c_int32), ("clip_eps", C.c_float), ("vf_coef", C.c_float), ("ent_coef", C.c_float),
                ("max_grad_norm", C.c_float), ("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float),
                ("adam_eps", C.c_float), ("optimizer", C.c_int32), ("rms_alpha", C.c_float), ("rho_bar", C.c_float),
                ("value_clip", C.c_float)]

    def __init__(self, algo=ALGO_A2C, clip_eps=0.1, vf_coef=0.5, ent_coef=0.01, max_grad_norm=0.0, lr=7e-4,
                 beta1=0.9, beta2=0.999, adam_eps=1e-5, optimizer=OPT_ADAM, rms_alpha=0.99, rho_bar=1.0,
                 value_clip=0.0):
        super().__init__(algo, clip_eps, vf_coef, ent_coef, max_grad_norm, lr, beta1, beta2, adam_eps, optimizer,
                         rms_alpha, rho_bar, value_clip)


class _OptStateC(C.Structure):
    _fields_ = [("m", C.c_void_p), ("v", C.c_void_p), ("step", C.c_int64)]


class OptState:
    """Adam moments (device fp32 [P]) and the host-side count of completed updates."""

    def __init__(self, m: torch.Tensor, v: torch.Tensor, step: int = 0):
        self.m, self.v, self.step = m, v, step


class _Rows(C.Structure):
    _fields_ = [("p", C.c_void_p), ("ld", C.c_int64)]


class _Steps(C.Structure):
    _fields_ = [("p", C.c_void_p), ("st", C.c_int64), ("sn", C.c_int64)]


class _LinearDesc(C.Structure):
    _fields_ = [(f, C.c_int32) for f in ("M", "N", "K", "precision", "act")]


class _ConvDesc(C.Structure):
    _fields_ = [(f, C.c_int32) for f in ("T", "N", "D", "W", "precision", "act")]


class _ScanDesc(C.Structure):
    _fields_ = [(f, C.c_int32) for f in ("T", "N", "D", "S", "G", "precision", "softplus")]


class _ScanInputs(C.Structure):
    _fields_ = [("x", _Steps), ("dt", _Steps), ("B", _Steps), ("C", _Steps), ("z", _Steps), ("A", C.c_void_p), ("skip", C.c_void_p),
                ("dt_bias", C.c_void_p), ("starts", C.c_void_p), ("lengths", C.c_void_p), ("h_in", C.c_void_p)]


class _ScanGrads(C.Structure):
    _fields_ = [("dx", _Steps), ("ddt", _Steps), ("dB", _Steps), ("dC", _Steps), ("dz", _Steps), ("dA", C.c_void_p), ("dskip", C.c_void_p),
                ("ddt_bias", C.c_void_p), ("dh_in", C.c_void_p)]


class _NormDesc(C.Structure):
    _fields_ = [("M", C.c_int32), ("F", C.c_int32), ("precision", C.c_int32), ("eps", C.c_float)]


class _DeltaDesc(C.Structure):
    _fields_ = [(f, C.c_int32) for f in ("T", "N", "H", "G", "K", "V", "precision", "normalize", "softplus")] + [("scale", C.c_float)]


class _DeltaInputs(C.Structure):
    _fields_ = [("q", _Steps), ("k", _Steps), ("v", _Steps), ("a", _Steps), ("b", _Steps), ("A", C.c_void_p), ("a_bias", C.c_void_p), ("starts", C.c_void_p),
                ("lengths", C.c_void_p), ("h_in", C.c_void_p)]


class _DeltaGrads(C.Structure):
    _fields_ = [("dq", _Steps), ("dk", _Steps), ("dv", _Steps), ("da", _Steps), ("db", _Steps), ("dA", C.c_void_p), ("da_bias", C.c_void_p), ("dh_in", C.c_void_p)]


class _AdamWTensorC(C.Structure):
    _fields_ = [(f, C.c_void_p) for f in ("p", "g", "m", "v", "m_scale", "v_scale", "copy")] + [("n", C.c_int64), ("weight_decay", C.c_float), ("lr_scale", C.c_float),
                                                                                                 ("grad_precision", C.c_int32), ("bits", C.c_int32)]


class AdamWHParams(C.Structure):
    """hts_adamw_hparams."""
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float), ("max_grad_norm", C.c_float), ("reserved", C.c_int32), ("seed", C.c_uint64)]

    def __init__(self, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, max_grad_norm=0.0, seed=0):
        super().__init__(lr, beta1, beta2, eps, max_grad_norm, 0, seed)


STATS_FIELDS = ("policy_loss", "value_loss", "entropy", "grad_norm", "clip_frac", "approx_kl", "nonfinite")

_lib = None


def load_library():
    """Load libhts.so; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise HtsError(f"{LIB_PATH} not found: build it with `python -m paper_2012_09849_amd.build`")
        lib = C.CDLL(LIB_PATH)
        lib.hts_param_count.restype = C.c_int64
        lib.hts_param_count.argtypes = [C.POINTER(NetDesc)]
        lib.hts_strerror.restype = C.c_char_p
        lib.hts_strerror.argtypes = [C.c_int32]
        lib.hts_create.argtypes = [C.POINTER(NetDesc), C.c_int32, C.c_int32, C.c_void_p, C.POINTER(C.c_void_p)]
        lib.hts_destroy.argtypes = [C.c_void_p]
        lib.hts_act.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_uint64, C.c_uint32, C.c_int32, C.c_int32,
                                C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.hts_sync_params.argtypes = [C.c_void_p, C.c_void_p]
        lib.hts_track_params.argtypes = [C.c_void_p, C.c_int32]
        lib.hts_sample_from_logits.argtypes = [C.c_void_p, C.c_void_p, C.c_uint64, C.c_uint32, C.c_int32, C.c_int32,
                                               C.c_void_p, C.c_void_p]
        lib.hts_returns_gae.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float, C.c_float,
                                        C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        lib.hts_normalize_advantages.argtypes = [C.c_void_p, C.c_void_p, C.c_int64]
        lib.hts_learner_step.argtypes = [C.c_void_p, C.POINTER(Buffer), C.c_void_p, C.POINTER(_OptStateC),
                                         C.POINTER(HParams), C.c_void_p]
        lib.hts_learner_step_delayed.argtypes = [C.c_void_p, C.POINTER(Buffer), C.c_void_p, C.c_void_p, C.POINTER(_OptStateC),
                                                 C.POINTER(HParams), C.c_void_p]
        lib.hts_loss_and_grads.argtypes = [C.c_void_p, C.POINTER(Buffer), C.c_void_p, C.POINTER(HParams), C.c_void_p,
                                           C.c_void_p]
        lib.hts_adam_apply.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(_OptStateC), C.POINTER(HParams),
                                       C.c_int64]
        lib.hts_adam_apply_static.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(_OptStateC), C.POINTER(HParams),
                                              C.c_int64, C.c_void_p]
        lib.hts_test_gemm.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                      C.c_int32]
        lib.hts_profile_site_name.restype = C.c_char_p
        lib.hts_profile_site_name.argtypes = [C.c_int32]
        lib.hts_profile_begin.argtypes = [C.c_void_p, C.c_int32]
        lib.hts_profile_begin_sampled.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
        lib.hts_profile_end.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_double)]
        lib.hts_profile_overhead.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_double)]
        lib.hts_stream_create_cu_range.argtypes = [C.c_int32, C.c_int32, C.POINTER(C.c_void_p)]
        lib.hts_stream_destroy.argtypes = [C.c_void_p]
        vp, rows, steps = C.c_void_p, _Rows, _Steps
        lib.hts_seq_create.argtypes = [C.c_int64, vp, C.POINTER(vp)]
        lib.hts_seq_destroy.argtypes = [vp]
        for f, desc in (("hts_linear_workspace", _LinearDesc), ("hts_short_conv_workspace", _ConvDesc), ("hts_selective_scan_workspace", _ScanDesc),
                        ("hts_selective_scan_states", _ScanDesc)):
            getattr(lib, f).restype = C.c_int64
            getattr(lib, f).argtypes = [C.POINTER(desc)]
        lib.hts_linear.argtypes = [vp, C.POINTER(_LinearDesc), rows, rows, vp, rows, rows, rows]
        lib.hts_linear_backward.argtypes = [vp, C.POINTER(_LinearDesc), rows, rows, rows, rows, rows, rows, vp, vp]
        lib.hts_short_conv.argtypes = [vp, C.POINTER(_ConvDesc), steps, vp, vp, vp, vp, vp, steps, vp]
        lib.hts_short_conv_backward.argtypes = [vp, C.POINTER(_ConvDesc), steps, vp, vp, vp, vp, vp, steps, vp, steps, vp, vp, vp]
        lib.hts_selective_scan.argtypes = [vp, C.POINTER(_ScanDesc), C.POINTER(_ScanInputs), steps, vp, vp]
        lib.hts_selective_scan_backward.argtypes = [vp, C.POINTER(_ScanDesc), C.POINTER(_ScanInputs), steps, vp, vp, C.POINTER(_ScanGrads)]
        for f, desc in (("hts_layer_norm_workspace", _NormDesc), ("hts_delta_rule_workspace", _DeltaDesc), ("hts_delta_rule_states", _DeltaDesc)):
            getattr(lib, f).restype = C.c_int64
            getattr(lib, f).argtypes = [C.POINTER(desc)]
        lib.hts_layer_norm.argtypes = [vp, C.POINTER(_NormDesc), rows, vp, vp, rows]
        lib.hts_layer_norm_backward.argtypes = [vp, C.POINTER(_NormDesc), rows, vp, rows, rows, rows, vp, vp]
        lib.hts_delta_rule.argtypes = [vp, C.POINTER(_DeltaDesc), C.POINTER(_DeltaInputs), steps, vp, vp]
        lib.hts_delta_rule_backward.argtypes = [vp, C.POINTER(_DeltaDesc), C.POINTER(_DeltaInputs), steps, vp, vp, C.POINTER(_DeltaGrads)]
        lib.hts_adamw_create.argtypes = [C.POINTER(_AdamWTensorC), C.c_int32, vp, C.POINTER(vp)]
        lib.hts_adamw_destroy.argtypes = [vp]
        lib.hts_adamw_step.argtypes = [vp, C.POINTER(AdamWHParams), C.POINTER(C.c_int64), vp]
        _lib = lib
    return _lib


def _check(rc: int, what: str):
    if rc != 0:
        lib = load_library()
        raise HtsError(f"{what}: {lib.hts_strerror(rc).decode()} (code {rc}, hip {lib.hts_last_hip_error()})")


def param_count(C_in: int, H: int, W: int, A: int, precision: int = PRECISION_FP32) -> int:
    d = NetDesc(C_in, H, W, A, precision)
    n = load_library().hts_param_count(C.byref(d))
    if n < 0:
        _check(int(n), "hts_param_count")
    return int(n)


def _ptr(t, dtype, name):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise HtsError(f"{name}: expected a contiguous {dtype} device tensor")
    return t.data_ptr()          # (every entry declares its argument types, so the address itself is enough)


def hts_adam_apply_static(params, grads, opt: OptState, hp: HParams, stream=None):
    """Clip + optimiser step through the library's static scratch array: no context, no allocation."""
    lib = load_library()
    stream = stream if stream is not None else torch.cuda.current_stream()
    oc = _OptStateC(_ptr(opt.m, torch.float32, "m"), _ptr(opt.v, torch.float32, "v"), opt.step)
    _check(lib.hts_adam_apply_static(_ptr(params, torch.float32, "params"), _ptr(grads, torch.float32, "grads"),
                                     C.byref(oc), C.byref(hp), params.numel(), C.c_void_p(stream.cuda_stream)),
           "hts_adam_apply_static")
    opt.step = oc.step


class AdamWTensor:
    """A tensor of an AdamW plan: p float32, g float32 or bfloat16, m and v float32, or uint8 with m_scale and v_scale (adamw_scales(n) float32 each), copy
    bfloat16 or None; all contiguous device tensors of p's number of entries."""

    def __init__(self, p, g, m, v, m_scale=None, v_scale=None, copy=None, weight_decay=0.0, lr_scale=1.0):
        self.p, self.g, self.m, self.v, self.m_scale, self.v_scale, self.copy, self.weight_decay, self.lr_scale = p, g, m, v, m_scale, v_scale, copy, weight_decay, lr_scale


def adamw_scales(n: int) -> int:
    """Scales of a moment of n entries that is held in 8 bits: one for every 256 of them."""
    return -(-n // 256)


class AdamW:
    """Owns an hts_adamw plan over AdamWTensors, bound to a torch stream (default: the current stream at construction); keeps the tensors alive.
    step: updates done."""

    def __init__(self, tensors, stream=None):
        self.lib = load_library()
        self._h = C.c_void_p()
        if not torch.cuda.is_available():
            raise HtsError("no GPU visible: the library has no CPU path")
        self.tensors, self.step = list(tensors), 0
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        table = (_AdamWTensorC * max(1, len(self.tensors)))()
        for i, t in enumerate(self.tensors):
            table[i] = self._entry(t, f"tensor {i}: ")
        self.stream.synchronize()                              # (the tensors' contents may still be on their way; the plan's tables are there when create returns)
        _check(self.lib.hts_adamw_create(table, len(self.tensors), C.c_void_p(self.stream.cuda_stream), C.byref(self._h)), "hts_adamw_create")

    @staticmethod
    def _entry(t, name):
        if not isinstance(t.p, torch.Tensor) or t.p.numel() == 0:
            raise HtsError(name + "p: expected a contiguous torch.float32 device tensor")
        n, f = t.p.numel(), torch.float32
        eight = isinstance(t.m, torch.Tensor) and t.m.dtype is torch.uint8
        state, half = torch.uint8 if eight else f, isinstance(t.g, torch.Tensor) and t.g.dtype is torch.bfloat16
        given = [(t.p, f, n, "p"), (t.g, torch.bfloat16 if half else f, n, "g"), (t.m, state, n, "m"), (t.v, state, n, "v")]
        given += [(t.m_scale, f, adamw_scales(n), "m_scale"), (t.v_scale, f, adamw_scales(n), "v_scale")] if eight else []
        for x, dtype, count, what in given + ([(t.copy, torch.bfloat16, n, "copy")] if t.copy is not None else []):
            if x is None or _ptr(x, dtype, name + what) is None or x.numel() != count:
                raise HtsError(f"{name}{what}: expected {count} entries of {dtype}")
        scales = (t.m_scale.data_ptr(), t.v_scale.data_ptr()) if eight else (None, None)
        return _AdamWTensorC(t.p.data_ptr(), t.g.data_ptr(), t.m.data_ptr(), t.v.data_ptr(), *scales, t.copy.data_ptr() if t.copy is not None else None, n, t.weight_decay,
                             t.lr_scale, PRECISION_BF16 if half else PRECISION_FP32, 8 if eight else 32)

    def hts_adamw_step(self, hp: AdamWHParams, grad_norm=None):
        """One update of all tensors; grad_norm (float32 [1]) receives the gradients' norm before clipping."""
        step = C.c_int64(self.step)
        _check(self.lib.hts_adamw_step(self._h, C.byref(hp), C.byref(step), _array(grad_norm, torch.float32, (1,), "grad_norm") or None), "hts_adamw_step")
        self.step = step.value

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            self.stream.synchronize()
            self.lib.hts_adamw_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class CuRangeStream:
    """hts_stream_create_cu_range: a stream whose kernels run on compute units [first_cu, first_cu + n_cus) only, wrapped
    as a torch stream (`.stream`).  close() synchronises and destroys it."""

    def __init__(self, first_cu: int, n_cus: int):
        lib = load_library()
        h = C.c_void_p()
        _check(lib.hts_stream_create_cu_range(first_cu, n_cus, C.byref(h)), "hts_stream_create_cu_range")
        self._h = h
        self.stream = torch.cuda.ExternalStream(h.value)

    def close(self):
        if self._h is not None and self._h.value:
            _check(load_library().hts_stream_destroy(self._h), "hts_stream_destroy")
            self._h = None


class Context:
    """Owns an hts_ctx bound to a torch stream (default: the current stream at construction)."""

    def __init__(self, C_in, H, W, A, precision=PRECISION_FP32, max_act_batch=0, max_learn_batch=0, stream=None):
        self.lib = load_library()
        if not torch.cuda.is_available():
            raise HtsError("no GPU visible: the library has no CPU path")
        self.desc = NetDesc(C_in, H, W, A, precision)
        self.A = A
        self.P = param_count(C_in, H, W, A, precision)
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self._h = C.c_void_p()
        _check(self.lib.hts_create(C.byref(self.desc), max_act_batch, max_learn_batch,
                                   C.c_void_p(self.stream.cuda_stream), C.byref(self._h)), "hts_create")

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            self.stream.synchronize()
            self.lib.hts_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- the three calls of the hot path ------------------------------------------------------------------
    def hts_act(self, obs, params, seed, step, env_offset, actions, logp, values, logits=None):
        N = obs.shape[0]
        _check(self.lib.hts_act(self._h, _ptr(obs, torch.uint8, "obs"), _ptr(params, torch.float32, "params"),
                                C.c_uint64(seed), C.c_uint32(step), N, env_offset,
                                _ptr(actions, torch.int32, "actions"), _ptr(logp, torch.float32, "logp"),
                                _ptr(values, torch.float32, "values"), _ptr(logits, torch.float32, "logits")),
               "hts_act")

    def act_rows(self, obs, actions, logp, values, logits=None):
        """Pre-marshalled hts_act arguments, one entry per leading index s of obs [S,N,C,H,W], actions / logp / values
        [S,N] (and logits [S,N,A]): the tensors are checked once and only raw device addresses are kept."""
        S, N = obs.shape[0], obs.shape[1]
        for t, dt, nm in ((obs, torch.uint8, "obs"), (actions, torch.int32, "actions"), (logp, torch.float32, "logp"),
                          (values, torch.float32, "values"), (logits, torch.float32, "logits")):
            if t is not None:
                _ptr(t, dt, nm)
                if t.shape[0] != S or t.shape[1] != N:
                    raise HtsError(f"{nm}: leading dimensions must be [{S},{N}]")
        ob, so = obs.data_ptr(), obs[0].numel()
        ab, lb, vb = actions.data_ptr(), logp.data_ptr(), values.data_ptr()
        gb, sg = (logits.data_ptr(), 4 * logits[0].numel()) if logits is not None else (0, 0)
        rows = [(ob + s * so, ab + 4 * s * N, lb + 4 * s * N, vb + 4 * s * N, (gb + s * sg) if gb else None)
                for s in range(S)]
        return (N, rows, (obs, actions, logp, values, logits))

    def hts_act_rows(self, act_rows, params, seed, step0, env_offset, first=0, last=None):
        """One hts_act call per entry [first, last) of act_rows (see act_rows); entry s is step step0 + s.  The
        parameters are passed to entry 0 only (the actors keep one parameter version for a whole storage)."""
        N, rows, _keep = act_rows
        fn, h = self.lib.hts_act, self._h
        pp = _ptr(params, torch.float32, "params")
        last = len(rows) if last is None else last
        for s in range(first, last):
            o, a, l, v, g = rows[s]
            rc = fn(h, o, pp if s == 0 else None, seed, step0 + s, N, env_offset, a, l, v, g)
            if rc != 0:
                _check(rc, "hts_act")

    def hts_track_params(self, on: bool):
        _check(self.lib.hts_track_params(self._h, 1 if on else 0), "hts_track_params")

    def hts_sync_params(self, params):
        _check(self.lib.hts_sync_params(self._h, _ptr(params, torch.float32, "params")), "hts_sync_params")

    def hts_sample_from_logits(self, logits, seed, step, env_offset, actions, logp):
        N = logits.shape[0]
        _check(self.lib.hts_sample_from_logits(self._h, _ptr(logits, torch.float32, "logits"), C.c_uint64(seed),
                                               C.c_uint32(step), N, env_offset,
                                               _ptr(actions, torch.int32, "actions"),
                                               _ptr(logp, torch.float32, "logp")), "hts_sample_from_logits")

    def hts_returns_gae(self, rewards, values, dones, gamma, lam, advantages, returns):
        T, N = rewards.shape
        if tuple(values.shape) != (T + 1, N) or tuple(dones.shape) != (T, N):
            raise HtsError("hts_returns_gae: values must be [T+1,N] and dones [T,N]")
        _check(self.lib.hts_returns_gae(self._h, _ptr(rewards, torch.float32, "rewards"),
                                        _ptr(values, torch.float32, "values"), _ptr(dones, torch.uint8, "dones"),
                                        gamma, lam, T, N, _ptr(advantages, torch.float32, "advantages"),
                                        _ptr(returns, torch.float32, "returns")), "hts_returns_gae")

    def hts_normalize_advantages(self, adv):
        _check(self.lib.hts_normalize_advantages(self._h, _ptr(adv, torch.float32, "adv"), adv.numel()),
               "hts_normalize_advantages")

    def _buffer(self, obs, actions, old_logp, advantages, returns, index, B, old_values=None):
        count = obs.shape[0]
        if B is None:
            B = count if index is None else index.numel()
        keep = (obs, actions, old_logp, advantages, returns, index, old_values)
        return Buffer(_ptr(obs, torch.uint8, "obs"), _ptr(actions, torch.int32, "actions"),
                      _ptr(old_logp, torch.float32, "old_logp"), _ptr(old_values, torch.float32, "old_values"),
                      _ptr(advantages, torch.float32, "advantages"), _ptr(returns, torch.float32, "returns"), count,
                      _ptr(index, torch.int32, "index"), B), keep

    def hts_learner_step(self, obs, actions, old_logp, advantages, returns, params, opt: OptState, hp: HParams,
                         index=None, B=None, stats=None, old_values=None):
        buf, _keep = self._buffer(obs, actions, old_logp, advantages, returns, index, B, old_values)
        oc = _OptStateC(_ptr(opt.m, torch.float32, "m"), _ptr(opt.v, torch.float32, "v"), opt.step)
        _check(self.lib.hts_learner_step(self._h, C.byref(buf), _ptr(params, torch.float32, "params"), C.byref(oc),
                                         C.byref(hp), _ptr(stats, torch.float32, "stats")), "hts_learner_step")
        opt.step = oc.step

    def hts_learner_step_delayed(self, obs, actions, old_logp, advantages, returns, params_behaviour, params_target,
                                 opt: OptState, hp: HParams, index=None, B=None, stats=None, old_values=None):
        buf, _keep = self._buffer(obs, actions, old_logp, advantages, returns, index, B, old_values)
        oc = _OptStateC(_ptr(opt.m, torch.float32, "m"), _ptr(opt.v, torch.float32, "v"), opt.step)
        _check(self.lib.hts_learner_step_delayed(self._h, C.byref(buf),
                                                 _ptr(params_behaviour, torch.float32, "params_behaviour"),
                                                 _ptr(params_target, torch.float32, "params_target"), C.byref(oc),
                                                 C.byref(hp), _ptr(stats, torch.float32, "stats")),
               "hts_learner_step_delayed")
        opt.step = oc.step

    def hts_loss_and_grads(self, obs, actions, old_logp, advantages, returns, params, hp: HParams, grads, index=None,
                           B=None, stats=None, old_values=None):
        buf, _keep = self._buffer(obs, actions, old_logp, advantages, returns, index, B, old_values)
        _check(self.lib.hts_loss_and_grads(self._h, C.byref(buf), _ptr(params, torch.float32, "params"), C.byref(hp),
                                           _ptr(grads, torch.float32, "grads"), _ptr(stats, torch.float32, "stats")),
               "hts_loss_and_grads")

    def hts_adam_apply(self, params, grads, opt: OptState, hp: HParams):
        oc = _OptStateC(_ptr(opt.m, torch.float32, "m"), _ptr(opt.v, torch.float32, "v"), opt.step)
        _check(self.lib.hts_adam_apply(self._h, _ptr(params, torch.float32, "params"),
                                       _ptr(grads, torch.float32, "grads"), C.byref(oc), C.byref(hp), params.numel()),
               "hts_adam_apply")
        opt.step = oc.step

    def hts_test_gemm(self, precision, A, B, out):
        M, K = A.shape
        N = B.shape[0]
        _check(self.lib.hts_test_gemm(self._h, precision, _ptr(A, torch.float32, "A"), _ptr(B, torch.float32, "B"),
                                      _ptr(out, torch.float32, "out"), M, N, K), "hts_test_gemm")

    def profile_sites(self):
        return [self.lib.hts_profile_site_name(i).decode() for i in range(self.lib.hts_profile_site_count())]

    def hts_profile_begin(self, site: int):
        _check(self.lib.hts_profile_begin(self._h, site), "hts_profile_begin")

    def hts_profile_begin_sampled(self, site: int, every: int):
        _check(self.lib.hts_profile_begin_sampled(self._h, site, every), "hts_profile_begin_sampled")

    def hts_profile_end(self):
        """-> (timed launches, total milliseconds)."""
        n, ms = C.c_int32(), C.c_double()
        _check(self.lib.hts_profile_end(self._h, C.byref(n), C.byref(ms)), "hts_profile_end")
        return n.value, ms.value

    def hts_profile_overhead(self, reps=256):
        """-> mean milliseconds of an empty event bracket."""
        ms = C.c_double()
        _check(self.lib.hts_profile_overhead(self._h, reps, C.byref(ms)), "hts_profile_overhead")
        return ms.value

    @staticmethod
    def new_stats(device="cuda"):
        """Device buffer for hts_stats (6 floats + 1 int32, viewed as 7 float32 words)."""
        return torch.zeros(7, dtype=torch.float32, device=device)

    @staticmethod
    def read_stats(stats) -> dict:
        h = stats.cpu()
        d = {k: float(h[i]) for i, k in enumerate(STATS_FIELDS[:6])}
        d["nonfinite"] = int(h[6:7].view(torch.int32)[0])
        return d


# ---- sequence memory --------------------------------------------------------------------------------------------------
_DTYPE = {PRECISION_FP32: torch.float32, PRECISION_BF16: torch.bfloat16}
_Tensor = torch.Tensor


def _size(what: str, rc: int) -> int:
    if rc < 0:
        _check(rc, what)
    return rc


def linear_workspace(M: int, N: int, K: int, precision: int = PRECISION_FP32, act: int = ACT_NONE) -> int:
    """Bytes of workspace that hts_linear_backward needs for M rows, N outputs and K inputs (hts_linear needs none)."""
    return _size("hts_linear_workspace", load_library().hts_linear_workspace(C.byref(_LinearDesc(M, N, K, precision, act))))


def short_conv_workspace(T: int, N: int, D: int, W: int, precision: int = PRECISION_FP32) -> int:
    return _size("hts_short_conv_workspace", load_library().hts_short_conv_workspace(C.byref(_ConvDesc(T, N, D, W, precision, ACT_NONE))))


def selective_scan_workspace(T: int, N: int, D: int, S: int, G: int = 1, precision: int = PRECISION_FP32) -> int:
    return _size("hts_selective_scan_workspace", load_library().hts_selective_scan_workspace(C.byref(_ScanDesc(T, N, D, S, G, precision, 1))))


def selective_scan_states(T: int, N: int, D: int, S: int, G: int = 1) -> int:
    """Floats of the `states` that a training forward call hands to its backward call."""
    return _size("hts_selective_scan_states", load_library().hts_selective_scan_states(C.byref(_ScanDesc(T, N, D, S, G, PRECISION_FP32, 1))))


def layer_norm_workspace(M: int, F: int, precision: int = PRECISION_FP32) -> int:
    """Bytes of workspace that hts_layer_norm_backward needs for M rows of F entries (hts_layer_norm needs none)."""
    return _size("hts_layer_norm_workspace", load_library().hts_layer_norm_workspace(C.byref(_NormDesc(M, F, precision, 0.0))))


def delta_rule_workspace(T: int, N: int, H: int, G: int, K: int, V: int, precision: int = PRECISION_FP32) -> int:
    return _size("hts_delta_rule_workspace", load_library().hts_delta_rule_workspace(C.byref(_DeltaDesc(T, N, H, G, K, V, precision, 1, 1, 1.0))))


def delta_rule_states(T: int, N: int, H: int, K: int, V: int) -> int:
    """Floats of the `states` that a training forward call hands to its backward call."""
    return _size("hts_delta_rule_states", load_library().hts_delta_rule_states(C.byref(_DeltaDesc(T, N, H, H, K, V, PRECISION_FP32, 1, 1, 1.0))))


# A small call's time is the host's, and these run for each of its operands: one look at a tensor's properties, no calls between them.
def _precision(t, name, dims=None):
    if not isinstance(t, torch.Tensor) or t.dtype not in (torch.float32, torch.bfloat16) or (dims is not None and t.dim() != dims):
        raise HtsError(f"{name}: expected a float32 or bfloat16 device tensor" + (f" of {dims} dimensions" if dims else ""))
    return PRECISION_BF16 if t.dtype is torch.bfloat16 else PRECISION_FP32


def _last(t, name):
    """The length of a tensor's last dimension, from which a call takes a size."""
    if not isinstance(t, _Tensor) or t.dim() < 2:
        raise HtsError(f"{name}: expected a device tensor of two dimensions or more")
    return t.shape[-1]


def _wrong(dtype, shape, name, what=""):
    return HtsError(f"{name}: expected a {what}{dtype} device tensor of shape {tuple(shape)}")


def _rows(t, dtype, shape, name):
    """(address, distance of rows) of a [M, K] operand whose rows are contiguous, at any distance."""
    if t is None:
        return 0, 0
    if not (isinstance(t, _Tensor) and t.dtype is dtype and t.is_cuda and t.shape == shape):
        raise _wrong(dtype, shape, name)
    ld, one = t.stride()
    if one != 1 and shape[1] > 1:
        raise HtsError(f"{name}: rows must be contiguous")
    return t.data_ptr(), ld


def _steps(t, dtype, shape, name):
    """(address, distances of steps and of sequences) of a [T, N, ...] operand whose steps are contiguous, at any distance."""
    if t is None:
        return 0, 0, 0
    if not (isinstance(t, _Tensor) and t.dtype is dtype and t.is_cuda and t.shape == shape):
        raise _wrong(dtype, shape, name)
    st = t.stride()
    if len(st) > 3 or st[2] != 1:
        inner = 1
        for size, stride in zip(shape[:1:-1], st[:1:-1]):
            if stride != inner and size > 1:
                raise HtsError(f"{name}: steps must be contiguous")
            inner *= size
    return t.data_ptr(), st[0], st[1]


def _array(t, dtype, shape, name):
    """The address of a contiguous array of that shape, 0 for None."""
    if t is None:
        return 0
    if not (isinstance(t, _Tensor) and t.dtype is dtype and t.is_cuda and t.shape == shape and t.is_contiguous()):
        raise _wrong(dtype, shape, name, "contiguous ")
    return t.data_ptr()


class _Arguments:
    """Structures of a call over one piece of memory that a call fills at once (a small call's time is the host's)."""

    def __init__(self, *kinds):
        size = sum(C.sizeof(k) for k in kinds)
        self._memory, self._fill, self.of = bytearray(size), struct.Struct(f"{size // 8}q").pack_into, []      # of: the structures, at: the first one's address
        at = 0
        for k in kinds:
            self.of.append(k.from_buffer(self._memory, at))
            at += C.sizeof(k)
        self.at = C.byref(self.of[0])

    def set(self, *words):
        self._fill(self._memory, 0, *words)
        return self.of


class SeqContext:
    """Owns an hts_seq_ctx bound to a torch stream (default: the current stream at construction): the operators of a sequence memory.
    workspace_bytes: the most that any of its calls needs (linear_workspace, short_conv_workspace, selective_scan_workspace, layer_norm_workspace, delta_rule_workspace)."""

    def __init__(self, workspace_bytes=0, stream=None):
        self.lib = load_library()
        if not torch.cuda.is_available():
            raise HtsError("no GPU visible: the library has no CPU path")
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        self._linear, self._linear_back, self._conv, self._conv_back = (_Arguments(*[k] * n) for k, n in ((_Rows, 5), (_Rows, 6), (_Steps, 2), (_Steps, 3)))
        self._norm, self._norm_back = _Arguments(*[_Rows] * 2), _Arguments(*[_Rows] * 4)
        self._delta_in, self._delta_grads = _Arguments(_DeltaInputs), _Arguments(_DeltaGrads)
        self._scan_in, self._scan_grads, self._one, self._descs = _Arguments(_ScanInputs), _Arguments(_ScanGrads), _Arguments(_Steps), {}
        self._h = C.c_void_p()
        _check(self.lib.hts_seq_create(workspace_bytes, C.c_void_p(self.stream.cuda_stream), C.byref(self._h)), "hts_seq_create")

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            self.stream.synchronize()
            self.lib.hts_seq_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _desc(self, kind, *sizes):
        """A call's sizes as the library reads them, made once."""
        key = kind, sizes
        d = self._descs.get(key)
        if d is None:
            if len(self._descs) > 256:
                self._descs.clear()
            d = self._descs[key] = C.byref(kind(*sizes))
        return d

    def hts_linear(self, x, w, y, bias=None, residual=None, pre=None, act=ACT_NONE):
        """y = act(x w^T + bias) + residual; pre receives x w^T + bias."""
        prec = _precision(x, "x", 2)
        _precision(w, "w", 2)
        dt, (M, K), N = _DTYPE[prec], x.shape, w.shape[0]
        xs, ws, rs, ys, ps = self._linear.set(*_rows(x, dt, (M, K), "x"), *_rows(w, dt, (N, K), "w"), *_rows(residual, dt, (M, N), "residual"), *_rows(y, dt, (M, N), "y"),
                                              *_rows(pre, dt, (M, N), "pre"))
        rc = self.lib.hts_linear(self._h, self._desc(_LinearDesc, M, N, K, prec, act), xs, ws, _array(bias, torch.float32, (N,), "bias"), rs, ys, ps)
        if rc:
            _check(rc, "hts_linear")

    def hts_linear_backward(self, x, w, dy, pre=None, act=ACT_NONE, add=None, dx=None, dw=None, db=None):
        """With g = dy act'(pre): dx = g w + add, dw = g^T x, db = column sums of g; each of the three only where it is given."""
        prec = _precision(dy, "dy", 2)
        _precision(w, "w", 2)
        dt, (M, N), K, f = _DTYPE[prec], dy.shape, w.shape[1], torch.float32
        a = self._linear_back.set(*_rows(x, dt, (M, K), "x"), *_rows(w, dt, (N, K), "w"), *_rows(pre, dt, (M, N), "pre"), *_rows(dy, dt, (M, N), "dy"),
                                  *_rows(add, dt, (M, K), "add"), *_rows(dx, dt, (M, K), "dx"))
        rc = self.lib.hts_linear_backward(self._h, self._desc(_LinearDesc, M, N, K, prec, act), *a, _array(dw, f, (N, K), "dw"), _array(db, f, (N,), "db"))
        if rc:
            _check(rc, "hts_linear_backward")

    @staticmethod
    def _sequences(starts, lengths, T, N):
        return _array(starts, torch.uint8, (T, N), "starts"), _array(lengths, torch.int32, (N,), "lengths")

    def hts_short_conv(self, x, w, y, bias=None, act=ACT_NONE, starts=None, lengths=None, state_in=None, state_out=None):
        """y_t = act(bias + sum_j w[:, j] x_{t-W+1+j}) over the steps of t's episode; state_in and state_out (which may be one) hold the last W - 1 inputs."""
        prec = _precision(x, "x", 3)
        cells, W, f = x.shape, _last(w, "w"), torch.float32
        (T, N, D), dt = cells, _DTYPE[prec]
        state = (N, W - 1, D)
        xs, ys = self._conv.set(*_steps(x, dt, cells, "x"), *_steps(y, dt, cells, "y"))
        rc = self.lib.hts_short_conv(self._h, self._desc(_ConvDesc, T, N, D, W, prec, act), xs, _array(w, f, (D, W), "w"), _array(bias, f, (D,), "bias"),
                                     *self._sequences(starts, lengths, T, N), _array(state_in, f, state, "state_in"), ys, _array(state_out, f, state, "state_out"))
        if rc:
            _check(rc, "hts_short_conv")

    def hts_short_conv_backward(self, x, w, dy, dx, dw, db=None, bias=None, act=ACT_NONE, starts=None, lengths=None, state_in=None, dstate_out=None,
                                dstate_in=None):
        """The gradients dx, dw, db and dstate_in of dy and dstate_out."""
        prec = _precision(x, "x", 3)
        cells, W, f = x.shape, _last(w, "w"), torch.float32
        (T, N, D), dt = cells, _DTYPE[prec]
        state = (N, W - 1, D)
        xs, gs, ds = self._conv_back.set(*_steps(x, dt, cells, "x"), *_steps(dy, dt, cells, "dy"), *_steps(dx, dt, cells, "dx"))
        rc = self.lib.hts_short_conv_backward(self._h, self._desc(_ConvDesc, T, N, D, W, prec, act), xs, _array(w, f, (D, W), "w"), _array(bias, f, (D,), "bias"),
                                              *self._sequences(starts, lengths, T, N), _array(state_in, f, state, "state_in"), gs,
                                              _array(dstate_out, f, state, "dstate_out"), ds, _array(dw, f, (D, W), "dw"), _array(db, f, (D,), "db"),
                                              _array(dstate_in, f, state, "dstate_in"))
        if rc:
            _check(rc, "hts_short_conv_backward")

    def _scan(self, x, dt, A, B, C_, z, skip, dt_bias, softplus, starts, lengths, h_in):
        prec, f = _precision(x, "x", 3), torch.float32
        cells, S, ty = x.shape, _last(A, "A"), _DTYPE[prec]
        T, N, D = cells
        G, held = 1, (N, D, S)
        pair = (T, N, S)
        _last(B, "B")
        if B.dim() == 4:
            G = B.shape[2]
            pair = (T, N, G, S)
        st, le = self._sequences(starts, lengths, T, N)
        self._scan_in.set(*_steps(x, ty, cells, "x"), *_steps(dt, ty, cells, "dt"), *_steps(B, ty, pair, "B"), *_steps(C_, ty, pair, "C"), *_steps(z, ty, cells, "z"),
                          _array(A, f, (D, S), "A"), _array(skip, f, (D,), "skip"), _array(dt_bias, f, (D,), "dt_bias"), st, le, _array(h_in, f, held, "h_in"))
        return self._desc(_ScanDesc, T, N, D, S, G, prec, 1 if softplus else 0), self._scan_in.at, ty, cells, pair, held

    def hts_selective_scan(self, x, dt, A, B, C_, y, z=None, skip=None, dt_bias=None, softplus=True, starts=None, lengths=None, h_in=None, h_out=None,
                           states=None):
        """h_t = exp(delta A) h_{t-1} + delta x B, y = (C h + skip x) silu(z), delta = softplus(dt + dt_bias).  B, C: [T, N, S] or [T, N, G, S].  h_in and
        h_out may be one; states (selective_scan_states floats) is for a backward call."""
        desc, inputs, ty, cells, _, held = self._scan(x, dt, A, B, C_, z, skip, dt_bias, softplus, starts, lengths, h_in)
        if states is not None and (not isinstance(states, _Tensor) or states.numel() < self.lib.hts_selective_scan_states(desc)):
            raise HtsError("states: too few entries (selective_scan_states)")
        rc = self.lib.hts_selective_scan(self._h, desc, inputs, self._one.set(*_steps(y, ty, cells, "y"))[0], _array(h_out, torch.float32, held, "h_out"),
                                         _ptr(states, torch.float32, "states"))
        if rc:
            _check(rc, "hts_selective_scan")

    def hts_selective_scan_backward(self, x, dt, A, B, C_, dy, states, dx, ddt, dB, dC, dA, z=None, dz=None, skip=None, dskip=None, dt_bias=None,
                                    ddt_bias=None, softplus=True, starts=None, lengths=None, h_in=None, dh_out=None, dh_in=None):
        """The gradients of dy and dh_out; states as the forward call on the same inputs left it."""
        desc, inputs, ty, cells, pair, held = self._scan(x, dt, A, B, C_, z, skip, dt_bias, softplus, starts, lengths, h_in)
        if not isinstance(states, _Tensor) or states.numel() < self.lib.hts_selective_scan_states(desc):
            raise HtsError("states: too few entries (selective_scan_states)")
        f, (_, D, S) = torch.float32, held
        self._scan_grads.set(*_steps(dx, ty, cells, "dx"), *_steps(ddt, ty, cells, "ddt"), *_steps(dB, ty, pair, "dB"), *_steps(dC, ty, pair, "dC"),
                             *_steps(dz, ty, cells, "dz"), _array(dA, f, (D, S), "dA"), _array(dskip, f, (D,), "dskip"), _array(ddt_bias, f, (D,), "ddt_bias"),
                             _array(dh_in, f, held, "dh_in"))
        rc = self.lib.hts_selective_scan_backward(self._h, desc, inputs, self._one.set(*_steps(dy, ty, cells, "dy"))[0], _array(dh_out, f, held, "dh_out"),
                                                  _ptr(states, f, "states"), self._scan_grads.at)
        if rc:
            _check(rc, "hts_selective_scan_backward")

    def hts_layer_norm(self, x, y, w=None, b=None, eps=1e-5):
        """y = (x - mean) / sqrt(var + eps) w + b over the rows of x [M, F]; y may be x."""
        prec = _precision(x, "x", 2)
        shape, dt, f = x.shape, _DTYPE[prec], torch.float32
        xs, ys = self._norm.set(*_rows(x, dt, shape, "x"), *_rows(y, dt, shape, "y"))
        rc = self.lib.hts_layer_norm(self._h, self._desc(_NormDesc, *shape, prec, eps), xs, _array(w, f, shape[1:], "w"), _array(b, f, shape[1:], "b"), ys)
        if rc:
            _check(rc, "hts_layer_norm")

    def hts_layer_norm_backward(self, x, dy, w=None, add=None, dx=None, dw=None, db=None, eps=1e-5):
        """The gradients of dy: dx (and add), dw, db; each of the three only where it is given.  dx may be dy, add or x."""
        prec = _precision(x, "x", 2)
        shape, dt, f = x.shape, _DTYPE[prec], torch.float32
        xs, gs, adds, ds = self._norm_back.set(*_rows(x, dt, shape, "x"), *_rows(dy, dt, shape, "dy"), *_rows(add, dt, shape, "add"), *_rows(dx, dt, shape, "dx"))
        rc = self.lib.hts_layer_norm_backward(self._h, self._desc(_NormDesc, *shape, prec, eps), xs, _array(w, f, shape[1:], "w"), gs, adds, ds, _array(dw, f, shape[1:], "dw"),
                                              _array(db, f, shape[1:], "db"))
        if rc:
            _check(rc, "hts_layer_norm_backward")

    def _delta(self, q, k, v, a, b, A, a_bias, scale, normalize, softplus, starts, lengths, h_in):
        prec, f = _precision(q, "q", 4), torch.float32
        _precision(v, "v", 4)
        keys, values, ty = q.shape, v.shape, _DTYPE[prec]
        T, N, G, K = keys
        H, V = values[2:]
        gates, held = (T, N, H), (N, H, K, V)
        st, le = self._sequences(starts, lengths, T, N)
        self._delta_in.set(*_steps(q, ty, keys, "q"), *_steps(k, ty, keys, "k"), *_steps(v, ty, (T, N, H, V), "v"), *_steps(a, ty, gates, "a"), *_steps(b, ty, gates, "b"),
                           _array(A, f, (H,), "A"), _array(a_bias, f, (H,), "a_bias"), st, le, _array(h_in, f, held, "h_in"))
        return self._desc(_DeltaDesc, T, N, H, G, K, V, prec, 1 if normalize else 0, 1 if softplus else 0, scale), self._delta_in.at, ty, keys, values, gates, held

    def hts_delta_rule(self, q, k, v, a, b, A, y, a_bias=None, scale=1.0, normalize=True, softplus=True, starts=None, lengths=None, h_in=None, h_out=None, states=None):
        """z = v - alpha S^T k, S = alpha S + beta k z^T, y = scale S^T q; alpha = exp(A softplus(a + a_bias)), beta = sigmoid(b).  q, k [T, N, G, K], v, y [T, N, H, V],
        a, b [T, N, H].  h_in and h_out (float32 [N, H, K, V]) may be one; states (delta_rule_states floats) is for a backward call."""
        desc, inputs, ty, _, values, _, held = self._delta(q, k, v, a, b, A, a_bias, scale, normalize, softplus, starts, lengths, h_in)
        if states is not None and (not isinstance(states, _Tensor) or states.numel() < _size("hts_delta_rule_states", self.lib.hts_delta_rule_states(desc))):
            raise HtsError("states: too few entries (delta_rule_states)")
        rc = self.lib.hts_delta_rule(self._h, desc, inputs, self._one.set(*_steps(y, ty, values, "y"))[0], _array(h_out, torch.float32, held, "h_out"),
                                     _ptr(states, torch.float32, "states"))
        if rc:
            _check(rc, "hts_delta_rule")

    def hts_delta_rule_backward(self, q, k, v, a, b, A, dy, states, dq, dk, dv, da, db, dA, a_bias=None, da_bias=None, scale=1.0, normalize=True, softplus=True, starts=None,
                                lengths=None, h_in=None, dh_out=None, dh_in=None):
        """The gradients of dy and dh_out; states as the forward call on the same inputs left it."""
        desc, inputs, ty, keys, values, gates, held = self._delta(q, k, v, a, b, A, a_bias, scale, normalize, softplus, starts, lengths, h_in)
        if not isinstance(states, _Tensor) or states.numel() < _size("hts_delta_rule_states", self.lib.hts_delta_rule_states(desc)):
            raise HtsError("states: too few entries (delta_rule_states)")
        f, heads = torch.float32, held[1:2]
        self._delta_grads.set(*_steps(dq, ty, keys, "dq"), *_steps(dk, ty, keys, "dk"), *_steps(dv, ty, values, "dv"), *_steps(da, ty, gates, "da"), *_steps(db, ty, gates, "db"),
                              _array(dA, f, heads, "dA"), _array(da_bias, f, heads, "da_bias"), _array(dh_in, f, held, "dh_in"))
        rc = self.lib.hts_delta_rule_backward(self._h, desc, inputs, self._one.set(*_steps(dy, ty, values, "dy"))[0], _array(dh_out, f, held, "dh_out"), _ptr(states, f, "states"),
                                              self._delta_grads.at)
        if rc:
            _check(rc, "hts_delta_rule_backward")
