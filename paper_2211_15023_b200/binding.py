"""ctypes binding of libaccerl.so: same names and argument order as include/accerl.h."""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None
_CALLS = None

FLAG_KEEP_ACTIVATIONS = 1
FLAG_FORCE_GENERIC = 2
FLAG_TAP_FUSED = 4
FLAG_VALUE_HEAD = 8
FLAG_TEST_NO_FASTDIV = 16
FLAG_TEST_NO_AFFINE = 32
RELU_IN, RELU_OUT, LOGITS = 1, 2, 4
_KINDS = {"conv": 0, "fc": 1, "maxpool": 2}
STATUS = {0: "OK", 1: "INVALID_ARG", 2: "UNSUPPORTED", 3: "BATCH_TOO_LARGE", 4: "OOM", 5: "CUDA",
          6: "TIMEOUT"}


class AccerlError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("accerl %s: %s" % (STATUS.get(status, status), message))
        self.status = status


class LayerDesc(C.Structure):
    _fields_ = [("kind", C.c_int32), ("flags", C.c_uint32),
                ("in_c", C.c_int32), ("in_h", C.c_int32), ("in_w", C.c_int32),
                ("out_c", C.c_int32), ("kh", C.c_int32), ("kw", C.c_int32),
                ("stride", C.c_int32), ("pad", C.c_int32),
                ("s_in", C.c_float), ("s_out", C.c_float),
                ("w", C.c_void_p), ("s_w", C.c_void_p), ("bias", C.c_void_p),
                ("skip_from", C.c_int32), ("skip_mul", C.c_void_p)]


class LayerFp32(C.Structure):
    _fields_ = [("kind", C.c_int32), ("flags", C.c_uint32),
                ("in_c", C.c_int32), ("in_h", C.c_int32), ("in_w", C.c_int32),
                ("out_c", C.c_int32), ("kh", C.c_int32), ("kw", C.c_int32),
                ("stride", C.c_int32), ("pad", C.c_int32),
                ("w", C.c_void_p), ("bias", C.c_void_p), ("skip_from", C.c_int32)]


def library_path() -> str:
    return os.path.join(_HERE, "libaccerl.so")


def library() -> C.CDLL:
    """Load libaccerl.so; there is no fallback if it has not been built."""
    global _LIB
    if _LIB is None:
        path = library_path()
        if not os.path.exists(path):
            raise ImportError("%s is missing: build it with `python -m paper_2211_15023_b200.build`"
                              % path)
        lib = C.CDLL(path)
        vp, i32, f32 = C.c_void_p, C.c_int32, C.c_float
        lib.accerl_policy_create.argtypes = [C.POINTER(vp), i32, C.POINTER(i32), f32,
                                             C.POINTER(LayerDesc), i32, i32, C.c_uint32, i32]
        lib.accerl_policy_act.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp]
        lib.accerl_policy_act_timed.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp, i32]
        lib.accerl_policy_act_noalloc.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp]
        lib.accerl_policy_act_host.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp]
        lib.accerl_policy_read_activation.argtypes = [vp, i32, i32, vp, C.c_size_t]
        lib.accerl_policy_check.argtypes = [vp]
        lib.accerl_policy_info.argtypes = [vp, i32, C.POINTER(i32), C.POINTER(C.c_size_t),
                                           C.POINTER(i32), C.c_char_p, C.c_size_t]
        lib.accerl_policy_act_ex.argtypes = [vp, vp, vp, i32, vp, vp, vp, vp, vp, vp]
        lib.accerl_policy_kl.argtypes = [vp, vp, i32, i32, vp, vp, vp]
        lib.accerl_policy_act_mixed.argtypes = [vp, vp, vp, vp, vp, f32, i32, vp, vp, vp, vp, vp, vp, vp]
        lib.accerl_vtrace.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, f32, f32, f32, vp, vp, vp]
        for f in ("accerl_policy_act_ex", "accerl_policy_kl", "accerl_policy_act_mixed", "accerl_vtrace"):
            getattr(lib, f).restype = C.c_int
        lib.accerl_policy_create_fp32.argtypes = [C.POINTER(vp), i32, C.POINTER(i32), C.POINTER(LayerFp32), i32, vp,
                                                  i32, i32, i32, C.c_uint32, i32]
        lib.accerl_policy_create_fp32.restype = C.c_int
        lib.accerl_policy_export.argtypes = [vp, i32, vp, C.c_size_t, vp, vp, C.POINTER(f32), C.POINTER(f32)]
        lib.accerl_policy_export.restype = C.c_int
        lib.accerl_policy_selftest_wait.argtypes = [vp, i32, vp]
        lib.accerl_policy_selftest_wait.restype = C.c_int
        lib.accerl_tc_probe_i8.argtypes = [i32, i32, i32, i32, i32, i32, i32, i32, C.POINTER(f32), C.POINTER(f32)]
        lib.accerl_tc_probe_i8.restype = C.c_int
        lib.accerl_policy_loss.argtypes, lib.accerl_policy_loss.restype = [C.POINTER(PolicyLossArgs), vp], C.c_int
        i64 = C.c_int64
        lib.accerl_ckpt_save.argtypes = [vp, i64, i32, i64, i32, i32, vp, i64, vp, i64, vp, i64, vp]
        lib.accerl_ckpt_load.argtypes = [vp, i64, vp, i64, i64, i32, vp, i64, i32, vp]
        lib.accerl_ckpt_act_backward.argtypes = [vp, i64, i32, vp, i64, vp, i64, i64, i32, i32, vp, i64, vp]
        for f in ("ckpt_save", "ckpt_load", "ckpt_act_backward"):
            getattr(lib, "accerl_" + f).restype = C.c_int
        lib.accerl_quant_rows.argtypes, lib.accerl_quant_rows.restype = [vp, i64, i32, i64, i32, vp, i64, vp, vp], C.c_int
        lib.accerl_linear_i8.argtypes, lib.accerl_linear_i8.restype = [C.POINTER(LinearI8Args), vp], C.c_int
        lib.accerl_linear_i8_workspace.argtypes, lib.accerl_linear_i8_workspace.restype = [i32, i32, i32], i64
        lib.accerl_device_check.argtypes, lib.accerl_device_check.restype = [], C.c_int
        lib.accerl_ckpt_weight_grad.argtypes = [C.POINTER(WeightGradArgs), vp]
        lib.accerl_ckpt_weight_grad.restype = C.c_int
        lib.accerl_ckpt_weight_grad_workspace.argtypes = [C.POINTER(WeightGradArgs)]
        lib.accerl_ckpt_weight_grad_workspace.restype = i64
        lib.accerl_policy_destroy.argtypes = [vp]
        lib.accerl_policy_destroy.restype = None
        lib.accerl_trim.argtypes, lib.accerl_trim.restype = [], None
        lib.accerl_last_error.restype = C.c_char_p
        lib.accerl_version.restype = C.c_char_p
        for f in ("create", "act", "act_timed", "act_noalloc", "act_host", "read_activation", "check", "info"):
            getattr(lib, "accerl_policy_" + f).restype = C.c_int
        _LIB = lib
    return _LIB


def _calls():
    """The native module behind the hot calls (csrc/torch_calls.cpp); built with the library."""
    global _CALLS
    if _CALLS is None:
        import torch  # noqa: F401  (its libraries have to be loaded first)
        library()
        from . import _calls as native
        _CALLS = native
    return _CALLS


def _check(status: int):
    if status != 0:
        raise AccerlError(status, library().accerl_last_error().decode())


def _done(r):
    """The results of a native call, or the error its status code stands for."""
    if type(r) is int:
        _check(r)
    return r


def _out_hw(l):
    if l["kind"] == "fc":
        return 1, 1
    return ((l["in_h"] + 2 * l["pad"] - l["kh"]) // l["stride"] + 1,
            (l["in_w"] + 2 * l["pad"] - l["kw"]) // l["stride"] + 1)


def tc_probe_i8(n: int, issuing_warps: int = 1, mmas_per_warp: int = 4096, ctas: int = 148,
                layout: int = 128, a_shift_rows: int = 0, commit_every: int = 0, device: int = 0) -> dict:
    """accerl_tc_probe_i8: cost of an M = 128, N = n int8 MMA; returns ms, cycles_per_mma, tops."""
    ms, cyc = C.c_float(), C.c_float()
    _check(library().accerl_tc_probe_i8(device, n, issuing_warps, mmas_per_warp, ctas, layout, a_shift_rows, commit_every,
                                        C.byref(ms), C.byref(cyc)))
    ops = ctas * issuing_warps * mmas_per_warp * 2.0 * 128 * n * 32
    return dict(n=n, issuing_warps=issuing_warps, mmas_per_warp=mmas_per_warp, ctas=ctas, layout=layout, a_shift_rows=a_shift_rows, commit_every=commit_every,
                ms=ms.value, cycles_per_mma=cyc.value, tops=ops / (ms.value * 1e-3) / 1e12)


def trim():
    """accerl_trim: give back the memory kept for the next policy."""
    library().accerl_trim()


def _stream_of(t, stream):
    import torch
    return torch.cuda.current_stream(t.device).cuda_stream if stream is None else stream


class _Memory:
    """Where a call's memory comes from: the pool of the stream that it runs on.  What torch's current stream has given back
    may be in use by work that waits there, and a stream that was named does not wait for it.  Results are the caller's, who
    may give them back while its current stream still reads them."""

    def __init__(self, like, stream):
        import torch
        self._torch, self._device, self._caller = torch, like.device, None
        if stream is not None and like.is_cuda:
            at, current = int(getattr(stream, "value", stream) or 0), self._torch.cuda.current_stream(like.device)
            if at != current.cuda_stream:
                self._caller = current
                self._named = self._torch.cuda.ExternalStream(at, device=like.device) if at else \
                    self._torch.cuda.default_stream(like.device)

    def _made(self, make):
        if self._caller is None:
            return make()
        with self._torch.cuda.stream(self._named):
            return make()

    def result(self, shape, dtype, stride=None):
        t = self._made(lambda: self._torch.empty(shape, dtype=dtype, device=self._device) if stride is None else
                       self._torch.empty_strided(shape, stride, dtype=dtype, device=self._device))
        if self._caller is not None and t.numel():
            t.record_stream(self._caller)
        return t

    def workspace(self, nbytes):
        return self._made(lambda: self._torch.empty(nbytes, dtype=self._torch.uint8, device=self._device)) if nbytes else None


def _check_batch(frames, obs, *per_state):
    """What a kernel reads as a batch of observations and floats per state must be that, on the device."""
    import torch
    assert obs.is_cuda and obs.is_contiguous() and \
        (obs.element_size() == 1 if frames else obs.dtype == torch.float32)
    for t in per_state:
        assert t.device == obs.device and t.is_contiguous() and t.dtype == torch.float32 and t.numel() >= obs.shape[0]


def kl(logits_original, logits_smaller, stream=None):
    """accerl_policy_kl on two CUDA fp32 [B, A] tensors; returns (kl [B], mean_max [2]) tensors."""
    r = (_CALLS or _calls()).kl(logits_original, logits_smaller, stream)
    if r is not None:
        return _done(r)
    import torch
    assert logits_original.shape == logits_smaller.shape and logits_original.is_contiguous() and \
        logits_smaller.is_contiguous() and logits_original.dtype == logits_smaller.dtype == torch.float32 and \
        logits_original.is_cuda and logits_smaller.is_cuda
    b, a = logits_original.shape
    memory = _Memory(logits_original, stream)
    out, stats = memory.result(b, torch.float32), memory.result(2, torch.float32)
    _check(library().accerl_policy_kl(logits_original.data_ptr(), logits_smaller.data_ptr(), b, a,
                                      out.data_ptr(), stats.data_ptr(), _stream_of(out, stream)))
    return out, stats


def vtrace(logp_smaller, logp_original, rewards, values, bootstrap, gamma, rho_hat=1.0, c_hat=1.0,
           discounts=None, stream=None, out=None, checked=True):
    """accerl_vtrace on CUDA fp32 time-major [n, B] tensors; returns (vs, adv) tensors [n, B]."""
    if out is None:
        r = (_CALLS or _calls()).vtrace(logp_smaller, logp_original, rewards, values, bootstrap, discounts, gamma,
                                        rho_hat, c_hat, stream)
        if r is not None:
            return _done(r)
    import torch
    n, b = logp_smaller.shape
    if checked:
        for t in (logp_smaller, logp_original, rewards, values):
            assert t.shape == (n, b) and t.is_contiguous() and t.dtype == torch.float32 and t.is_cuda
        assert bootstrap.shape == (b,) and bootstrap.is_contiguous() and bootstrap.dtype == torch.float32 and \
            bootstrap.is_cuda
        assert discounts is None or (discounts.shape == (n, b) and discounts.is_contiguous() and
                                     discounts.dtype == torch.float32 and discounts.is_cuda)
    memory = _Memory(values, stream) if out is None else None
    vs, adv = (memory.result(values.shape, values.dtype), memory.result(values.shape, values.dtype)) if out is None else out
    _check(library().accerl_vtrace(logp_smaller.data_ptr(), logp_original.data_ptr(), rewards.data_ptr(),
                                   values.data_ptr(), bootstrap.data_ptr(),
                                   None if discounts is None else discounts.data_ptr(), n, b,
                                   float(gamma), float(rho_hat), float(c_hat), vs.data_ptr(),
                                   adv.data_ptr(), _stream_of(vs, stream)))
    return vs, adv


def act_mixed(smaller, original, obs, uniforms, select_uniforms, alpha, stream=None):
    """accerl_policy_act_mixed; returns dict(logits, actions, logp, entropy, use_smaller[, value])."""
    r = (_CALLS or _calls()).act_mixed(smaller._raw, original._raw, smaller.n_actions, smaller.in_kind == "u8",
                                       smaller.value_head and original.value_head, obs, uniforms, select_uniforms,
                                       alpha, stream)
    if r is not None:
        return _done(r)
    import torch
    _check_batch(smaller.in_kind == "u8", obs, uniforms, select_uniforms)
    b, memory = int(obs.shape[0]), _Memory(obs, stream)
    out = dict(logits=memory.result((b, smaller.n_actions), torch.float32), actions=memory.result(b, torch.int32),
               logp=memory.result(b, torch.float32), entropy=memory.result(b, torch.float32),
               use_smaller=memory.result(b, torch.uint8))
    if smaller.value_head and original.value_head:
        out["value"] = memory.result(b, torch.float32)
    _check(library().accerl_policy_act_mixed(
        smaller._h, original._h, obs.data_ptr(), uniforms.data_ptr(), select_uniforms.data_ptr(),
        float(alpha), b, out["logits"].data_ptr(), out["actions"].data_ptr(), out["logp"].data_ptr(),
        out["value"].data_ptr() if "value" in out else None, out["entropy"].data_ptr(),
        out["use_smaller"].data_ptr(), _stream_of(obs, stream)))
    return out


# -- operators of the Learner's side ---------------------------------------------------------------
_DTYPES = ("float32", "bfloat16", "float16")  # in the order of accerl_dtype


class PolicyLossArgs(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("logits", "logits_ref", "actions", "logp_old", "advantages", "logp_ref",
                                          "weights")] + \
        [(n, C.c_int64) for n in ("ld_logits", "ld_logits_ref", "ld_grad")] + \
        [(n, C.c_int32) for n in ("rows", "n_actions", "dtype", "actions64")] + \
        [(n, C.c_float) for n in ("clip_low", "clip_high", "kl_coef", "entropy_coef")] + \
        [(n, C.c_void_p) for n in ("grad", "logp", "kl", "entropy", "stats", "terms")]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _dtype_code(dtype):
    import torch
    for i, n in enumerate(_DTYPES):
        if dtype is getattr(torch, n):
            return i
    raise AssertionError("dtype %s is none of %s" % (dtype, ", ".join(_DTYPES)))


def _check_rows(t, like=None, dtype=None):
    """A CUDA matrix whose rows lie one after another (any distance between them); on the device of `like`."""
    assert t.is_cuda and t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1) and \
        (t.stride(0) >= t.shape[1] or t.shape[0] == 1), "rows of a CUDA matrix, the elements of a row adjacent"
    assert like is None or t.device == like.device, "tensors on different devices"
    assert dtype is None or t.dtype == dtype, "expected %s" % dtype


def _ld(t):
    """Distance of two rows (torch leaves the stride of a single row open)."""
    return t.stride(0) if t.shape[0] > 1 else max(int(t.shape[1]), t.stride(0))


def _check_vector(t, n, like, *dtypes):
    assert t.is_cuda and t.device == like.device and t.dim() == 1 and t.shape[0] == n and t.is_contiguous() and \
        t.dtype in dtypes, "a contiguous CUDA vector of %d %s" % (n, " or ".join(map(str, dtypes)))


class _on_device_of:
    """Makes the device of a tensor the current one, where it is not."""

    def __init__(self, t):
        import torch
        self.guard = None if t.device.index == torch.cuda.current_device() else torch.cuda.device(t.device)

    def __enter__(self):
        if self.guard:
            self.guard.__enter__()

    def __exit__(self, *a):
        if self.guard:
            self.guard.__exit__(*a)


def policy_loss(logits, actions, logp_old, advantages, weights=None, logits_ref=None, logp_ref=None, clip=0.2,
                kl_coef=0.0, entropy_coef=0.0, grad=True, stream=None) -> dict:
    """accerl_policy_loss on CUDA rows of logits [T, A] (fp32, bf16 or fp16).

    ``actions`` int32 or int64 [T]; ``logp_old``, ``advantages``, ``weights`` (None: 1 / T each), ``logp_ref`` fp32 [T];
    ``logits_ref`` like ``logits``; ``clip`` a number or (low, high).  ``grad``: True for a new tensor, a tensor to write
    (``logits`` itself among them), False for none.  Returns dict(stats [8], logp [T], kl [T], entropy [T], grad):
    ``stats`` holds the loss, the weighted sums of the clipped objective, KL, entropy and clipped rows, the sum of
    weights, the largest KL and the weighted sum of ratios.
    """
    low, high = clip if isinstance(clip, (tuple, list)) else (clip, clip)
    r = (_CALLS or _calls()).policy_loss(logits, actions, logp_old, advantages, weights, logits_ref, logp_ref, low, high,
                                         kl_coef, entropy_coef, grad, stream)
    if r is not None:
        return _done(r)
    import torch
    code = _dtype_code(logits.dtype)
    _check_rows(logits)
    t, v = int(logits.shape[0]), int(logits.shape[1])
    if logits_ref is not None:
        _check_rows(logits_ref, logits, logits.dtype)
        assert logits_ref.shape == logits.shape
    _check_vector(actions, t, logits, torch.int32, torch.int64)
    for x in (logp_old, advantages, weights, logp_ref):
        if x is not None:
            _check_vector(x, t, logits, torch.float32)
    assert logp_old is not None and advantages is not None
    memory = _Memory(logits, stream)
    if grad is True:
        # rows as far apart as the logits', which then lie alike to 16 bytes; but not those of the last token of sequences
        grad = memory.result(logits.shape, logits.dtype, (_ld(logits) if _ld(logits) < 2 * v else -(-v // 8) * 8, 1))
    elif grad is False:
        grad = None
    if grad is not None:
        _check_rows(grad, logits, logits.dtype)
        assert grad.shape == logits.shape
    f = memory.result(8 + 5 * t, torch.float32)
    out = dict(stats=f[:8], logp=f[8 + 2 * t:8 + 3 * t], kl=f[8 + 3 * t:8 + 4 * t], entropy=f[8 + 4 * t:], grad=grad)
    a = PolicyLossArgs(_ptr(logits), _ptr(logits_ref), _ptr(actions), _ptr(logp_old), _ptr(advantages), _ptr(logp_ref),
                       _ptr(weights), _ld(logits), 0 if logits_ref is None else _ld(logits_ref),
                       0 if grad is None else _ld(grad), t, v, code, int(actions.dtype == torch.int64), float(low),
                       float(high), float(kl_coef), float(entropy_coef), _ptr(grad), _ptr(out["logp"]),
                       _ptr(out["kl"]), _ptr(out["entropy"]), _ptr(f), _ptr(f[8:]))
    with _on_device_of(logits):
        _check(library().accerl_policy_loss(C.byref(a), _stream_of(logits, stream)))
    return out


_ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}


def _check_ckpt(ckpt, rows, cols, like):
    """(q int8 [rows, >= cols32], e uint8 [rows, >= cols32 / 32]) as ckpt_save makes them."""
    import torch
    q, e = ckpt
    cols32 = -(-cols // 32) * 32
    _check_rows(q, like, torch.int8)
    _check_rows(e, like, torch.uint8)
    assert q.shape[0] == e.shape[0] == rows and q.shape[1] >= cols32 and e.shape[1] >= cols32 // 32, \
        "a checkpoint of %d rows of %d" % (rows, cols)
    return q, e


def ckpt_save(x, act="none", out=None, stream=None):
    """accerl_ckpt_save of CUDA rows x [T, K] (fp32, bf16, fp16): returns (y, (q, e)) with y = act(x), act one of "none"
    (y is x), "relu", "gelu", "silu".  ``out``: where to write y, x itself among the choices.  The checkpoint is
    q int8 [T, K32], e uint8 [T, K32 / 32], K32 = K rounded up to 32."""
    if out is None:
        r = (_CALLS or _calls()).ckpt_save(x, _ACTS[act], stream)
        if r is not None:
            return _done(r)
    import torch
    code = _dtype_code(x.dtype)
    _check_rows(x)
    t, k = int(x.shape[0]), int(x.shape[1])
    k32 = -(-k // 32) * 32
    memory = _Memory(x, stream)
    q, e = memory.result((t, k32), torch.int8), memory.result((t, k32 // 32), torch.uint8)
    if out is not None:
        _check_rows(out, x, x.dtype)
        assert out.shape == x.shape
    y = out if out is not None else x if act == "none" else memory.result((t, k), x.dtype)
    with _on_device_of(x):
        _check(library().accerl_ckpt_save(_ptr(x), _ld(x), code, t, k, _ACTS[act],
                                          None if act == "none" and out is None else _ptr(y), _ld(y), _ptr(q), k32, _ptr(e),
                                          k32 // 32, _stream_of(x, stream)))
    return y, (q, e)


def ckpt_load(ckpt, cols, dtype, out=None, stream=None):
    """accerl_ckpt_load: the values [T, cols] that a checkpoint stands for, in ``dtype`` (or into ``out``)."""
    if out is None:
        r = (_CALLS or _calls()).ckpt_load(ckpt, cols, dtype, stream)
        if r is not None:
            return _done(r)
    import torch
    t = int(ckpt[0].shape[0])
    if out is None:
        out = _Memory(ckpt[0], stream).result((t, cols), dtype)
    code = _dtype_code(out.dtype)
    _check_rows(out)
    assert out.dtype == dtype and tuple(out.shape) == (t, cols)
    q, e = _check_ckpt(ckpt, t, cols, out)
    with _on_device_of(out):
        _check(library().accerl_ckpt_load(_ptr(q), _ld(q), _ptr(e), _ld(e), t, cols, _ptr(out), _ld(out), code,
                                          _stream_of(out, stream)))
    return out


def ckpt_act_backward(dy, ckpt, act, out=None, stream=None):
    """accerl_ckpt_act_backward: dx = dy act'(x^) for CUDA rows dy [T, K]; ``out`` may be dy."""
    if out is None:
        r = (_CALLS or _calls()).ckpt_act_backward(dy, ckpt, _ACTS[act], stream)
        if r is not None:
            return _done(r)
    import torch
    code = _dtype_code(dy.dtype)
    _check_rows(dy)
    t, k = int(dy.shape[0]), int(dy.shape[1])
    q, e = _check_ckpt(ckpt, t, k, dy)
    if out is None:
        out = _Memory(dy, stream).result((t, k), dy.dtype)
    _check_rows(out, dy, dy.dtype)
    assert out.shape == dy.shape
    with _on_device_of(dy):
        _check(library().accerl_ckpt_act_backward(_ptr(dy), _ld(dy), code, _ptr(q), _ld(q), _ptr(e), _ld(e), t, k, _ACTS[act],
                                                  _ptr(out), _ld(out), _stream_of(dy, stream)))
    return out


class WeightGradArgs(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("dy", "q", "e", "dw", "db", "workspace")] + \
        [(n, C.c_int64) for n in ("ld_dy", "ld_q", "ld_e", "ld_dw", "workspace_bytes")] + \
        [(n, C.c_int32) for n in ("tokens", "n", "k", "dy_dtype", "out_dtype", "accumulate")]


def ckpt_weight_grad(dy, ckpt, cols, out_dtype=None, bias=True, out=None, accumulate=False, stream=None):
    """accerl_ckpt_weight_grad: (dw [N, K], db [N] or None) from CUDA rows dy [T, N] (bf16 or fp16) and the checkpoint of
    the layer's input [T, K = cols].  ``out_dtype`` fp32 or dy's type (the default); ``out`` = (dw, db) to write, or with
    ``accumulate`` (fp32) to add to; db None leaves it out, as does ``bias`` False."""
    if out is None and not accumulate:
        r = (_CALLS or _calls()).ckpt_weight_grad(dy, ckpt, cols, out_dtype, bias, stream)
        if r is not None:
            return _done(r)
    import torch
    code = _dtype_code(dy.dtype)
    _check_rows(dy)
    t, n, k = int(dy.shape[0]), int(dy.shape[1]), int(cols)
    q, e = _check_ckpt(ckpt, t, k, dy)
    assert out is not None or not accumulate, "accumulate adds to `out`"
    memory = _Memory(dy, stream)
    if out is None:
        dt = out_dtype or dy.dtype
        out = memory.result((n, k), dt), memory.result(n, dt) if bias else None
    dw, db = out
    _check_rows(dw, dy)
    assert tuple(dw.shape) == (n, k) and (out_dtype is None or dw.dtype == out_dtype)
    if db is not None:
        _check_vector(db, n, dy, dw.dtype)
    a = WeightGradArgs(_ptr(dy), _ptr(q), _ptr(e), _ptr(dw), _ptr(db), None, _ld(dy), _ld(q), _ld(e), _ld(dw), 0, t, n, k,
                       code, _dtype_code(dw.dtype), int(accumulate))
    lib = library()
    need = lib.accerl_ckpt_weight_grad_workspace(C.byref(a))
    mem = memory.workspace(need)
    if need:
        a.workspace, a.workspace_bytes = _ptr(mem), need
    with _on_device_of(dy):
        _check(lib.accerl_ckpt_weight_grad(C.byref(a), _stream_of(dy, stream)))
    return dw, db


class LinearI8Args(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("x", "x_scale", "w", "w_scale", "bias", "y", "workspace")] + \
        [(n, C.c_int64) for n in ("ld_x", "ld_w", "ld_y", "workspace_bytes")] + \
        [(n, C.c_int32) for n in ("tokens", "n", "k", "x_dtype", "y_dtype", "relu")]


def quant_rows(x, stream=None):
    """accerl_quant_rows of CUDA rows x [T, K] (fp32, bf16, fp16): (q int8 [T, K], scale fp32 [T]), one scale a row: the
    tokens of a batch of activations, or the channels of weights [out, in].  The rows of q start at multiples of 16
    bytes (its row stride is K rounded up to 16), as linear_i8 reads them."""
    r = (_CALLS or _calls()).quant_rows(x, stream)
    if r is not None:
        return _done(r)
    import torch
    code = _dtype_code(x.dtype)
    _check_rows(x)
    t, k = int(x.shape[0]), int(x.shape[1])
    k16 = -(-k // 16) * 16
    memory = _Memory(x, stream)
    q, scale = memory.result((t, k16), torch.int8), memory.result(t, torch.float32)
    with _on_device_of(x):
        _check(library().accerl_quant_rows(_ptr(x), _ld(x), code, t, k, _ptr(q), k16, _ptr(scale), _stream_of(x, stream)))
    return q[:, :k], scale


def _check_q_rows(q, scale, like):
    import torch
    _check_rows(q, like, torch.int8)
    _check_vector(scale, int(q.shape[0]), like, torch.float32)
    assert (q.stride(0) % 16 == 0 or q.shape[0] == 1) and q.data_ptr() % 16 == 0, "rows of q at multiples of 16 bytes (quant_rows)"


def _ld16(q):
    return q.stride(0) if q.shape[0] > 1 else -(-max(int(q.shape[1]), q.stride(0)) // 16) * 16


def linear_i8(x, weight, bias=None, relu=False, out_dtype=None, out=None, stream=None):
    """accerl_linear_i8: y [T, N] = (x quantised per token) times weight = (q int8 [N, K], scale fp32 [N]) as quant_rows
    makes it of [N, K], plus ``bias`` fp32 [N], through a ReLU where asked.  x is CUDA rows [T, K] (fp32, bf16, fp16),
    or a pair (q, scale) of quant_rows; y has x's type (fp32 for a pair) or ``out_dtype``, or is ``out``."""
    wq, ws = weight
    if out is None:
        r = (_CALLS or _calls()).linear_i8(x, wq, ws, bias, relu, out_dtype, stream)
        if r is not None:
            return _done(r)
    import torch
    given = isinstance(x, (tuple, list))
    xq, xs = x if given else (x, None)
    code = 3 if given else _dtype_code(xq.dtype)
    if given:
        _check_q_rows(xq, xs, xq)
    else:
        _check_rows(xq)
    _check_q_rows(wq, ws, xq)
    t, k, n = int(xq.shape[0]), int(xq.shape[1]), int(wq.shape[0])
    assert wq.shape[1] == k, "weights of rows of %d for tokens of %d" % (wq.shape[1], k)
    if bias is not None:
        _check_vector(bias, n, xq, torch.float32)
    memory = _Memory(xq, stream)
    if out is None:
        out = memory.result((t, n), out_dtype or (torch.float32 if given else xq.dtype))
    _check_rows(out, xq)
    assert tuple(out.shape) == (t, n) and (out_dtype is None or out.dtype == out_dtype)
    lib = library()
    need = lib.accerl_linear_i8_workspace(t, k, code)
    ws_mem = memory.workspace(need)
    a = LinearI8Args(_ptr(xq), _ptr(xs), _ptr(wq), _ptr(ws), _ptr(bias), _ptr(out), _ptr(ws_mem),
                     _ld16(xq) if given else _ld(xq), _ld16(wq), _ld(out), need, t, n, k, code, _dtype_code(out.dtype), int(relu))
    with _on_device_of(xq):
        _check(lib.accerl_linear_i8(C.byref(a), _stream_of(xq, stream)))
    return out


def device_check():
    """accerl_device_check: waits for the current device; raises if a bounded wait of these operators gave up."""
    _check(library().accerl_device_check())


class Policy:
    """An int8 policy resident on one GPU.

    ``policy`` is a dict with ``in_kind`` ("u8" | "f32"), ``in_shape`` (C, H, W),
    ``s_input`` and ``layers``: dicts with kind, in_c, in_h, in_w, out_c, kh, kw, stride, pad,
    relu_in, relu_out, logits, skip_from, s_in, s_out and numpy arrays w (int8 OIHW), s_w, bias,
    skip_mul (or None).
    """

    @classmethod
    def from_fp32(cls, in_kind: str, in_shape, layers, params, calib_obs, max_batch: int,
                  prune24: bool = False, flags: int = 0, device: int = 0) -> "Policy":
        """accerl_policy_create_fp32: quantise and calibrate on the device.  ``layers`` are
        architecture dicts, ``params`` the matching fp32 {w, bias} (None for max-pool)."""
        lib = library()
        self = cls.__new__(cls)
        self._h = C.c_void_p()
        n = len(layers)
        descs = (LayerFp32 * n)()
        keep = []
        for i, (l, pr) in enumerate(zip(layers, params)):
            d = descs[i]
            d.kind = _KINDS[l["kind"]]
            d.flags = (RELU_IN if l["relu_in"] else 0) | (RELU_OUT if l["relu_out"] else 0) | \
                (LOGITS if l["logits"] else 0)
            for k in ("in_c", "in_h", "in_w", "out_c", "kh", "kw", "stride", "pad", "skip_from"):
                setattr(d, k, int(l[k]))
            if pr is not None:
                w, b = np.ascontiguousarray(pr["w"], np.float32), np.ascontiguousarray(pr["bias"], np.float32)
                keep += [w, b]
                d.w, d.bias = w.ctypes.data, b.ctypes.data
        shape = (C.c_int32 * 3)(*[int(v) for v in in_shape])
        calib = np.ascontiguousarray(calib_obs, np.uint8 if in_kind == "u8" else np.float32)
        self.layers = [dict(l) for l in layers]
        self.in_kind, self.in_shape = in_kind, tuple(int(v) for v in in_shape)
        self.max_batch, self.device = int(max_batch), int(device)
        self.value_head = bool(layers[-1].get("value"))
        if self.value_head:
            flags = int(flags) | FLAG_VALUE_HEAD
        _check(lib.accerl_policy_create_fp32(C.byref(self._h), 0 if in_kind == "u8" else 1, shape, descs, n,
                                             calib.ctypes.data, int(calib.shape[0]), int(bool(prune24)),
                                             self.max_batch, int(flags), self.device))
        self._raw = self._h.value
        self.n_actions = int(layers[-1]["out_c"]) - (1 if self.value_head else 0)
        return self

    def export(self, layer: int) -> dict:
        """accerl_policy_export: the quantised parameters of one layer of a from_fp32 policy."""
        l = self.layers[layer]
        s_in, s_out = C.c_float(), C.c_float()
        if l["kind"] == "maxpool":
            _check(library().accerl_policy_export(self._h, layer, None, 0, None, None, C.byref(s_in), C.byref(s_out)))
            return dict(w=None, s_w=None, skip_mul=None, s_in=np.float32(s_in.value), s_out=np.float32(s_out.value))
        w = np.empty((l["out_c"], l["in_c"], l["kh"], l["kw"]), np.int8)
        s_w = np.empty(l["out_c"], np.float32)
        sm = np.empty(l["out_c"], np.int32) if l["skip_from"] >= 0 else None
        _check(library().accerl_policy_export(self._h, layer, w.ctypes.data, w.nbytes, s_w.ctypes.data,
                                              None if sm is None else sm.ctypes.data, C.byref(s_in),
                                              C.byref(s_out)))
        return dict(w=w, s_w=s_w, skip_mul=sm, s_in=np.float32(s_in.value), s_out=np.float32(s_out.value))

    def __init__(self, policy: dict, max_batch: int, flags: int = 0, device: int = 0):
        lib = library()
        self._h = C.c_void_p()
        self.layers = policy["layers"]
        n = len(self.layers)
        descs = (LayerDesc * n)()
        keep = []  # host arrays must outlive the create call only
        for i, l in enumerate(self.layers):
            d = descs[i]
            d.kind = _KINDS[l["kind"]]
            d.flags = (RELU_IN if l["relu_in"] else 0) | (RELU_OUT if l["relu_out"] else 0) | \
                (LOGITS if l["logits"] else 0)
            for k in ("in_c", "in_h", "in_w", "out_c", "kh", "kw", "stride", "pad", "skip_from"):
                setattr(d, k, int(l[k]))
            d.s_in, d.s_out = float(l["s_in"]), float(l["s_out"])
            for k, dt in (("w", np.int8), ("s_w", np.float32), ("bias", np.float32),
                          ("skip_mul", np.int32)):
                if l.get(k) is not None:
                    a = np.ascontiguousarray(l[k], dt)
                    keep.append(a)
                    setattr(d, k, a.ctypes.data)
        shape = (C.c_int32 * 3)(*[int(v) for v in policy["in_shape"]])
        self.in_kind = policy["in_kind"]
        self.in_shape = tuple(int(v) for v in policy["in_shape"])
        self.max_batch = int(max_batch)
        self.device = int(device)
        if self.layers[-1].get("value"):
            flags = int(flags) | FLAG_VALUE_HEAD
        _check(lib.accerl_policy_create(C.byref(self._h), 0 if self.in_kind == "u8" else 1, shape,
                                        float(policy["s_input"]), descs, n, self.max_batch,
                                        int(flags), self.device))
        self._raw = self._h.value
        self.value_head = bool(self.layers[-1].get("value"))
        self.n_actions = int(self.layers[-1]["out_c"]) - (1 if self.value_head else 0)

    # -- the hot call ---------------------------------------------------------------------
    def act(self, obs, uniforms, out=None, stream=None):
        """obs, uniforms: CUDA torch tensors.  Returns (logits, actions, logp) CUDA tensors."""
        r = (_CALLS or _calls()).act(self._raw, self.n_actions, self.in_kind == "u8", obs, uniforms, out, stream)
        if r is not None:
            return _done(r)
        # not what the native call takes: say what is wrong, or go through ctypes
        import torch
        b = int(obs.shape[0])
        if out is None:
            memory = _Memory(obs, stream)
            out = (memory.result((b, self.n_actions), torch.float32), memory.result(b, torch.int32),
                   memory.result(b, torch.float32))
        if stream is None:
            stream = torch.cuda.current_stream(obs.device).cuda_stream
        assert obs.is_contiguous() and uniforms.is_contiguous() and obs.is_cuda and uniforms.is_cuda
        assert obs.dtype == (torch.uint8 if self.in_kind == "u8" else torch.float32)
        assert uniforms.dtype == torch.float32 and uniforms.numel() == b
        _check(library().accerl_policy_act(self._h, obs.data_ptr(), uniforms.data_ptr(), b,
                                           out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(),
                                           stream))
        return out

    def act_ex(self, obs, uniforms, stream=None) -> dict:
        """accerl_policy_act_ex: dict(logits, actions, logp, entropy[, value]) of CUDA tensors."""
        r = (_CALLS or _calls()).act_ex(self._raw, self.n_actions, self.in_kind == "u8", self.value_head, obs, uniforms,
                                        stream)
        if r is not None:
            return _done(r)
        import torch
        _check_batch(self.in_kind == "u8", obs, uniforms)
        b, memory = int(obs.shape[0]), _Memory(obs, stream)
        out = dict(logits=memory.result((b, self.n_actions), torch.float32), actions=memory.result(b, torch.int32),
                   logp=memory.result(b, torch.float32), entropy=memory.result(b, torch.float32))
        if self.value_head:
            out["value"] = memory.result(b, torch.float32)
        _check(library().accerl_policy_act_ex(
            self._h, obs.data_ptr(), uniforms.data_ptr(), b, out["logits"].data_ptr(),
            out["actions"].data_ptr(), out["logp"].data_ptr(),
            out["value"].data_ptr() if self.value_head else None, out["entropy"].data_ptr(),
            _stream_of(obs, stream)))
        return out

    def act_timed(self, obs, uniforms, out, stream=None) -> np.ndarray:
        """One step with CUDA events around every launch; returns milliseconds per launch."""
        import torch
        if stream is None:
            stream = torch.cuda.current_stream(obs.device).cuda_stream
        n = self.info()["launches_per_act"]
        ms = np.zeros(n, np.float32)
        _check(library().accerl_policy_act_timed(self._h, obs.data_ptr(), uniforms.data_ptr(),
                                                 int(obs.shape[0]), out[0].data_ptr(),
                                                 out[1].data_ptr(), out[2].data_ptr(), stream,
                                                 ms.ctypes.data, n))
        return ms

    def act_noalloc_raw(self, obs_ptr, u_ptr, batch, logits_ptr, actions_ptr, logp_ptr,
                        stream=0) -> int:
        """accerl_policy_act_noalloc with raw device addresses; returns the status code."""
        r = (_CALLS or _calls()).act_noalloc(self._raw, obs_ptr, u_ptr, batch, logits_ptr, actions_ptr, logp_ptr,
                                             stream)
        if r is not None:
            return r
        return library().accerl_policy_act_noalloc(self._h, obs_ptr, u_ptr, batch, logits_ptr, actions_ptr, logp_ptr,
                                                   stream)

    def act_raw(self, obs_ptr, u_ptr, batch, logits_ptr, actions_ptr, logp_ptr, stream=0) -> int:
        """Unchecked pass-through returning the status code (for ABI tests)."""
        return library().accerl_policy_act(self._h, obs_ptr, u_ptr, batch, logits_ptr, actions_ptr,
                                           logp_ptr, stream)

    def act_host(self, obs, uniforms, out, stream=0):
        """obs, uniforms, out=(logits, actions, logp): host tensors/arrays (pinned is faster)."""
        ptr = lambda a: a.data_ptr() if hasattr(a, "data_ptr") else a.ctypes.data  # noqa: E731
        _check(library().accerl_policy_act_host(self._h, ptr(obs), ptr(uniforms), int(obs.shape[0]),
                                                ptr(out[0]), ptr(out[1]), ptr(out[2]), stream))
        return out

    # -- parity taps and introspection --------------------------------------------------------
    def read_activation(self, layer: int, batch: int) -> np.ndarray:
        if layer < 0:
            shape = (batch,) + self.in_shape
        else:
            l = self.layers[layer]
            shape = (batch, l["out_c"]) + _out_hw(l)
        dst = np.empty(shape, np.int8)
        _check(library().accerl_policy_read_activation(self._h, layer, batch, dst.ctypes.data,
                                                       dst.nbytes))
        return dst

    def check(self):
        _check(library().accerl_policy_check(self._h))

    def selftest_wait(self, poll_limit: int = 200, stream=0):
        """accerl_policy_selftest_wait: makes a bounded device-side wait run out on purpose."""
        _check(library().accerl_policy_selftest_wait(self._h, poll_limit, stream))

    def info(self, batch: int | None = None) -> dict:
        na, ws, nl = C.c_int32(), C.c_size_t(), C.c_int32()
        buf = C.create_string_buffer(1 << 16)
        _check(library().accerl_policy_info(self._h, batch or self.max_batch, C.byref(na),
                                            C.byref(ws), C.byref(nl), buf, len(buf)))
        return dict(n_actions=na.value, workspace_bytes=ws.value, launches_per_act=nl.value,
                    plan=buf.value.decode())

    def close(self):
        if self._h:
            library().accerl_policy_destroy(self._h)
            self._h = C.c_void_p()
            self._raw = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
