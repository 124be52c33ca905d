"""Thin ctypes binding over libbagel.so (C ABI in include/bagel.h).

Argument marshalling only: every function below checks shapes / dtypes / device of the torch
tensors it is given and passes their device pointers through.  PyTorch supplies device memory
and the stream; all computation happens inside the library's HIP kernels.  There is no
fallback: if the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbagel.so")

OK, EINVAL, ENOTPREPARED, ENOMEM, ENOTPD, EHIP = 0, -1, -2, -3, -4, -5
_NAMES = {EINVAL: "BAGEL_EINVAL", ENOTPREPARED: "BAGEL_ENOTPREPARED", ENOMEM: "BAGEL_ENOMEM",
          ENOTPD: "BAGEL_ENOTPD", EHIP: "BAGEL_EHIP"}

EXPORTS = ["bagel_num_params", "bagel_create", "bagel_destroy", "bagel_workspace_bytes",
           "bagel_prepare_samples", "bagel_set_samples", "bagel_rollout_loss",
           "bagel_rollout_loss_grad", "bagel_sample_eval", "bagel_last_error", "bagel_adam_step", "bagel_optimize",
           "bagel_hyper_lml_grad", "bagel_hyper_fit", "bagel_prepare_posterior", "bagel_posterior_rollout_loss", "bagel_posterior_rollout_loss_grad",
           "bagel_profile_enable", "bagel_profile_read", "bagel_sample_eval_static",
           "bagel_block_join", "bagel_block_join_grad", "bagel_block_join_workspace",
           "bagel_recurrence", "bagel_recurrence_grad", "bagel_recurrence_step", "bagel_recurrence_workspace",
           "bagel_recurrence_carry_rows", "bagel_adamw_step"]


class BagelError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{_NAMES.get(code, code)}: {msg}")
        self.code = code


class Dims(C.Structure):
    _fields_ = [
        ("d_s", C.c_int32), ("d_a", C.c_int32), ("d_g", C.c_int32),
        ("N", C.c_int32), ("L", C.c_int32), ("S", C.c_int32), ("B", C.c_int32), ("H", C.c_int32),
        ("n_hidden", C.c_int32), ("hidden", C.c_int32 * 2),
        ("act_bound", C.c_float),
        ("tracked", C.c_int32 * 8), ("q", C.c_float * 8),
        ("ckpt_interval", C.c_int32), ("cost_kind", C.c_int32), ("sigma_r", C.c_float),
    ]


def make_dims(*, d_s, d_a, d_g, N, L, S, B, H, hidden: Sequence[int], act_bound=0.0, tracked=None,
              q=None, ckpt_interval=0, cost_kind=0, sigma_r=1.0) -> Dims:
    dm = Dims()
    dm.d_s, dm.d_a, dm.d_g = d_s, d_a, d_g
    dm.N, dm.L, dm.S, dm.B, dm.H = N, L, S, B, H
    dm.n_hidden = len(hidden)
    for i, h in enumerate(list(hidden)[:2]):
        dm.hidden[i] = h
    dm.act_bound = float(act_bound)
    tracked = list(range(d_g)) if tracked is None else list(tracked)
    q = [1.0] * d_g if q is None else list(q)
    for j in range(min(d_g, 8)):
        dm.tracked[j] = tracked[j]
        dm.q[j] = q[j]
    dm.ckpt_interval, dm.cost_kind, dm.sigma_r = ckpt_interval, cost_kind, float(sigma_r)
    return dm


def dims_from_config(cfg, S: Optional[int] = None, **kw) -> Dims:
    kw.setdefault("ckpt_interval", cfg.ckpt_interval)
    return make_dims(d_s=cfg.d_s, d_a=cfg.d_a, d_g=cfg.d_g, N=cfg.N, L=cfg.L,
                     S=cfg.B if S is None else S, B=cfg.B, H=cfg.H, hidden=cfg.hidden,
                     act_bound=cfg.act_bound, tracked=cfg.tracked, q=cfg.q, **kw)


def _matrices(*names):
    return [f for n in names for f in ((n, C.c_void_p), (n + "_stride", C.c_int64))]


class _Join(C.Structure):
    _fields_ = [("rows", C.c_int64), ("width", C.c_int32), ("dtype", C.c_int32), ("act", C.c_int32), ("eps", C.c_float),
                *_matrices("branch", "gate", "resid", "out", "normed"),
                ("post_weight", C.c_void_p), ("scale", C.c_void_p), ("pre_weight", C.c_void_p),
                *_matrices("d_out", "d_normed", "d_branch", "d_gate", "d_resid"),
                ("d_post_weight", C.c_void_p), ("d_scale", C.c_void_p), ("d_pre_weight", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)]


class _Recurrence(C.Structure):
    _fields_ = [("rows", C.c_int64), ("width", C.c_int32), ("dtype", C.c_int32), ("sequences", C.c_int32), ("offsets", C.c_void_p),
                *_matrices("value", "forget", "hidden"),
                ("bias", C.c_void_p), ("initial", C.c_void_p), ("final", C.c_void_p), ("carry", C.c_void_p), ("state", C.c_void_p),
                *_matrices("d_hidden", "d_value", "d_forget"),
                ("d_final", C.c_void_p), ("d_initial", C.c_void_p), ("d_bias", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)]


class _AdamWTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("copy", C.c_void_p), ("count", C.c_int64), ("weight_decay", C.c_double)]


class _AdamW(C.Structure):
    _fields_ = [("step", C.c_int64), ("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("grad_scale", C.c_void_p), ("grad_dtype", C.c_int32), ("copy_dtype", C.c_int32), ("state_bits", C.c_int32),
                ("seed", C.c_uint32), ("draws", C.c_int32)]


_lib = None


def load():
    """Load libbagel.so; raises if it has not been built (python -m paper_2202_13638_amd.build)."""
    global _lib
    if _lib is None:
        # torch first: the library must bind to the HIP runtime that torch has already loaded, so
        # that device pointers and streams handed over belong to the same runtime instance
        import torch  # noqa: F401
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2202_13638_amd.build`")
        L = C.CDLL(LIB_PATH)
        fp, vp = C.c_void_p, C.c_void_p
        L.bagel_num_params.restype = C.c_int
        L.bagel_num_params.argtypes = [C.POINTER(Dims)]
        L.bagel_create.restype = C.c_int
        L.bagel_create.argtypes = [C.POINTER(vp), C.POINTER(Dims), vp]
        L.bagel_destroy.restype = C.c_int
        L.bagel_destroy.argtypes = [vp]
        L.bagel_workspace_bytes.restype = C.c_int64
        L.bagel_workspace_bytes.argtypes = [vp]
        L.bagel_prepare_samples.restype = C.c_int
        L.bagel_prepare_samples.argtypes = [vp] + [fp] * 10
        L.bagel_set_samples.restype = C.c_int
        L.bagel_set_samples.argtypes = [vp] + [fp] * 7
        L.bagel_rollout_loss.restype = C.c_int
        L.bagel_rollout_loss.argtypes = [vp] + [fp] * 6
        L.bagel_rollout_loss_grad.restype = C.c_int
        L.bagel_rollout_loss_grad.argtypes = [vp] + [fp] * 8
        L.bagel_sample_eval.restype = C.c_int
        L.bagel_sample_eval.argtypes = [vp] + [fp] * 3
        L.bagel_profile_enable.restype = C.c_int
        L.bagel_profile_enable.argtypes = [vp, C.c_int]
        L.bagel_profile_read.restype = C.c_int
        L.bagel_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_int)]
        L.bagel_prepare_posterior.restype = C.c_int
        L.bagel_prepare_posterior.argtypes = [vp] + [fp] * 5
        L.bagel_posterior_rollout_loss.restype = C.c_int
        L.bagel_posterior_rollout_loss.argtypes = [vp] + [fp] * 7
        L.bagel_posterior_rollout_loss_grad.restype = C.c_int
        L.bagel_posterior_rollout_loss_grad.argtypes = [vp] + [fp] * 9
        L.bagel_hyper_lml_grad.restype = C.c_int
        L.bagel_hyper_lml_grad.argtypes = [vp] + [fp] * 5
        L.bagel_hyper_fit.restype = C.c_int
        L.bagel_hyper_fit.argtypes = [vp] + [fp] * 5 + [C.c_int] * 2 + [C.c_float] * 4 + [fp]
        L.bagel_adam_step.restype = C.c_int
        L.bagel_adam_step.argtypes = [vp] + [fp] * 4 + [C.c_int] + [C.c_float] * 4
        L.bagel_optimize.restype = C.c_int
        L.bagel_optimize.argtypes = [vp] + [fp] * 5 + [C.c_int] * 3 + [C.c_float] * 4 + [fp]
        L.bagel_sample_eval_static.restype = C.c_int
        L.bagel_sample_eval_static.argtypes = [C.POINTER(Dims), vp] + [fp] * 10
        L.bagel_block_join_workspace.restype = L.bagel_recurrence_workspace.restype = L.bagel_recurrence_carry_rows.restype = C.c_int64
        L.bagel_block_join_workspace.argtypes = L.bagel_recurrence_workspace.argtypes = [C.c_int64, C.c_int32]
        L.bagel_recurrence_carry_rows.argtypes = [C.c_int64]
        for name in ("bagel_block_join", "bagel_block_join_grad", "bagel_recurrence", "bagel_recurrence_grad", "bagel_recurrence_step"):
            getattr(L, name).restype, getattr(L, name).argtypes = C.c_int, [vp, vp]
        L.bagel_adamw_step.restype = C.c_int
        L.bagel_adamw_step.argtypes = [vp, C.c_int32, vp, vp]
        L.bagel_last_error.restype = C.c_char_p
        L.bagel_last_error.argtypes = [vp]
        # The message is thread-local.  Until a thread has touched it, glibc looks up the thread-local data of every library the long way, the
        # HIP runtime's too: 0.27 us of a launch.
        L.bagel_last_error(None)
        _lib = L
    return _lib


def bagel_num_params(dims: Dims) -> int:
    return int(load().bagel_num_params(C.byref(dims)))


_Tensor = _float32 = None        # torch's, looked up once: a call checks up to eleven tensors


def _ptr(t, shape, name, optional=False):
    global _Tensor, _float32
    if t is None:
        if optional:
            return None
        raise ValueError(f"{name} is required")
    if _float32 is None:         # (the one that is set last: another thread may come in between)
        from torch import Tensor as _Tensor, float32 as _float32
    if not isinstance(t, _Tensor) or not t.is_cuda or t.dtype is not _float32 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 tensor on the GPU")
    if t.shape != shape and tuple(t.shape) != tuple(shape):      # (the tuples are made only for what is no tuple itself)
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t.data_ptr()


def bagel_sample_eval_static(dims: Dims, X, lengthscale, signal_var, omega, phase, w, v, x, f, jac=None, stream=None):
    """The context-free, allocation-free sample evaluation (see include/bagel.h)."""
    import torch
    lib = load()
    M, D = dims.d_s, dims.d_s + dims.d_a
    if stream is None:
        stream = torch.cuda.current_stream()
    rc = lib.bagel_sample_eval_static(
        C.byref(dims), C.c_void_p(stream.cuda_stream), _ptr(X, (dims.N, D), "X"),
        _ptr(lengthscale, (M, D), "lengthscale"), _ptr(signal_var, (M,), "signal_var"),
        _ptr(omega, (M, dims.L, D), "omega"), _ptr(phase, (M, dims.L), "phase"), _ptr(w, (dims.S, M, dims.L), "w"),
        _ptr(v, (dims.S, M, dims.N), "v"), _ptr(x, (dims.B, D), "x"), _ptr(f, (dims.B, M), "f"),
        _ptr(jac, (dims.B, M, D), "jac", optional=True))
    if rc != OK:
        raise BagelError(rc, lib.bagel_last_error(None).decode())


# ---------------------------------------------------------------------------- operators of a policy with memory
# Outputs are tensors of the caller; what is None is left out.  `stream` None: torch's current one.  All tensors are on the current device.
# Calls of a few rows take as long on the host as on the GPU, so the tensors are checked and packed by compiled code (csrc/marshal.cpp), which
# makes the structures above as bytes.
JOIN_MAX_WIDTH, RECURRENCE_SPAN, ADAMW_BLOCK = 16384, 128, 256
_ACTS = {"none": 0, "identity": 1, "logistic": 2, "silu": 3}
_JOIN_HEAD, _RECURRENCE_HEAD, _ADAMW_OPTIONS, _WORKSPACE = (struct.Struct(f) for f in ("qiiif", "qiii4xP", "qddddPiiiIi4x", "Pq"))
assert (_JOIN_HEAD.size, _RECURRENCE_HEAD.size, _ADAMW_OPTIONS.size) == (_Join.branch.offset, _Recurrence.value.offset, C.sizeof(_AdamW))
_NOTHING = bytes(256)
_JOIN_FIELDS, _RECURRENCE_FIELDS = ("rows", "width", "dtype", "act", "eps"), ("rows", "width", "dtype", "offsets", "offsets")
_STEP_FIELDS, _ADAMW_FIELDS = ("", "width", "dtype", "rows"), ("step", "lr", "beta1", "beta2", "eps", "grad_scale", "grads", "copy", "m")
_torch = _marshal = _raw_stream = None


def _load():
    """The library, with torch and the compiled checks looked up once."""
    global _torch, _marshal, _raw_stream
    if _raw_stream is None:
        import torch as _torch
        from . import _marshal
        # the handle of the current stream, in 0.1 us where torch.cuda.current_stream() takes 2.7
        _raw_stream = getattr(_torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: _torch.cuda.current_stream(device).cuda_stream)
    return _lib or load()


_UNFIT = (struct.error, OverflowError, TypeError, ValueError)


def _unfit(form, fields, *values):
    """What is wrong with values that could not be packed: a ValueError that names the first of them that does not fit its field."""
    for code, name, value in zip((c for c in form.format if c in "qifdPI"), fields, values):
        try:
            struct.pack(code, value if code in "fd" else int(value) & 0xFFFFFFFF if code == "I" else int(value))
        except _UNFIT:
            return ValueError(f"{name} must be a {'number' if code in 'fd' else 'whole number'} that fits its field, not {value!r}")
    return ValueError("an argument does not fit its field")


def _stream(stream):
    """(handle of the call's stream, current device)"""
    device = _torch.cuda.current_device() if _torch.cuda.is_initialized() or _torch.cuda.is_available() else -1
    if stream is None:
        return _raw_stream(device) if device >= 0 else 0, device
    if stream.device_index != device:
        raise ValueError("the stream must be one of the current GPU")
    return stream.cuda_stream, device


def _workspace(workspace, need, device, stream):
    """The caller's work space, or one from torch's allocator on the call's stream (`stream` as the caller gave it)."""
    if workspace is None:
        if need <= 0:                                                 # none, or sizes that the library refuses
            return None, bytes(16)
        if stream is None:
            workspace = _torch.empty(need, dtype=_torch.uint8, device=device)
        else:
            with _torch.cuda.stream(stream):
                workspace = _torch.empty(need, dtype=_torch.uint8, device=device)
    elif not isinstance(workspace, _torch.Tensor) or workspace.dtype != _torch.uint8 or not workspace.is_contiguous() or workspace.get_device() != device:
        raise ValueError(f"workspace must be a contiguous uint8 tensor on cuda:{device}")
    return workspace, _WORKSPACE.pack(workspace.data_ptr(), workspace.numel())


def _done(lib, rc):
    if rc != OK:
        raise BagelError(rc, lib.bagel_last_error(None).decode())


def bagel_block_join_workspace(rows: int, width: int) -> int:
    """Bytes of work space of bagel_block_join_grad."""
    return int(load().bagel_block_join_workspace(rows, width))


def _act(act):
    if act not in _ACTS:
        raise ValueError(f"act must be one of {sorted(_ACTS)}")
    return _ACTS[act]


_FORWARD, _BACKWARD = ("branch", "gate", "resid", "out", "normed"), ("d_out", "d_normed", "d_branch", "d_gate", "d_resid")
_VECTORS, _D_VECTORS = ("post_weight", "scale", "pre_weight"), ("d_post_weight", "d_scale", "d_pre_weight")


def bagel_block_join(branch, resid, out=None, normed=None, *, gate=None, act="none", post_weight=None, scale=None, pre_weight=None, eps=1e-6,
                     stream=None):
    """out = resid + scale * act(gate) * (R(branch) * post_weight), normed = R(out) * pre_weight (see include/bagel.h)."""
    lib = _load()
    kind = _act(act)
    on, device = _stream(stream)
    like, name = (resid, "resid") if resid is not None else (branch, "branch")
    rows, width, code = _marshal.first(like, name, device)
    try:
        head = _JOIN_HEAD.pack(rows, width, code, kind, eps)
    except _UNFIT:
        raise _unfit(_JOIN_HEAD, _JOIN_FIELDS, rows, width, code, kind, eps) from None
    args = (head + _marshal.matrices(like, _FORWARD, (branch, gate, resid, out, normed)) +
            _marshal.vectors(device, (width,), _VECTORS, (post_weight, scale, pre_weight)) + _NOTHING)
    _done(lib, lib.bagel_block_join(args, on))


def bagel_block_join_grad(branch, out, d_out=None, d_normed=None, *, gate=None, act="none", post_weight=None, scale=None, pre_weight=None,
                          eps=1e-6, d_branch=None, d_gate=None, d_resid=None, d_post_weight=None, d_scale=None, d_pre_weight=None,
                          workspace=None, stream=None):
    """The gradient of bagel_block_join at the `out` it stored (see include/bagel.h)."""
    lib = _load()
    kind = _act(act)
    on, device = _stream(stream)
    rows, width, code = _marshal.first(out, "out", device)
    sums = d_post_weight is not None or d_scale is not None or d_pre_weight is not None
    workspace, space = _workspace(workspace, lib.bagel_block_join_workspace(rows, width) if sums else 0, device, stream)
    try:
        head = _JOIN_HEAD.pack(rows, width, code, kind, eps)
    except _UNFIT:
        raise _unfit(_JOIN_HEAD, _JOIN_FIELDS, rows, width, code, kind, eps) from None
    args = (head + _marshal.matrices(out, _FORWARD, (branch, gate, None, out, None)) +
            _marshal.vectors(device, (width,), _VECTORS, (post_weight, scale, pre_weight)) +
            _marshal.matrices(out, _BACKWARD, (d_out, d_normed, d_branch, d_gate, d_resid)) +
            _marshal.vectors(device, (width,), _D_VECTORS, (d_post_weight, d_scale, d_pre_weight)) + space)
    _done(lib, lib.bagel_block_join_grad(args, on))


def bagel_recurrence_carry_rows(rows: int) -> int:
    """Rows of `carry`, the part of the forward pass that bagel_recurrence_grad needs, for so many rows of activations."""
    return int(load().bagel_recurrence_carry_rows(rows))


def bagel_recurrence_workspace(rows: int, width: int) -> int:
    """Bytes of work space of bagel_recurrence and bagel_recurrence_grad."""
    return int(load().bagel_recurrence_workspace(rows, width))


def _sequences(offsets, device):
    """(number of sequences, pointer of their offsets): an int32 tensor on the GPU, or the number of sequences of equal length."""
    if not isinstance(offsets, _torch.Tensor):
        try:
            return int(offsets), 0
        except _UNFIT:
            raise ValueError(f"offsets must be an int32 tensor or the number of sequences, not {offsets!r}") from None
    if offsets.dtype != _torch.int32 or offsets.dim() != 1 or offsets.numel() < 1 or not offsets.is_contiguous() or offsets.get_device() != device:
        raise ValueError(f"offsets must be a contiguous int32 tensor of one dimension on cuda:{device}, or the number of sequences")
    return offsets.numel() - 1, offsets.data_ptr()


def _needed(t, name):
    if t is None:
        raise ValueError(f"{name} is required")
    return t


def bagel_recurrence(value, forget, hidden, offsets, *, bias=None, initial=None, final=None, carry=None, workspace=None, stream=None):
    """h_t = h_{t-1} + q_t (value_t - h_{t-1}), q_t = 1 / (1 + exp(forget_t + bias)), along packed sequences (see include/bagel.h)."""
    lib = _load()
    on, device = _stream(stream)
    rows, width, code = _marshal.first(value, "value", device)
    n, at = _sequences(offsets, device)
    workspace, space = _workspace(workspace, lib.bagel_recurrence_workspace(rows, width), device, stream)
    try:
        head = _RECURRENCE_HEAD.pack(rows, width, code, n, at)
    except _UNFIT:
        raise _unfit(_RECURRENCE_HEAD, _RECURRENCE_FIELDS, rows, width, code, n, at) from None
    args = (head +
            _marshal.matrices(value, ("value", "forget", "hidden"), (value, _needed(forget, "forget"), _needed(hidden, "hidden"))) +
            _marshal.vectors(device, (width,), ("bias",), (bias,)) + _marshal.vectors(device, (n, width), ("initial", "final"), (initial, final)) +
            _marshal.vectors(device, (lib.bagel_recurrence_carry_rows(rows), width), ("carry",), (carry,)) + bytes(8 + 3 * 16 + 3 * 8) + space)
    _done(lib, lib.bagel_recurrence(args, on))


def bagel_recurrence_grad(value, forget, d_hidden, d_value, d_forget, offsets, carry, *, bias=None, initial=None, d_final=None, d_initial=None,
                          d_bias=None, workspace=None, stream=None):
    """The gradient of bagel_recurrence, with the `carry` it wrote (see include/bagel.h)."""
    lib = _load()
    on, device = _stream(stream)
    rows, width, code = _marshal.first(value, "value", device)
    n, at = _sequences(offsets, device)
    workspace, space = _workspace(workspace, lib.bagel_recurrence_workspace(rows, width), device, stream)
    try:
        head = _RECURRENCE_HEAD.pack(rows, width, code, n, at)
    except _UNFIT:
        raise _unfit(_RECURRENCE_HEAD, _RECURRENCE_FIELDS, rows, width, code, n, at) from None
    args = (head +
            _marshal.matrices(value, ("value", "forget", "hidden"), (value, _needed(forget, "forget"), None)) +
            _marshal.vectors(device, (width,), ("bias",), (bias,)) + _marshal.vectors(device, (n, width), ("initial", "final"), (initial, None)) +
            _marshal.vectors(device, (lib.bagel_recurrence_carry_rows(rows), width), ("carry",), (_needed(carry, "carry"),)) + bytes(8) +
            _marshal.matrices(value, ("d_hidden", "d_value", "d_forget"), (_needed(d_hidden, "d_hidden"), d_value, d_forget)) +
            _marshal.vectors(device, (n, width), ("d_final", "d_initial"), (d_final, d_initial)) +
            _marshal.vectors(device, (width,), ("d_bias",), (d_bias,)) + space)
    _done(lib, lib.bagel_recurrence_grad(args, on))


def bagel_recurrence_step(value, forget, state, hidden=None, *, bias=None, stream=None):
    """One step of as many sequences as there are rows, the float32 state updated in place (see include/bagel.h)."""
    lib = _load()
    on, device = _stream(stream)
    rows, width, code = _marshal.first(value, "value", device)
    try:
        head = _RECURRENCE_HEAD.pack(0, width, code, rows, 0)
    except _UNFIT:
        raise _unfit(_RECURRENCE_HEAD, _STEP_FIELDS, 0, width, code, rows, 0) from None
    args = (head +
            _marshal.matrices(value, ("value", "forget", "hidden"), (value, _needed(forget, "forget"), hidden)) +
            _marshal.vectors(device, (width,), ("bias",), (bias,)) + bytes(3 * 8) +
            _marshal.vectors(device, (rows, width), ("state",), (_needed(state, "state"),)) + _NOTHING)
    _done(lib, lib.bagel_recurrence_step(args, on))


def bagel_adamw_step(params, grads, m, v, step, *, m_scale=None, v_scale=None, copy=None, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8,
                     weight_decay=0.01, grad_scale=None, seed=None, run=0, stream=None):
    """One update of a list of tensors (see include/bagel.h).

    params: contiguous float32 tensors; grads, m, v, copy (None: none): lists of tensors of the same shapes.  grads are all of one
    type, and so are the entries of copy.  m and v are float32, or float8_e4m3fn with m_scale and v_scale, lists of float32 tensors
    with an entry for every ADAMW_BLOCK values.  weight_decay: a number, or one for every tensor.

    The draws that round moments in 8 bits are independent from place to place, tensor to tensor and update to update.  `run` tells runs apart, and
    calls that share an update.  seed: for a caller that computes the draws itself (see BAGEL_DRAWS_GIVEN), another one for every update."""
    lib = _load()
    on, device = _stream(stream)
    n, table, grad_type, copy_type, bits = _marshal.adamw(device, params, grads, m, v, m_scale, v_scale, copy, weight_decay)
    scale = 0
    if grad_scale is not None:
        if not isinstance(grad_scale, _torch.Tensor) or grad_scale.numel() != 1 or grad_scale.dtype != _torch.float32 or grad_scale.get_device() != device:
            raise ValueError("grad_scale must hold one float32 value and be on the current GPU")
        scale = grad_scale.data_ptr()
    draws, given = (run, 0) if seed is None else (seed, 1)
    try:
        options = _ADAMW_OPTIONS.pack(int(step), lr, beta1, beta2, eps, scale, grad_type, copy_type, bits, int(draws) & 0xFFFFFFFF, given)
    except _UNFIT:
        fields = _ADAMW_FIELDS + ("run" if seed is None else "seed",)
        raise _unfit(_ADAMW_OPTIONS, fields, step, lr, beta1, beta2, eps, scale, grad_type, copy_type, bits, draws) from None
    _done(lib, lib.bagel_adamw_step(table, n, options, on))


class Bagel:
    """One context = one set of dims on the current device and stream."""

    def __init__(self, dims: Dims, stream=None):
        import torch
        self._lib = load()
        self.dims = dims
        self._h = C.c_void_p()
        if stream is None:
            stream = torch.cuda.current_stream()
        self.stream = stream
        rc = self._lib.bagel_create(C.byref(self._h), C.byref(dims), C.c_void_p(stream.cuda_stream))
        if rc != OK:
            msg = self._lib.bagel_last_error(None).decode()
            self._h = C.c_void_p()
            raise BagelError(rc, msg)
        self.P = bagel_num_params(dims)
        self.M = dims.d_s
        self.D = dims.d_s + dims.d_a

    # -- helpers -------------------------------------------------------------------------
    def _check(self, rc: int):
        if rc != OK:
            raise BagelError(rc, self._lib.bagel_last_error(self._h).decode())

    def workspace_bytes(self) -> int:
        return int(self._lib.bagel_workspace_bytes(self._h))

    def close(self):
        if self._h:
            self._lib.bagel_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the entry points, same names as the C ABI --------------------------------------------
    def bagel_prepare_samples(self, X, y, lengthscale, signal_var, noise_var, omega, phase, w, eps, v_out=None):
        d, M, D = self.dims, self.M, self.D
        self._check(self._lib.bagel_prepare_samples(
            self._h, _ptr(X, (d.N, D), "X"), _ptr(y, (M, d.N), "y"), _ptr(lengthscale, (M, D), "lengthscale"),
            _ptr(signal_var, (M,), "signal_var"), _ptr(noise_var, (M,), "noise_var"),
            _ptr(omega, (M, d.L, D), "omega"), _ptr(phase, (M, d.L), "phase"), _ptr(w, (d.S, M, d.L), "w"),
            _ptr(eps, (d.S, M, d.N), "eps"), _ptr(v_out, (d.S, M, d.N), "v_out", optional=True)))

    def bagel_set_samples(self, X, lengthscale, signal_var, omega, phase, w, v):
        d, M, D = self.dims, self.M, self.D
        self._check(self._lib.bagel_set_samples(
            self._h, _ptr(X, (d.N, D), "X"), _ptr(lengthscale, (M, D), "lengthscale"),
            _ptr(signal_var, (M,), "signal_var"), _ptr(omega, (M, d.L, D), "omega"),
            _ptr(phase, (M, d.L), "phase"), _ptr(w, (d.S, M, d.L), "w"), _ptr(v, (d.S, M, d.N), "v")))

    def bagel_rollout_loss(self, theta, s0, goals, loss, loss_per_traj=None, states=None):
        d = self.dims
        self._check(self._lib.bagel_rollout_loss(
            self._h, _ptr(theta, (self.P,), "theta"), _ptr(s0, (d.B, d.d_s), "s0"),
            _ptr(goals, (d.H, d.B, d.d_g), "goals"), _ptr(loss, (1,), "loss"),
            _ptr(loss_per_traj, (d.B,), "loss_per_traj", optional=True),
            _ptr(states, (d.H + 1, d.B, d.d_s), "states", optional=True)))

    def bagel_rollout_loss_grad(self, theta, s0, goals, loss, grad_theta, loss_per_traj=None, states=None,
                                grad_s0=None):
        d = self.dims
        self._check(self._lib.bagel_rollout_loss_grad(
            self._h, _ptr(theta, (self.P,), "theta"), _ptr(s0, (d.B, d.d_s), "s0"),
            _ptr(goals, (d.H, d.B, d.d_g), "goals"), _ptr(loss, (1,), "loss"),
            _ptr(grad_theta, (self.P,), "grad_theta"),
            _ptr(loss_per_traj, (d.B,), "loss_per_traj", optional=True),
            _ptr(states, (d.H + 1, d.B, d.d_s), "states", optional=True),
            _ptr(grad_s0, (d.B, d.d_s), "grad_s0", optional=True)))

    def bagel_prepare_posterior(self, X, y, lengthscale, signal_var, noise_var):
        d, M, D = self.dims, self.M, self.D
        self._check(self._lib.bagel_prepare_posterior(
            self._h, _ptr(X, (d.N, D), "X"), _ptr(y, (M, d.N), "y"), _ptr(lengthscale, (M, D), "lengthscale"),
            _ptr(signal_var, (M,), "signal_var"), _ptr(noise_var, (M,), "noise_var")))

    def bagel_posterior_rollout_loss(self, theta, s0, goals, xi, loss, loss_per_traj=None, states=None):
        d = self.dims
        self._check(self._lib.bagel_posterior_rollout_loss(
            self._h, _ptr(theta, (self.P,), "theta"), _ptr(s0, (d.B, d.d_s), "s0"),
            _ptr(goals, (d.H, d.B, d.d_g), "goals"), _ptr(xi, (d.H, d.B, self.M), "xi"), _ptr(loss, (1,), "loss"),
            _ptr(loss_per_traj, (d.B,), "loss_per_traj", optional=True),
            _ptr(states, (d.H + 1, d.B, d.d_s), "states", optional=True)))

    def bagel_posterior_rollout_loss_grad(self, theta, s0, goals, xi, loss, grad_theta, loss_per_traj=None,
                                          states=None, grad_s0=None):
        d = self.dims
        self._check(self._lib.bagel_posterior_rollout_loss_grad(
            self._h, _ptr(theta, (self.P,), "theta"), _ptr(s0, (d.B, d.d_s), "s0"),
            _ptr(goals, (d.H, d.B, d.d_g), "goals"), _ptr(xi, (d.H, d.B, self.M), "xi"), _ptr(loss, (1,), "loss"),
            _ptr(grad_theta, (self.P,), "grad_theta"),
            _ptr(loss_per_traj, (d.B,), "loss_per_traj", optional=True),
            _ptr(states, (d.H + 1, d.B, d.d_s), "states", optional=True),
            _ptr(grad_s0, (d.B, d.d_s), "grad_s0", optional=True)))

    def bagel_hyper_lml_grad(self, X, y, log_hyp, lml, grad=None):
        d, M, D = self.dims, self.M, self.D
        self._check(self._lib.bagel_hyper_lml_grad(
            self._h, _ptr(X, (d.N, D), "X"), _ptr(y, (M, d.N), "y"), _ptr(log_hyp, (M, D + 2), "log_hyp"),
            _ptr(lml, (M,), "lml"), _ptr(grad, (M, D + 2), "grad", optional=True)))

    def bagel_hyper_fit(self, X, y, log_hyp, adam_m, adam_v, n_iters, lml_history, first_step=1, lr=1e-2, beta1=0.9,
                        beta2=0.999, eps=1e-8):
        d, M, D = self.dims, self.M, self.D
        self._check(self._lib.bagel_hyper_fit(
            self._h, _ptr(X, (d.N, D), "X"), _ptr(y, (M, d.N), "y"), _ptr(log_hyp, (M, D + 2), "log_hyp"),
            _ptr(adam_m, (M, D + 2), "adam_m"), _ptr(adam_v, (M, D + 2), "adam_v"), int(n_iters), int(first_step),
            lr, beta1, beta2, eps, _ptr(lml_history, (int(n_iters), M), "lml_history")))

    def bagel_adam_step(self, theta, grad, adam_m, adam_v, step, lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8):
        P = (self.P,)
        self._check(self._lib.bagel_adam_step(
            self._h, _ptr(theta, P, "theta"), _ptr(grad, P, "grad"), _ptr(adam_m, P, "adam_m"),
            _ptr(adam_v, P, "adam_v"), int(step), lr, beta1, beta2, eps))

    def bagel_optimize(self, theta, adam_m, adam_v, s0_sets, goal_sets, n_iters, loss_history, first_step=1,
                       lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8):
        d, P = self.dims, (self.P,)
        n_sets = int(s0_sets.shape[0]) if hasattr(s0_sets, "shape") and len(s0_sets.shape) == 3 else 0
        self._check(self._lib.bagel_optimize(
            self._h, _ptr(theta, P, "theta"), _ptr(adam_m, P, "adam_m"), _ptr(adam_v, P, "adam_v"),
            _ptr(s0_sets, (n_sets, d.B, d.d_s), "s0_sets"), _ptr(goal_sets, (n_sets, d.H, d.B, d.d_g), "goal_sets"),
            n_sets, int(n_iters), int(first_step), lr, beta1, beta2, eps,
            _ptr(loss_history, (int(n_iters),), "loss_history")))

    def bagel_profile_enable(self, every: int):
        self._check(self._lib.bagel_profile_enable(self._h, int(every)))

    def bagel_profile_read(self):
        ms, n = C.c_double(), C.c_int()
        self._check(self._lib.bagel_profile_read(self._h, C.byref(ms), C.byref(n)))
        return ms.value, n.value

    def bagel_sample_eval(self, x, f, jac=None):
        d = self.dims
        self._check(self._lib.bagel_sample_eval(
            self._h, _ptr(x, (d.B, self.D), "x"), _ptr(f, (d.B, self.M), "f"),
            _ptr(jac, (d.B, self.M, self.D), "jac", optional=True)))
