"""Thin ctypes binding of ``libcountdown.so`` (declared in ``include/countdown.h``).

The functions carry the C names and only marshal arguments: torch tensors
become device pointers, ``stream`` defaults to torch's current HIP stream,
and a non-OK status raises :class:`CountdownError`. All compute runs in the
library's HIP kernels; there is no fallback when the library or the GPU is
missing.
"""
from __future__ import annotations

import array
import ctypes as C
import os

PKG = os.path.dirname(os.path.abspath(__file__))
# CD_LIBRARY names another build of the library to load (the sanitizer test of
# the host code loads an instrumented build this way)
LIB_PATH = os.environ.get("CD_LIBRARY") or os.path.join(PKG, "libcountdown.so")

CD_OK, CD_EINVAL, CD_EUNSUPPORTED, CD_EHIP, CD_ENOMEM = 0, -1, -2, -3, -4
CD_VARIANT_MONO, CD_VARIANT_DUAL_IDEAL, CD_VARIANT_DUAL_PRED, CD_VARIANT_DENSE = 0, 1, 2, 3
CD_VARIANT_CATS, CD_VARIANT_DUAL_TERN = 4, 5
CD_PLAN_KEEP_COEF, CD_PLAN_DETERMINISTIC = 1, 2
CD_PHASE_COEF, CD_PHASE_DOWN, CD_PHASE_ALL = 1, 2, 3
CD_TYPE_F32, CD_TYPE_BF16 = 0, 1
CD_ADAPTERS_TRAIN = 1

# every symbol include/countdown.h declares
EXPORTS = (
    "countdown_plan_create", "countdown_plan_destroy", "countdown_ffn_mono", "countdown_ffn_dual",
    "countdown_ffn_mono_noalloc",
    "countdown_ffn_dense", "countdown_ffn_cats", "countdown_ffn_topk", "countdown_ffn_residual",
    "countdown_calibrate", "countdown_ffn_tern", "countdown_ffn_tern_topk",
    "countdown_calibrate_tern", "countdown_ternary_words", "countdown_ternary_pack",
    "countdown_export_active",
    "countdown_plan_set_phases", "countdown_stream_read", "countdown_check_args",
    "countdown_check_shape", "countdown_status_string", "countdown_abi_version",
    "countdown_adapters_create", "countdown_adapters_destroy", "countdown_adapters_project",
    "countdown_adapters_add", "countdown_adapters_backward",
    "countdown_clip_create", "countdown_clip_destroy", "countdown_clip_grads",
)

_lib = None


class CountdownError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: {status_string(status)}")
        self.status = status


def load_library(path: str = LIB_PATH):
    """Load the built library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with __graft_entry__.build() "
                           "(python -m paper_2505_17701_amd.build)")
    lib = C.CDLL(path)
    vp, i, u, f, d = C.c_void_p, C.c_int, C.c_uint, C.c_float, C.c_double
    z = C.c_size_t
    sig = {
        "countdown_plan_create": (i, [i, i, i, i, u, C.POINTER(vp)]),
        "countdown_plan_destroy": (i, [vp]),
        "countdown_ffn_mono": (i, [vp, vp, i, vp, vp, vp, f, vp, vp]),
        "countdown_ffn_dual": (i, [vp, vp, i, vp, vp, vp, vp, vp, f, vp, vp]),
        "countdown_ffn_mono_noalloc": (i, [vp, i, vp, vp, vp, i, i, f, vp, vp]),
        "countdown_ffn_dense": (i, [vp, vp, i, vp, vp, vp, vp, vp]),
        "countdown_ffn_cats": (i, [vp, vp, i, vp, vp, vp, f, vp, vp]),
        "countdown_ffn_residual": (i, [vp, i, vp, vp, vp, f, vp, i, vp, vp, vp, vp, vp, f, vp,
                                       vp]),
        "countdown_ffn_topk": (i, [vp, i, vp, i, vp, vp, vp, vp, vp, d, vp, vp, vp]),
        "countdown_calibrate": (i, [vp, i, vp, i, vp, vp, vp, vp, d, vp, vp, vp]),
        "countdown_ffn_tern": (i, [vp, vp, i, vp, vp, vp, vp, f, vp, vp]),
        "countdown_ffn_tern_topk": (i, [vp, vp, i, vp, vp, vp, vp, d, vp, vp, vp]),
        "countdown_calibrate_tern": (i, [vp, vp, i, vp, d, vp, vp, vp]),
        "countdown_ternary_words": (C.c_size_t, [i, i]),
        "countdown_ternary_pack": (i, [vp, i, i, vp]),
        "countdown_export_active": (i, [vp, vp, vp, vp, vp, vp]),
        "countdown_plan_set_phases": (i, [vp, u]),
        "countdown_stream_read": (i, [vp, C.c_size_t, vp, vp]),
        "countdown_check_args": (i, [i, i, i, i, i, vp, i, vp, vp, vp, vp, vp, f, vp]),
        "countdown_check_shape": (i, [i, i, i, i]),
        "countdown_status_string": (C.c_char_p, [i]),
        "countdown_abi_version": (i, []),
        "countdown_adapters_create": (i, [i, i, i, i, i, u, C.POINTER(vp)]),
        "countdown_adapters_destroy": (i, [vp]),
        "countdown_adapters_project": (i, [vp, vp, z, i, vp, vp, vp, vp, vp, i, vp, z, vp]),
        "countdown_adapters_add": (i, [vp, vp, z, i, vp, vp, vp, vp, i, vp, z, vp, z, vp]),
        "countdown_adapters_backward": (i, [vp, vp, z, vp, z, i, vp, vp, vp, vp, i, vp, z, vp, z,
                                            vp, vp, vp]),
        "countdown_clip_create": (i, [i, C.POINTER(vp)]),
        "countdown_clip_destroy": (i, [vp]),
        "countdown_clip_grads": (i, [vp, vp, i, d, vp, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().countdown_status_string(int(status)).decode()


def _check(status: int, what: str) -> None:
    if status != CD_OK:
        raise CountdownError(status, what)


# A call of a small layer is bound by this module: 256 x 688 at one token took 15.4 us a
# call, 7 of them on the GPU. So torch and its dtypes are looked up once (the module can be
# imported without torch), each operand is checked and its pointer taken in one step, and
# the current stream's handle is read without building a Stream object.
_torch = None


def _use_torch():
    global _torch, _BF16, _F32, _TYPES, _raw_stream
    import torch

    _BF16, _F32 = torch.bfloat16, torch.float32
    _TYPES = {_F32: CD_TYPE_F32, _BF16: CD_TYPE_BF16}
    try:  # (device index) -> handle of its current stream
        raw, device = torch._C._cuda_getCurrentRawStream, torch.cuda.current_device

        def _raw_stream():
            return raw(device())
    except AttributeError:
        def _raw_stream():
            return torch.cuda.current_stream().cuda_stream
    _torch = torch
    return torch


def _ptr(t) -> int | None:
    """Device pointer of a torch tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("countdown tensors must live on the GPU")
    if not t.is_contiguous():
        raise ValueError("countdown tensors must be contiguous")
    return t.data_ptr()


def _stream(stream) -> int | None:
    if stream is None:
        if _torch is None:
            _use_torch()
        return _raw_stream()
    return int(stream) if not hasattr(stream, "cuda_stream") else stream.cuda_stream


def _bf16(t) -> int | None:
    """Device pointer of a bfloat16 tensor (None -> NULL)."""
    if t is None:
        return None
    if _torch is None:
        _use_torch()
    if t.dtype is not _BF16:
        raise TypeError(f"expected a bfloat16 tensor, got {t.dtype}")
    if t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    return _ptr(t)  # raises


def _f32(t):
    if _torch is None:
        _use_torch()
    if t.dtype is not _F32:
        raise TypeError(f"expected a float32 tensor, got {t.dtype}")
    return t


class Plan:
    """Owns a ``cd_plan``: shape, workspace, and optional timing/coefficient capture."""

    def __init__(self, d_model: int, d_ff: int, max_batch: int = 1, d_rank: int = 0,
                 keep_coef: bool = False, deterministic: bool = False):
        self.d_model, self.d_ff, self.max_batch, self.d_rank = d_model, d_ff, max_batch, d_rank
        flags = (CD_PLAN_KEEP_COEF if keep_coef else 0) | (
            CD_PLAN_DETERMINISTIC if deterministic else 0)
        h = C.c_void_p()
        _check(load_library().countdown_plan_create(d_model, d_ff, max_batch, d_rank, flags,
                                                    C.byref(h)), "countdown_plan_create")
        self.handle = h.value
        self.keep_coef = keep_coef
        self.last_batch = 0

    def close(self):
        if getattr(self, "handle", None):
            _check(load_library().countdown_plan_destroy(self.handle), "countdown_plan_destroy")
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def countdown_plan_create(d_model, d_ff, max_batch=1, d_rank=0, keep_coef=False,
                          deterministic=False):
    return Plan(d_model, d_ff, max_batch, d_rank, keep_coef, deterministic)


def countdown_plan_destroy(plan: Plan) -> None:
    plan.close()


def _shape(t, shape, name):
    """ValueError unless ``t`` (None is skipped) has exactly ``shape``."""
    if t is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")


def _layer_shapes(plan, x, W_gate=None, W_up=None, W_down=None, A_t=None, B_t=None,
                  theta_packed=None):
    """Check a call's tensors against the plan before any pointer is taken: the C ABI
    sees only pointers, and the kernels read exactly these extents."""
    xs = x.shape
    if len(xs) != 2 or xs[1] != plan.d_model:
        raise ValueError(f"x must be [B, {plan.d_model}], got {tuple(xs)}")
    shape = (plan.d_ff, plan.d_model)
    _shape(W_gate, shape, "W_gate")
    _shape(W_up, shape, "W_up")
    _shape(W_down, shape, "W_down")
    if A_t is not None or B_t is not None:
        _shape(A_t, (plan.d_rank, plan.d_model), "A_t")
        _shape(B_t, (plan.d_ff, plan.d_rank), "B_t")
    if theta_packed is not None:
        words = countdown_ternary_words(plan.d_model, plan.d_ff)
        if theta_packed.numel() * theta_packed.element_size() != 4 * words:
            raise ValueError(f"theta_packed must hold {words} 32-bit words "
                             f"(countdown_ternary_words), got {theta_packed.numel()} elements")


def _out(plan: Plan, x, y):
    B = x.shape[0]
    if y is None:
        if _torch is None:
            _use_torch()
        return B, _torch.empty((B, plan.d_model), dtype=_F32, device=x.device)
    _shape(y, (B, plan.d_model), "y")
    return B, _f32(y)


def countdown_ffn_mono(plan: Plan, x, W_gate, W_up, W_down, thld: float, y=None, stream=None):
    """M-CountDown FFN; returns y ``[B, d_model]`` fp32 (enqueued on ``stream``)."""
    _layer_shapes(plan, x, W_gate, W_up, W_down)
    B, y = _out(plan, x, y)
    _check(load_library().countdown_ffn_mono(
        plan.handle, _bf16(x), B, _bf16(W_gate), _bf16(W_up),
        _bf16(W_down), float(thld), _ptr(y), _stream(stream)), "countdown_ffn_mono")
    plan.last_batch = B
    return y


def countdown_ffn_mono_noalloc(x, W_gate, W_up, W_down, thld: float, y, stream=None):
    """M-CountDown without a plan (the library's static workspace); y [B, d_model] fp32
    must be given (nothing is allocated). Returns y."""
    for t, name in ((x, "x"), (W_gate, "W_gate"), (W_up, "W_up"), (W_down, "W_down")):
        if t is None or t.dim() != 2:
            raise ValueError(f"{name} must be a 2-D tensor")
    if y is None:
        raise ValueError("y must be given: countdown_ffn_mono_noalloc allocates nothing")
    B, dm = x.shape
    dff = W_up.shape[0]
    for t, name in ((W_gate, "W_gate"), (W_up, "W_up"), (W_down, "W_down")):
        _shape(t, (dff, dm), name)
    _shape(_f32(y), (B, dm), "y")
    _check(load_library().countdown_ffn_mono_noalloc(
        _bf16(x), B, _bf16(W_gate), _bf16(W_up), _bf16(W_down), dm, dff,
        float(thld), _ptr(y), _stream(stream)), "countdown_ffn_mono_noalloc")
    return y


def countdown_ffn_dual(plan: Plan, x, W_gate, W_up, W_down, thld: float, A_t=None, B_t=None,
                       y=None, stream=None):
    """D-CountDown FFN (ideal without a predictor, practical with ``A_t``/``B_t``)."""
    _layer_shapes(plan, x, W_gate, W_up, W_down, A_t, B_t)
    B, y = _out(plan, x, y)
    _check(load_library().countdown_ffn_dual(
        plan.handle, _bf16(x), B, _bf16(W_gate), _bf16(W_up),
        _bf16(W_down), _bf16(A_t), _bf16(B_t), float(thld), _ptr(y),
        _stream(stream)), "countdown_ffn_dual")
    plan.last_batch = B
    return y


def countdown_ffn_cats(plan: Plan, x, W_gate, W_up, W_down, thld: float, y=None, stream=None):
    """CATS (Eq. 6a): keep |SiLU(x.W_gate)| > thld, gather W_up on the kept neurons."""
    _layer_shapes(plan, x, W_gate, W_up, W_down)
    B, y = _out(plan, x, y)
    _check(load_library().countdown_ffn_cats(
        plan.handle, _bf16(x), B, _bf16(W_gate), _bf16(W_up),
        _bf16(W_down), float(thld), _ptr(y), _stream(stream)), "countdown_ffn_cats")
    plan.last_batch = B
    return y


def countdown_ffn_topk(plan: Plan, variant: int, x, W_gate, W_up, W_down, k: float, A_t=None,
                       B_t=None, y=None, thld_out=None, stream=None):
    """Per-token threshold: each token keeps the neurons above the k-quantile of its
    own coefficients (union over the batch). ``thld_out``: optional fp64 [B] device
    tensor for the thresholds. Returns y."""
    import torch

    _layer_shapes(plan, x, W_gate, W_up, W_down, A_t, B_t)
    B, y = _out(plan, x, y)
    if thld_out is not None and (thld_out.dtype != torch.float64 or thld_out.numel() < B):
        raise ValueError("thld_out must be a float64 device tensor with at least B entries")
    _check(load_library().countdown_ffn_topk(
        plan.handle, int(variant), _bf16(x), B, _bf16(W_gate), _bf16(W_up),
        _bf16(W_down), _bf16(A_t), _bf16(B_t), float(k), _ptr(thld_out),
        _ptr(y), _stream(stream)), "countdown_ffn_topk")
    plan.last_batch = B
    return y


def countdown_ffn_residual(plan: Plan, variant: int, h_in, y_prev, h_out, x_out, W_gate, W_up,
                           W_down, thld: float = 0.0, A_t=None, B_t=None, eps: float = 1e-5,
                           y=None, stream=None):
    """One layer of a residual stack: h_out = h_in + y_prev, x_out = bf16(RMSNorm(h_out)),
    then the ``variant`` FFN of x_out into ``y`` (returned). ``y_prev`` may be None or ``y``."""
    import torch

    B = h_in.shape[0]
    if y is None:
        y = torch.empty((B, plan.d_model), dtype=torch.float32, device=h_in.device)
    for t in (h_in, h_out, y) + (() if y_prev is None else (y_prev,)):
        if t.dtype != torch.float32 or not t.is_contiguous() or tuple(t.shape) != (B, plan.d_model):
            raise ValueError("h_in, y_prev, h_out and y must be contiguous fp32 [B, d_model]")
    if tuple(x_out.shape) != (B, plan.d_model) or not x_out.is_contiguous():
        raise ValueError("x_out must be a contiguous [B, d_model] bf16 tensor")
    _layer_shapes(plan, x_out, W_gate, W_up, W_down, A_t, B_t)
    _check(load_library().countdown_ffn_residual(
        plan.handle, int(variant), _ptr(h_in), _ptr(y_prev), _ptr(h_out), float(eps),
        _bf16(x_out), B, _bf16(W_gate), _bf16(W_up), _bf16(W_down),
        _bf16(A_t), _bf16(B_t), float(thld), _ptr(y), _stream(stream)),
        "countdown_ffn_residual")
    plan.last_batch = B
    return y


def countdown_ffn_dense(plan: Plan, x, W_gate, W_up, W_down, y=None, stream=None):
    """Dense Gated-MLP through the same kernels."""
    _layer_shapes(plan, x, W_gate, W_up, W_down)
    B, y = _out(plan, x, y)
    _check(load_library().countdown_ffn_dense(
        plan.handle, _bf16(x), B, _bf16(W_gate), _bf16(W_up),
        _bf16(W_down), _ptr(y), _stream(stream)), "countdown_ffn_dense")
    plan.last_batch = B
    return y


def countdown_calibrate(plan: Plan, variant: int, X, k: float, W_gate=None, W_up=None, A_t=None,
                        B_t=None, stream=None):
    """Layerwise threshold; returns ``(thld fp32 tensor [1], per-token quantiles fp64 [T])``."""
    import torch

    _layer_shapes(plan, X, W_gate, W_up, None, A_t, B_t)
    T = X.shape[0]
    thld = torch.empty(1, dtype=torch.float32, device=X.device)
    q = torch.empty(T, dtype=torch.float64, device=X.device)
    _check(load_library().countdown_calibrate(
        plan.handle, int(variant), _bf16(X), T, _bf16(W_gate), _bf16(W_up),
        _bf16(A_t), _bf16(B_t), float(k), _ptr(thld), _ptr(q), _stream(stream)),
        "countdown_calibrate")
    return thld, q


def _u32(t):
    import torch

    if t.dtype not in (torch.int32, torch.uint32):
        raise TypeError(f"expected a packed 32-bit tensor, got {t.dtype}")
    return t


def countdown_ternary_words(d_model: int, d_ff: int) -> int:
    """uint32 words of the packed ternary predictor of a shape (0 if rejected)."""
    return int(load_library().countdown_ternary_words(int(d_model), int(d_ff)))


def countdown_ternary_pack(theta_t):
    """Pack a host int8 ``theta_t [d_ff, d_model]`` (entries -1, 0, +1; theta transposed)
    into the kernels' layout; returns a host numpy uint32 array (move it to the GPU)."""
    import numpy as np

    t = np.ascontiguousarray(theta_t, dtype=np.int8)
    d_ff, d_model = t.shape
    n = countdown_ternary_words(d_model, d_ff)
    if n == 0:
        raise CountdownError(CD_EINVAL, "countdown_ternary_words")
    out = np.zeros(n, dtype=np.uint32)
    _check(load_library().countdown_ternary_pack(t.ctypes.data, d_model, d_ff, out.ctypes.data),
           "countdown_ternary_pack")
    return out


def countdown_ffn_tern(plan: Plan, x, W_gate, W_up, W_down, theta_packed, thld: float, y=None,
                       stream=None):
    """D-CountDown with the ternary predictor (``theta_packed``: device int32/uint32 tensor
    from :func:`countdown_ternary_pack`)."""
    _layer_shapes(plan, x, W_gate, W_up, W_down, theta_packed=theta_packed)
    B, y = _out(plan, x, y)
    _check(load_library().countdown_ffn_tern(
        plan.handle, _bf16(x), B, _bf16(W_gate), _bf16(W_up),
        _bf16(W_down), _ptr(_u32(theta_packed)), float(thld), _ptr(y), _stream(stream)),
        "countdown_ffn_tern")
    plan.last_batch = B
    return y


def countdown_ffn_tern_topk(plan: Plan, x, W_gate, W_up, W_down, theta_packed, k: float, y=None,
                            thld_out=None, stream=None):
    """Per-token threshold on the ternary predictor score; returns y."""
    import torch

    _layer_shapes(plan, x, W_gate, W_up, W_down, theta_packed=theta_packed)
    B, y = _out(plan, x, y)
    if thld_out is not None and (thld_out.dtype != torch.float64 or thld_out.numel() < B):
        raise ValueError("thld_out must be a float64 device tensor with at least B entries")
    _check(load_library().countdown_ffn_tern_topk(
        plan.handle, _bf16(x), B, _bf16(W_gate), _bf16(W_up),
        _bf16(W_down), _ptr(_u32(theta_packed)), float(k), _ptr(thld_out), _ptr(y),
        _stream(stream)), "countdown_ffn_tern_topk")
    plan.last_batch = B
    return y


def countdown_calibrate_tern(plan: Plan, X, theta_packed, k: float, stream=None):
    """Layerwise threshold of the ternary predictor score; returns ``(thld [1], q [T])``."""
    import torch

    _layer_shapes(plan, X, theta_packed=theta_packed)
    T = X.shape[0]
    thld = torch.empty(1, dtype=torch.float32, device=X.device)
    q = torch.empty(T, dtype=torch.float64, device=X.device)
    _check(load_library().countdown_calibrate_tern(
        plan.handle, _bf16(X), T, _ptr(_u32(theta_packed)), float(k), _ptr(thld), _ptr(q),
        _stream(stream)), "countdown_calibrate_tern")
    return thld, q


def countdown_export_active(plan: Plan, stream=None):
    """The last call's ``(IDX [n] int32, s_c [B, n] fp32, coef [B, d_ff] or None)`` as new
    device tensors. Synchronises the stream to read ``n``."""
    import torch

    dev = torch.device("cuda", torch.cuda.current_device())
    B = max(plan.last_batch, 1)
    idx = torch.empty(plan.d_ff, dtype=torch.int32, device=dev)
    n = torch.empty(1, dtype=torch.int32, device=dev)
    s = torch.empty((B, plan.d_ff), dtype=torch.float32, device=dev)
    coef = torch.empty((B, plan.d_ff), dtype=torch.float32, device=dev) if plan.keep_coef else None
    _check(load_library().countdown_export_active(plan.handle, _ptr(idx), _ptr(n), _ptr(s),
                                                  _ptr(coef), _stream(stream)),
           "countdown_export_active")
    m = int(n.item())  # .item() synchronises with the copy's stream
    return idx[:m], s[:, :m], coef


def countdown_plan_set_phases(plan: Plan, phases: int) -> None:
    """Launch only the kernels in ``phases`` (CD_PHASE_*) on later calls (measurement aid)."""
    _check(load_library().countdown_plan_set_phases(plan.handle, int(phases)),
           "countdown_plan_set_phases")


def countdown_stream_read(src, sink, stream=None) -> None:
    """Measurement aid: a plain streaming read of the whole of ``src`` (a contiguous
    device tensor) with the coefficient kernel's load pattern; ``sink`` is a one-word
    int32 / uint32 device tensor. Enqueued on ``stream``."""
    if sink.numel() * sink.element_size() < 4:
        raise ValueError("sink must hold at least one 32-bit word")
    _check(load_library().countdown_stream_read(
        _ptr(src), src.numel() * src.element_size(), _ptr(sink), _stream(stream)),
        "countdown_stream_read")


class Adapters:
    """Owns a ``cd_adapters``: the workspace of the calls on a pool of ``n_adapters`` low-rank
    adapters beside a ``d_in`` -> ``d_out`` projection, for up to ``max_tokens`` tokens a
    call (``train``: the backward call too). The weights stay with the caller:
    A [n_adapters, rank, d_in] and B [n_adapters, d_out, rank], bf16."""

    def __init__(self, d_in: int, d_out: int, rank: int, n_adapters: int, max_tokens: int,
                 train: bool = False):
        self.d_in, self.d_out, self.rank = d_in, d_out, rank
        self.n_adapters, self.max_tokens, self.train = n_adapters, max_tokens, train
        self._a_shape = (n_adapters, rank, d_in)
        self._b_shape = (n_adapters, d_out, rank)
        h = C.c_void_p()
        _check(load_library().countdown_adapters_create(
            d_in, d_out, rank, n_adapters, max_tokens, CD_ADAPTERS_TRAIN if train else 0,
            C.byref(h)), "countdown_adapters_create")
        self.handle = h.value
        self.device = (_torch or _use_torch()).cuda.current_device()

    def close(self):
        if getattr(self, "handle", None):
            _check(load_library().countdown_adapters_destroy(self.handle),
                   "countdown_adapters_destroy")
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def countdown_adapters_create(d_in, d_out, rank, n_adapters, max_tokens, train=False):
    return Adapters(d_in, d_out, rank, n_adapters, max_tokens, train)


def countdown_adapters_destroy(pool: Adapters) -> None:
    pool.close()


def _rows(t, n, width, name, device):
    """(pointer, row stride) of a [n, width] tensor whose rows are contiguous."""
    if t.shape != (n, width):
        raise ValueError(f"{name} must have shape {(n, width)}, got {tuple(t.shape)}")
    if t.get_device() != device:
        raise ValueError(f"{name} must live on GPU {device}, where the pool was created")
    row, col = t.stride()
    if n <= 1 or t.is_contiguous():  # (the stride of a single row says nothing)
        row = width
    if col != 1 and width > 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    return t.data_ptr(), row


def _whole(t, shape, dtype, name, device):
    """Pointer of a contiguous tensor of exactly this shape and type."""
    if t.dtype is not dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
    if t.get_device() != device:
        raise ValueError(f"{name} must live on GPU {device}, where the pool was created")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _row_type(t, name) -> int:
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise TypeError(f"{name}: expected float32 or bfloat16, got {t.dtype}")
    return kind


def _pool_args(pool: Adapters, x, ids, A, B, scale):
    if pool.handle is None:
        raise ValueError("the pool is closed")
    if x.dim() != 2 or x.dtype is not _BF16:
        raise TypeError(f"x must be a bfloat16 [T, {pool.d_in}] tensor")
    T, dev = x.shape[0], pool.device
    xp, ldx = _rows(x, T, pool.d_in, "x", dev)
    return (T, xp, ldx, _whole(ids, (T,), _torch.int32, "ids", dev),
            _whole(A, pool._a_shape, _BF16, "A", dev), _whole(B, pool._b_shape, _BF16, "B", dev),
            None if scale is None else _whole(scale, (pool.n_adapters,), _F32, "scale", dev))


def countdown_adapters_project(pool: Adapters, x, W, ids, A, B, scale=None, y=None, stream=None):
    """y = x W^T + each token's own adapter, for up to 16 tokens; returns y ``[T, d_out]``
    (fp32, or the type of the given fp32 / bf16 ``y``). ``ids`` int32 [T]: the adapter of
    each token (outside [0, n_adapters): none); ``scale`` fp32 [n_adapters] or None."""
    T, xp, ldx, ip, ap, bp, sp = _pool_args(pool, x, ids, A, B, scale)
    if y is None:
        y = _torch.empty((T, pool.d_out), dtype=_F32, device=x.device)
    yp, ldy = _rows(y, T, pool.d_out, "y", pool.device)
    _check(load_library().countdown_adapters_project(
        pool.handle, xp, ldx, T, _whole(W, (pool.d_out, pool.d_in), _BF16, "W", pool.device), ip,
        ap, bp, sp, _row_type(y, "y"), yp, ldy, _stream(stream)), "countdown_adapters_project")
    return y


def _base(base, out, T, width, out_name, dtype, device):
    """The output (made if None: of base's type, else dtype) and the pointers of base and output."""
    if out is None:
        out = _torch.empty((T, width), dtype=dtype if base is None else base.dtype,
                           device=f"cuda:{device}")
    op, ldo = _rows(out, T, width, out_name, device)
    if base is None:
        return out, None, 0, op, ldo
    if base.dtype is not out.dtype:
        raise TypeError(f"base and {out_name} must have one type, got {base.dtype} and {out.dtype}")
    bp, ldb = (op, ldo) if base is out else _rows(base, T, width, "base", device)
    return out, bp, ldb, op, ldo


def countdown_adapters_add(pool: Adapters, x, ids, A, B, scale=None, base=None, y=None,
                           stream=None):
    """y = base + each token's own adapter of x, for any number of tokens; returns y
    ``[T, d_out]``. ``base`` (fp32 or bf16, None: zeros) is what the shared projection gave,
    e.g. an FFN call's y; ``y`` may be ``base`` itself (in place), has its type, and is a new
    tensor if None."""
    T, xp, ldx, ip, ap, bp, sp = _pool_args(pool, x, ids, A, B, scale)
    y, basep, ldb, yp, ldy = _base(base, y, T, pool.d_out, "y", _F32, pool.device)
    _check(load_library().countdown_adapters_add(
        pool.handle, xp, ldx, T, ip, ap, bp, sp, _row_type(y, "y"), basep, ldb, yp, ldy,
        _stream(stream)), "countdown_adapters_add")
    return y


def countdown_adapters_backward(pool: Adapters, x, dy, ids, A, B, scale=None, base=None, dx=None,
                                dA=None, dB=None, need=(True, True, True), stream=None):
    """The gradients ``(dx, dA, dB)`` of the adapters' part for ``dy`` (bf16 [T, d_out]).
    dx = base + A^T (scale B^T dy) has base's type (bf16 without one); dA and dB are fp32 of
    A's and B's shapes, overwritten whole. ``need`` says which of the three are computed
    (None is returned for the others); given tensors are written, missing ones made."""
    T, xp, ldx, ip, ap, bp, sp = _pool_args(pool, x, ids, A, B, scale)
    dev = pool.device
    if dy.dtype is not _BF16:
        raise TypeError(f"dy: expected a bfloat16 tensor, got {dy.dtype}")
    dyp, lddy = _rows(dy, T, pool.d_out, "dy", dev)
    basep, ldb, dxp, lddx, dap, dbp, kind = None, 0, None, 0, None, None, CD_TYPE_BF16
    if need[0]:
        dx, basep, ldb, dxp, lddx = _base(base, dx, T, pool.d_in, "dx", _BF16, dev)
        kind = _row_type(dx, "dx")
    if need[1]:
        if dA is None:
            dA = _torch.empty(pool._a_shape, dtype=_F32, device=x.device)
        dap = _whole(dA, pool._a_shape, _F32, "dA", dev)
    if need[2]:
        if dB is None:
            dB = _torch.empty(pool._b_shape, dtype=_F32, device=x.device)
        dbp = _whole(dB, pool._b_shape, _F32, "dB", dev)
    _check(load_library().countdown_adapters_backward(
        pool.handle, xp, ldx, dyp, lddy, T, ip, ap, bp, sp, kind, basep, ldb, dxp, lddx, dap, dbp,
        _stream(stream)), "countdown_adapters_backward")
    return dx if need[0] else None, dA if need[1] else None, dB if need[2] else None


class GradClip:
    """Owns a ``cd_clip``: the workspace of :func:`countdown_clip_grads` for up to
    ``max_tensors`` gradients a call."""

    def __init__(self, max_tensors: int):
        self.max_tensors = max_tensors
        h = C.c_void_p()
        _check(load_library().countdown_clip_create(max_tensors, C.byref(h)),
               "countdown_clip_create")
        self.handle = h.value
        self.device = (_torch or _use_torch()).cuda.current_device()

    def close(self):
        if getattr(self, "handle", None):
            _check(load_library().countdown_clip_destroy(self.handle), "countdown_clip_destroy")
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def countdown_clip_create(max_tensors):
    return GradClip(max_tensors)


def countdown_clip_destroy(clip: GradClip) -> None:
    clip.close()


def countdown_clip_grads(clip: GradClip, grads, max_norm: float, out=None, norm=None, stream=None):
    """The global norm of a list of fp32 / bf16 gradients, as a new 0-dim fp64 device tensor (or
    into ``norm``, one fp64 element), and the gradients scaled by min(1, max_norm / norm): in place, or into the
    tensors of the list ``out``. ``max_norm`` inf scales nothing (without ``out`` only the norm
    is computed). A norm that is not finite leaves the gradients as they are."""
    if clip.handle is None:
        raise ValueError("the workspace is closed")
    if out is not None and len(out) != len(grads):
        raise ValueError(f"out must have as many tensors as grads ({len(grads)}), got {len(out)}")
    dev, words = clip.device, []  # cd_grad: three 64-bit words, the type in a fourth
    for i, g in enumerate(grads):
        if g.get_device() != dev or not g.is_contiguous():
            raise ValueError(f"gradients must be contiguous tensors on GPU {dev}")
        p, t = g.data_ptr(), g.dtype
        if t is not _F32 and t is not _BF16:
            raise TypeError(f"gradients must be float32 or bfloat16, got {t}")
        words += (p, p if out is None else _out_ptr(g, out[i], dev), g.numel(),
                  CD_TYPE_F32 if t is _F32 else CD_TYPE_BF16)
    words = array.array("Q", words)
    if norm is None:
        norm = _torch.empty((), dtype=_torch.float64, device=f"cuda:{dev}")
    elif norm.numel() != 1 or norm.dtype is not _torch.float64 or norm.get_device() != dev:
        raise ValueError(f"norm must be one float64 element on GPU {dev}")
    _check(load_library().countdown_clip_grads(
        clip.handle, words.buffer_info()[0], len(grads), float(max_norm), norm.data_ptr(),
        _stream(stream)), "countdown_clip_grads")
    return norm


def _out_ptr(g, o, device) -> int:
    if o.shape != g.shape or o.dtype is not g.dtype:
        raise ValueError("an output must have its gradient's shape and type")
    if o.get_device() != device or not o.is_contiguous():
        raise ValueError(f"outputs must be contiguous tensors on GPU {device}")
    return o.data_ptr()


def countdown_check_args(variant, d_model, d_ff, max_batch, d_rank, x, B, W_gate, W_up, W_down,
                         A_t, B_t, thld, y) -> int:
    """Host-only argument validation (integer pointers); returns the status code."""
    return load_library().countdown_check_args(variant, d_model, d_ff, max_batch, d_rank, x, B,
                                               W_gate, W_up, W_down, A_t, B_t, float(thld), y)


def countdown_check_shape(d_model, d_ff, max_batch, d_rank) -> int:
    return load_library().countdown_check_shape(d_model, d_ff, max_batch, d_rank)


def max_batch_for(d_model: int, d_ff: int = 8, d_rank: int = 0) -> int:
    """Largest max_batch countdown_check_shape accepts for this shape (0 if none)."""
    for b in range(8, 0, -1):
        if countdown_check_shape(d_model, d_ff, b, d_rank) == CD_OK:
            return b
    return 0


def countdown_abi_version() -> int:
    return load_library().countdown_abi_version()
