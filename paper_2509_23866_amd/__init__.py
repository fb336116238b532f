"""Python binding of libdart (the C ABI declared in include/dart.h).

Argument marshalling only: every step of the path runs in the HIP kernels under
``csrc/``. torch supplies device memory and the stream. The library must
be built (``__graft_entry__.build()``); if it is missing, importing a function
raises — there is no CPU fallback. Calls whose arguments are plain tensors, with
the outputs left to the call and on the current stream, are marshalled natively
(``csrc/binding.cpp``, where it is built); all others, and every complaint about an
argument, here.

Functions carry the C names: ``dart_tok_stats``, ``dart_step_select``,
``dart_tis_loss_fwd_bwd`` (and its halves ``dart_tis_loss_fwd`` /
``dart_tis_grad``), the ``_ex`` variants (inverse temperature, the KL term,
aggregation and ratio level, zero-row skipping), ``dart_tis_loss_workspace_bytes``,
``dart_kept_steps`` and ``dart_status_string``. ``policy_update`` chains the
device calls. From the LM head's inputs: ``dart_lmhead_tok_stats`` and
``dart_lmhead_backward``; its supervised loss, ``dart_lmhead_xent_fwd`` and, with
the gradients, ``dart_lmhead_xent_fwd_bwd``; and the head in four bits,
``dart_mxfp4_quantize`` (an ``Mxfp4``), ``dart_mxfp4_dequantize``,
``dart_mxfp4_matmul`` and ``dart_lmhead_mxfp4_tok_stats``. With ``stream`` these last
two sets run as under ``torch.cuda.stream(stream)``: what they allocate, results
included, is that stream's.
"""

from __future__ import annotations

import contextlib
import ctypes
import importlib
import os
import warnings
from typing import NamedTuple

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdart.so")

DART_OK = 0
DART_ERR_INVALID_ARG = 1
DART_ERR_UNSUPPORTED = 2
DART_ERR_HIP = 3
DART_F32 = 0
DART_BF16 = 1

DART_KL = {"none": 0, "k1": 1, "k2": 2, "k3": 3}
DART_AGG = {"token_mean": 0, "token_mean_all": 1, "step_mean": 2}
DART_RATIO = {"token": 0, "step_geomean": 1, "step_product": 2}
DART_XENT = {"mean": 0, "sum": 1}
DART_GRAD_SKIP_ZERO_ROWS = 1
DART_LMHEAD_SKIP_ZERO_ROWS = 1
DART_LMHEAD_BF16_GRADS = 4

EXPORTED = ("dart_tok_stats", "dart_step_select", "dart_tis_loss_fwd_bwd", "dart_tis_loss_fwd",
            "dart_tis_grad", "dart_tis_loss_fwd_bwd_noalloc", "dart_select_tis_loss_fwd",
            "dart_tok_stats_ex", "dart_tis_loss_fwd_ex", "dart_tis_grad_ex",
            "dart_grpo_advantage", "dart_step_select_groups", "dart_tis_loss_workspace_bytes",
            "dart_tis_loss_split_workspace_bytes",
            "dart_lmhead_tok_stats", "dart_lmhead_tok_stats_ex", "dart_lmhead_stats_workspace_bytes",
            "dart_lmhead_dlogits", "dart_lmhead_dlogits_ex",
            "dart_lmhead_backward", "dart_lmhead_backward_workspace_bytes",
            "dart_lmhead_backward_ex", "dart_lmhead_backward_ex_workspace_bytes",
            "dart_lmhead_backward_split_workspace_bytes",
            "dart_lmhead_xent_fwd", "dart_lmhead_xent_fwd_workspace_bytes",
            "dart_lmhead_xent_fwd_bwd", "dart_lmhead_xent_workspace_bytes", "dart_grad_scale",
            "dart_mxfp4_bytes", "dart_mxfp4_quantize", "dart_mxfp4_dequantize",
            "dart_mxfp4_matmul", "dart_lmhead_mxfp4_tok_stats",
            "dart_lmhead_mxfp4_stats_workspace_bytes",
            "dart_kept_steps",
            "dart_status_string")


class dart_loss_config_t(ctypes.Structure):
    """Mirror of the C struct dart_loss_config_t."""

    _fields_ = [("eps_low", ctypes.c_float), ("eps_high", ctypes.c_float), ("C", ctypes.c_float),
                ("kl", ctypes.c_int32), ("beta", ctypes.c_float), ("aggregation", ctypes.c_int32),
                ("ratio", ctypes.c_int32)]


class dart_xent_config_t(ctypes.Structure):
    """Mirror of the C struct dart_xent_config_t."""

    _fields_ = [("label_smoothing", ctypes.c_float), ("z_loss", ctypes.c_float),
                ("reduction", ctypes.c_int32)]


class DartError(RuntimeError):
    def __init__(self, fn, code):
        super().__init__(f"{fn} failed: {dart_status_string(code)} ({code})")
        self.code = code


_lib = None
_P = ctypes.c_void_p
_I64 = ctypes.c_int64


def load_library():
    """Open libdart.so (raises if it is not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build()")
        try:
            _torch()  # its HIP runtime first: libdart.so alone would bring another
        except ImportError:
            pass  # the host helpers do without
        lib = ctypes.CDLL(LIB_PATH)
        lib.dart_tok_stats.restype = ctypes.c_int
        lib.dart_tok_stats.argtypes = [_P, ctypes.c_int, _I64, _I64, _I64, _P, _P, _P, _P, _P]
        lib.dart_step_select.restype = ctypes.c_int
        lib.dart_step_select.argtypes = [_P, _I64, _P, _I64, ctypes.c_double, _P, _P, _P, _P]
        lib.dart_tis_loss_fwd_bwd.restype = ctypes.c_int
        lib.dart_tis_loss_fwd_bwd.argtypes = [
            _P, ctypes.c_int, _I64, _I64, _I64, _P, _P, _P, _P, _P, _P, _P, _I64, _P,
            ctypes.c_float, ctypes.c_float, ctypes.c_float, _P, _I64, _P, _P, _P, _P,
            ctypes.c_size_t, _P]
        lib.dart_tis_loss_fwd_bwd_noalloc.restype = ctypes.c_int
        lib.dart_tis_loss_fwd_bwd_noalloc.argtypes = [
            _P, ctypes.c_int, _I64, _I64, _I64, _P, _P, _P, _P, _P, _P, _P, _I64, _P,
            ctypes.c_float, ctypes.c_float, ctypes.c_float, _P, _I64, _P, _P, _P, _P]
        lib.dart_tis_loss_fwd.restype = ctypes.c_int
        lib.dart_tis_loss_fwd.argtypes = [_I64, _P, _P, _P, _P, _P, _I64, _P, ctypes.c_float,
                                          ctypes.c_float, ctypes.c_float, _P, _P, _P, _P,
                                          ctypes.c_size_t, _P]
        lib.dart_select_tis_loss_fwd.restype = ctypes.c_int
        lib.dart_select_tis_loss_fwd.argtypes = [
            _I64, _P, _P, _P, _P, _P, _P, _I64, ctypes.c_double, ctypes.c_float, ctypes.c_float,
            ctypes.c_float, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]
        lib.dart_tis_loss_workspace_bytes.restype = ctypes.c_size_t
        lib.dart_tis_loss_workspace_bytes.argtypes = [_I64]
        lib.dart_tis_loss_split_workspace_bytes.restype = ctypes.c_size_t
        lib.dart_tis_loss_split_workspace_bytes.argtypes = [_I64]
        lib.dart_tis_grad.restype = ctypes.c_int
        lib.dart_tis_grad.argtypes = [_P, ctypes.c_int, _I64, _I64, _I64, _P, _P, _P, _P, _P,
                                      _I64, _P]
        lib.dart_tok_stats_ex.restype = ctypes.c_int
        lib.dart_tok_stats_ex.argtypes = [_P, ctypes.c_int, _I64, _I64, _I64, _P, ctypes.c_float,
                                          _P, _P, _P, _P]
        lib.dart_tis_loss_fwd_ex.restype = ctypes.c_int
        lib.dart_tis_loss_fwd_ex.argtypes = [_I64, _P, _P, _P, _P, _P, _P, _I64, _P,
                                             ctypes.POINTER(dart_loss_config_t), _P, _P, _P, _P,
                                             ctypes.c_size_t, _P]
        lib.dart_tis_grad_ex.restype = ctypes.c_int
        lib.dart_tis_grad_ex.argtypes = [_P, ctypes.c_int, _I64, _I64, _I64, _P, _P, _P, _P,
                                         ctypes.c_float, ctypes.c_uint32, _P, _I64, _P]
        lib.dart_grpo_advantage.restype = ctypes.c_int
        lib.dart_grpo_advantage.argtypes = [_P, _I64, _P, _P, _I64, _P, _I64, _I64, _P, _P, _P, _P]
        lib.dart_step_select_groups.restype = ctypes.c_int
        lib.dart_step_select_groups.argtypes = [_P, _I64, _P, _I64, _P, _I64, ctypes.c_double, _P,
                                                _P, _P, _P]
        lib.dart_lmhead_tok_stats.restype = ctypes.c_int
        lib.dart_lmhead_tok_stats.argtypes = [_P, _I64, _I64, _I64, _P, _I64, _I64, _P, _P, _P, _P,
                                              _P, ctypes.c_size_t, _P]
        lib.dart_lmhead_tok_stats_ex.restype = ctypes.c_int
        lib.dart_lmhead_tok_stats_ex.argtypes = [_P, _I64, _I64, _I64, _P, _I64, _I64, _P,
                                                 ctypes.c_float, _P, _P, _P, _P, ctypes.c_size_t,
                                                 _P]
        lib.dart_lmhead_stats_workspace_bytes.restype = ctypes.c_size_t
        lib.dart_lmhead_stats_workspace_bytes.argtypes = [_I64, _I64]
        lib.dart_lmhead_dlogits.restype = ctypes.c_int
        lib.dart_lmhead_dlogits.argtypes = [_P, _I64, _I64, _I64, _P, _I64, _I64, _P, _P, _P, _P,
                                            _P, _I64, _P]
        lib.dart_lmhead_dlogits_ex.restype = ctypes.c_int
        lib.dart_lmhead_dlogits_ex.argtypes = [_P, _I64, _I64, _I64, _P, _I64, _I64, _P, _P, _P,
                                               _P, ctypes.c_float, _P, _I64, _P]
        lib.dart_lmhead_backward.restype = ctypes.c_int
        lib.dart_lmhead_backward.argtypes = [_P, _I64, _I64, _I64, _P, _I64, _I64, _P, _P, _P, _P,
                                             _P, _I64, _P, _I64, _I64, _P, ctypes.c_size_t, _P]
        lib.dart_lmhead_backward_workspace_bytes.restype = ctypes.c_size_t
        lib.dart_lmhead_backward_workspace_bytes.argtypes = [_I64, _I64]
        lib.dart_lmhead_backward_ex.restype = ctypes.c_int
        lib.dart_lmhead_backward_ex.argtypes = [_P, _I64, _I64, _I64, _P, _I64, _I64, _P, _P, _P,
                                                _P, ctypes.c_float, _P, _I64, _P, _I64, _I64,
                                                _I64, ctypes.c_uint32, _P, ctypes.c_size_t, _P]
        lib.dart_lmhead_backward_ex_workspace_bytes.restype = ctypes.c_size_t
        lib.dart_lmhead_backward_ex_workspace_bytes.argtypes = [_I64, _I64, _I64, _I64, _I64,
                                                                ctypes.c_uint32]
        lib.dart_lmhead_backward_split_workspace_bytes.restype = ctypes.c_size_t
        lib.dart_lmhead_backward_split_workspace_bytes.argtypes = [_I64, _I64, _I64, _I64, _I64,
                                                                   ctypes.c_uint32]
        lib.dart_lmhead_xent_fwd.restype = ctypes.c_int
        lib.dart_lmhead_xent_fwd.argtypes = [_P, _I64, _I64, _I64, _P, _I64, _I64, _P,
                                             ctypes.POINTER(dart_xent_config_t), _P, _P, _P, _P,
                                             ctypes.c_size_t, _P]
        lib.dart_lmhead_xent_fwd_workspace_bytes.restype = ctypes.c_size_t
        lib.dart_lmhead_xent_fwd_workspace_bytes.argtypes = [_I64, _I64, _I64]
        lib.dart_lmhead_xent_fwd_bwd.restype = ctypes.c_int
        lib.dart_lmhead_xent_fwd_bwd.argtypes = [_P, _I64, _I64, _I64, _P, _I64, _I64, _P,
                                                 ctypes.POINTER(dart_xent_config_t), _P, _P, _P,
                                                 _P, _I64, _P, _I64, _I64, _P, ctypes.c_size_t, _P]
        lib.dart_lmhead_xent_workspace_bytes.restype = ctypes.c_size_t
        lib.dart_lmhead_xent_workspace_bytes.argtypes = [_I64, _I64, _I64, _I64]
        lib.dart_grad_scale.restype = ctypes.c_int
        lib.dart_grad_scale.argtypes = [_P, ctypes.c_int, _I64, _I64, _I64, _P, _P]
        lib.dart_mxfp4_bytes.restype = ctypes.c_size_t
        lib.dart_mxfp4_bytes.argtypes = [_I64, _I64]
        lib.dart_mxfp4_quantize.restype = ctypes.c_int
        lib.dart_mxfp4_quantize.argtypes = [_P, ctypes.c_int, _I64, _I64, _I64, _P, _P]
        lib.dart_mxfp4_dequantize.restype = ctypes.c_int
        lib.dart_mxfp4_dequantize.argtypes = [_P, _I64, _I64, ctypes.c_int, _P, _I64, _P]
        lib.dart_mxfp4_matmul.restype = ctypes.c_int
        lib.dart_mxfp4_matmul.argtypes = [_P, _I64, _P, _I64, _I64, ctypes.c_int, _P, _I64, _P]
        lib.dart_lmhead_mxfp4_tok_stats.restype = ctypes.c_int
        lib.dart_lmhead_mxfp4_tok_stats.argtypes = [_P, _I64, _P, _I64, _I64, _P, ctypes.c_float, _P,
                                                    _P, _P, _P, ctypes.c_size_t, _P]
        lib.dart_lmhead_mxfp4_stats_workspace_bytes.restype = ctypes.c_size_t
        lib.dart_lmhead_mxfp4_stats_workspace_bytes.argtypes = [_I64, _I64]
        lib.dart_kept_steps.restype = _I64
        lib.dart_kept_steps.argtypes = [_I64, ctypes.c_double]
        lib.dart_status_string.restype = ctypes.c_char_p
        lib.dart_status_string.argtypes = [ctypes.c_int]
        _lib = lib
    return _lib


_native = None


class _NoNative:
    """Stands for the native marshalling where it is not built: takes no call."""

    def __getattr__(self, name):
        return lambda *args: None


def _nat(required=False):
    """The native marshalling. Without it (only libdart.so is built, or _native.so
    was built against another torch) every call is marshalled in Python, which is
    said once; with ``required`` that raises."""
    global _native
    if _native is None or required and isinstance(_native, _NoNative):
        load_library()
        try:
            native = importlib.import_module("._native", __name__)
        except ImportError as e:
            if required:
                raise RuntimeError("_native.so is not built; run __graft_entry__.build()") from e
            warnings.warn(f"calls are marshalled in Python (an update: 46 us of host time in place "
                          f"of 19): {e}; run __graft_entry__.build()", RuntimeWarning, stacklevel=3)
            native = _NoNative()
        else:
            native.open(LIB_PATH)
        _native = native
    return _native


def _made(out, *names):
    """What a native call made, or DartError for the C call that failed."""
    if type(out) is int:
        raise DartError(names[out >> 8], out & 255)
    return out


def dart_status_string(code: int) -> str:
    return load_library().dart_status_string(int(code)).decode()


def dart_kept_steps(S: int, rho: float) -> int:
    return int(load_library().dart_kept_steps(int(S), float(rho)))


def _torch():
    import torch

    return torch


def _stream_handle(stream, device):
    """The HIP stream a call enqueues on: for None the current stream of the
    inputs' device (not of the current device); a torch stream, which must
    belong to the inputs' device; or a raw hipStream_t handle, taken as given."""
    torch = _torch()
    if stream is None:
        return torch.cuda.current_stream(device).cuda_stream
    if hasattr(stream, "cuda_stream"):
        if torch.device(stream.device) != torch.device(device):
            raise ValueError(f"the stream is on {stream.device}, the inputs on {device}")
        return stream.cuda_stream
    return int(stream)


def _ptr(t):
    return None if t is None else t.data_ptr()


def dart_tis_loss_workspace_bytes(T: int) -> int:
    return int(load_library().dart_tis_loss_workspace_bytes(int(T)))


def dart_tis_loss_split_workspace_bytes(T: int) -> int:
    return int(load_library().dart_tis_loss_split_workspace_bytes(int(T)))


def _workspace(workspace, T, device, stream):
    """(pointer, bytes, tensor) for the loss workspace: "auto" allocates one
    from torch's caching allocator (kept for the stream the call runs on),
    None passes NULL (one-workgroup loss), a uint8 tensor is used as given."""
    torch = _torch()
    if workspace is None:
        return None, 0, None
    if isinstance(workspace, str):
        if workspace != "auto":
            raise ValueError('workspace must be "auto", None or a uint8 device tensor')
        workspace = torch.empty(dart_tis_loss_split_workspace_bytes(T), dtype=torch.uint8,
                                device=device)
        if isinstance(stream, torch.cuda.Stream):
            workspace.record_stream(stream)
    if (not isinstance(workspace, torch.Tensor) or workspace.dtype != torch.uint8
            or workspace.device != device or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous uint8 tensor on the device of the inputs")
    return workspace.data_ptr(), workspace.numel(), workspace


def _check_vec(name, t, dtype, n, device):
    torch = _torch()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype != dtype or t.device != device or t.dim() != 1 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} vector of {n} elements on {device}")


def _logits_meta(logits):
    torch = _torch()
    if logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError("logits must be a 2-D tensor with contiguous rows")
    if logits.dtype == torch.bfloat16:
        dt = DART_BF16
    elif logits.dtype == torch.float32:
        dt = DART_F32
    else:
        raise TypeError("logits must be bfloat16 or float32")
    if not logits.is_cuda:
        raise ValueError("logits must be on a GPU")
    return dt, logits.shape[0], logits.shape[1], logits.stride(0)


def dart_tok_stats(logits, target, logp=None, entropy=None, lse=None, stream=None, inv_temp=1.0):
    """Per-token log-prob of the target, entropy and log-normaliser (float32 [T]
    each) of softmax(inv_temp * logits)."""
    if logp is None and entropy is None and lse is None and stream is None:
        out = _nat().tok_stats(logits, target, inv_temp)
        if out is not None:
            return _made(out, "dart_tok_stats", "dart_tok_stats_ex")
    torch = _torch()
    dt, T, V, ld = _logits_meta(logits)
    dev = logits.device
    _check_vec("target", target, torch.int32, T, dev)
    logp = torch.empty(T, dtype=torch.float32, device=dev) if logp is None else logp
    entropy = torch.empty(T, dtype=torch.float32, device=dev) if entropy is None else entropy
    lse = torch.empty(T, dtype=torch.float32, device=dev) if lse is None else lse
    for n, v in (("logp", logp), ("entropy", entropy), ("lse", lse)):
        _check_vec(n, v, torch.float32, T, dev)
    if inv_temp == 1.0:
        rc = load_library().dart_tok_stats(logits.data_ptr(), dt, T, V, ld, target.data_ptr(),
                                           logp.data_ptr(), entropy.data_ptr(), lse.data_ptr(),
                                           _stream_handle(stream, dev))
        name = "dart_tok_stats"
    else:
        rc = load_library().dart_tok_stats_ex(logits.data_ptr(), dt, T, V, ld, target.data_ptr(),
                                              float(inv_temp), logp.data_ptr(),
                                              entropy.data_ptr(), lse.data_ptr(),
                                              _stream_handle(stream, dev))
        name = "dart_tok_stats_ex"
    if rc != DART_OK:
        raise DartError(name, rc)
    return logp, entropy, lse


def dart_step_select(entropy, step_offsets, rho, step_entropy=None, step_mask=None,
                     n_kept_steps=None, stream=None):
    """Per-step mean entropy (float32 [S]), kept-step mask (uint8 [S]) and the
    kept count (int32 [1])."""
    torch = _torch()
    dev = entropy.device
    T = entropy.numel()
    S = step_offsets.numel() - 1
    _check_vec("entropy", entropy, torch.float32, T, dev)
    _check_vec("step_offsets", step_offsets, torch.int32, S + 1, dev)
    step_entropy = torch.empty(S, dtype=torch.float32, device=dev) if step_entropy is None else step_entropy
    step_mask = torch.empty(S, dtype=torch.uint8, device=dev) if step_mask is None else step_mask
    n_kept_steps = torch.empty(1, dtype=torch.int32, device=dev) if n_kept_steps is None else n_kept_steps
    _check_vec("step_entropy", step_entropy, torch.float32, S, dev)
    _check_vec("step_mask", step_mask, torch.uint8, S, dev)
    _check_vec("n_kept_steps", n_kept_steps, torch.int32, 1, dev)
    rc = load_library().dart_step_select(entropy.data_ptr(), T, step_offsets.data_ptr(), S,
                                         float(rho), step_entropy.data_ptr(), step_mask.data_ptr(),
                                         n_kept_steps.data_ptr(), _stream_handle(stream, dev))
    if rc != DART_OK:
        raise DartError("dart_step_select", rc)
    return step_entropy, step_mask, n_kept_steps


def dart_tis_loss_fwd_bwd(logits, target, logp, lse, logp_old, logp_rollout, adv, step_offsets,
                          step_mask, eps_low, eps_high, C, dlogits=None, loss=None, tok_coef=None,
                          stats=None, with_stats=True, stream=None, workspace="auto"):
    """Loss (float64 [1]), dlogits (dtype and shape of logits; pass ``dlogits=logits``
    for the in-place gradient), per-token coefficient (float32 [T]) and stats
    (float32 [4]: clip fraction, mean TIS weight, capped fraction, N).
    ``workspace``: "auto" (allocated here), None (one-workgroup loss, no
    workspace) or a uint8 device tensor of dart_tis_loss_workspace_bytes(T), or of
    dart_tis_loss_split_workspace_bytes(T), as "auto" allocates."""
    torch = _torch()
    dt, T, V, ld = _logits_meta(logits)
    dev = logits.device
    S = step_offsets.numel() - 1
    _check_vec("target", target, torch.int32, T, dev)
    for n, v in (("logp", logp), ("lse", lse), ("logp_old", logp_old),
                 ("logp_rollout", logp_rollout), ("adv", adv)):
        _check_vec(n, v, torch.float32, T, dev)
    _check_vec("step_offsets", step_offsets, torch.int32, S + 1, dev)
    _check_vec("step_mask", step_mask, torch.uint8, S, dev)
    if dlogits is None:
        dlogits = torch.empty((T, V), dtype=logits.dtype, device=dev)
    if (dlogits.dtype != logits.dtype or dlogits.dim() != 2 or tuple(dlogits.shape) != (T, V)
            or dlogits.stride(1) != 1 or dlogits.device != dev):
        raise ValueError("dlogits must match logits in dtype and shape, with contiguous rows")
    loss = torch.empty(1, dtype=torch.float64, device=dev) if loss is None else loss
    tok_coef = torch.empty(T, dtype=torch.float32, device=dev) if tok_coef is None else tok_coef
    if stats is None and with_stats:
        stats = torch.empty(4, dtype=torch.float32, device=dev)
    _check_vec("loss", loss, torch.float64, 1, dev)
    _check_vec("tok_coef", tok_coef, torch.float32, T, dev)
    if stats is not None:
        _check_vec("stats", stats, torch.float32, 4, dev)
    ws, ws_bytes, _ws = _workspace(workspace, T, dev, stream)
    rc = load_library().dart_tis_loss_fwd_bwd(
        logits.data_ptr(), dt, T, V, ld, target.data_ptr(), logp.data_ptr(), lse.data_ptr(),
        logp_old.data_ptr(), logp_rollout.data_ptr(), adv.data_ptr(), step_offsets.data_ptr(), S,
        step_mask.data_ptr(), float(eps_low), float(eps_high), float(C), dlogits.data_ptr(),
        dlogits.stride(0), loss.data_ptr(), tok_coef.data_ptr(), _ptr(stats), ws, ws_bytes,
        _stream_handle(stream, dev))
    if rc != DART_OK:
        raise DartError("dart_tis_loss_fwd_bwd", rc)
    return loss, dlogits, tok_coef, stats


def dart_tis_loss_fwd_bwd_noalloc(logits, target, logp, lse, logp_old, logp_rollout, adv,
                                  step_offsets, step_mask, eps_low, eps_high, C, dlogits=None,
                                  loss=None, tok_coef=None, stats=None, with_stats=True,
                                  stream=None):
    """dart_tis_loss_fwd_bwd with the loss workspace in the library's fixed
    per-GPU scratch array (the C call allocates nothing; outputs not given are
    allocated here by torch). Calls on one GPU that may overlap race."""
    torch = _torch()
    dt, T, V, ld = _logits_meta(logits)
    dev = logits.device
    S = step_offsets.numel() - 1
    _check_vec("target", target, torch.int32, T, dev)
    for n, v in (("logp", logp), ("lse", lse), ("logp_old", logp_old),
                 ("logp_rollout", logp_rollout), ("adv", adv)):
        _check_vec(n, v, torch.float32, T, dev)
    _check_vec("step_offsets", step_offsets, torch.int32, S + 1, dev)
    _check_vec("step_mask", step_mask, torch.uint8, S, dev)
    if dlogits is None:
        dlogits = torch.empty((T, V), dtype=logits.dtype, device=dev)
    if (dlogits.dtype != logits.dtype or dlogits.dim() != 2 or tuple(dlogits.shape) != (T, V)
            or dlogits.stride(1) != 1 or dlogits.device != dev):
        raise ValueError("dlogits must match logits in dtype and shape, with contiguous rows")
    loss = torch.empty(1, dtype=torch.float64, device=dev) if loss is None else loss
    tok_coef = torch.empty(T, dtype=torch.float32, device=dev) if tok_coef is None else tok_coef
    if stats is None and with_stats:
        stats = torch.empty(4, dtype=torch.float32, device=dev)
    _check_vec("loss", loss, torch.float64, 1, dev)
    _check_vec("tok_coef", tok_coef, torch.float32, T, dev)
    if stats is not None:
        _check_vec("stats", stats, torch.float32, 4, dev)
    rc = load_library().dart_tis_loss_fwd_bwd_noalloc(
        logits.data_ptr(), dt, T, V, ld, target.data_ptr(), logp.data_ptr(), lse.data_ptr(),
        logp_old.data_ptr(), logp_rollout.data_ptr(), adv.data_ptr(), step_offsets.data_ptr(), S,
        step_mask.data_ptr(), float(eps_low), float(eps_high), float(C), dlogits.data_ptr(),
        dlogits.stride(0), loss.data_ptr(), tok_coef.data_ptr(), _ptr(stats),
        _stream_handle(stream, dev))
    if rc != DART_OK:
        raise DartError("dart_tis_loss_fwd_bwd_noalloc", rc)
    return loss, dlogits, tok_coef, stats


def dart_tis_loss_fwd(logp, logp_old, logp_rollout, adv, step_offsets, step_mask, eps_low,
                      eps_high, C, loss=None, tok_coef=None, stats=None, with_stats=True,
                      stream=None, workspace="auto"):
    """Loss (float64 [1]), per-token coefficient (float32 [T]) and stats; the
    logits are not needed. ``workspace`` as for dart_tis_loss_fwd_bwd."""
    torch = _torch()
    dev = logp.device
    T = logp.numel()
    S = step_offsets.numel() - 1
    for n, v in (("logp", logp), ("logp_old", logp_old), ("logp_rollout", logp_rollout),
                 ("adv", adv)):
        _check_vec(n, v, torch.float32, T, dev)
    _check_vec("step_offsets", step_offsets, torch.int32, S + 1, dev)
    _check_vec("step_mask", step_mask, torch.uint8, S, dev)
    loss = torch.empty(1, dtype=torch.float64, device=dev) if loss is None else loss
    tok_coef = torch.empty(T, dtype=torch.float32, device=dev) if tok_coef is None else tok_coef
    if stats is None and with_stats:
        stats = torch.empty(4, dtype=torch.float32, device=dev)
    _check_vec("loss", loss, torch.float64, 1, dev)
    _check_vec("tok_coef", tok_coef, torch.float32, T, dev)
    if stats is not None:
        _check_vec("stats", stats, torch.float32, 4, dev)
    ws, ws_bytes, _ws = _workspace(workspace, T, dev, stream)
    rc = load_library().dart_tis_loss_fwd(
        T, logp.data_ptr(), logp_old.data_ptr(), logp_rollout.data_ptr(), adv.data_ptr(),
        step_offsets.data_ptr(), S, step_mask.data_ptr(), float(eps_low), float(eps_high),
        float(C), loss.data_ptr(), tok_coef.data_ptr(), _ptr(stats), ws, ws_bytes,
        _stream_handle(stream, dev))
    if rc != DART_OK:
        raise DartError("dart_tis_loss_fwd", rc)
    return loss, tok_coef, stats


def dart_select_tis_loss_fwd(entropy, logp, logp_old, logp_rollout, adv, step_offsets, rho,
                             eps_low, eps_high, C, step_entropy=None, step_mask=None,
                             n_kept_steps=None, loss=None, tok_coef=None, stats=None,
                             with_stats=True, stream=None, workspace="auto"):
    """dart_step_select then dart_tis_loss_fwd in one call (one launch up to
    4096 tokens and 80 steps). Returns (step_entropy, step_mask,
    n_kept_steps, loss, tok_coef, stats). ``workspace`` as for
    dart_tis_loss_fwd_bwd."""
    if (step_entropy is None and step_mask is None and n_kept_steps is None and loss is None
            and tok_coef is None and stats is None and stream is None
            and isinstance(workspace, str) and workspace == "auto"):
        out = _nat().select_tis_loss_fwd(entropy, logp, logp_old, logp_rollout, adv, step_offsets,
                                         rho, eps_low, eps_high, C, bool(with_stats))
        if out is not None:
            return _made(out, "dart_select_tis_loss_fwd")
    torch = _torch()
    dev = logp.device
    T = logp.numel()
    S = step_offsets.numel() - 1
    for n, v in (("entropy", entropy), ("logp", logp), ("logp_old", logp_old),
                 ("logp_rollout", logp_rollout), ("adv", adv)):
        _check_vec(n, v, torch.float32, T, dev)
    _check_vec("step_offsets", step_offsets, torch.int32, S + 1, dev)
    step_entropy = torch.empty(S, dtype=torch.float32, device=dev) if step_entropy is None else step_entropy
    step_mask = torch.empty(S, dtype=torch.uint8, device=dev) if step_mask is None else step_mask
    n_kept_steps = torch.empty(1, dtype=torch.int32, device=dev) if n_kept_steps is None else n_kept_steps
    loss = torch.empty(1, dtype=torch.float64, device=dev) if loss is None else loss
    tok_coef = torch.empty(T, dtype=torch.float32, device=dev) if tok_coef is None else tok_coef
    if stats is None and with_stats:
        stats = torch.empty(4, dtype=torch.float32, device=dev)
    _check_vec("step_entropy", step_entropy, torch.float32, S, dev)
    _check_vec("step_mask", step_mask, torch.uint8, S, dev)
    _check_vec("n_kept_steps", n_kept_steps, torch.int32, 1, dev)
    _check_vec("loss", loss, torch.float64, 1, dev)
    _check_vec("tok_coef", tok_coef, torch.float32, T, dev)
    if stats is not None:
        _check_vec("stats", stats, torch.float32, 4, dev)
    ws, ws_bytes, _ws = _workspace(workspace, T, dev, stream)
    rc = load_library().dart_select_tis_loss_fwd(
        T, entropy.data_ptr(), logp.data_ptr(), logp_old.data_ptr(), logp_rollout.data_ptr(),
        adv.data_ptr(), step_offsets.data_ptr(), S, float(rho), float(eps_low), float(eps_high),
        float(C), step_entropy.data_ptr(), step_mask.data_ptr(), n_kept_steps.data_ptr(),
        loss.data_ptr(), tok_coef.data_ptr(), _ptr(stats), ws, ws_bytes,
        _stream_handle(stream, dev))
    if rc != DART_OK:
        raise DartError("dart_select_tis_loss_fwd", rc)
    return step_entropy, step_mask, n_kept_steps, loss, tok_coef, stats


def dart_tis_loss_fwd_ex(logp, logp_old, logp_rollout, adv, step_offsets, step_mask, eps_low,
                         eps_high, C, logp_ref=None, kl="none", beta=0.0, aggregation="token_mean",
                         ratio="token", loss=None, tok_coef=None, stats=None, with_stats=True,
                         stream=None, workspace="auto"):
    """The loss with the KL term, aggregation and ratio level selectable.
    Returns (loss float64 [1], tok_coef float32 [T], stats float32 [6]).
    ``workspace`` as for dart_tis_loss_fwd_bwd."""
    if (loss is None and tok_coef is None and stats is None and stream is None
            and isinstance(workspace, str) and workspace == "auto"):
        out = _nat().tis_loss_fwd_ex(logp, logp_old, logp_rollout, adv, step_offsets, step_mask,
                                     logp_ref, eps_low, eps_high, C, DART_KL[kl], beta,
                                     DART_AGG[aggregation], DART_RATIO[ratio], bool(with_stats))
        if out is not None:
            return _made(out, "dart_tis_loss_fwd_ex")
    torch = _torch()
    dev = logp.device
    T = logp.numel()
    S = step_offsets.numel() - 1
    for n, v in (("logp", logp), ("logp_old", logp_old), ("logp_rollout", logp_rollout),
                 ("adv", adv)):
        _check_vec(n, v, torch.float32, T, dev)
    if DART_KL[kl] != 0:
        _check_vec("logp_ref", logp_ref, torch.float32, T, dev)
    _check_vec("step_offsets", step_offsets, torch.int32, S + 1, dev)
    _check_vec("step_mask", step_mask, torch.uint8, S, dev)
    loss = torch.empty(1, dtype=torch.float64, device=dev) if loss is None else loss
    tok_coef = torch.empty(T, dtype=torch.float32, device=dev) if tok_coef is None else tok_coef
    if stats is None and with_stats:
        stats = torch.empty(6, dtype=torch.float32, device=dev)
    _check_vec("loss", loss, torch.float64, 1, dev)
    _check_vec("tok_coef", tok_coef, torch.float32, T, dev)
    if stats is not None:
        _check_vec("stats", stats, torch.float32, 6, dev)
    cfg = dart_loss_config_t(float(eps_low), float(eps_high), float(C), DART_KL[kl], float(beta),
                             DART_AGG[aggregation], DART_RATIO[ratio])
    ws, ws_bytes, _ws = _workspace(workspace, T, dev, stream)
    rc = load_library().dart_tis_loss_fwd_ex(
        T, logp.data_ptr(), logp_old.data_ptr(), logp_rollout.data_ptr(),
        None if DART_KL[kl] == 0 else logp_ref.data_ptr(), adv.data_ptr(),
        step_offsets.data_ptr(), S, step_mask.data_ptr(), ctypes.byref(cfg), loss.data_ptr(),
        tok_coef.data_ptr(), _ptr(stats), ws, ws_bytes, _stream_handle(stream, dev))
    if rc != DART_OK:
        raise DartError("dart_tis_loss_fwd_ex", rc)
    return loss, tok_coef, stats


def dart_tis_grad(logits, target, logp, lse, tok_coef, dlogits=None, stream=None, inv_temp=1.0,
                  skip_zero_rows=False):
    """dlogits = inv_temp * tok_coef * (onehot(target) - softmax(inv_temp * logits)),
    dtype of logits; ``skip_zero_rows`` writes rows with a zero coefficient
    without reading them."""
    if stream is None:
        out = _nat().tis_grad(logits, target, logp, lse, tok_coef, dlogits, inv_temp,
                              bool(skip_zero_rows))
        if out is not None:
            return _made(out, "dart_tis_grad", "dart_tis_grad_ex")
    torch = _torch()
    dt, T, V, ld = _logits_meta(logits)
    dev = logits.device
    _check_vec("target", target, torch.int32, T, dev)
    for n, v in (("logp", logp), ("lse", lse), ("tok_coef", tok_coef)):
        _check_vec(n, v, torch.float32, T, dev)
    if dlogits is None:
        dlogits = torch.empty((T, V), dtype=logits.dtype, device=dev)
    if (dlogits.dtype != logits.dtype or dlogits.dim() != 2 or tuple(dlogits.shape) != (T, V)
            or dlogits.stride(1) != 1 or dlogits.device != dev):
        raise ValueError("dlogits must match logits in dtype and shape, with contiguous rows")
    if inv_temp == 1.0 and not skip_zero_rows:
        rc = load_library().dart_tis_grad(
            logits.data_ptr(), dt, T, V, ld, target.data_ptr(), logp.data_ptr(), lse.data_ptr(),
            tok_coef.data_ptr(), dlogits.data_ptr(), dlogits.stride(0), _stream_handle(stream, dev))
        name = "dart_tis_grad"
    else:
        rc = load_library().dart_tis_grad_ex(
            logits.data_ptr(), dt, T, V, ld, target.data_ptr(), logp.data_ptr(), lse.data_ptr(),
            tok_coef.data_ptr(), float(inv_temp),
            DART_GRAD_SKIP_ZERO_ROWS if skip_zero_rows else 0, dlogits.data_ptr(),
            dlogits.stride(0), _stream_handle(stream, dev))
        name = "dart_tis_grad_ex"
    if rc != DART_OK:
        raise DartError(name, rc)
    return dlogits


def dart_grpo_advantage(reward, traj_step_offsets, group_traj_offsets, step_offsets, T=None,
                        adv=None, group_mean=None, group_std=None, stream=None):
    """Step-wise GRPO advantage per token (float32 [T]) and per-group mean/std."""
    if adv is None and group_mean is None and group_std is None and stream is None:
        out = _nat().grpo_advantage(reward, traj_step_offsets, group_traj_offsets, step_offsets, T)
        if out is not None:
            return _made(out, "dart_grpo_advantage")
    torch = _torch()
    dev = reward.device
    n_traj = reward.numel()
    G = group_traj_offsets.numel() - 1
    S = step_offsets.numel() - 1
    _check_vec("reward", reward, torch.float32, n_traj, dev)
    _check_vec("traj_step_offsets", traj_step_offsets, torch.int32, n_traj + 1, dev)
    _check_vec("group_traj_offsets", group_traj_offsets, torch.int32, G + 1, dev)
    _check_vec("step_offsets", step_offsets, torch.int32, S + 1, dev)
    if T is None:
        T = int(step_offsets[-1].item())
    adv = torch.empty(T, dtype=torch.float32, device=dev) if adv is None else adv
    group_mean = torch.empty(G, dtype=torch.float32, device=dev) if group_mean is None else group_mean
    group_std = torch.empty(G, dtype=torch.float32, device=dev) if group_std is None else group_std
    _check_vec("adv", adv, torch.float32, T, dev)
    rc = load_library().dart_grpo_advantage(
        reward.data_ptr(), n_traj, traj_step_offsets.data_ptr(), group_traj_offsets.data_ptr(), G,
        step_offsets.data_ptr(), S, T, adv.data_ptr(), _ptr(group_mean), _ptr(group_std),
        _stream_handle(stream, dev))
    if rc != DART_OK:
        raise DartError("dart_grpo_advantage", rc)
    return adv, group_mean, group_std


def dart_step_select_groups(entropy, step_offsets, group_step_offsets, rho, step_entropy=None,
                            step_mask=None, n_kept_steps=None, stream=None):
    """Per-step entropy, mask and kept count per group (top ceil(rho S_g) of each group)."""
    if step_entropy is None and step_mask is None and n_kept_steps is None and stream is None:
        out = _nat().step_select_groups(entropy, step_offsets, group_step_offsets, rho)
        if out is not None:
            return _made(out, "dart_step_select_groups")
    torch = _torch()
    dev = entropy.device
    T = entropy.numel()
    S = step_offsets.numel() - 1
    G = group_step_offsets.numel() - 1
    _check_vec("entropy", entropy, torch.float32, T, dev)
    _check_vec("step_offsets", step_offsets, torch.int32, S + 1, dev)
    _check_vec("group_step_offsets", group_step_offsets, torch.int32, G + 1, dev)
    step_entropy = torch.empty(S, dtype=torch.float32, device=dev) if step_entropy is None else step_entropy
    step_mask = torch.empty(S, dtype=torch.uint8, device=dev) if step_mask is None else step_mask
    n_kept_steps = torch.empty(G, dtype=torch.int32, device=dev) if n_kept_steps is None else n_kept_steps
    rc = load_library().dart_step_select_groups(
        entropy.data_ptr(), T, step_offsets.data_ptr(), S, group_step_offsets.data_ptr(), G,
        float(rho), step_entropy.data_ptr(), step_mask.data_ptr(), n_kept_steps.data_ptr(),
        _stream_handle(stream, dev))
    if rc != DART_OK:
        raise DartError("dart_step_select_groups", rc)
    return step_entropy, step_mask, n_kept_steps


def dart_lmhead_stats_workspace_bytes(T: int, V: int) -> int:
    return int(load_library().dart_lmhead_stats_workspace_bytes(int(T), int(V)))


def _matrix_bf16(name, t, device=None):
    torch = _torch()
    if not isinstance(t, torch.Tensor) or t.dtype != torch.bfloat16 or t.dim() != 2:
        raise TypeError(f"{name} must be a 2-D bfloat16 tensor")
    if t.stride(1) != 1 or t.stride(0) % 8 or t.data_ptr() % 16 or not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU with contiguous rows, a row stride that is a "
                         "multiple of 8 and a 16-byte aligned base")
    if device is not None and t.device != device:
        raise ValueError(f"{name} must be on {device}")


def dart_lmhead_tok_stats(hidden, weight, target, logp=None, entropy=None, lse=None,
                          workspace="auto", stream=None):
    """(logp, entropy, lse) float32 [T] of softmax(hidden @ weight^T) without
    materialising the logits: hidden [T, d] and weight [V, d] bfloat16 (d a
    multiple of 8). ``workspace``: "auto" (allocated here) or a uint8 device
    tensor of dart_lmhead_stats_workspace_bytes(T, V) bytes."""
    return _lmhead_tok_stats(None, hidden, weight, target, logp, entropy, lse, workspace, stream)


def dart_lmhead_tok_stats_ex(hidden, weight, target, inv_temp, logp=None, entropy=None,
                             lse=None, workspace="auto", stream=None):
    """dart_lmhead_tok_stats of softmax(inv_temp * hidden @ weight^T)."""
    return _lmhead_tok_stats(float(inv_temp), hidden, weight, target, logp, entropy, lse,
                             workspace, stream)


def _lmhead_tok_stats(inv_temp, hidden, weight, target, logp, entropy, lse, workspace, stream):
    if (logp is None and entropy is None and lse is None and stream is None
            and isinstance(workspace, str) and workspace == "auto"):
        out = _nat().lmhead_tok_stats(hidden, weight, target, inv_temp)
        if out is not None:
            return _made(out, "dart_lmhead_tok_stats" + ("" if inv_temp is None else "_ex"))
    torch = _torch()
    _matrix_bf16("hidden", hidden)
    dev = hidden.device
    _matrix_bf16("weight", weight, dev)
    T, d = hidden.shape
    V = weight.shape[0]
    if weight.shape[1] != d:
        raise ValueError("hidden and weight must have the same inner size d")
    _check_vec("target", target, torch.int32, T, dev)
    logp = torch.empty(T, dtype=torch.float32, device=dev) if logp is None else logp
    entropy = torch.empty(T, dtype=torch.float32, device=dev) if entropy is None else entropy
    lse = torch.empty(T, dtype=torch.float32, device=dev) if lse is None else lse
    for n, v in (("logp", logp), ("entropy", entropy), ("lse", lse)):
        _check_vec(n, v, torch.float32, T, dev)
    if isinstance(workspace, str):
        if workspace != "auto":
            raise ValueError('workspace must be "auto" or a uint8 device tensor')
        workspace = torch.empty(dart_lmhead_stats_workspace_bytes(T, V), dtype=torch.uint8,
                                device=dev)
        if isinstance(stream, torch.cuda.Stream):
            workspace.record_stream(stream)
    if (not isinstance(workspace, torch.Tensor) or workspace.dtype != torch.uint8
            or workspace.device != dev or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous uint8 tensor on the device of the inputs")
    args = [hidden.data_ptr(), T, d, hidden.stride(0), weight.data_ptr(), V, weight.stride(0),
            target.data_ptr()]
    name = "dart_lmhead_tok_stats"
    if inv_temp is not None:
        args.append(inv_temp)
        name += "_ex"
    args += [logp.data_ptr(), entropy.data_ptr(), lse.data_ptr(), workspace.data_ptr(),
             workspace.numel(), _stream_handle(stream, dev)]
    rc = getattr(load_library(), name)(*args)
    if rc != DART_OK:
        raise DartError(name, rc)
    return logp, entropy, lse


def dart_lmhead_backward_workspace_bytes(chunk_rows: int, V: int) -> int:
    return int(load_library().dart_lmhead_backward_workspace_bytes(int(chunk_rows), int(V)))


def dart_lmhead_backward_ex_workspace_bytes(T: int, d: int, V: int, chunk_rows: int,
                                            chunk_cols: int, flags: int) -> int:
    return int(load_library().dart_lmhead_backward_ex_workspace_bytes(
        int(T), int(d), int(V), int(chunk_rows), int(chunk_cols), int(flags)))


def dart_lmhead_backward_split_workspace_bytes(T: int, d: int, V: int, chunk_rows: int,
                                               chunk_cols: int, flags: int) -> int:
    return int(load_library().dart_lmhead_backward_split_workspace_bytes(
        int(T), int(d), int(V), int(chunk_rows), int(chunk_cols), int(flags)))


def _lmhead_common(hidden, weight, target, lse, logp, tok_coef):
    torch = _torch()
    _matrix_bf16("hidden", hidden)
    dev = hidden.device
    _matrix_bf16("weight", weight, dev)
    T, d = hidden.shape
    if weight.shape[1] != d:
        raise ValueError("hidden and weight must have the same inner size d")
    _check_vec("target", target, torch.int32, T, dev)
    for n, v in (("lse", lse), ("logp", logp), ("tok_coef", tok_coef)):
        _check_vec(n, v, torch.float32, T, dev)
    return dev, T, d, weight.shape[0]


def dart_lmhead_dlogits(hidden, weight, target, lse, logp, tok_coef, dlogits=None, stream=None,
                        inv_temp=None):
    """bfloat16 [T, V] dlogits = tok_coef (onehot - softmax(hidden @ weight^T)), the
    logits recomputed on the matrix cores; lse and logp from dart_lmhead_tok_stats.
    With inv_temp (dart_lmhead_dlogits_ex): inv_temp tok_coef (onehot -
    softmax(inv_temp hidden @ weight^T)), lse and logp from dart_lmhead_tok_stats_ex."""
    torch = _torch()
    dev, T, d, V = _lmhead_common(hidden, weight, target, lse, logp, tok_coef)
    if dlogits is None:
        dlogits = torch.empty((T, V), dtype=torch.bfloat16, device=dev)
    _matrix_bf16("dlogits", dlogits, dev)
    if tuple(dlogits.shape) != (T, V):
        raise ValueError(f"dlogits must have shape ({T}, {V})")
    args = [hidden.data_ptr(), T, d, hidden.stride(0), weight.data_ptr(), V, weight.stride(0),
            target.data_ptr(), lse.data_ptr(), logp.data_ptr(), tok_coef.data_ptr()]
    name = "dart_lmhead_dlogits"
    if inv_temp is not None:
        args.append(float(inv_temp))
        name += "_ex"
    args += [dlogits.data_ptr(), dlogits.stride(0), _stream_handle(stream, dev)]
    rc = getattr(load_library(), name)(*args)
    if rc != DART_OK:
        raise DartError(name, rc)
    return dlogits


def _lmhead_backward(name, flags, hidden, weight, target, lse, logp, tok_coef, chunk_rows,
                     chunk_cols, dhidden, dweight, workspace, stream, inv_temp=1.0):
    torch = _torch()
    dev, T, d, V = _lmhead_common(hidden, weight, target, lse, logp, tok_coef)
    f = 0 if flags is None else int(flags)
    chunk_rows = max(1, min(int(chunk_rows), T))
    chunk_cols = max(1, min(int(chunk_cols), V))
    gdt = torch.bfloat16 if f & DART_LMHEAD_BF16_GRADS else torch.float32
    dhidden = torch.empty((T, d), dtype=gdt, device=dev) if dhidden is None else dhidden
    dweight = torch.empty((V, d), dtype=gdt, device=dev) if dweight is None else dweight
    for n, m, shape in (("dhidden", dhidden, (T, d)), ("dweight", dweight, (V, d))):
        if (not isinstance(m, torch.Tensor) or m.dtype != gdt or m.device != dev
                or tuple(m.shape) != shape or m.stride(1) != 1):
            raise ValueError(f"{n} must be a {gdt} {shape} tensor on {dev} with contiguous rows")
    if isinstance(workspace, str):
        if workspace != "auto":
            raise ValueError('workspace must be "auto" or a uint8 device tensor')
        nbytes = dart_lmhead_backward_split_workspace_bytes(T, d, V, chunk_rows, chunk_cols, f)
        if nbytes == 0:
            raise ValueError(f"{name}: bad sizes or flags")
        try:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        except torch.OutOfMemoryError:
            # the least that does: up to 192 MiB less, slower
            nbytes = dart_lmhead_backward_ex_workspace_bytes(T, d, V, chunk_rows, chunk_cols, f)
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        if isinstance(stream, torch.cuda.Stream):
            workspace.record_stream(stream)
    if (not isinstance(workspace, torch.Tensor) or workspace.dtype != torch.uint8
            or workspace.device != dev or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous uint8 tensor on the device of the inputs")
    args = [hidden.data_ptr(), T, d, hidden.stride(0), weight.data_ptr(), V, weight.stride(0),
            target.data_ptr(), lse.data_ptr(), logp.data_ptr(), tok_coef.data_ptr()]
    if flags is not None:
        args.append(float(inv_temp))
    args += [dhidden.data_ptr(), dhidden.stride(0), dweight.data_ptr(), dweight.stride(0),
             chunk_rows]
    if flags is not None:
        args += [chunk_cols, f]
    args += [workspace.data_ptr(), workspace.numel(), _stream_handle(stream, dev)]
    rc = getattr(load_library(), name)(*args)
    if rc != DART_OK:
        raise DartError(name, rc)
    return dhidden, dweight


def dart_lmhead_backward(hidden, weight, target, lse, logp, tok_coef, chunk_rows=1024,
                         dhidden=None, dweight=None, workspace="auto", stream=None):
    """(dhidden float32 [T, d], dweight float32 [V, d]) of the loss through the LM
    head, dlogits formed chunk_rows rows at a time in ``workspace`` ("auto" or a
    uint8 device tensor of dart_lmhead_backward_workspace_bytes(min(chunk_rows, T), V)
    bytes)."""
    return _lmhead_backward("dart_lmhead_backward", None, hidden, weight, target, lse, logp,
                            tok_coef, chunk_rows, weight.shape[0], dhidden, dweight, workspace,
                            stream)


def dart_lmhead_backward_ex(hidden, weight, target, lse, logp, tok_coef, chunk_rows=None,
                            chunk_cols=None, flags=0, dhidden=None, dweight=None,
                            workspace="auto", stream=None, inv_temp=1.0):
    """dart_lmhead_backward in blocks of chunk_rows rows x chunk_cols vocabulary
    entries (both None: lmhead_backward_plan's block), at inverse temperature
    inv_temp (lse and logp from dart_lmhead_tok_stats_ex at the same value),
    with flags (bitwise or):
    DART_LMHEAD_BF16_GRADS: dhidden and dweight in bfloat16;
    DART_LMHEAD_SKIP_ZERO_ROWS: the GEMMs over the rows with tok_coef != 0 only
    (their count is read on the device: the call stays asynchronous).
    ``workspace`` is "auto" or a uint8 device tensor of
    dart_lmhead_backward_ex_workspace_bytes(T, d, V, chunk_rows, chunk_cols, flags)
    bytes; one of dart_lmhead_backward_split_workspace_bytes(...), as "auto" allocates where
    there is the memory, is faster where a block has few rows, and leaves zero rows out of
    large calls unasked."""
    if chunk_rows is None and chunk_cols is None:
        chunk_rows, chunk_cols = lmhead_backward_plan(hidden.shape[0], weight.shape[0])
    elif chunk_rows is None or chunk_cols is None:
        raise ValueError("give both chunk_rows and chunk_cols, or neither")
    return _lmhead_backward("dart_lmhead_backward_ex", int(flags), hidden, weight, target, lse,
                            logp, tok_coef, chunk_rows, chunk_cols, dhidden, dweight, workspace,
                            stream, inv_temp)


def lmhead_backward_plan(T: int, V: int, budget_bytes: int = 512 << 20):
    """(chunk_rows, chunk_cols) for dart_lmhead_backward_ex: the block whose bf16
    dlogits fit budget_bytes and that rewrites the summed outputs least. Each of
    the ceil(T / rows) row blocks rewrites the [V, d] dweight and each of the
    ceil(V / cols) vocabulary blocks the [T, d] dhidden, so the cost is
    ceil(T / rows) V + ceil(V / cols) T; blocks are whole 256-wide tiles (or all
    of T, V). All rows when T << V, square blocks when T ~ V."""
    T, V = int(T), int(V)
    elems = max(budget_bytes // 2, 256 * 256)
    best = None
    for rows in sorted({T} | set(range(256, T, 256))):
        cols = V if rows * V <= elems else (elems // rows) // 256 * 256
        if cols < 256:
            continue
        cost = -(-T // rows) * V + -(-V // cols) * T
        if best is None or cost < best[0]:
            best = (cost, rows, cols)
    if best is None:
        return min(T, 256), min(V, 256)
    return best[1], best[2]


def _on(stream, device):
    """A context in which ``stream`` (as _stream_handle takes it) is the current one of ``device``,
    and that the current device: the null stream is the current device's, and what is allocated in
    it is handed out, and again after it, in the order of the stream whose kernels use it."""
    torch = _torch()
    if stream is None:
        here = torch.cuda.current_device() == device.index
        return contextlib.nullcontext() if here else torch.cuda.device(device)
    handle = _stream_handle(stream, device)
    if not isinstance(stream, torch.cuda.Stream):  # (a handle of 0 would make a new stream)
        stream = (torch.cuda.ExternalStream(handle, device=device) if handle
                  else torch.cuda.default_stream(device))
    return torch.cuda.stream(stream)


def _enqueue(name, device, *args):
    """The C call ``name`` on the current stream of ``device``, inside _on."""
    rc = getattr(load_library(), name)(*args, _stream_handle(None, device))
    if rc != DART_OK:
        raise DartError(name, rc)


def _out_matrix(name, out, shape, dtype, device):
    """``out``, or a new tensor, of this shape and type, with contiguous rows that do not overlap."""
    torch = _torch()
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if (not isinstance(out, torch.Tensor) or out.dtype != dtype or out.device != device
            or tuple(out.shape) != shape or (shape[1] > 1 and out.stride(1) != 1)
            or (shape[0] > 1 and out.stride(0) < shape[1])):
        raise ValueError(f"{name} must be a {dtype} {shape} tensor on {device} with contiguous rows")
    return out


def _span(t):
    """The addresses [first, end) between which a matrix or a vector lies."""
    last = (t.shape[0] - 1) * t.stride(0) + t.shape[1] if t.ndim == 2 else t.numel()
    return t.data_ptr(), t.data_ptr() + last * t.element_size()


def _share_memory(x, y):
    """Whether any byte is in both. Columns of one wider matrix lie between each other's rows: with
    rows equally far apart, their places in a row decide."""
    (a, a_end), (b, b_end) = _span(x), _span(y)
    if a >= b_end or b >= a_end:
        return False
    if x.ndim == y.ndim == 2 and min(x.shape[0], y.shape[0]) > 1:
        pitch, wx, wy = (n * t.element_size() for n, t in ((x.stride(0), x), (x.shape[1], x),
                                                            (y.shape[1], y)))
        if pitch == y.stride(0) * y.element_size() and max(wx, wy) <= pitch:
            return (b - a) % pitch < wx or (a - b) % pitch < wy
    return True


def _check_apart(writes, reads):
    """Refuses a tensor that the call writes (name -> tensor, or None) where it shares memory with
    another of them or with one that the call reads."""
    done = [(n, t) for n, t in reads.items() if t is not None]
    for name, out in writes.items():
        if out is None:
            continue
        for other_name, other in done:
            if _share_memory(out, other):
                raise ValueError(f"the memory of {name} and {other_name} must not overlap")
        done.append((name, out))


def _ld(t):
    """The row stride of a matrix (of one row: its length)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _byte_workspace(workspace, nbytes, device):
    """``workspace``, or for "auto" a new uint8 tensor of nbytes."""
    torch = _torch()
    if isinstance(workspace, str):
        if workspace != "auto":
            raise ValueError('workspace must be "auto" or a uint8 device tensor')
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
    if (not isinstance(workspace, torch.Tensor) or workspace.dtype != torch.uint8
            or workspace.device != device or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous uint8 tensor on the device of the inputs")
    return workspace


def dart_lmhead_xent_fwd_workspace_bytes(T: int, d: int, V: int) -> int:
    return int(load_library().dart_lmhead_xent_fwd_workspace_bytes(int(T), int(d), int(V)))


def dart_lmhead_xent_workspace_bytes(T: int, d: int, V: int, chunk_rows: int) -> int:
    return int(load_library().dart_lmhead_xent_workspace_bytes(int(T), int(d), int(V),
                                                               int(chunk_rows)))


def lmhead_xent_plan(T: int, V: int, budget_bytes: int = 2 << 30) -> int:
    """chunk_rows for dart_lmhead_xent_fwd_bwd: all rows where their exponentials fit
    budget_bytes, else as many whole tiles of 256 as do, the chunks of one size: each chunk reads
    and rewrites the [V, d] sum of dweight."""
    T, V = int(T), max(int(V), 1)  # (sizes of 0 are the call's to refuse)
    most = max(budget_bytes // (2 * ((V + 7) // 8 * 8)), 256)
    if T <= most:
        return T
    most = most // 256 * 256
    chunks = -(-T // most)
    return min(most, -(-T // chunks // 256) * 256)


def _xent_inputs(hidden, weight, target, label_smoothing, z_loss, reduction):
    torch = _torch()
    _matrix_bf16("hidden", hidden)
    dev = hidden.device
    _matrix_bf16("weight", weight, dev)
    T, d = hidden.shape
    if weight.shape[1] != d:
        raise ValueError("hidden and weight must have the same inner size d")
    _check_vec("target", target, torch.int32, T, dev)
    if reduction not in DART_XENT:
        raise ValueError(f"reduction must be one of {sorted(DART_XENT)}")
    config = dart_xent_config_t(float(label_smoothing), float(z_loss), DART_XENT[reduction])
    return dev, T, d, weight.shape[0], config


def dart_lmhead_xent_fwd(hidden, weight, target, label_smoothing=0.0, z_loss=0.0, reduction="mean",
                         workspace="auto", stream=None):
    """(loss float32 [1], tok_loss float32 [T], n_valid int32 [1]): the cross entropy of
    softmax(hidden @ weight^T) with the targets, without materialising the logits; hidden [T, d] and
    weight [V, d] bfloat16 (d a multiple of 8), target int32 [T]. Rows whose target is negative
    (-100, say) have a loss of 0 and do not count. Per row, with eps = label_smoothing:
    (1 - eps) (lse - z_y) + eps (lse - mean z) + z_loss lse^2; ``reduction``: "mean" over the rows
    that count, or "sum". ``workspace``: "auto" (allocated here) or a uint8 device tensor of
    dart_lmhead_xent_fwd_workspace_bytes(T, d, V) bytes."""
    if stream is None and isinstance(workspace, str) and workspace == "auto":
        out = _nat().lmhead_xent_fwd(hidden, weight, target, label_smoothing, z_loss,
                                     DART_XENT.get(reduction))
        if out is not None:
            return _made(out, "dart_lmhead_xent_fwd")
    torch = _torch()
    dev, T, d, V, config = _xent_inputs(hidden, weight, target, label_smoothing, z_loss, reduction)
    with _on(stream, dev):
        loss = torch.empty(1, dtype=torch.float32, device=dev)
        tok = torch.empty(T, dtype=torch.float32, device=dev)
        n = torch.empty(1, dtype=torch.int32, device=dev)
        workspace = _byte_workspace(workspace, dart_lmhead_xent_fwd_workspace_bytes(T, d, V), dev)
        _check_apart(dict(workspace=workspace), dict(hidden=hidden, weight=weight, target=target))
        _enqueue("dart_lmhead_xent_fwd", dev, hidden.data_ptr(), T, d, _ld(hidden),
                 weight.data_ptr(), V, _ld(weight), target.data_ptr(), ctypes.byref(config),
                 loss.data_ptr(), tok.data_ptr(), n.data_ptr(), workspace.data_ptr(),
                 workspace.numel())
    return loss, tok, n


def dart_lmhead_xent_fwd_bwd(hidden, weight, target, label_smoothing=0.0, z_loss=0.0,
                             reduction="mean", chunk_rows=None, dhidden=None, dweight=None,
                             want=(True, True), workspace="auto", stream=None):
    """dart_lmhead_xent_fwd's (loss, tok_loss, n_valid) and the loss's gradients (dhidden [T, d],
    dweight [V, d]) in bfloat16, the logits formed once: chunk_rows rows of their exponentials at a
    time are kept in the workspace (default: lmhead_xent_plan's; fewer than 32 take more workspace,
    not less). ``want`` says which gradients to form (None is returned for the other); ``dhidden``
    and ``dweight`` are matrices to write them to, apart from the inputs. ``workspace``: "auto"
    (allocated here) or a uint8 device tensor of dart_lmhead_xent_workspace_bytes(T, d, V, chunk_rows)
    bytes."""
    want_h, want_w = map(bool, want)
    if not (want_h or want_w):
        raise ValueError("want at least one gradient")
    if (stream is None and dhidden is None and dweight is None and isinstance(workspace, str)
            and workspace == "auto" and getattr(hidden, "ndim", 0) == getattr(weight, "ndim", 0) == 2):
        T, V = hidden.shape[0], weight.shape[0]
        rows = lmhead_xent_plan(T, V) if chunk_rows is None else max(1, min(int(chunk_rows), T))
        out = _nat().lmhead_xent_fwd_bwd(hidden, weight, target, label_smoothing, z_loss,
                                         DART_XENT.get(reduction), rows, want_h, want_w)
        if out is not None:
            return _made(out, "dart_lmhead_xent_fwd_bwd")
    torch = _torch()
    dev, T, d, V, config = _xent_inputs(hidden, weight, target, label_smoothing, z_loss, reduction)
    bf16 = torch.bfloat16
    chunk_rows = lmhead_xent_plan(T, V) if chunk_rows is None else max(1, min(int(chunk_rows), T))
    with _on(stream, dev):
        dhidden = _out_matrix("dhidden", dhidden, (T, d), bf16, dev) if want_h else None
        dweight = _out_matrix("dweight", dweight, (V, d), bf16, dev) if want_w else None
        loss = torch.empty(1, dtype=torch.float32, device=dev)
        tok = torch.empty(T, dtype=torch.float32, device=dev)
        n = torch.empty(1, dtype=torch.int32, device=dev)
        nbytes = dart_lmhead_xent_workspace_bytes(T, d, V, chunk_rows)
        workspace = _byte_workspace(workspace, nbytes, dev)
        _check_apart(dict(dhidden=dhidden, dweight=dweight, workspace=workspace),
                     dict(hidden=hidden, weight=weight, target=target))
        _enqueue("dart_lmhead_xent_fwd_bwd", dev, hidden.data_ptr(), T, d, _ld(hidden),
                 weight.data_ptr(), V, _ld(weight), target.data_ptr(), ctypes.byref(config),
                 loss.data_ptr(), tok.data_ptr(), n.data_ptr(), _ptr(dhidden),
                 _ld(dhidden) if want_h else 0, _ptr(dweight), _ld(dweight) if want_w else 0,
                 chunk_rows, workspace.data_ptr(), workspace.numel())
    return loss, tok, n, dhidden, dweight


def dart_grad_scale(x, factor, stream=None):
    """x *= factor in place for a 2-D bfloat16 or float32 tensor with contiguous rows and a float32
    scalar on the same GPU; where the factor is 1, x is not touched. Returns x."""
    torch = _torch()
    if not isinstance(x, torch.Tensor) or str(x.dtype) not in _FLOATS or x.dim() != 2:
        raise TypeError("x must be a 2-D float32 or bfloat16 tensor")
    if not x.is_cuda or x.numel() == 0:
        raise ValueError("x must be on a GPU and not empty")
    _out_matrix("x", x, tuple(x.shape), x.dtype, x.device)
    if (not isinstance(factor, torch.Tensor) or factor.dtype != torch.float32
            or factor.device != x.device or factor.numel() != 1):
        raise ValueError(f"factor must be a float32 tensor of one element on {x.device}")
    _check_apart(dict(x=x), dict(factor=factor.reshape(1)))
    with _on(stream, x.device):
        _enqueue("dart_grad_scale", x.device, x.data_ptr(), _FLOATS[str(x.dtype)], x.shape[0],
                 x.shape[1], _ld(x), factor.data_ptr())
    return x


_FLOATS = {"torch.float32": DART_F32, "torch.bfloat16": DART_BF16}


class Mxfp4(NamedTuple):
    """A rows x cols matrix in blocks of 32 four-bit values with a power-of-two scale, as
    dart_mxfp4_quantize makes it: ``data`` uint8 [dart_mxfp4_bytes(rows, cols)] (include/dart.h says
    which byte is which)."""

    data: object
    rows: int
    cols: int


def dart_mxfp4_bytes(R: int, K: int) -> int:
    return int(load_library().dart_mxfp4_bytes(int(R), int(K)))


def dart_lmhead_mxfp4_stats_workspace_bytes(T: int, V: int) -> int:
    return int(load_library().dart_lmhead_mxfp4_stats_workspace_bytes(int(T), int(V)))


def _check_mxfp4(name, q, device=None):
    torch = _torch()
    if not isinstance(q, Mxfp4):
        raise TypeError(f"{name} must be an Mxfp4")
    t, n = q.data, dart_mxfp4_bytes(q.rows, q.cols)
    if (not isinstance(t, torch.Tensor) or t.dtype != torch.uint8 or not t.is_contiguous()
            or n == 0 or t.numel() != n or not t.is_cuda or t.data_ptr() % 16):
        raise ValueError(f"{name}.data must be a contiguous, 16-byte aligned uint8 tensor of {n} bytes "
                         "on a GPU")
    if device is not None and t.device != device:
        raise ValueError(f"{name} must be on {device}")


def dart_mxfp4_quantize(x, out=None, stream=None):
    """The Mxfp4 of a 2-D float32 or bfloat16 tensor with contiguous rows: along a row, blocks of 32
    values share the scale 2^max(floor(log2 of the largest size) - 2, -127), and each becomes the
    nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times it (ties to the even code, larger ones 6). A block
    with an infinity or a NaN stands for NaN. ``out``: an Mxfp4 of the same shape to write to."""
    if out is None and stream is None:
        made = _nat().mxfp4_quantize(x)
        if made is not None:
            return Mxfp4(_made(made, "dart_mxfp4_quantize")[0], *x.shape)
    torch = _torch()
    if not isinstance(x, torch.Tensor) or str(x.dtype) not in _FLOATS:
        raise TypeError("x must be a float32 or bfloat16 tensor")
    if x.dim() != 2 or not x.is_cuda or x.numel() == 0 or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError("x must be a 2-D tensor on a GPU, not empty, with contiguous rows")
    R, K = x.shape
    ld = _ld(x)
    if ld < K:
        raise ValueError("the rows of x must not overlap")
    if out is not None:
        _check_mxfp4("out", out, x.device)
        if (out.rows, out.cols) != (R, K):
            raise ValueError(f"out must be {R} x {K}")
        _check_apart(dict(out=out.data), dict(x=x))
    with _on(stream, x.device):
        if out is None:
            out = Mxfp4(torch.empty(dart_mxfp4_bytes(R, K), dtype=torch.uint8, device=x.device), R, K)
        _enqueue("dart_mxfp4_quantize", x.device, x.data_ptr(), _FLOATS[str(x.dtype)], R, K, ld,
                 out.data.data_ptr())
    return out


def dart_mxfp4_dequantize(q, dtype=None, out=None, stream=None):
    """The values that an Mxfp4 stands for, as a [rows, cols] bfloat16 (default) or float32 tensor."""
    if out is None and stream is None:
        made = _nat().mxfp4_dequantize(q, dtype)
        if made is not None:
            return _made(made, "dart_mxfp4_dequantize")[0]
    torch = _torch()
    _check_mxfp4("q", q)
    dtype = (torch.bfloat16 if out is None else out.dtype) if dtype is None else dtype
    if str(dtype) not in _FLOATS:
        raise TypeError("dtype must be float32 or bfloat16")
    with _on(stream, q.data.device):
        out = _out_matrix("out", out, (q.rows, q.cols), dtype, q.data.device)
        _check_apart(dict(out=out), dict(q=q.data))
        _enqueue("dart_mxfp4_dequantize", out.device, q.data.data_ptr(), q.rows,
                 q.cols, _FLOATS[str(dtype)], out.data_ptr(), _ld(out))
    return out


def _rows_against(name, x, weight):
    """The rows of ``x``, an Mxfp4 or a float32 or bfloat16 matrix that fits the Mxfp4 ``weight``."""
    dev = weight.data.device
    if isinstance(x, Mxfp4):
        _check_mxfp4(name, x, dev)
        shape = (x.rows, x.cols)
    else:
        if str(getattr(x, "dtype", None)) not in _FLOATS:
            raise TypeError(f"{name} must be an Mxfp4 or a float32 or bfloat16 tensor")
        if x.device != dev:
            raise ValueError(f"{name} must be on {dev}")
        shape = tuple(x.shape)
    if len(shape) != 2 or shape[1] != weight.cols:
        raise ValueError(f"{name} must be a matrix of the weight's inner size, {weight.cols}")
    return shape[0]


def _as_mxfp4(x, stream):
    """``x`` itself where it is an Mxfp4, else (a float32 or bfloat16 matrix) quantised."""
    return x if isinstance(x, Mxfp4) else dart_mxfp4_quantize(x, stream=stream)


def dart_mxfp4_matmul(a, b, dtype=None, out=None, stream=None):
    """a @ b^T of Mxfp4 matrices a [M, K] and b [N, K], summed in float32, as a [M, N] bfloat16
    (default) or float32 tensor: the logits of tokens ``a`` under a head ``b`` kept in four bits.
    ``a`` may be a float32 or bfloat16 tensor, which is quantised first."""
    if out is None and stream is None:
        made = _nat().mxfp4_matmul(a, b, dtype)
        if made is not None:
            return _made(made, "dart_mxfp4_matmul", "dart_mxfp4_quantize")[0]
    torch = _torch()
    _check_mxfp4("b", b)
    dtype = (torch.bfloat16 if out is None else out.dtype) if dtype is None else dtype
    if str(dtype) not in _FLOATS:
        raise TypeError("dtype must be float32 or bfloat16")
    dev = b.data.device
    rows = _rows_against("a", a, b)
    with _on(stream, dev):
        out = _out_matrix("out", out, (rows, b.rows), dtype, dev)
        _check_apart(dict(out=out), dict(a=a.data if isinstance(a, Mxfp4) else a, b=b.data))
        a = _as_mxfp4(a, stream)
        _enqueue("dart_mxfp4_matmul", dev, a.data.data_ptr(), a.rows, b.data.data_ptr(), b.rows,
                 b.cols, _FLOATS[str(dtype)], out.data_ptr(), _ld(out))
    return out


def dart_lmhead_mxfp4_tok_stats(hidden, weight, target, inv_temp=1.0, logp=None, entropy=None,
                                lse=None, workspace="auto", stream=None):
    """(logp, entropy, lse) float32 [T] of softmax(inv_temp * hidden @ weight^T) for an Mxfp4 weight
    [V, d] and hidden states [T, d] in Mxfp4, or in float32 or bfloat16 and quantised first: the
    log-probs of a rollout policy whose head is kept in four bits, without materialising the logits.
    ``workspace``: "auto" (allocated here) or a uint8 device tensor of
    dart_lmhead_mxfp4_stats_workspace_bytes(T, V) bytes."""
    if (logp is None and entropy is None and lse is None and stream is None
            and isinstance(workspace, str) and workspace == "auto"):
        out = _nat().lmhead_mxfp4_tok_stats(hidden, weight, target, inv_temp)
        if out is not None:
            return _made(out, "dart_lmhead_mxfp4_tok_stats", "dart_mxfp4_quantize")
    torch = _torch()
    _check_mxfp4("weight", weight)
    dev = weight.data.device
    T, V = _rows_against("hidden", hidden, weight), weight.rows
    _check_vec("target", target, torch.int32, T, dev)
    with _on(stream, dev):
        logp = torch.empty(T, dtype=torch.float32, device=dev) if logp is None else logp
        entropy = torch.empty(T, dtype=torch.float32, device=dev) if entropy is None else entropy
        lse = torch.empty(T, dtype=torch.float32, device=dev) if lse is None else lse
        for n, v in (("logp", logp), ("entropy", entropy), ("lse", lse)):
            _check_vec(n, v, torch.float32, T, dev)
        workspace = _byte_workspace(workspace, dart_lmhead_mxfp4_stats_workspace_bytes(T, V), dev)
        _check_apart(dict(logp=logp, entropy=entropy, lse=lse, workspace=workspace),
                     dict(hidden=hidden.data if isinstance(hidden, Mxfp4) else hidden,
                          weight=weight.data, target=target))
        hidden = _as_mxfp4(hidden, stream)
        _enqueue("dart_lmhead_mxfp4_tok_stats", dev, hidden.data.data_ptr(), T,
                 weight.data.data_ptr(), V, weight.cols, target.data_ptr(), float(inv_temp),
                 logp.data_ptr(), entropy.data_ptr(), lse.data_ptr(), workspace.data_ptr(),
                 workspace.numel())
    return logp, entropy, lse


_UPDATE = ("logp", "entropy", "lse", "step_entropy", "step_mask", "n_kept_steps", "loss",
           "dlogits", "tok_coef", "stats")


def policy_update(logits, target, logp_old, logp_rollout, adv, step_offsets, rho, eps_low,
                  eps_high, C, dlogits=None, stream=None):
    """tok_stats -> select_tis_loss_fwd -> tis_grad on one stream. Returns a dict
    of device tensors (nothing is synchronised)."""
    if stream is None:
        out = _nat().policy_update(logits, target, logp_old, logp_rollout, adv, step_offsets, rho,
                                   eps_low, eps_high, C, dlogits)
        if out is not None:
            out = _made(out, "dart_tok_stats", "dart_select_tis_loss_fwd", "dart_tis_grad")
            return dict(zip(_UPDATE, out))
    logp, ent, lse = dart_tok_stats(logits, target, stream=stream)
    step_ent, mask, n_kept, loss, coef, stats = dart_select_tis_loss_fwd(
        ent, logp, logp_old, logp_rollout, adv, step_offsets, rho, eps_low, eps_high, C,
        stream=stream)
    dz = dart_tis_grad(logits, target, logp, lse, coef, dlogits, stream=stream)
    return dict(logp=logp, entropy=ent, lse=lse, step_entropy=step_ent, step_mask=mask,
                n_kept_steps=n_kept, loss=loss, dlogits=dz, tok_coef=coef, stats=stats)
