"""Binding of the worker-side entry points of libstar.so: losses on logits with their gradients, activations kept in 8
bits and the weight gradient formed from them.  Argument marshalling only, as in ``binding``; outputs are tensors that the
caller hands in.  A workspace, where a call needs one, is taken from torch's allocator on the call's stream, or
passed in (a uint8 tensor of at least the bytes the C header's ``*_workspace`` function returns)."""
from __future__ import annotations

import ctypes
import functools
from typing import Optional

import numpy as np

from .binding import BF16, F32, StarError, _stream_handle, last_error, load_library

_lib = None
_ERR_NULL = 1     # STAR_ERR_NULL


class _PolicyParams(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("clip_low", ctypes.c_float), ("clip_high", ctypes.c_float),
                ("kl_coef", ctypes.c_float), ("temperature", ctypes.c_float)]


class _PreferenceParams(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("beta", ctypes.c_float), ("label_smoothing", ctypes.c_float),
                ("temperature", ctypes.c_float)]


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        vp, i32, i64, size, f32, st = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float,
                                       ctypes.c_int)
        logits = [vp, st, i64, i64, i64, vp]
        signatures = {
            "star_token_logprobs": (st, logits + [f32, vp, vp, vp, size, vp]),
            "star_token_logprobs_grad": (st, logits + [f32, vp, vp, vp, i64, vp]),
            "star_policy_loss": (st, logits + [vp, vp, vp, vp, vp, vp, i64, vp, vp, vp, size, vp]),
            "star_preference_loss": (st, logits + [vp, vp, i32, vp, vp, vp, i64, vp, vp, vp, vp, size, vp]),
            "star_token_logprobs_workspace": (size, [st, i64, i64]),
            "star_policy_loss_workspace": (size, [st, i64, i64]),
            "star_preference_loss_workspace": (size, [st, i64, i64, i32]),
            "star_act_bytes": (size, [i64, i64]),
            "star_act_pack": (st, [vp, st, i64, i64, i64, vp, vp]),
            "star_act_unpack": (st, [vp, i64, i64, vp, st, i64, vp]),
            "star_act_weight_grad": (st, [vp, st, i64, i64, i64, vp, i64, vp, st, i32, vp, size, vp]),
            "star_act_weight_grad_workspace": (size, [st, i64, i64, i64]),
        }
        for name, (result, arguments) in signatures.items():
            f = getattr(lib, name)
            f.restype, f.argtypes = result, arguments
        _lib = lib
    return _lib


def _check(status: int):
    if status != 0:
        raise StarError(status, last_error())


# torch's own names, looked up once: these checks are most of what a call on a few rows costs the host (a call of
# star_token_logprobs on one row 6.4 us with them in their first form, the kernel itself 2).
_torch = _codes = _f32 = _i64 = None


def _names():
    global _torch, _codes, _f32, _i64
    import torch
    _torch, _f32, _i64 = torch, torch.float32, torch.int64
    _codes = {torch.float32: F32, torch.bfloat16: BF16}


def _dtype(x, what: str) -> int:
    if _codes is None:
        _names()
    code = _codes.get(x.dtype)
    if code is None:
        raise TypeError(f"{what} must be a float32 or bfloat16 tensor")
    return code


def _matrix(x, what: str, rows=None, columns=None):
    """(address, rows, columns, distance of the rows) of a 2-D tensor whose rows are contiguous."""
    if x.dim() != 2 or (rows is not None and (x.size(0) != rows or x.size(1) != columns)):
        raise ValueError(f"{what} must be a 2-D tensor" + ("" if rows is None else f" of shape ({rows}, {columns})"))
    rows, columns = x.shape
    if x.is_contiguous():
        return x.data_ptr(), rows, columns, columns
    step = x.stride(0) if rows > 1 else columns
    if (columns > 1 and x.stride(1) != 1) or step < columns:
        raise ValueError(f"the rows of {what} must be contiguous and must not overlap")
    return x.data_ptr(), rows, columns, step


def _vector(x, dtype, n: int, what: str, device: int):
    """Address of a contiguous vector of n; ``device``: the index of the logits' device."""
    if x is None:
        return None
    if x.dtype is not dtype or x.dim() != 1 or x.size(0) != n or not x.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} tensor [{n}]")
    if x.get_device() != device:
        raise ValueError(f"{what} must be on the first tensor's device")
    return x.data_ptr()


def _logits(logits, targets, dlogits=None):
    """What every call on logits begins with: (address, dtype code, tokens, vocab, ld, targets), its gradient's (address,
    ld), and the device's index."""
    code = _dtype(logits, "logits")
    x, tokens, vocab, ld = _matrix(logits, "logits")
    device = logits.get_device()
    out, ld_out = None, ld
    if dlogits is not None:
        if dlogits.dtype is not logits.dtype or dlogits.get_device() != device:
            raise TypeError("dlogits must have the logits' type and device")
        out, _, _, ld_out = _matrix(dlogits, "dlogits", tokens, vocab)
    return (x, code, tokens, vocab, ld, _vector(targets, _i64, tokens, "targets", device)), (out, ld_out), device


def _on_gpu(device: int):
    """A kernel must not be given the address of host memory, which it would fault on."""
    if device < 0:
        raise ValueError("the tensors must be in GPU memory")


@functools.lru_cache(maxsize=4096)
def _need(name: str, *sizes) -> int:
    """Workspace bytes of a call, by its sizes."""
    return getattr(_library(), name)(*sizes)


def _workspace(given, need: int, device: int, stream):
    """(address, bytes, the tensor to keep until the call is enqueued)."""
    if given is not None:
        if given.element_size() != 1 or not given.is_contiguous() or given.get_device() != device:
            raise ValueError("workspace must be a contiguous uint8 tensor on the same device")
        return given.data_ptr(), given.numel(), given
    if need == 0:
        return None, 0, None
    if stream is None:
        w = _torch.empty(need, dtype=_torch.uint8, device=device)
    else:
        # on the call's own stream, so that the memory is not handed out again before the call has run
        s = stream if isinstance(stream, _torch.cuda.Stream) else _torch.cuda.ExternalStream(int(stream), device=device)
        with _torch.cuda.stream(s):
            w = _torch.empty(need, dtype=_torch.uint8, device=device)
    return w.data_ptr(), need, w


def star_token_logprobs(logits, targets, logp_out, *, lse_out=None, temperature: float = 1.0, workspace=None,
                        stream=None) -> None:
    """``logp_out[t]`` = log-probability of ``targets[t]`` under softmax(logits[t] / temperature), ``lse_out[t]`` its
    normaliser (float32 [tokens]); both 0 where the target is outside the vocabulary.  ``logits``: float32 or bfloat16
    [tokens, vocab], rows at any distance; ``targets``: int64 [tokens]."""
    lib = _library()
    head, _, device = _logits(logits, targets)
    tokens = head[2]
    logp, lse = _vector(logp_out, _f32, tokens, "logp_out", device), _vector(lse_out, _f32, tokens, "lse_out", device)
    _on_gpu(device)
    w, size, _keep = _workspace(workspace, _need("star_token_logprobs_workspace", *head[1:4]), device, stream)
    _check(lib.star_token_logprobs(*head, temperature, logp, lse, w, size, _stream_handle(stream)))


def star_token_logprobs_grad(logits, targets, lse, dlogp, dlogits, *, temperature: float = 1.0, stream=None) -> None:
    """``dlogits`` of a function whose derivatives by the log-probabilities are ``dlogp`` (float32 [tokens]); ``lse`` as
    ``star_token_logprobs`` left it (beyond 64 in size, of bfloat16 rows 1024, where one fp32 number no longer holds it well enough, a row's sum is formed again).
    ``dlogits`` may be ``logits``."""
    lib = _library()
    head, out, device = _logits(logits, targets, dlogits)
    tokens = head[2]
    normaliser, slope = _vector(lse, _f32, tokens, "lse", device), _vector(dlogp, _f32, tokens, "dlogp", device)
    _on_gpu(device)
    _check(lib.star_token_logprobs_grad(*head, temperature, normaliser, slope, *out, _stream_handle(stream)))


def star_policy_loss(logits, targets, old_logp, advantages, stats_out, *, dlogits=None, ref_logp=None, weights=None,
                     scale: Optional[float] = None, clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0,
                     temperature: float = 1.0, logp_out=None, workspace=None, stream=None) -> None:
    """Clipped policy loss with a KL term and, if ``dlogits`` is given, its gradient.  ``stats_out``: float32 [4]: loss,
    KL estimate, clipped share, weight, each summed with ``scale * weights``.  ``scale``: None = 1 / tokens."""
    lib = _library()
    head, out, device = _logits(logits, targets, dlogits)
    n = head[2]
    p = _PolicyParams(1.0 / max(n, 1) if scale is None else scale, clip_low, clip_high, kl_coef, temperature)
    old, ref = _vector(old_logp, _f32, n, "old_logp", device), _vector(ref_logp, _f32, n, "ref_logp", device)
    adv, wts = _vector(advantages, _f32, n, "advantages", device), _vector(weights, _f32, n, "weights", device)
    logp, stats = _vector(logp_out, _f32, n, "logp_out", device), _vector(stats_out, _f32, 4, "stats_out", device)
    if kl_coef and ref is None:
        raise StarError(_ERR_NULL, "ref_logp is NULL and kl_coef is not 0")
    _on_gpu(device)
    w, size, _keep = _workspace(workspace, _need("star_policy_loss_workspace", *head[1:4]), device, stream)
    _check(lib.star_policy_loss(*head, old, ref, adv, wts, ctypes.byref(p), *out, logp, stats, w, size,
                                _stream_handle(stream)))


def star_preference_loss(logits, targets, ref_logp, offsets, loss_out, *, dlogits=None, weights=None,
                         scale: Optional[float] = None, beta: float = 0.1, label_smoothing: float = 0.0,
                         temperature: float = 1.0, logp_out=None, margins_out=None, workspace=None, stream=None) -> None:
    """Preference loss on pairs of answers and, if ``dlogits`` is given, its gradient.  ``offsets``: host sequence of
    2 pairs + 1 row numbers (preferred, other, preferred, ...); ``loss_out``: float32 [1]; ``margins_out``: float32
    [pairs].  ``scale``: None = 1 / pairs."""
    lib = _library()
    head, out, device = _logits(logits, targets, dlogits)
    n = head[2]
    at = np.ascontiguousarray(offsets, dtype=np.int64)
    if at.ndim != 1 or at.shape[0] % 2 != 1:
        raise ValueError("offsets must hold 2 pairs + 1 numbers")
    pairs = (at.shape[0] - 1) // 2
    p = _PreferenceParams(1.0 / max(pairs, 1) if scale is None else scale, beta, label_smoothing, temperature)
    ref, wts = _vector(ref_logp, _f32, n, "ref_logp", device), _vector(weights, _f32, n, "weights", device)
    logp, margins = _vector(logp_out, _f32, n, "logp_out", device), _vector(margins_out, _f32, pairs, "margins_out", device)
    loss = _vector(loss_out, _f32, 1, "loss_out", device)
    _on_gpu(device)
    w, size, _keep = _workspace(workspace, _need("star_preference_loss_workspace", *head[1:4], pairs), device, stream)
    _check(lib.star_preference_loss(*head, ref, wts, pairs, at.ctypes.data, ctypes.byref(p), *out, logp, margins, loss, w,
                                    size, _stream_handle(stream)))


def star_act_bytes(tokens: int, width: int) -> int:
    """Bytes of the packed form of activations [tokens, width]."""
    return _need("star_act_bytes", tokens, width)


def _packed(packed, tokens: int, width: int, device: int) -> int:
    if packed.element_size() != 1 or packed.dim() != 1 or not packed.is_contiguous() or packed.get_device() != device:
        raise ValueError("packed must be a contiguous 1-D uint8 tensor on the same device")
    if packed.size(0) < _need("star_act_bytes", tokens, width):
        raise ValueError("packed must hold star_act_bytes(tokens, width) bytes")
    return packed.data_ptr()


def star_act_pack(x, packed, *, stream=None) -> None:
    """Keeps ``x`` (float32 or bfloat16 [tokens, width], rows at any distance) in 8 bits in ``packed``, a uint8 tensor of
    ``star_act_bytes(tokens, width)`` bytes."""
    code = _dtype(x, "x")
    p, tokens, width, ld = _matrix(x, "x")
    device = x.get_device()
    to = _packed(packed, tokens, width, device)
    _on_gpu(device)
    _check(_library().star_act_pack(p, code, tokens, width, ld, to, _stream_handle(stream)))


def star_act_unpack(packed, out, *, stream=None) -> None:
    """The kept values of ``packed``, into ``out`` (float32 or bfloat16 [tokens, width])."""
    code = _dtype(out, "out")
    p, tokens, width, ld = _matrix(out, "out")
    device = out.get_device()
    source = _packed(packed, tokens, width, device)
    _on_gpu(device)
    _check(_library().star_act_unpack(source, tokens, width, p, code, ld, _stream_handle(stream)))


def star_act_weight_grad(dy, packed, dw, *, accumulate: bool = False, workspace=None, stream=None) -> None:
    """``dw`` [out, width] = (or, with ``accumulate``, +=) dy^T x for the activations x [tokens, width] in ``packed``.
    ``dy``: float32 or bfloat16 [tokens, out]; ``dw``: contiguous float32 or bfloat16, for example
    ``row[a:a + out * width].view(out, width)`` of a worker's gradient row."""
    lib = _library()
    dy_code, dw_code = _dtype(dy, "dy"), _dtype(dw, "dw")
    p, tokens, out, ld = _matrix(dy, "dy")
    if dw.dim() != 2 or dw.size(0) != out or not dw.is_contiguous():
        raise ValueError(f"dw must be a contiguous tensor [{out}, width]")
    device = dy.get_device()
    if dw.get_device() != device:
        raise ValueError("dw must be on dy's device")
    width = dw.size(1)
    kept = _packed(packed, tokens, width, device)
    _on_gpu(device)
    w, size, _keep = _workspace(workspace, _need("star_act_weight_grad_workspace", dy_code, tokens, out, width), device, stream)
    _check(lib.star_act_weight_grad(p, dy_code, tokens, out, ld, kept, width, dw.data_ptr(), dw_code,
                                    int(bool(accumulate)), w, size, _stream_handle(stream)))
