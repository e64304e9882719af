"""Binding of the worker-side entry points of libstar.so: losses on logits with their gradients, activations kept in 8
bits and the weight gradient formed from them.  Argument marshalling only, as in ``binding``; outputs are tensors that the
caller hands in.  A workspace, where a call needs one, is taken from torch's allocator on the call's stream, or
passed in (a uint8 tensor of at least the bytes the C header's ``*_workspace`` function returns)."""
from __future__ import annotations

import ctypes
from typing import Optional

import numpy as np

from .binding import BF16, F32, StarError, _stream_handle, last_error, load_library

_lib = None


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


_codes = None


def _dtype(x, what: str) -> int:
    global _codes
    if _codes is None:
        import torch
        _codes = {torch.float32: F32, torch.bfloat16: BF16}
    code = _codes.get(x.dtype)
    if code is None:
        raise TypeError(f"{what} must be a float32 or bfloat16 tensor")
    return code


def _matrix(x, what: str, shape=None):
    """(address, rows, columns, distance of the rows) of a 2-D tensor whose rows are contiguous."""
    if x.dim() != 2 or (shape is not None and tuple(x.shape) != shape):
        raise ValueError(f"{what} must be a 2-D tensor" + ("" if shape is None else f" of shape {shape}"))
    rows, columns = x.shape
    step = x.stride(0) if rows > 1 else columns
    if columns > 1 and x.stride(1) != 1 or step < columns:
        raise ValueError(f"the rows of {what} must be contiguous and must not overlap")
    return x.data_ptr(), rows, columns, step


def _floats(x, n: int, what: str, device):
    import torch
    if x is None:
        return None
    if x.dtype != torch.float32 or x.dim() != 1 or x.shape[0] != n or not x.is_contiguous():
        raise ValueError(f"{what} must be a contiguous float32 tensor [{n}]")
    if x.device != device:
        raise ValueError(f"{what} must be on the logits' device")
    return x.data_ptr()


def _logits(logits, targets, dlogits=None):
    """The arguments that every call on logits begins with, and those of its gradient."""
    import torch
    code = _dtype(logits, "logits")
    x, tokens, vocab, ld = _matrix(logits, "logits")
    if targets.dtype != torch.int64 or targets.dim() != 1 or targets.shape[0] != tokens or not targets.is_contiguous():
        raise ValueError(f"targets must be a contiguous int64 tensor [{tokens}]")
    if targets.device != logits.device:
        raise ValueError("targets must be on the logits' device")
    out, ld_out = None, ld
    if dlogits is not None:
        if dlogits.dtype != logits.dtype or dlogits.device != logits.device:
            raise TypeError("dlogits must have the logits' type and device")
        out, _, _, ld_out = _matrix(dlogits, "dlogits", (tokens, vocab))
        if out == x:
            ld_out = ld if tokens <= 1 else ld_out
    return (x, code, tokens, vocab, ld, targets.data_ptr()), (out, ld_out)


def _workspace(given, need: int, device, stream):
    """(address, bytes, the tensor to keep until the call is enqueued)."""
    if given is not None:
        if given.element_size() != 1 or not given.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 tensor")
        return given.data_ptr(), given.numel(), given
    if need == 0:
        return None, 0, None
    import torch
    if stream is None or device.type != "cuda":
        w = torch.empty(need, dtype=torch.uint8, device=device)
    else:
        # on the call's own stream, so that the memory is not handed out again before the call has run
        s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream), device=device)
        with torch.cuda.stream(s):
            w = torch.empty(need, dtype=torch.uint8, device=device)
    return w.data_ptr(), need, w


def star_token_logprobs(logits, targets, logp_out, *, lse_out=None, temperature: float = 1.0, workspace=None,
                        stream=None) -> None:
    """``logp_out[t]`` = log-probability of ``targets[t]`` under softmax(logits[t] / temperature), ``lse_out[t]`` its
    normaliser (float32 [tokens]); both 0 where the target is outside the vocabulary.  ``logits``: float32 or bfloat16
    [tokens, vocab], rows at any distance; ``targets``: int64 [tokens]."""
    lib = _library()
    head, _ = _logits(logits, targets)
    _, code, tokens, vocab, _, _ = head
    logp, lse = _floats(logp_out, tokens, "logp_out", logits.device), _floats(lse_out, tokens, "lse_out", logits.device)
    w, size, _keep = _workspace(workspace, lib.star_token_logprobs_workspace(code, tokens, vocab), logits.device, stream)
    _check(lib.star_token_logprobs(*head, temperature, logp, lse, w, size, _stream_handle(stream)))


def star_token_logprobs_grad(logits, targets, lse, dlogp, dlogits, *, temperature: float = 1.0, stream=None) -> None:
    """``dlogits`` of a function whose derivatives by the log-probabilities are ``dlogp`` (float32 [tokens]); ``lse`` as
    ``star_token_logprobs`` left it.  ``dlogits`` may be ``logits``."""
    lib = _library()
    head, out = _logits(logits, targets, dlogits)
    tokens = head[2]
    _check(lib.star_token_logprobs_grad(*head, temperature, _floats(lse, tokens, "lse", logits.device),
                                        _floats(dlogp, tokens, "dlogp", logits.device), *out, _stream_handle(stream)))


def star_policy_loss(logits, targets, old_logp, advantages, stats_out, *, dlogits=None, ref_logp=None, weights=None,
                     scale: Optional[float] = None, clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0,
                     temperature: float = 1.0, logp_out=None, workspace=None, stream=None) -> None:
    """Clipped policy loss with a KL term and, if ``dlogits`` is given, its gradient.  ``stats_out``: float32 [4]: loss,
    KL estimate, clipped share, weight, each summed with ``scale * weights``.  ``scale``: None = 1 / tokens."""
    lib = _library()
    head, out = _logits(logits, targets, dlogits)
    _, code, tokens, vocab, _, _ = head
    device = logits.device
    p = _PolicyParams(1.0 / max(tokens, 1) if scale is None else scale, clip_low, clip_high, kl_coef, temperature)
    old, ref = _floats(old_logp, tokens, "old_logp", device), _floats(ref_logp, tokens, "ref_logp", device)
    adv, wts = _floats(advantages, tokens, "advantages", device), _floats(weights, tokens, "weights", device)
    logp, stats = _floats(logp_out, tokens, "logp_out", device), _floats(stats_out, 4, "stats_out", device)
    w, size, _keep = _workspace(workspace, lib.star_policy_loss_workspace(code, tokens, vocab), device, stream)
    _check(lib.star_policy_loss(*head, old, ref, adv, wts, ctypes.byref(p), *out, logp, stats, w, size,
                                _stream_handle(stream)))


def star_preference_loss(logits, targets, ref_logp, offsets, loss_out, *, dlogits=None, weights=None,
                         scale: Optional[float] = None, beta: float = 0.1, label_smoothing: float = 0.0,
                         temperature: float = 1.0, logp_out=None, margins_out=None, workspace=None, stream=None) -> None:
    """Preference loss on pairs of answers and, if ``dlogits`` is given, its gradient.  ``offsets``: host sequence of
    2 pairs + 1 row numbers (preferred, other, preferred, ...); ``loss_out``: float32 [1]; ``margins_out``: float32
    [pairs].  ``scale``: None = 1 / pairs."""
    lib = _library()
    head, out = _logits(logits, targets, dlogits)
    _, code, tokens, vocab, _, _ = head
    device = logits.device
    at = np.ascontiguousarray(offsets, dtype=np.int64)
    if at.ndim != 1 or at.shape[0] % 2 != 1:
        raise ValueError("offsets must hold 2 pairs + 1 numbers")
    pairs = (at.shape[0] - 1) // 2
    p = _PreferenceParams(1.0 / max(pairs, 1) if scale is None else scale, beta, label_smoothing, temperature)
    ref, wts = _floats(ref_logp, tokens, "ref_logp", device), _floats(weights, tokens, "weights", device)
    logp, margins = _floats(logp_out, tokens, "logp_out", device), _floats(margins_out, pairs, "margins_out", device)
    loss = _floats(loss_out, 1, "loss_out", device)
    w, size, _keep = _workspace(workspace, lib.star_preference_loss_workspace(code, tokens, vocab, pairs), device, stream)
    _check(lib.star_preference_loss(*head, ref, wts, pairs, at.ctypes.data, ctypes.byref(p), *out, logp, margins, loss, w,
                                    size, _stream_handle(stream)))


def star_act_bytes(tokens: int, width: int) -> int:
    """Bytes of the packed form of activations [tokens, width]."""
    return int(_library().star_act_bytes(tokens, width))


def _packed(packed, tokens: int, width: int, device) -> int:
    if packed.element_size() != 1 or packed.dim() != 1 or not packed.is_contiguous() or packed.device != device:
        raise ValueError("packed must be a contiguous 1-D uint8 tensor on the same device")
    if packed.shape[0] < star_act_bytes(tokens, width):
        raise ValueError("packed must hold star_act_bytes(tokens, width) bytes")
    return packed.data_ptr()


def star_act_pack(x, packed, *, stream=None) -> None:
    """Keeps ``x`` (float32 or bfloat16 [tokens, width], rows at any distance) in 8 bits in ``packed``, a uint8 tensor of
    ``star_act_bytes(tokens, width)`` bytes."""
    code = _dtype(x, "x")
    p, tokens, width, ld = _matrix(x, "x")
    _check(_library().star_act_pack(p, code, tokens, width, ld, _packed(packed, tokens, width, x.device),
                                    _stream_handle(stream)))


def star_act_unpack(packed, out, *, stream=None) -> None:
    """The kept values of ``packed``, into ``out`` (float32 or bfloat16 [tokens, width])."""
    code = _dtype(out, "out")
    p, tokens, width, ld = _matrix(out, "out")
    _check(_library().star_act_unpack(_packed(packed, tokens, width, out.device), tokens, width, p, code, ld,
                                      _stream_handle(stream)))


def star_act_weight_grad(dy, packed, dw, *, accumulate: bool = False, workspace=None, stream=None) -> None:
    """``dw`` [out, width] = (or, with ``accumulate``, +=) dy^T x for the activations x [tokens, width] in ``packed``.
    ``dy``: float32 or bfloat16 [tokens, out]; ``dw``: contiguous float32 or bfloat16, for example
    ``row[a:a + out * width].view(out, width)`` of a worker's gradient row."""
    lib = _library()
    dy_code, dw_code = _dtype(dy, "dy"), _dtype(dw, "dw")
    p, tokens, out, ld = _matrix(dy, "dy")
    if dw.dim() != 2 or dw.shape[0] != out or not dw.is_contiguous():
        raise ValueError(f"dw must be a contiguous tensor [{out}, width]")
    if dw.device != dy.device:
        raise ValueError("dw must be on dy's device")
    width = dw.shape[1]
    w, size, _keep = _workspace(workspace, lib.star_act_weight_grad_workspace(dy_code, tokens, out, width), dy.device, stream)
    _check(lib.star_act_weight_grad(p, dy_code, tokens, out, ld, _packed(packed, tokens, width, dy.device), width,
                                    dw.data_ptr(), dw_code, int(bool(accumulate)), w, size, _stream_handle(stream)))
