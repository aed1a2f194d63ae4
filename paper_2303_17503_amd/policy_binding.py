"""ctypes binding of the policy entry points of libpgxgo.so; names follow include/pgxpolicy.h.

Between an environment's outputs and its next actions: adjust_logits (pgxpolicy_logits), sample_actions (pgxpolicy_sample) and,
for a learner of recorded moves, policy_loss (pgxpolicy_loss).  All run on the current stream of the logits' device.
"""
import contextlib
import ctypes as C

import torch

from . import binding
from .binding import PgxGoError, _address, _ptr, lib as _golib

TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
MAX_ACTIONS, MAX_RECORD = 8192, 65535
_ready = False
_fast = None   # as in binding.py: checks the arguments, makes the outputs and calls, or leaves the call to the Python lines
_calls = {}


class _Adjust(C.Structure):
    _fields_ = [("mask", C.c_void_p), ("mask_pitch", C.c_int64), ("bias", C.c_void_p), ("bias_pitch", C.c_int64),
                ("record", C.c_void_p), ("record_row_stride", C.c_int64), ("record_ply_stride", C.c_int64), ("record_len", C.c_int32),
                ("repetition", C.c_float), ("frequency", C.c_float), ("presence", C.c_float), ("begin", C.c_void_p), ("end", C.c_void_p),
                ("temperature_row", C.c_void_p), ("temperature", C.c_float)]


def lib():
    """The shared library with the pgxpolicy_* prototypes declared; raises if it has not been built (no fallback)."""
    global _ready, _fast
    L = _golib()
    if not _ready:
        vp, i32, i64, f32, adj = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.POINTER(_Adjust)
        L.pgxpolicy_logits.argtypes = [i32, i32, vp, i32, i64, adj, i32, vp, i64, vp]
        L.pgxpolicy_sample.argtypes = [i32, i32, vp, i32, i64, adj, vp, i64, vp, vp, vp]
        L.pgxpolicy_loss.argtypes = [i32, i32, vp, i32, i64, adj, vp, i64, vp, vp, f32, f32, vp, vp, vp, i64, vp]
        L.pgxpolicy_strerror.restype = C.c_char_p
        L.pgxpolicy_strerror.argtypes = [C.c_int]
        L.pgxpolicy_last_hip_error.restype = C.c_int
        _calls.update({n: _address(getattr(L, "pgxpolicy_" + n)) for n in ("logits", "sample", "loss")})
        _fast = binding._fast
        if _fast is not None:
            _fast.set_raw_stream(torch._C._cuda_getCurrentRawStream)
        _ready = True
    return L


def _check(rc, what):
    if rc != 0:
        L = lib()
        raise PgxGoError(f"{what}: {L.pgxpolicy_strerror(rc).decode()} (code {rc}, hip error {L.pgxpolicy_last_hip_error()})")


def _on(t, device, dtypes, shape, name):
    """A tensor of one of the types on the device, of the shape (None: any size), its last dimension dense."""
    dtypes = dtypes if isinstance(dtypes, tuple) else (dtypes,)
    if (not isinstance(t, torch.Tensor) or t.dtype not in dtypes or t.device != device or t.dim() != len(shape)
            or any(want is not None and want != size for want, size in zip(shape, t.shape)) or (t.numel() > 0 and t.shape[-1] > 1 and t.stride(-1) != 1)):
        got = f"{t.dtype} {tuple(t.shape)} of strides {t.stride()} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
        raise PgxGoError(f"{name}: expected {' or '.join(map(str, dtypes))} tensor of shape {shape} on {device} with a dense last dimension, got {got}")
    return t


def _rows(t, device, dtype, rows, name):   # one value per row
    return _on(t, device, dtype, (rows,), name)


def _logits(logits):
    if not isinstance(logits, torch.Tensor) or not logits.is_cuda or logits.dtype not in TYPES or logits.dim() != 2 or (logits.shape[1] > 1 and logits.numel() and logits.stride(1) != 1):
        raise PgxGoError("logits: expected a cuda tensor [rows][actions] of float32, float16 or bfloat16 with dense rows")
    rows, actions = logits.shape
    if not 1 <= actions <= MAX_ACTIONS or rows >= 2 ** 31:
        raise PgxGoError(f"logits: 1 to {MAX_ACTIONS} actions and fewer than 2^31 rows, got {actions} and {rows}")
    return rows, actions


def _adjust(logits, rows, actions, mask, bias, record, begin, end, repetition, frequency, presence, temperature):
    dev, a = logits.device, _Adjust()
    if mask is not None:
        _on(mask, dev, (torch.uint8, torch.bool), (rows, None), "mask")
        if mask.shape[1] < actions:
            raise PgxGoError(f"mask: rows of {mask.shape[1]} bytes for {actions} actions")
        a.mask, a.mask_pitch = mask.data_ptr(), mask.stride(0)
    if bias is not None:
        _on(bias, dev, torch.float32, (actions,) if getattr(bias, "ndim", 2) == 1 else (rows, actions), "bias")
        a.bias, a.bias_pitch = bias.data_ptr(), 0 if bias.dim() == 1 else bias.stride(0)
    a.repetition, a.frequency, a.presence = repetition, frequency, presence
    if not 0.0 < a.repetition < float("inf"):
        raise PgxGoError(f"repetition: above 0, got {repetition}")
    if record is not None:
        if not isinstance(record, torch.Tensor) or record.dtype is not torch.int32 or record.device != dev or record.dim() != 2 or record.shape[0] != rows:
            raise PgxGoError(f"record: expected int32 tensor [{rows}][plies] on {dev} (a trajectory [plies][games] as its transpose)")
        if record.shape[1] > MAX_RECORD:
            raise PgxGoError(f"record: at most {MAX_RECORD} plies, got {record.shape[1]}")
        a.record, a.record_len = record.data_ptr(), record.shape[1]
        a.record_row_stride, a.record_ply_stride = record.stride()
        if begin is not None: a.begin = _rows(begin, dev, torch.int32, rows, "begin").data_ptr()
        if end is not None: a.end = _rows(end, dev, torch.int32, rows, "end").data_ptr()
    elif begin is not None or end is not None or repetition != 1.0 or frequency != 0.0 or presence != 0.0:
        raise PgxGoError("begin, end, repetition, frequency and presence are about a record: none was given")
    if isinstance(temperature, torch.Tensor):
        a.temperature_row = _rows(temperature, dev, torch.float32, rows, "temperature").data_ptr()
    elif temperature is not None:
        a.temperature = temperature
        if not 0.0 < a.temperature < float("inf"):
            raise PgxGoError(f"temperature: a number above 0, or a tensor with one per row (0: greedy), got {temperature}")
    return a


@contextlib.contextmanager
def _current(device):
    with torch.cuda.device(device):
        yield torch.cuda.current_stream(device).cuda_stream


def adjust_logits(logits, mask=None, bias=None, record=None, begin=None, end=None, repetition=1.0, frequency=0.0, presence=0.0, temperature=None,
                  normalize=False, out=None):
    """Adjusted logits, float32 [rows][actions] (include/pgxpolicy.h states the formula): penalties for the moves of the record,
    plus the bias, over the temperature, -inf where the mask is 0; with normalize their log-probabilities.

    logits float32, float16 or bfloat16 [rows][actions]; mask uint8 or bool [rows][>= actions], as GoEnv.new_mask; bias float32 [actions] or
    [rows][actions]; record int32 [rows][plies] of any strides, of which plies begin[b] <= t < end[b] count (int32 [rows]);
    repetition above 1, frequency and presence above 0 make repeated moves less likely; temperature a number or float32 [rows]."""
    if not _ready: lib()
    if _fast is not None:
        got = _fast.policy_logits(_calls["logits"], logits, mask, bias, record, begin, end, repetition, frequency, presence, temperature, normalize, out)
        if type(got) is tuple: return got[0]
        if got is not None: _check(got, "pgxpolicy_logits")
    rows, actions = _logits(logits)
    a = _adjust(logits, rows, actions, mask, bias, record, begin, end, repetition, frequency, presence, temperature)
    if out is None:
        out = torch.empty((rows, actions), dtype=torch.float32, device=logits.device)
    _on(out, logits.device, torch.float32, (rows, actions), "out")
    with _current(logits.device) as stream:
        _check(lib().pgxpolicy_logits(rows, actions, _ptr(logits), TYPES[logits.dtype], logits.stride(0), C.byref(a), int(bool(normalize)), _ptr(out),
                                      out.stride(0), stream), "pgxpolicy_logits")
    return out


def sample_actions(logits, noise=None, mask=None, bias=None, record=None, begin=None, end=None, repetition=1.0, frequency=0.0, presence=0.0,
                   temperature=None, out=None, logp=None):
    """(int32 [rows] actions, float32 [rows] their log-probabilities): the possible action with the largest adjusted logit plus noise.
    With Gumbel noise (float32 [rows][actions]) a draw from the adjusted distribution, without it the most likely action; rows
    of temperature 0 are greedy.  -1 and 0 where nothing is possible.  Other arguments as for adjust_logits."""
    if not _ready: lib()
    if _fast is not None:
        got = _fast.policy_sample(_calls["sample"], logits, noise, mask, bias, record, begin, end, repetition, frequency, presence, temperature, out, logp)
        if type(got) is tuple: return got
        if got is not None: _check(got, "pgxpolicy_sample")
    rows, actions = _logits(logits)
    a = _adjust(logits, rows, actions, mask, bias, record, begin, end, repetition, frequency, presence, temperature)
    dev = logits.device
    if noise is not None: _on(noise, dev, torch.float32, (rows, actions), "noise")
    out = torch.empty(rows, dtype=torch.int32, device=dev) if out is None else _rows(out, dev, torch.int32, rows, "out")
    logp = torch.empty(rows, dtype=torch.float32, device=dev) if logp is None else _rows(logp, dev, torch.float32, rows, "logp")
    with _current(dev) as stream:
        _check(lib().pgxpolicy_sample(rows, actions, _ptr(logits), TYPES[logits.dtype], logits.stride(0), C.byref(a), _ptr(noise),
                                      0 if noise is None else noise.stride(0), _ptr(out), _ptr(logp), stream), "pgxpolicy_sample")
    return out, logp


def policy_loss(logits, target, weight=None, entropy=0.0, grad_scale=1.0, mask=None, bias=None, record=None, begin=None, end=None, repetition=1.0,
                frequency=0.0, presence=0.0, temperature=None, grad=None):
    """(loss, entropies, gradient) of a learner's policy term: per row the cross entropy of the adjusted distribution against the target, times
    weight (float32 [rows]), less `entropy` times its entropy; the gradient of grad_scale times the sum of the losses for the logits,
    in their type, comes with it (logits.backward(gradient) goes on from there).  target: float32 [rows][actions], a search's visit
    shares, or int32 [rows], a move each (-1: none).  Other arguments as for adjust_logits."""
    if not _ready: lib()
    if _fast is not None:
        got = _fast.policy_loss(_calls["loss"], logits, target, weight, entropy, grad_scale, mask, bias, record, begin, end, repetition, frequency, presence,
                                temperature, grad)
        if type(got) is tuple: return got
        if got is not None: _check(got, "pgxpolicy_loss")
    rows, actions = _logits(logits)
    a = _adjust(logits, rows, actions, mask, bias, record, begin, end, repetition, frequency, presence, temperature)
    dev = logits.device
    moves = isinstance(target, torch.Tensor) and target.dtype is torch.int32
    if moves: _rows(target, dev, torch.int32, rows, "target")
    else: _on(target, dev, torch.float32, (rows, actions), "target")
    if weight is not None: _rows(weight, dev, torch.float32, rows, "weight")
    loss, entropies = torch.empty((2, rows), dtype=torch.float32, device=dev).unbind(0)
    grad = torch.empty((rows, actions), dtype=logits.dtype, device=dev) if grad is None else _on(grad, dev, logits.dtype, (rows, actions), "grad")
    with _current(dev) as stream:
        _check(lib().pgxpolicy_loss(rows, actions, _ptr(logits), TYPES[logits.dtype], logits.stride(0), C.byref(a), None if moves else _ptr(target),
                                    0 if moves else target.stride(0), _ptr(target) if moves else None, _ptr(weight), entropy, grad_scale, _ptr(loss),
                                    _ptr(entropies), _ptr(grad), grad.stride(0), stream), "pgxpolicy_loss")
    return loss, entropies, grad
