"""ctypes binding of the rotary positions' entry point of libpgxgo.so; names follow include/pgxrotary.h (pgxrotary_turn -> rotate).

Runs on the current stream of the tensors' device."""
import ctypes as C
import math

import torch

from . import binding
from .binding import PgxGoError, _address, lib as _golib
from .policy_binding import TYPES, _current

MAX_HEAD_DIM = 1024
_ready = False
_fast = None   # as in binding.py
_call = None


class _Part(C.Structure):
    _fields_ = ([("in_", C.c_void_p)] + [(n, C.c_int64) for n in ("in_entry", "in_token", "in_head")] + [("out", C.c_void_p)]
                + [(n, C.c_int64) for n in ("out_entry", "out_token", "out_head")] + [("heads", C.c_int32)])


def lib():
    """The shared library with the pgxrotary_* prototypes declared; raises if it has not been built (no fallback)."""
    global _ready, _fast, _call
    L = _golib()
    if not _ready:
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        L.pgxrotary_turn.argtypes = [i32, i32, i32, i32, i32, vp, i64, i64, vp, C.c_float, i32, i32, i32, C.POINTER(_Part), vp]
        L.pgxrotary_strerror.restype = C.c_char_p
        L.pgxrotary_strerror.argtypes = [C.c_int]
        L.pgxrotary_last_hip_error.restype = C.c_int
        _call = _address(L.pgxrotary_turn)
        _fast = binding._fast
        if _fast is not None:
            _fast.set_raw_stream(torch._C._cuda_getCurrentRawStream)
        _ready = True
    return L


def _check(rc, what):
    if rc != 0:
        L = lib()
        raise PgxGoError(f"{what}: {L.pgxrotary_strerror(rc).decode()} (code {rc}, hip error {L.pgxrotary_last_hip_error()})")


def rotary_frequencies(rotary_dim, base=10000.0, scaling=None, factor=1.0, original=None, low=1.0, high=32.0, device="cuda:0"):
    """Radians per position of each pair, float64 [rotary_dim / 2] on the device: base ** (-2 j / rotary_dim); to be made once and kept.
    For contexts `factor` times as long as those that a model was trained on (of `original` positions), scaling is
      "linear"  every frequency over factor
      "base"    the base times factor ** (rotary_dim / (rotary_dim - 2)): the slowest pair is slowed by factor, the fastest stays
      "parts"   pairs that turn at least `high` times within `original` positions stay, those that turn at most `low` times are slowed by factor, between them
                the two are mixed by the number of turns (0.1 ln factor + 1 is then a usual `magnitude` for rotate)."""
    R = rotary_dim
    if not isinstance(R, int) or isinstance(R, bool) or not 2 <= R <= MAX_HEAD_DIM or R % 2:
        raise PgxGoError(f"rotary_dim: an even number from 2 to {MAX_HEAD_DIM}, got {rotary_dim}")
    if not (0 < base < math.inf and 0 < factor < math.inf):
        raise PgxGoError(f"base and factor: above 0, got {base} and {factor}")
    if scaling not in (None, "linear", "base", "parts"):
        raise PgxGoError(f"scaling: None, 'linear', 'base' or 'parts', got {scaling!r}")
    if scaling is None and factor != 1.0:
        raise PgxGoError("factor is about a scaling: none was given")
    if scaling == "base":
        if R == 2:
            raise PgxGoError("scaling 'base' needs a rotary_dim of 4 or more")
        try:
            base = base * factor ** (R / (R - 2))
        except OverflowError:
            base = math.inf
        if not 0 < base < math.inf:
            raise PgxGoError(f"scaling 'base': base and factor make a base of {base}")
    f = torch.tensor(base, dtype=torch.float64) ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
    if scaling == "linear":
        f = f / factor
    elif scaling == "parts":
        if original is None or not original > 0 or not low < high:
            raise PgxGoError(f"scaling 'parts' needs original above 0 and low below high, got {original}, {low} and {high}")
        keep = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
    if not torch.isfinite(f).all():
        raise PgxGoError("frequencies would not be finite")
    return f.to(device)


def rotate(x, positions, frequencies, interleaved=False, magnitude=1.0, inverse=False, out=None):
    """x with the first R = 2 * len(frequencies) elements of each head turned by their token's position, the others as they are
    (include/pgxrotary.h states the formula).  x: [n][heads][head_dim], or [n][tokens][heads][head_dim], of float32, float16 or bfloat16 with a dense last
    dimension, or a pair of them (queries and keys) that differ in their heads alone, for which one launch is enough; positions: int32 [n] or [n][tokens];
    frequencies: float64 [R / 2] (rotary_frequencies).  interleaved: pairs are neighbours, otherwise R / 2 apart.  inverse: turned back, times the
    magnitude, which takes the result's gradient to x's.  out: as x, or x itself.  Returns a tensor, or a pair.
    The call makes no graph of its own: while one is being made, tensors that require gradients are refused (call it under torch.no_grad(), or in an autograd.Function
    whose backward is the call with inverse=True)."""
    if not _ready: lib()
    if _fast is not None:
        got = _fast.rotate(_call, x, positions, frequencies, interleaved, magnitude, inverse, out)
        if type(got) is tuple: return got if type(x) is tuple or type(x) is list else got[0]
        if got is not None: _check(got, "pgxrotary_turn")
    pair = isinstance(x, (tuple, list))
    xs = tuple(x) if pair else (x,)
    if not 1 <= len(xs) <= 2:
        raise PgxGoError(f"x: a tensor or two of them, got {len(xs)}")
    first = xs[0]
    for t in xs:
        if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in TYPES or t.dim() not in (3, 4) or (t.numel() and t.stride(-1) != 1 and t.shape[-1] > 1):
            raise PgxGoError("x: expected cuda tensors [n][heads][head_dim] or [n][tokens][heads][head_dim] of float32, float16 or bfloat16 with a dense last dimension")
        if t.dtype is not first.dtype or t.device != first.device or t.shape[:-2] != first.shape[:-2] or t.shape[-1] != first.shape[-1]:
            raise PgxGoError("x: the two tensors may differ in their number of heads alone")
    lead, D, dev = first.shape[:-2], first.shape[-1], first.device
    if not isinstance(positions, torch.Tensor) or positions.dtype is not torch.int32 or positions.device != dev or positions.shape != lead:
        raise PgxGoError(f"positions: expected int32 {list(lead)} on {dev}")
    if not isinstance(frequencies, torch.Tensor) or frequencies.dtype is not torch.float64 or frequencies.device != dev or frequencies.dim() != 1 or not frequencies.is_contiguous():
        raise PgxGoError(f"frequencies: expected contiguous float64 [rotary_dim / 2] on {dev} (rotary_frequencies)")
    R = 2 * frequencies.shape[0]
    if not 2 <= R <= D or D > MAX_HEAD_DIM:
        raise PgxGoError(f"frequencies: {R // 2} pairs for heads of {D} elements (at most {MAX_HEAD_DIM})")
    if not math.isfinite(magnitude):
        raise PgxGoError(f"magnitude: a finite number, got {magnitude}")
    if out is None:
        outs = tuple(torch.empty(t.shape, dtype=t.dtype, device=dev) for t in xs)
    else:
        outs = tuple(out) if isinstance(out, (tuple, list)) else (out,)
        if len(outs) != len(xs) or any(not isinstance(o, torch.Tensor) or o.dtype is not t.dtype or o.device != dev or o.shape != t.shape or (o.numel() and D > 1 and o.stride(-1) != 1)
                                       for o, t in zip(outs, xs)):
            raise PgxGoError("out: expected tensors as x")
    if torch.is_grad_enabled() and any(t.requires_grad for t in xs + outs):
        raise PgxGoError("x: gradients would be lost, the call makes no graph; under torch.no_grad(), or in an autograd.Function whose backward is rotate(gradient, ..., inverse=True)")
    n, T = lead[0], lead[1] if len(lead) == 2 else 1
    if n * T >= 2 ** 31:
        raise PgxGoError(f"x: fewer than 2^31 tokens, got {n * T}")
    strides = lambda t: (t.stride(0), t.stride(1) if t.dim() == 4 else 0, t.stride(-2))  # noqa: E731
    parts = (_Part * len(xs))(*[_Part(t.data_ptr(), *strides(t), o.data_ptr(), *strides(o), t.shape[-2]) for t, o in zip(xs, outs)])
    with _current(dev) as stream:
        _check(lib().pgxrotary_turn(n, T, D, R, TYPES[first.dtype], positions.data_ptr(), positions.stride(0), positions.stride(1) if len(lead) == 2 else 0,
                                    frequencies.data_ptr(), magnitude, int(bool(interleaved)), int(bool(inverse)), len(xs), parts, stream), "pgxrotary_turn")
    if out is not None:   # what autograd has kept of them is no longer what it was
        torch.autograd.graph.increment_version([o for o in outs if not o.is_inference()])
    return outs if pair else outs[0]
