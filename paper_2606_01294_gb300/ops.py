"""Python binding of include/ccq_ops.h: the operators around the CCQ token mixer.

The embedding lookup and its gradient, the rotation of queries and keys by their positions, linear attention with a
decay for each head (prompts, their gradients, single tokens), the (gated) group norm after the mixer's read and its
gradient, the clipped policy loss with its gradient, the token log-probabilities, and the AdamW update of many tensors.  As in
:mod:`.ccq`, this is argument marshalling only: tensors are CUDA tensors (there is no CPU path), outputs
and workspaces are allocated with torch on the inputs' device, and every computation runs in the
library's kernels on the current stream.  ``stream=`` makes a call as within ``torch.cuda.stream(stream)``: what
it allocates belongs to that stream, which waits for the inputs, and is waited for, as torch's streams do; what
it returns may be used on the caller's stream after such a wait, and dropped there.

Tensors of rows need contiguous rows; the rows themselves may lie apart (a slice of a wider projection), as
long as one stride reaches them all.
"""
from __future__ import annotations

import ctypes
import functools
import math
import struct
from dataclasses import dataclass
from itertools import chain
from typing import List, Optional

import torch

from . import ccq
from .ccq import _check, _dtype_code, _on_stream, _ptr, _stream

ACTIVATION = {"none": 0, "silu": 1, "sigmoid": 2}
ADAMW_BLOCK = 256
_CODE = {torch.bfloat16: ccq.BF16, torch.float32: ccq.FP32}

_VP, _I, _L, _F, _D, _Z = (ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_double,
                           ctypes.c_size_t)


class _PolicyParams(ctypes.Structure):
    _fields_ = [("clip_low", _F), ("clip_high", _F), ("kl_coef", _F), ("temperature", _F), ("grad_scale", _F)]


class _AdamWParams(ctypes.Structure):
    _fields_ = [("lr", _D), ("beta1", _D), ("beta2", _D), ("eps", _D), ("weight_decay", _D), ("step", _L)]


_lib = None


def _library() -> ctypes.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    lib = ccq.load_library()
    size = ctypes.POINTER(_Z)
    for name, args in {
            # table, dtype, stride | ids, id_bytes, n, rows, width, scale | out, stride | stream
            "ccq_embed": [_VP, _I, _L, _VP, _I, _L, _L, _I, _F, _VP, _L, _VP],
            # dout, dtype, stride | ids, id_bytes, n, rows, width, scale, padding | dtable, dtype, stride | ws | stream
            "ccq_embed_grad": [_VP, _I, _L, _VP, _I, _L, _L, _I, _F, _L, _VP, _I, _L, _VP, _Z, _VP],
            "ccq_embed_grad_workspace_size": [_L, _L, _I, size],
            # x, gate (strides), weight, bias, dtypes, y, stride | tokens, channels, groups, centered, eps, act | stream
            "ccq_group_norm": [_VP, _L, _VP, _L, _VP, _VP, _I, _I, _VP, _L, _L, _I, _I, _I, _F, _I, _VP],
            # x, gate, weight, bias, dy, dtypes | dx, dgate, dweight, dbias | sizes, centered, eps, act | ws | stream
            "ccq_group_norm_bwd": [_VP, _L, _VP, _L, _VP, _VP, _VP, _L, _I, _I, _VP, _L, _VP, _L, _VP, _VP, _L, _I,
                                   _I, _I, _F, _I, _VP, _Z, _VP],
            "ccq_group_norm_bwd_workspace_size": [_L, _I, _I, _I, size],
            # logits, dtype, stride | actions, id_bytes | old, ref, adv, weights | n, vocab, params | loss, logp,
            # dlogits, stride | ws | stream
            "ccq_policy_loss": [_VP, _I, _L, _VP, _I, _VP, _VP, _VP, _VP, _L, _I, ctypes.POINTER(_PolicyParams), _VP,
                                _VP, _VP, _L, _VP, _Z, _VP],
            "ccq_policy_loss_workspace_size": [_L, size],
            "ccq_token_logp": [_VP, _I, _L, _VP, _I, _L, _I, _F, _VP, _VP],
            # x, dtype | T, width | cu, cu_bytes, num_seqs | stream
            "ccq_zero_outside": [_VP, _I, _L, _I, _VP, _I, _L, _VP],
            # x, y (arrays), count, dtype | B, T, width, part | positions, bytes | freqs, amplitude, interleaved, inverse | stream
            "ccq_rotary": [_VP, _VP, _I, _I, _L, _L, _I, _I, _VP, _I, _VP, _F, _I, _I, _VP],
            # q, k, v, dtype | log_decay, scale, S0 | o, ST | B, T, H, d | cu, cu_bytes, num_seqs | ws | stream
            "ccq_decay_attention": [_VP, _VP, _VP, _I, _VP, _F, _VP, _VP, _VP, _L, _L, _I, _I, _VP, _I, _L, _VP, _Z, _VP],
            # q, k, v, dtype | log_decay, scale, S0 | dout, dST | dq, dk, dv, dS0 | B, T, H, d | cu, cu_bytes, num_seqs | ws
            # | stream
            "ccq_decay_attention_bwd": [_VP, _VP, _VP, _I, _VP, _F, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _L, _L, _I, _I, _VP, _I,
                                        _L, _VP, _Z, _VP],
            "ccq_decay_attention_workspace_size": [_L, _L, _I, _I, _L, _I, size],
            "ccq_decay_attention_bwd_workspace_size": [_L, _L, _I, _I, _I, _I, _I, _L, _I, size],
            # q, k, v, dtype | log_decay, scale, state, rows, slots, slot_bytes | o | B, H, d | stream
            "ccq_decay_attention_step": [_VP, _VP, _VP, _I, _VP, _F, _VP, _L, _VP, _I, _VP, _L, _I, _I, _VP],
            "ccq_adamw_step": [_VP, _I, _I, _I, _I, ctypes.POINTER(_AdamWParams), _VP, _VP]}.items():
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, _I
    lib.ccq_default_policy_params.argtypes = [ctypes.POINTER(_PolicyParams)]
    lib.ccq_default_policy_params.restype = None
    _lib = lib
    return lib


@functools.lru_cache(maxsize=256)
def _size(fn, device, *args):
    """Bytes from a workspace query: a function of the sizes (and of the device's SM count)."""
    need = _Z(0)
    _check(getattr(_library(), fn)(*args, ctypes.byref(need)))
    return need.value


def _workspace(workspace, need, device):
    if workspace is None and not need:
        return None, 0
    if workspace is None:
        return torch.empty(max(need, 16), dtype=torch.uint8, device=device), max(need, 16)
    _dense(workspace, "workspace", device)
    return workspace, workspace.numel() * workspace.element_size()


def _cuda(t, name, device=None):
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise ValueError(f"{name} must be a CUDA tensor (there is no CPU path)")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    return t


def _dense(t, name, device, dtype=None, shape=None):
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.device == device and t.is_contiguous()
            and (dtype is None or t.dtype is dtype) and (shape is None or t.shape == shape)):
        return t
    _cuda(t, name, device)
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _rows(t, name, device=None, dtype=None, shape=None):
    """The stride between the rows of a [..., width] tensor with contiguous rows.  (A tensor as most are passes on one
    expression: the small cases' time is the host's.)"""
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous() and (device is None or t.device == device)
            and (dtype is None or t.dtype is dtype) and (shape is None or t.shape == shape) and t.dim() > 0):
        return t.shape[-1]
    _cuda(t, name, device)
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.dim() < 1:
        raise ValueError(f"{name} must have at least one dimension")
    if t.is_contiguous():
        return t.shape[-1]
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name} must have contiguous rows (its last dimension)")
    step, reach = None, 0
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if step is None:
            step, reach = stride, stride * size
        elif stride == reach:
            reach = stride * size
        else:
            raise ValueError(f"{name}: one stride must reach all of its rows")
    if step is not None and step < t.shape[-1]:
        raise ValueError(f"{name}: its rows overlap")
    return t.shape[-1] if step is None else step


def _ids(t, name, device):
    if isinstance(t, torch.Tensor) and t.device == device and t.is_cuda and t.is_contiguous():
        if t.dtype is torch.int64:
            return 8
        if t.dtype is torch.int32:
            return 4
    if t.dtype not in (torch.int64, torch.int32):
        raise TypeError(f"{name} must be int64 or int32, got {t.dtype}")
    _dense(t, name, device)
    return t.element_size()


# ---------------------------------------------------------------- embedding


def embed(table, ids, *, scale: float = 1.0, out=None, stream=None):
    """``scale * table[ids]`` (ccq_embed): table [rows, width] bf16 or fp32, ids int64 or int32 of any
    shape; returns [*ids.shape, width].  An id outside the table gives a zero row and CCQ_ERR_INDEX
    from :func:`ccq.device_status`."""
    if stream is not None:
        return _on_stream(stream, embed, table, ids, scale=scale, out=out)
    ts = _rows(table, "table")
    if table.dim() != 2:
        raise ValueError("table must be [rows, width]")
    dev = table.device
    id_bytes = _ids(ids, "ids", dev)
    rows, width = table.shape
    if out is None:
        out, os = torch.empty((*ids.shape, width), dtype=table.dtype, device=dev), width
    else:
        os = _rows(out, "out", dev, table.dtype, ids.shape + (width,))
    _check(_library().ccq_embed(table.data_ptr(), _dtype_code(table), ts, ids.data_ptr(), id_bytes, ids.numel(), rows,
                                width, scale, out.data_ptr(), os, _stream(dev, None)))
    return out


def embed_grad(dout, ids, rows: int, *, scale: float = 1.0, padding_id: Optional[int] = None, dtype=None, out=None,
               workspace=None, stream=None):
    """Gradient of :func:`embed`'s table (ccq_embed_grad): row r is ``scale`` times the sum of dout over
    the tokens with id r, summed in fp32 in a fixed order; rows without a token (and ``padding_id``'s) are zero.
    dout [*ids.shape, width]; returns [rows, width] in ``dtype`` (dout's when not given) or ``out``."""
    if stream is not None:
        return _on_stream(stream, embed_grad, dout, ids, rows, scale=scale, padding_id=padding_id, dtype=dtype, out=out,
                          workspace=workspace)
    _rows(dout, "dout")
    dev = dout.device
    id_bytes = _ids(ids, "ids", dev)
    width, n = dout.shape[-1], ids.numel()
    ds = _rows(dout, "dout", dev, None, ids.shape + (width,))
    if out is None:
        out, os = torch.empty((rows, width), dtype=dtype or dout.dtype, device=dev), width
    else:
        os = _rows(out, "out", dev, dtype, (rows, width))
    if padding_id is not None and not 0 <= padding_id < rows:
        raise ValueError(f"padding_id {padding_id} is outside the table of {rows} rows")
    workspace, nbytes = _workspace(workspace, _size("ccq_embed_grad_workspace_size", -1, n, rows, width), dev)
    _check(_library().ccq_embed_grad(dout.data_ptr(), _dtype_code(dout), ds, ids.data_ptr(), id_bytes, n, rows, width,
                                     scale, -1 if padding_id is None else padding_id, out.data_ptr(), _dtype_code(out),
                                     os, _ptr(workspace), nbytes, _stream(dev, None)))
    return out


# ---------------------------------------------------------------- heads of tokens


# A call on small tensors costs the host more than the GPU, so what follows from shapes, strides and types alone is formed once
# for each combination of them (bounded caches of plain values).  A plan is None where a check fails: the call then goes the way
# that makes the checks one by one and says what is wrong.
_FIVE = struct.Struct("5q").pack
_INDEX = {torch.int64: 8, torch.int32: 4}


def _strides(shape, stride):
    """(batch, token, head stride, heads) of [batch, tokens, heads, width] or [rows, heads, width]; None: not contiguous channels."""
    if stride[-1] != 1 and shape[-1] > 1:
        return None
    return (*stride[:3], shape[2]) if len(shape) == 4 else (stride[0], stride[0], stride[1], shape[1])


def _dense_strides(shape):
    B, T, n, width = shape if len(shape) == 4 else (1, *shape)
    return T * n * width, n * width, width, n


def _is_dense(shape, stride):
    step = 1
    for n, s in zip(reversed(shape), reversed(stride)):
        if n != 1 and s != step:
            return 0 in shape
        step *= n
    return True


@functools.lru_cache(maxsize=512)
def _rotary_plan(q, k, positions, freqs):
    (dtype, shape, _), (kdtype, kshape, _) = q, k
    if len(shape) not in (3, 4) or len(kshape) != len(shape):
        return None
    xq, xk = _strides(*q[1:]), _strides(*k[1:])
    if (kdtype != dtype or dtype not in _CODE or not xq or not xk
            or kshape[:-2] != shape[:-2] or kshape[-1] != shape[-1] or positions[0] not in _INDEX or positions[1] != shape[:-2]
            or not _is_dense(*positions[1:]) or freqs[0] is not torch.float64 or not _is_dense(*freqs[1:])):
        return None
    B, T = shape[:2] if len(shape) == 4 else (1, shape[0])
    return xq, xk, _dense_strides(shape), _dense_strides(kshape), (2, _CODE[dtype], B, T, shape[-1], 2 * math.prod(freqs[1])), _INDEX[positions[0]]


@functools.lru_cache(maxsize=512)
def _decay_plan(q, k, v, log_decay, cu, states, index, dout=None):
    """Of decay_attention (dout None) and its gradients: (strides of q, k, v[, dout]), of o, its shape, the states' shape, the
    arguments from B on, type code and workspace bytes.  ``states``: shapes, strides and types of the states that are given."""
    dtype, shape, _ = q
    if dtype not in _CODE or len(shape) != 4 or log_decay[0] is not torch.float32 or len(log_decay[1]) != 1 or not _is_dense(*log_decay[1:]):
        return None
    B, T, _, d = shape
    H = log_decay[1][0]
    out = (B, T, H, d)
    tails = []
    for t in (q, k, v) + ((dout,) if dout else ()):
        x = _strides(*t[1:]) if len(t[1]) == 4 else None
        if t[0] != dtype or not x or tuple(t[1][:2]) != (B, T) or t[1][3] != d or t[1][2] < 1 or H % t[1][2] or (t is dout and t[1][2] != H):
            return None
        tails.append(x)
    seqs, cu_bytes = B, 8
    if cu is not None:
        if cu[0] not in _INDEX or len(cu[1]) != 1 or cu[1][0] < 1 or not _is_dense(*cu[1:]) or B != 1:
            return None
        seqs, cu_bytes = cu[1][0] - 1, _INDEX[cu[0]]
    state = (seqs, H, d, d)
    if any(t[0] is not torch.float32 or tuple(t[1]) != state or not _is_dense(*t[1:]) for t in states):
        return None
    code = _CODE[dtype]
    if dout:
        need = _size("ccq_decay_attention_bwd_workspace_size", index, B, T, H, shape[2], k[1][2], v[1][2], d, seqs, code)
    else:
        need = _size("ccq_decay_attention_workspace_size", index, B, T, H, d, seqs, code)
    return tails, _dense_strides(out), out, state, (B, T, H, d), (cu_bytes, seqs), code, need, d ** -0.5


@functools.lru_cache(maxsize=512)
def _step_plan(q, k, v, log_decay, state, slots):
    dtype, shape, _ = q
    if dtype not in _CODE or len(shape) != 3 or log_decay[0] is not torch.float32 or len(log_decay[1]) != 1 or not _is_dense(*log_decay[1:]):
        return None
    B, _, d = shape
    H = log_decay[1][0]
    tails = []
    for t in (q, k, v):
        x = _strides(*t[1:]) if len(t[1]) == 3 else None
        if t[0] != dtype or not x or t[1][0] != B or t[1][2] != d or t[1][1] < 1 or H % t[1][1]:
            return None
        tails.append(x)
    if state[0] is not torch.float32 or len(state[1]) != 4 or tuple(state[1][1:]) != (H, d, d) or not _is_dense(*state[1:]):
        return None
    if slots is None:
        if state[1][0] != B:
            return None
    elif slots[0] not in _INDEX or tuple(slots[1]) != (B,) or not _is_dense(*slots[1:]):
        return None
    return tails, (H * d, d, d, H), (B, H, d), _CODE[dtype], state[1][0], 4 if slots is None else _INDEX[slots[0]], d ** -0.5


def _like(t):
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _meta(t):
    return None if t is None else (t.dtype, t.shape, t.stride())


def _heads(t, name, device=None, dtype=None, shape=None, heads=None):
    """A ccq_heads of a [batch, tokens, heads, width] tensor (or [rows, heads, width]: one batch row of tokens, a batch
    of one token for the step).  Any strides but the channels', which are contiguous."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and (device is None or t.device == device)):
        _cuda(t, name, device)
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if heads is not None and (t.shape[-2] < 1 or heads % t.shape[-2]):
        raise ValueError(f"{name} has {t.shape[-2]} heads, no divisor of {heads}")
    strides = t.stride()
    if strides[-1] != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name} must have contiguous channels (its last dimension)")
    if len(strides) == 4:
        return _FIVE(t.data_ptr(), strides[0], strides[1], strides[2], t.shape[2])
    return _FIVE(t.data_ptr(), strides[0], strides[0], strides[1], t.shape[1])


def rotary_frequencies(part: int, *, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                       original_length: int = 4096, fast: float = 32.0, slow: float = 1.0, device="cuda"):
    """Frequencies for :func:`rotary`, fp64 [part / 2] radians a position, and the amplitude that goes with them.
    ``base ** (-2 i / part)``, for contexts ``factor`` times as long by ``scaling``: "linear" divides positions by the
    factor; "ntk" raises the base so that the slowest pair is stretched by it and the fastest is kept; "yarn" stretches the
    pairs that turn fewer than ``slow`` times in the ``original_length``, keeps those that turn more than ``fast`` times,
    blends those between, and raises the amplitude to ``0.1 log(factor) + 1``."""
    if part < 2 or part % 2:
        raise ValueError(f"part={part}: an even number of channels")
    if not (base > 1 and factor >= 1 and math.isfinite(base) and math.isfinite(factor)):
        raise ValueError(f"base={base}, factor={factor}: a base above 1 and a factor from 1 on")
    if scaling not in ("none", "linear", "ntk", "yarn"):
        raise ValueError(f"unknown scaling {scaling!r}: none, linear, ntk or yarn")
    if scaling == "none" and factor != 1:
        raise ValueError(f"factor={factor} without a scaling")
    if scaling == "ntk" and part > 2:
        base *= factor ** (part / (part - 2))
    freqs = base ** (-torch.arange(0, part, 2, dtype=torch.float64) / part)
    if scaling == "linear":
        freqs = freqs / factor
    if scaling != "yarn":
        return freqs.to(device), 1.0
    if not (original_length > 0 and fast >= slow > 0):
        raise ValueError(f"original_length={original_length}, fast={fast}, slow={slow}: positive, and fast >= slow")
    # the pair that turns so many times in the original length, as a fraction of an index
    lo, hi = (part * math.log(original_length / (2 * math.pi * turns)) / (2 * math.log(base)) for turns in (fast, slow))
    lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), part - 1)
    stretched = ((torch.arange(part // 2, dtype=torch.float64) - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
    return (freqs * (1 - stretched) + freqs / factor * stretched).to(device), 0.1 * math.log(factor) + 1.0


def _rotary(q, k, positions, freqs, interleaved, amplitude, inverse, out):
    if out is None and all(isinstance(t, torch.Tensor) and t.is_cuda for t in (q, k, positions, freqs)):
        dev = q.device
        plan = _rotary_plan((q.dtype, q.shape, q.stride()), (k.dtype, k.shape, k.stride()), _meta(positions), _meta(freqs))
        if plan is not None and k.device == dev and positions.device == dev and freqs.device == dev:
            xq, xk, yq, yk, sizes, index = plan
            a, b = _like(q), _like(k)
            _check(_library().ccq_rotary(_FIVE(q.data_ptr(), *xq) + _FIVE(k.data_ptr(), *xk),
                                         _FIVE(a.data_ptr(), *yq) + _FIVE(b.data_ptr(), *yk), *sizes, positions.data_ptr(), index,
                                         freqs.data_ptr(), amplitude, interleaved, inverse, _stream(dev, None)))
            return a, b
    if not isinstance(q, torch.Tensor) or q.dim() not in (3, 4):
        raise ValueError("q must be a CUDA tensor of [batch, tokens, heads, width] or [tokens, heads, width]")
    x = _heads(q, "q")
    dev, shape, width = q.device, q.shape, q.shape[-1]
    B, T = shape[:2] if q.dim() == 4 else (1, shape[0])
    outs = []
    y = b""
    for i, t in enumerate((q, k)):
        if t is None:
            break
        name = "qk"[i]
        if i:
            if not isinstance(t, torch.Tensor) or t.dim() != q.dim():
                raise ValueError(f"k must be a CUDA tensor of {q.dim()} dimensions, as q is")
            x += _heads(t, name, dev, q.dtype, shape[:-2] + (t.shape[-2], width))
        o = None if out is None else out[i]
        if o is None:
            n = t.shape[-2]
            o = _like(t)
            y += _FIVE(o.data_ptr(), T * n * width, n * width, width, n)
        else:
            y += _heads(o, "out", dev, t.dtype, t.shape)
        outs.append(o)
    _dense(freqs, "freqs", dev, torch.float64)
    bytes_ = _ids(positions, "positions", dev)
    if positions.shape != shape[:-2]:
        raise ValueError(f"positions have shape {tuple(positions.shape)}, expected {tuple(shape[:-2])}")
    _check(_library().ccq_rotary(x, y, len(outs), _dtype_code(q), B, T, width, 2 * freqs.numel(), positions.data_ptr(), bytes_,
                                 freqs.data_ptr(), amplitude, interleaved, inverse, _stream(dev, None)))
    return (outs[0], outs[1]) if k is not None else outs[0]


def rotary(q, k, positions, freqs, *, interleaved: bool = False, amplitude: float = 1.0, out=None, stream=None):
    """Rotation of queries and keys by their positions (ccq_rotary).  q [batch, tokens, heads, width] (or [tokens, heads,
    width]) and k, with heads of its own, bf16 or fp32 with any strides (slices of one projection); k may be None.
    positions int64 or int32 of the tokens' shape; freqs fp64 [part / 2] radians a position, as from
    :func:`rotary_frequencies`: the first ``part`` channels of a head turn, in pairs (i, i + part / 2) or
    (2 i, 2 i + 1) with ``interleaved``, the rest is copied.  Returns new (q, k), or q without k; ``out`` (a pair) may hold
    their tensors, the inputs themselves among them."""
    if stream is not None:
        return _on_stream(stream, rotary, q, k, positions, freqs, interleaved=interleaved, amplitude=amplitude, out=out)
    return _rotary(q, k, positions, freqs, bool(interleaved), amplitude, 0, out)


def rotary_bwd(dq, dk, positions, freqs, *, interleaved: bool = False, amplitude: float = 1.0, out=None, stream=None):
    """Gradients of :func:`rotary`'s q and k, of those of what it returned: the same rotation, the other way."""
    if stream is not None:
        return _on_stream(stream, rotary_bwd, dq, dk, positions, freqs, interleaved=interleaved, amplitude=amplitude, out=out)
    return _rotary(dq, dk, positions, freqs, bool(interleaved), amplitude, 1, out)


# ---------------------------------------------------------------- linear attention, a decay for each head


def _decay_args(q, k, v, log_decay, scale, cu_seqlens):
    if not isinstance(q, torch.Tensor) or q.dim() != 4:
        raise ValueError("q must be a CUDA tensor of [batch, tokens, heads, d]")
    B, T, _, d = q.shape
    dev = _cuda(q, "q").device
    _dense(log_decay, "log_decay", dev, torch.float32)
    if log_decay.dim() != 1:
        raise ValueError("log_decay must be [heads]")
    H = log_decay.shape[0]
    packed = [_heads(q, "q", heads=H)]
    for name, t in (("k", k), ("v", v)):
        if not isinstance(t, torch.Tensor) or t.dim() != 4:
            raise ValueError(f"{name} must be a CUDA tensor of [batch, tokens, heads, d]")
        packed.append(_heads(t, name, dev, q.dtype, (B, T, t.shape[2], d), H))
    cu, cu_bytes, seqs = None, 8, B
    if cu_seqlens is not None:
        cu_bytes = _ids(cu_seqlens, "cu_seqlens", dev)
        if B != 1 or cu_seqlens.dim() != 1 or cu_seqlens.shape[0] < 1:
            raise ValueError("cu_seqlens must be [sequences + 1] offsets into a batch of one row of packed tokens")
        cu, seqs = cu_seqlens.data_ptr(), cu_seqlens.shape[0] - 1
    return dev, B, T, H, d, packed, (cu, cu_bytes, seqs), d ** -0.5 if scale is None else scale


def decay_attention(q, k, v, log_decay, *, scale: Optional[float] = None, state=None, cu_seqlens=None, out=None,
                    final_state=None, return_state: bool = True, workspace=None, stream=None):
    """Linear attention with a constant decay for each head (ccq_decay_attention): with S = exp(log_decay) S + k v^T token by
    token, o = scale S^T q.  q, k, v [B, T, heads, d], d 64 or 128, bf16 or fp32 with any strides; fewer heads
    than log_decay's (fp32 [H], <= 0, a constant of the layer) are shared by consecutive ones.  ``scale``: d ** -0.5.
    ``cu_seqlens``: CUDA offsets [N + 1] of sequences packed in one row (tokens of none are zero in a new output, and left as
    they are in ``out``).
    ``state`` [B or N, H, d, d] fp32: the states before the first tokens.  Returns (o [B, T, H, d], the states after the
    last tokens; None without ``return_state``); ``final_state`` may be ``state``, ``out`` shares no element with an input.

    bf16 tensors whose addresses and strides are multiples of 16 bytes run on the tensor cores in chunks of 128 tokens: the products
    of queries and keys, and the copy of the state that queries read, are rounded to bf16 (outputs are off by 2.3e-3 of their
    size, where rounding exact ones alone gives 1.7e-3); the state itself is fp32, of terms in 24 bits where one is handed out, 17 where
    none is.  There a value that is not finite reaches the outputs of its whole chunk, those of earlier tokens too.  fp32 tensors,
    and bf16 ones that lie otherwise, are computed in fp32, 8 x 4096 x 16 x 128 about 30 times as long; there it reaches no earlier token."""
    if stream is not None:
        return _on_stream(stream, decay_attention, q, k, v, log_decay, scale=scale, state=state, cu_seqlens=cu_seqlens, out=out,
                          final_state=final_state, return_state=return_state, workspace=workspace)
    given = [t for t in (state, final_state) if t is not None]
    if out is None and all(isinstance(t, torch.Tensor) and t.is_cuda for t in (q, k, v, log_decay, *given)) and (
            cu_seqlens is None or (isinstance(cu_seqlens, torch.Tensor) and cu_seqlens.is_cuda)):
        dev = q.device
        raw = _stream(dev, None)
        plan = _decay_plan((q.dtype, q.shape, q.stride()), (k.dtype, k.shape, k.stride()), (v.dtype, v.shape, v.stride()),
                           _meta(log_decay), _meta(cu_seqlens), tuple(map(_meta, given)), dev.index)
        if plan is not None and k.device == dev and v.device == dev and log_decay.device == dev and all(
                t.device == dev for t in given) and (cu_seqlens is None or cu_seqlens.device == dev):
            (xq, xk, xv), xo, shape, state_shape, sizes, (cu_bytes, seqs), code, need, root = plan
            out = _like(q) if q.shape == shape else torch.empty(shape, dtype=q.dtype, device=dev)
            if final_state is None and return_state:
                final_state = torch.empty(state_shape, dtype=torch.float32, device=dev)
            workspace, nbytes = _workspace(workspace, need, dev)
            _check(_library().ccq_decay_attention(
                _FIVE(q.data_ptr(), *xq), _FIVE(k.data_ptr(), *xk), _FIVE(v.data_ptr(), *xv), code, log_decay.data_ptr(),
                root if scale is None else scale, _ptr(state), _FIVE(out.data_ptr(), *xo), _ptr(final_state), *sizes,
                _ptr(cu_seqlens), cu_bytes, seqs, _ptr(workspace), nbytes, raw))
            if cu_seqlens is not None:
                _check(_library().ccq_zero_outside(_FIVE(out.data_ptr(), *xo), code, shape[1], shape[3], cu_seqlens.data_ptr(), cu_bytes,
                                                   seqs, raw))
            return out, final_state
    dev, B, T, H, d, (hq, hk, hv), cu, scale = _decay_args(q, k, v, log_decay, scale, cu_seqlens)
    shape = (cu[2], H, d, d)
    if state is not None:
        _dense(state, "state", dev, torch.float32, shape)
    if final_state is not None:
        _dense(final_state, "final_state", dev, torch.float32, shape)
    elif return_state:
        final_state = torch.empty(shape, dtype=torch.float32, device=dev)
    new = out is None
    if new:
        out = torch.empty((B, T, H, d), dtype=q.dtype, device=dev)
        ho = _FIVE(out.data_ptr(), T * H * d, H * d, d, H)
    else:
        ho = _heads(out, "out", dev, q.dtype, (B, T, H, d))
    raw = _stream(dev, None)  # (before the workspace's size is asked for: a function of the current device's SMs)
    code = _dtype_code(q)
    workspace, nbytes = _workspace(workspace, _size("ccq_decay_attention_workspace_size", dev.index, B, T, H, d, cu[2], code),
                                   dev)
    _check(_library().ccq_decay_attention(hq, hk, hv, code, log_decay.data_ptr(), scale, _ptr(state),
                                          ho, _ptr(final_state), B, T, H, d, *cu,
                                          _ptr(workspace), nbytes, raw))
    if new and cu_seqlens is not None:
        _check(_library().ccq_zero_outside(ho, code, T, d, *cu, raw))
    return out, final_state


def decay_attention_bwd(q, k, v, log_decay, dout, *, scale: Optional[float] = None, state=None, dfinal_state=None,
                        cu_seqlens=None, out: Optional[dict] = None, workspace=None, stream=None):
    """Gradients of :func:`decay_attention` (ccq_decay_attention_bwd): a dict of dq, dk, dv (with q's, k's and v's heads) and,
    with ``state`` or ``dfinal_state`` (the gradient of the states that the forward returned), dstate.  Tokens that no packed
    sequence holds get zeros.  Only the forward's inputs are needed.  ``out`` may hold preallocated tensors under those names,
    apart from the inputs and each other.  Arithmetic as in :func:`decay_attention`: a gradient's two products over pairs of tokens are
    rounded to bf16 between them on the tensor cores, and so is the state that it reads."""
    if stream is not None:
        return _on_stream(stream, decay_attention_bwd, q, k, v, log_decay, dout, scale=scale, state=state,
                          dfinal_state=dfinal_state, cu_seqlens=cu_seqlens, out=out, workspace=workspace)
    given = [t for t in (state, dfinal_state) if t is not None]
    if not out and all(isinstance(t, torch.Tensor) and t.is_cuda for t in (q, k, v, log_decay, dout, *given)) and (
            cu_seqlens is None or (isinstance(cu_seqlens, torch.Tensor) and cu_seqlens.is_cuda)):
        dev = q.device
        raw = _stream(dev, None)
        plan = _decay_plan((q.dtype, q.shape, q.stride()), (k.dtype, k.shape, k.stride()), (v.dtype, v.shape, v.stride()),
                           _meta(log_decay), _meta(cu_seqlens), tuple(map(_meta, given)), dev.index, _meta(dout))
        if plan is not None and all(t.device == dev for t in (k, v, log_decay, dout, *given)) and (
                cu_seqlens is None or cu_seqlens.device == dev):
            (xq, xk, xv, xo), _, _, state_shape, sizes, (cu_bytes, seqs), code, need, root = plan
            dq, dk, dv = _like(q), _like(k), _like(v)
            g = {"dq": dq, "dk": dk, "dv": dv}
            if given:
                g["dstate"] = torch.empty(state_shape, dtype=torch.float32, device=dev)
            workspace, nbytes = _workspace(workspace, need, dev)
            _check(_library().ccq_decay_attention_bwd(
                _FIVE(q.data_ptr(), *xq), _FIVE(k.data_ptr(), *xk), _FIVE(v.data_ptr(), *xv), code, log_decay.data_ptr(),
                root if scale is None else scale, _ptr(state), _FIVE(dout.data_ptr(), *xo), _ptr(dfinal_state),
                *(_FIVE(t.data_ptr(), *_dense_strides(t.shape)) for t in (dq, dk, dv)), _ptr(g.get("dstate")), *sizes,
                _ptr(cu_seqlens), cu_bytes, seqs, _ptr(workspace), nbytes, raw))
            return g
    dev, B, T, H, d, (hq, hk, hv), cu, scale = _decay_args(q, k, v, log_decay, scale, cu_seqlens)
    shape = (cu[2], H, d, d)
    ho = _heads(dout, "dout", dev, q.dtype, (B, T, H, d))
    g = dict(out or {})
    if state is not None:
        _dense(state, "state", dev, torch.float32, shape)
    if dfinal_state is not None:
        _dense(dfinal_state, "dfinal_state", dev, torch.float32, shape)
    if g.get("dstate") is not None:
        _dense(g["dstate"], "dstate", dev, torch.float32, shape)
    elif state is not None or dfinal_state is not None:
        g["dstate"] = torch.empty(shape, dtype=torch.float32, device=dev)
    heads = []
    for name, like in (("dq", q), ("dk", k), ("dv", v)):
        if g.get(name) is None:
            n = like.shape[2]
            g[name] = _like(like)
            heads.append(_FIVE(g[name].data_ptr(), T * n * d, n * d, d, n))
        else:
            heads.append(_heads(g[name], name, dev, like.dtype, like.shape))
    raw = _stream(dev, None)
    code = _dtype_code(q)
    workspace, nbytes = _workspace(workspace, _size("ccq_decay_attention_bwd_workspace_size", dev.index, B, T, H, q.shape[2],
                                                    k.shape[2], v.shape[2], d, cu[2], code), dev)
    _check(_library().ccq_decay_attention_bwd(hq, hk, hv, code, log_decay.data_ptr(), scale, _ptr(state), ho,
                                              _ptr(dfinal_state), *heads, _ptr(g.get("dstate")), B, T, H, d, *cu,
                                              _ptr(workspace), nbytes, raw))
    return g


def decay_attention_step(q, k, v, log_decay, state, *, scale: Optional[float] = None, slots=None, out=None, stream=None):
    """One token of every sequence (ccq_decay_attention_step): q, k, v [B, heads, d] as for :func:`decay_attention`; ``state``
    fp32 [B, H, d, d], or [rows, H, d, d] with ``slots`` (int32 or int64 [B]: the row of each; negative: none, a zero
    output), is updated in place.  Returns o [B, H, d].  A slot outside the rows, or that an earlier row of the
    batch has, gives a zero output, changes nothing and leaves CCQ_ERR_INDEX for :func:`ccq.device_status`."""
    if stream is not None:
        return _on_stream(stream, decay_attention_step, q, k, v, log_decay, state, scale=scale, slots=slots, out=out)
    if out is None and all(isinstance(t, torch.Tensor) and t.is_cuda for t in (q, k, v, log_decay, state)) and (
            slots is None or (isinstance(slots, torch.Tensor) and slots.is_cuda)):
        dev = q.device
        plan = _step_plan((q.dtype, q.shape, q.stride()), (k.dtype, k.shape, k.stride()), (v.dtype, v.shape, v.stride()),
                          _meta(log_decay), _meta(state), _meta(slots))
        if plan is not None and k.device == dev and v.device == dev and log_decay.device == dev and state.device == dev and (
                slots is None or slots.device == dev):
            (xq, xk, xv), xo, shape, code, rows, slot_bytes, root = plan
            out = _like(q) if q.shape == shape else torch.empty(shape, dtype=q.dtype, device=dev)
            _check(_library().ccq_decay_attention_step(
                _FIVE(q.data_ptr(), *xq), _FIVE(k.data_ptr(), *xk), _FIVE(v.data_ptr(), *xv), code, log_decay.data_ptr(),
                root if scale is None else scale, state.data_ptr(), rows, _ptr(slots), slot_bytes, _FIVE(out.data_ptr(), *xo),
                *shape, _stream(dev, None)))
            return out
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a CUDA tensor of [batch, heads, d]")
    B, _, d = q.shape
    dev = _cuda(q, "q").device
    _dense(log_decay, "log_decay", dev, torch.float32)
    if log_decay.dim() != 1:
        raise ValueError("log_decay must be [heads]")
    H = log_decay.shape[0]
    packed = [_heads(q, "q", heads=H)]
    for name, t in (("k", k), ("v", v)):
        if not isinstance(t, torch.Tensor) or t.dim() != 3:
            raise ValueError(f"{name} must be a CUDA tensor of [batch, heads, d]")
        packed.append(_heads(t, name, dev, q.dtype, (B, t.shape[1], d), H))
    _dense(state, "state", dev, torch.float32)
    if state.dim() != 4 or state.shape[1:] != (H, d, d) or (slots is None and state.shape[0] != B):
        raise ValueError(f"state has shape {tuple(state.shape)}, expected {(B if slots is None else 'rows', H, d, d)}")
    slot_bytes = 4
    if slots is not None:
        slot_bytes = _ids(slots, "slots", dev)
        if slots.shape != (B,):
            raise ValueError(f"slots have shape {tuple(slots.shape)}, expected {(B,)}")
    if out is None:
        out = torch.empty((B, H, d), dtype=q.dtype, device=dev)
        ho = _FIVE(out.data_ptr(), H * d, d, d, H)
    else:
        ho = _heads(out, "out", dev, q.dtype, (B, H, d))
    _check(_library().ccq_decay_attention_step(*packed, _dtype_code(q), log_decay.data_ptr(), d ** -0.5 if scale is None else scale,
                                               state.data_ptr(), state.shape[0], _ptr(slots), slot_bytes,
                                               ho, B, H, d, _stream(dev, None)))
    return out


# ---------------------------------------------------------------- group norm


def _norm_args(x, weight, bias, gate, groups, activation):
    xs = _rows(x, "x")
    dev, channels = x.device, x.shape[-1]
    if groups < 1 or channels % groups:
        raise ValueError(f"{channels} channels do not divide into {groups} groups")
    if activation not in ACTIVATION:
        raise ValueError(f"unknown activation {activation!r}: one of {sorted(ACTIVATION)}")
    gs = 0 if gate is None else _rows(gate, "gate", dev, x.dtype, x.shape)
    param = weight if weight is not None else bias
    pdt = _dtype_code(param) if param is not None else ccq.FP32
    if weight is not None:
        _dense(weight, "weight", dev, param.dtype, (channels,))
    if bias is not None:
        _dense(bias, "bias", dev, param.dtype, (channels,))
    return dev, xs, gs, channels, pdt, x.numel() // channels if channels else 0


def group_norm(x, weight=None, bias=None, gate=None, *, groups: int, activation: str = "silu", centered: bool = True,
               eps: float = 1e-5, out=None, stream=None):
    """Group norm of every token's channels and an activation (ccq_group_norm): with ``groups`` = heads, what
    follows the mixer's read.  x [..., channels] bf16 or fp32; weight, bias [channels] (None: 1 and
    0); ``u * act(gate)`` with a gate of x's shape, ``act(u)`` without.  ``centered=False`` leaves the mean in
    (a root-mean-square norm)."""
    if stream is not None:
        return _on_stream(stream, group_norm, x, weight, bias, gate, groups=groups, activation=activation,
                          centered=centered, eps=eps, out=out)
    dev, xs, gs, channels, pdt, tokens = _norm_args(x, weight, bias, gate, groups, activation)
    if out is None:
        out, os = torch.empty(x.shape, dtype=x.dtype, device=dev), channels
    else:
        os = _rows(out, "out", dev, x.dtype, x.shape)
    _check(_library().ccq_group_norm(x.data_ptr(), xs, _ptr(gate), gs, _ptr(weight), _ptr(bias), _dtype_code(x), pdt,
                                     out.data_ptr(), os, tokens, channels, groups, int(bool(centered)), eps,
                                     ACTIVATION[activation], _stream(dev, None)))
    return out


def group_norm_bwd(x, weight, bias, gate, dout, *, groups: int, activation: str = "silu", centered: bool = True,
                   eps: float = 1e-5, out: Optional[dict] = None, workspace=None, stream=None):
    """Gradients of :func:`group_norm` (ccq_group_norm_bwd): a dict of dx, dgate (where there is a gate), dweight
    and dbias (where there are those).  Only the forward's inputs are needed.  ``out`` may hold preallocated
    tensors under those names."""
    if stream is not None:
        return _on_stream(stream, group_norm_bwd, x, weight, bias, gate, dout, groups=groups, activation=activation,
                          centered=centered, eps=eps, out=out, workspace=workspace)
    dev, xs, gs, channels, pdt, tokens = _norm_args(x, weight, bias, gate, groups, activation)
    ds = _rows(dout, "dout", dev, x.dtype, x.shape)
    for name, like in (("dgate", gate), ("dweight", weight), ("dbias", bias)):
        if like is None and out and out.get(name) is not None:
            raise ValueError(f"out has {name}, but there is no {name[1:]}")
    raw = _stream(dev, None)  # (before the workspace's size is asked for: a function of the current device's SMs)
    g = dict(out or {})
    strides = {"dgate": 0}
    for name, like in (("dx", x), ("dgate", gate)):
        if like is not None:
            if g.get(name) is None:
                g[name], strides[name] = torch.empty(x.shape, dtype=x.dtype, device=dev), channels
            else:
                strides[name] = _rows(g[name], name, dev, x.dtype, x.shape)
    for name, like in (("dweight", weight), ("dbias", bias)):
        if like is not None:
            if g.get(name) is None:
                g[name] = torch.empty(like.shape, dtype=like.dtype, device=dev)
            else:
                _dense(g[name], name, dev, like.dtype, like.shape)
    workspace, nbytes = _workspace(workspace, _size("ccq_group_norm_bwd_workspace_size", dev.index, tokens, channels,
                                                    groups, _dtype_code(x)), dev)
    _check(_library().ccq_group_norm_bwd(
        x.data_ptr(), xs, _ptr(gate), gs, _ptr(weight), _ptr(bias), dout.data_ptr(), ds, _dtype_code(x), pdt,
        g["dx"].data_ptr(), strides["dx"], _ptr(g.get("dgate")), strides["dgate"], _ptr(g.get("dweight")),
        _ptr(g.get("dbias")), tokens, channels, groups, int(bool(centered)), eps, ACTIVATION[activation],
        _ptr(workspace), nbytes, raw))
    return g


# ---------------------------------------------------------------- policy loss


def _tokens(logits, actions):
    ls = _rows(logits, "logits")
    dev = logits.device
    id_bytes = _ids(actions, "actions", dev)
    if actions.shape != logits.shape[:-1]:
        raise ValueError(f"actions have shape {tuple(actions.shape)}, expected {tuple(logits.shape[:-1])}")
    return dev, ls, id_bytes


def policy_loss(logits, actions, old_logp, advantages, *, ref_logp=None, weights=None, clip=(0.2, 0.2),
                kl_coef: float = 0.0, temperature: float = 1.0, grad_scale: float = 1.0, grad: bool = True,
                dlogits=None, workspace=None, stream=None):
    """Clipped policy loss with a KL term and its gradient (ccq_policy_loss).  logits [..., vocab] bf16 or fp32;
    actions [...] int64 or int32; old_logp, advantages, ref_logp (None: no KL term), weights (None: 1 / n)
    [...] fp32.  A token of weight 0 is masked: nothing of it counts, whatever it holds.  ``clip`` is (low, high), the ratio is held
    in [1 - low, 1 + high].  Returns a dict of loss (a scalar tensor), logp [...] (0 where masked) and,
    with ``grad``, dlogits (``grad_scale`` times the loss's gradient; ``dlogits`` may be the logits)."""
    if stream is not None:
        return _on_stream(stream, policy_loss, logits, actions, old_logp, advantages, ref_logp=ref_logp, weights=weights,
                          clip=clip, kl_coef=kl_coef, temperature=temperature, grad_scale=grad_scale, grad=grad,
                          dlogits=dlogits, workspace=workspace)
    dev, ls, id_bytes = _tokens(logits, actions)
    shape, vocab = actions.shape, logits.shape[-1]
    _dense(old_logp, "old_logp", dev, torch.float32, shape)
    _dense(advantages, "advantages", dev, torch.float32, shape)
    if ref_logp is not None:
        _dense(ref_logp, "ref_logp", dev, torch.float32, shape)
    if weights is not None:
        _dense(weights, "weights", dev, torch.float32, shape)
    loss = torch.empty((), dtype=torch.float32, device=dev)
    logp = torch.empty(shape, dtype=torch.float32, device=dev)
    gs = 0
    if grad:
        if dlogits is None:
            dlogits, gs = torch.empty(logits.shape, dtype=logits.dtype, device=dev), vocab
        else:
            gs = _rows(dlogits, "dlogits", dev, logits.dtype, logits.shape)
    elif dlogits is not None:
        raise ValueError("dlogits is given but grad is False")
    n = actions.numel()
    p = _PolicyParams(clip[0], clip[1], kl_coef, temperature, grad_scale)
    workspace, nbytes = _workspace(workspace, _size("ccq_policy_loss_workspace_size", -1, n), dev)
    _check(_library().ccq_policy_loss(
        logits.data_ptr(), _dtype_code(logits), ls, actions.data_ptr(), id_bytes, old_logp.data_ptr(), _ptr(ref_logp),
        advantages.data_ptr(), _ptr(weights), n, vocab, ctypes.byref(p), loss.data_ptr(), logp.data_ptr(),
        _ptr(dlogits), gs, _ptr(workspace), nbytes, _stream(dev, None)))
    return {"loss": loss, "logp": logp, "dlogits": dlogits} if grad else {"loss": loss, "logp": logp}


def token_logp(logits, actions, *, temperature: float = 1.0, out=None, stream=None):
    """``log_softmax(logits / temperature)`` at the actions (ccq_token_logp), fp32 [...]: the old and reference
    log-probabilities of a policy loss."""
    if stream is not None:
        return _on_stream(stream, token_logp, logits, actions, temperature=temperature, out=out)
    dev, ls, id_bytes = _tokens(logits, actions)
    if out is None:
        out = torch.empty(actions.shape, dtype=torch.float32, device=dev)
    else:
        _dense(out, "out", dev, torch.float32, actions.shape)
    _check(_library().ccq_token_logp(logits.data_ptr(), _dtype_code(logits), ls, actions.data_ptr(), id_bytes,
                                     actions.numel(), logits.shape[-1], temperature, out.data_ptr(),
                                     _stream(dev, None)))
    return out


# ---------------------------------------------------------------- AdamW


@dataclass
class AdamWState:
    """Moments of a list of parameters: m and v as fp32 tensors, or as float8_e4m3fn tensors that hold m and the
    square root of v over ``scale`` (fp32 [blocks, 2] per parameter, one row for ADAMW_BLOCK consecutive elements);
    ``master`` the fp32 copies of bf16 parameters (None: none)."""
    m: List[torch.Tensor]
    v: List[torch.Tensor]
    scale: Optional[List[torch.Tensor]] = None
    master: Optional[List[torch.Tensor]] = None


def adamw_state(params, *, bits: int = 32, master: bool = False) -> AdamWState:
    """Zero moments for ``params`` (in 32 or 8 bits), and fp32 master copies of them where asked for."""
    if bits not in (8, 32):
        raise ValueError(f"bits={bits}: 8 or 32")
    dtype = torch.float32 if bits == 32 else torch.float8_e4m3fn

    def zeros(p):
        return torch.zeros(p.shape, dtype=torch.float32 if bits == 32 else torch.uint8, device=p.device).view(dtype)

    scale = None
    if bits == 8:
        scale = [torch.full((-(-p.numel() // ADAMW_BLOCK), 2), 2.0 ** -100, device=p.device) for p in params]
    return AdamWState([zeros(p) for p in params], [zeros(p) for p in params], scale,
                      [p.detach().float().clone() for p in params] if master else None)


def _adamw_list(ts, name, count, index, dtype, numels):
    """The addresses of a list that goes with the parameters.  (One expression a tensor: with a hundred of them the
    host's work is most of a call.)"""
    if len(ts) != count:
        raise ValueError(f"{name} has {len(ts)} tensors for {count} parameters")
    at = [t.data_ptr() for t, n in zip(ts, numels)
          if t.dtype is dtype and t.get_device() == index and t.numel() == n and t.is_contiguous()]
    if len(at) != count:
        for i, (t, n) in enumerate(zip(ts, numels)):
            if t.dtype != dtype:
                raise TypeError(f"{name}[{i}] must be {dtype}, got {t.dtype}")
            if t.numel() != n or not t.is_contiguous() or t.get_device() != index:
                raise ValueError(f"{name}[{i}] must be a contiguous tensor of {n} elements on cuda:{index}")
    return at


def adamw_step(params, grads, state: AdamWState, step: int, *, lr: float, betas=(0.9, 0.999), eps: float = 1e-8,
               weight_decay: float = 0.01, grad_scale: Optional[torch.Tensor] = None, stream=None):
    """One AdamW update of all ``params`` (ccq_adamw_step), in place, with the moments of ``state``; ``step`` counts
    from 1.  params and grads: lists of contiguous bf16 or fp32 tensors (one type for all params, one for all
    grads).  ``grad_scale``: a CUDA fp32 scalar that multiplies the gradients (as from clipping their norm).  ``step``
    and ``lr`` are the host's: a CUDA graph that has captured the call keeps them (and what follows from the step) at
    every replay, so it is made outside of one."""
    if not params:
        return
    first = _cuda(params[0], "params[0]")
    dev, index, count = first.device, first.get_device(), len(params)
    numels = [p.numel() for p in params]
    bits = 32 if state.scale is None else 8
    dtype = torch.float32 if bits == 32 else torch.float8_e4m3fn
    none = [0] * count
    rows = zip(_adamw_list(params, "params", count, index, first.dtype, numels),
               _adamw_list(grads, "grads", count, index, grads[0].dtype if grads else None, numels),
               _adamw_list(state.m, "state.m", count, index, dtype, numels),
               _adamw_list(state.v, "state.v", count, index, dtype, numels),
               none if bits == 32 else _adamw_list(state.scale, "state.scale", count, index, torch.float32,
                                                   [-(-n // ADAMW_BLOCK) * 2 for n in numels]),
               none if state.master is None else _adamw_list(state.master, "state.master", count, index, torch.float32,
                                                             numels), numels)
    table = struct.pack(f"{7 * count}q", *chain.from_iterable(rows))
    if grad_scale is not None:
        _dense(grad_scale, "grad_scale", dev, torch.float32)
        if grad_scale.numel() != 1:
            raise ValueError("grad_scale must be a scalar")
    p = _AdamWParams(lr, betas[0], betas[1], eps, weight_decay, step)
    _check(_library().ccq_adamw_step(table, count, _dtype_code(first), _dtype_code(grads[0]), bits,
                                     ctypes.byref(p), _ptr(grad_scale), _stream(dev, stream)))
