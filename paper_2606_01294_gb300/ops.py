"""Python binding of include/ccq_ops.h: the operators around the CCQ token mixer.

The embedding lookup and its gradient, the (gated) group norm after the mixer's read and its gradient, the
clipped policy loss with its gradient, the token log-probabilities, and the AdamW update of many tensors.  As in
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
import struct
from dataclasses import dataclass
from itertools import chain
from typing import List, Optional

import torch

from . import ccq
from .ccq import _check, _dtype_code, _on_stream, _ptr, _stream

ACTIVATION = {"none": 0, "silu": 1, "sigmoid": 2}
ADAMW_BLOCK = 256

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
