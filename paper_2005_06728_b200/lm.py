"""Language-model operators around the update: argument marshalling for the odsgd_embed_*, odsgd_token_logprob,
odsgd_policy_loss, odsgd_grad_set_*, odsgd_gated_*, odsgd_dropout and odsgd_verify_* calls of libodsgd.so.

What a worker runs on either side of its model, and in it, when the parameter set is a language model's:

* `embed_lookup` / `embed_grad`: token rows out of the weight arena, and their gradient into the
  gradient arena (`arena[a:b].view(vocab, dim)` is a table);
* `token_logprob`: the score of each taken token (acting policy, reference policy, evaluation);
* `policy_loss`: the clipped policy loss with a KL term, and its gradient, in one pass;
* `GradSet`: norm and clipping of a list of gradient tensors, laid out into the arenas the server
  reads;
* `gated_ffn` / `gated_ffn_grad`: the gated feed-forward block up to its gated product h, on 16-bit activations, and its
  gradients (the product that leads back to the model's width is the caller's); `stalled_waits`: whether any was cut short;
* `dropout`: onto a residual, by a mask that is a function of a seed; its own gradient;
* `verify_draft`: drafted tokens accepted under the current policy, one more drawn, and their scores.

include/odsgd.h has the formulas and the treatment of padding, masks and special values.  Every
call is asynchronous on `stream` (default: the current stream), on the current device; results are
new tensors, in memory of that stream, unless a buffer is given.  With another stream than the one a
tensor belongs to, ordering the two and keeping the memory (record_stream) are the caller's.  Tensors may be strided in their leading axes (a shifted
view, an expanded value) as long as the last axis is contiguous and the leading ones fold into two
levels.  There is no CPU fallback and no autograd: the gradient calls are the backward pass.  Tensors that a
caller hands over to be written (out, dtable, dlogits, arenas, gradients clipped in place) count as changed in
place, so that a backward pass of torch that saved one of them fails; replays of a captured graph do not count.
"""
from __future__ import annotations

import ctypes
import struct
from typing import NamedTuple, Optional, Sequence, Tuple

import torch
from torch.autograd.graph import increment_version

from . import binding
from .binding import OK, OdsgdError

F32, BF16, F16, I32, I64 = 0, 1, 2, 3, 4
MAX_TOKENS = 1 << 24

_FLOATS = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
_FLOAT32 = {torch.float32: F32}
_INTS = {torch.int32: I32, torch.int64: I64}
_HALVES = {torch.bfloat16: BF16, torch.float16: F16}
_SAME = {t: {t: c} for t, c in _FLOATS.items()}                             # a tensor of the same type
_OR_FLOAT32 = {t: {t: c, torch.float32: F32} for t, c in _HALVES.items()}  # or of 32 bits
_ACTIVATIONS = {"silu": 0, "gelu": 1}

# odsgd_embed_desc, odsgd_policy_desc and odsgd_grad_tensor of include/odsgd.h, packed by struct: a call is
# a few microseconds, and filling a ctypes structure would be one of them.
_EMBED = struct.Struct("3P4i10qf4x")
_POLICY = struct.Struct("10P2i17q5f4x")
_GRAD_TENSOR = struct.Struct("PNN2i")
_GATED = struct.Struct("9P5i4x18q")
_DROPOUT = struct.Struct("4P2i9q2Qd")
_VERIFY = struct.Struct("7P2i11q2f")


class TokenLogprob(NamedTuple):
    logp: torch.Tensor  # float32, the labels' shape
    lse: torch.Tensor   # float32, the same


class PolicyLoss(NamedTuple):
    stats: torch.Tensor    # float32 [4]: loss, policy term, KL term (without its coefficient), weight of clipped tokens
    logp: torch.Tensor     # float32, the labels' shape
    dlogits: torch.Tensor  # the logits' shape and type

    @property
    def loss(self) -> torch.Tensor:
        return self.stats[0]


class GatedFfn(NamedTuple):
    h: torch.Tensor               # [..., width], x's type
    gate: Optional[torch.Tensor]  # the projections before the activation, the same; None unless kept
    up: Optional[torch.Tensor]


class GatedFfnGrad(NamedTuple):
    dx: Optional[torch.Tensor]       # x's shape and type
    dw_gate: Optional[torch.Tensor]  # the weights' shape
    dw_up: Optional[torch.Tensor]


class Verified(NamedTuple):
    accepted: torch.Tensor  # int32 [batch]: drafts accepted
    tokens: torch.Tensor    # [batch, drafts + 1] of the drafts' type: those, the drawn token, -1
    logp: torch.Tensor      # float32 [batch, drafts + 1]: under the target, 0 behind the drawn token


# --------------------------------------------------------------------------- checks

def _check(rc: int) -> None:
    if rc != OK:
        raise OdsgdError(rc, binding.load_library().odsgd_last_error(None).decode())


def _need(t: torch.Tensor, name: str, codes: dict, dev: int) -> int:
    """The code of a tensor of one of the types of `codes` on the current device, `dev`."""
    if isinstance(t, torch.Tensor):
        code = codes.get(t.dtype)
        if code is not None:
            if t.get_device() == dev:
                return code
            if t.is_cuda:
                raise ValueError(f"{name} is on {t.device}, the current device is cuda:{dev}")
    raise TypeError(f"{name}: need a CUDA tensor of {' / '.join(str(d) for d in codes)}")


def _shape(t: torch.Tensor, shape, name: str) -> None:
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")


# Tensors are passed to the library as [outer][inner], or [outer][inner][last], with two strides.

def _sizes(shape) -> Tuple[int, int]:
    """(outer, inner) of leading axes."""
    if len(shape) == 2:
        return shape
    outer = 1
    for n in shape[:-1]:
        outer *= n
    return outer, shape[-1] if len(shape) else 1


def _levels(t: torch.Tensor, lead: int, name: str) -> Tuple[int, int]:
    """Strides of the two levels that the first `lead` axes make."""
    stride = t.stride()
    if lead == 2:
        return stride[:2]
    if lead < 2:
        return (0, stride[0]) if lead else (0, 0)
    if 0 in t.shape[:lead]:
        return 0, 0  # no element, no stride
    outer, step = 1, 0  # all but the last leading axis fold into one level
    for n, s in reversed(list(zip(t.shape[:lead - 1], stride[:lead - 1]))):
        if n == 1:
            continue
        if outer == 1:
            step = s
        elif s != outer * step:
            raise ValueError(f"{name}: its leading axes do not fold into two strided levels (make it contiguous)")
        outer *= n
    return step, stride[lead - 1]


def _rows(t: torch.Tensor, lead: int, name: str) -> Tuple[int, int]:
    """The same of a tensor with one more axis, which has to be contiguous."""
    stride = t.stride()
    if stride[-1] != 1 and t.shape[-1] != 1:
        raise ValueError(f"{name}: the last axis must be contiguous")
    if lead == 2:
        return stride[:2]
    if lead == 1:
        return 0, stride[0]
    return _levels(t, lead, name)


def _dense(shape) -> Tuple[int, int]:
    """Strides of the rows of new memory of this shape."""
    n = len(shape)
    if n < 2:
        return 0, 0
    return (0 if n == 2 else shape[-2] * shape[-1]), shape[-1]


# Memory of the current device and stream without what a factory function looks at besides (0.7 us instead of 1.9): taken where that
# is nothing, so not under a dispatch or function mode, nor where new memory is filled (deterministic algorithms).
_empty_strided = getattr(getattr(getattr(torch._C, "_dynamo", None), "guards", None), "_empty_strided_cuda", None)
_dispatch_modes = getattr(torch._C, "_len_torch_dispatch_stack", None)
_function_modes = getattr(torch._C, "_len_torch_function_stack", None)
if _dispatch_modes is None or _function_modes is None:
    _empty_strided = None


def _new(like: torch.Tensor, shape, dtype, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    """Contiguous memory of the stream that the work runs on (`like` is on the current device); `shape` None: like's."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return _new(like, shape, dtype, None)
    if _empty_strided is None or _dispatch_modes() or _function_modes() or torch.are_deterministic_algorithms_enabled():
        if shape is None:
            return torch.empty_like(like, dtype=dtype, memory_format=torch.contiguous_format)
        return like.new_empty(shape, dtype=dtype)
    if shape is None:
        shape = like.shape
    elif type(shape) is int:
        return _empty_strided((shape,), (1,), dtype or like.dtype)
    strides, step = (), 1
    for n in reversed(shape):
        strides = (step, *strides)
        step *= n or 1
    return _empty_strided(tuple(shape), strides, dtype or like.dtype)


# The current stream's handle without the Stream object around it (a third of a small call).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _handle(stream: Optional[torch.cuda.Stream], dev: int) -> int:
    if stream is None and _raw_stream is not None:
        return _raw_stream(dev)
    return binding._stream_handle(stream)


def _table(table: torch.Tensor, name: str) -> Tuple[int, int, int]:
    if table.dim() != 2:
        raise ValueError(f"{name}: need [vocab, dim]")
    vocab, dim = table.shape
    stride, last = table.stride()
    if last != 1 and dim != 1:
        raise ValueError(f"{name}: the last axis must be contiguous")
    return vocab, dim, stride if vocab > 1 else max(dim, stride)


# --------------------------------------------------------------------------- embedding

def embed_lookup(tokens: torch.Tensor, table: torch.Tensor, *, scale: float = 1.0, dtype: Optional[torch.dtype] = None,
                 out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """scale * table[tokens], rounded once to `dtype` (default: the table's).  A token outside
    [0, vocab), such as the -1 that pads a ragged batch, gives a row of zeros."""
    dev = torch.cuda.current_device()
    token_type = _need(tokens, "tokens", _INTS, dev)
    table_type = _need(table, "table", _FLOATS, dev)
    vocab, dim, stride = _table(table, "table")
    shape = (*tokens.shape, dim)
    given = out is not None
    if not given:
        out = _new(table, shape, table.dtype if dtype is None else dtype, stream)
    elif dtype is not None and out.dtype != dtype:
        raise ValueError("out and dtype disagree")
    out_type = _need(out, "out", _FLOATS, dev)
    _shape(out, shape, "out")
    lead = tokens.dim()
    d = _EMBED.pack(tokens.data_ptr(), out.data_ptr(), table.data_ptr(), token_type, out_type, table_type, 0,
                    *_sizes(tokens.shape), *_levels(tokens, lead, "tokens"), *_rows(out, lead, "out"), vocab, dim, stride, -1, scale)
    _check(binding.load_library().odsgd_embed_lookup(d, _handle(stream, dev)))
    if given:
        increment_version(out)
    return out


def embed_grad(tokens: torch.Tensor, grad: torch.Tensor, dtable: torch.Tensor, *, scale: float = 1.0,
               padding_token: Optional[int] = None, accumulate: bool = False, workspace: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """dtable[v] = scale * sum of grad over the positions of token v, zeros where there is none
    (accumulate: added to what is there).  `dtable` is float32, normally a view of the worker's
    gradient arena.  Tokens outside [0, vocab) and `padding_token` contribute nothing."""
    dev = torch.cuda.current_device()
    token_type = _need(tokens, "tokens", _INTS, dev)
    grad_type = _need(grad, "grad", _FLOATS, dev)
    _need(dtable, "dtable", _FLOAT32, dev)
    vocab, dim, stride = _table(dtable, "dtable")
    _shape(grad, (*tokens.shape, dim), "grad")
    lead = tokens.dim()
    d = _EMBED.pack(tokens.data_ptr(), grad.data_ptr(), dtable.data_ptr(), token_type, grad_type, F32, 1 if accumulate else 0,
                    *_sizes(tokens.shape), *_levels(tokens, lead, "tokens"), *_rows(grad, lead, "grad"), vocab, dim, stride,
                    -1 if padding_token is None else padding_token, scale)
    lib = binding.load_library()
    if workspace is None:
        need = ctypes.c_size_t()
        _check(lib.odsgd_embed_grad_workspace(d, ctypes.byref(need)))
        workspace = _new(grad, max(16, need.value), torch.uint8, stream)
    elif not workspace.is_contiguous() or workspace.get_device() != dev:
        raise ValueError("workspace: need a contiguous tensor on the current device")
    _check(lib.odsgd_embed_grad(d, workspace.data_ptr(), workspace.nbytes, _handle(stream, dev)))
    increment_version(dtable)
    return dtable


def embed_grad_workspace(tokens: torch.Tensor, grad: torch.Tensor, dtable: torch.Tensor) -> int:
    """Bytes of workspace that embed_grad needs for tensors of these shapes and types."""
    d = _EMBED.pack(0, 0, 0, _INTS[tokens.dtype], _FLOATS[grad.dtype], F32, 0, *_sizes(tokens.shape), 0, 0, 0, 0,
                    dtable.shape[0], dtable.shape[1], dtable.shape[1], -1, 1.0)
    need = ctypes.c_size_t()
    _check(binding.load_library().odsgd_embed_grad_workspace(d, ctypes.byref(need)))
    return need.value


# --------------------------------------------------------------------------- scores and policy loss

def token_logprob(logits: torch.Tensor, labels: torch.Tensor, *, inv_temp: float = 1.0,
                  stream: Optional[torch.cuda.Stream] = None) -> TokenLogprob:
    """log softmax(inv_temp * logits)[label] and the row's log of summed exponentials, in float32;
    zeros where the label is outside [0, vocab)."""
    dev = torch.cuda.current_device()
    kind = _need(logits, "logits", _FLOATS, dev)
    label_type = _need(labels, "labels", _INTS, dev)
    shape, whole = labels.shape, logits.shape
    lead = len(shape)
    if len(whole) != lead + 1 or whole[:-1] != shape:
        raise ValueError(f"labels: shape {tuple(shape)}, expected {tuple(whole[:-1])}")
    strides = (*_rows(logits, lead, "logits"), *_levels(labels, lead, "labels"))
    logp, lse = _new(labels, None, torch.float32, stream), _new(labels, None, torch.float32, stream)
    d = _POLICY.pack(logits.data_ptr(), labels.data_ptr(), 0, 0, 0, 0, 0, logp.data_ptr(), lse.data_ptr(), 0, kind, label_type,
                     *_sizes(shape), whole[-1], *strides, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, inv_temp, 0.0, 0.0, 0.0, 0.0)
    _check(binding.load_library().odsgd_token_logprob(d, _handle(stream, dev)))
    return TokenLogprob(logp, lse)


def policy_loss(logits: torch.Tensor, labels: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor,
                weights: torch.Tensor, *, ref_logp: Optional[torch.Tensor] = None, clip_low: float = 0.2,
                clip_high: float = 0.2, kl_coef: float = 0.0, inv_temp: float = 1.0, grad_scale: float = 1.0,
                dlogits: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> PolicyLoss:
    """The clipped policy loss with a KL term, and its gradient, over rows of logits.

    `old_logp`, `ref_logp`, `advantages` and `weights` are float32 of the labels' shape (expanded
    views welcome); a weight is mask and normalisation in one.  `dlogits` may be `logits` itself.
    """
    dev = torch.cuda.current_device()
    kind = _need(logits, "logits", _FLOATS, dev)
    label_type = _need(labels, "labels", _INTS, dev)
    shape, whole = labels.shape, logits.shape
    lead = len(shape)
    if len(whole) != lead + 1 or whole[:-1] != shape:
        raise ValueError(f"labels: shape {tuple(shape)}, expected {tuple(whole[:-1])}")

    def vector(t, name):
        _need(t, name, _FLOAT32, dev)
        if t.shape != shape:
            _shape(t, shape, name)
        return t.stride() if lead == 2 else _levels(t, lead, name)

    strides = (*_rows(logits, lead, "logits"), *_levels(labels, lead, "labels"), *vector(old_logp, "old_logp"),
               *((0, 0) if ref_logp is None else vector(ref_logp, "ref_logp")),
               *vector(advantages, "advantages"), *vector(weights, "weights"))
    given = dlogits is not None
    if not given:
        dlogits = _new(logits, None, None, stream)
    else:
        _need(dlogits, "dlogits", {logits.dtype: kind}, dev)
        _shape(dlogits, whole, "dlogits")
    outer, inner = _sizes(shape)
    n = outer * inner
    stats, logp = _new(logits, 4, torch.float32, stream), _new(labels, None, torch.float32, stream)
    workspace = _new(logits, max(4, 3 * n), torch.float32, stream)  # 12 bytes a row
    d = _POLICY.pack(logits.data_ptr(), labels.data_ptr(), old_logp.data_ptr(), 0 if ref_logp is None else ref_logp.data_ptr(),
                     advantages.data_ptr(), weights.data_ptr(), dlogits.data_ptr(), logp.data_ptr(), 0, stats.data_ptr(), kind, label_type,
                     outer, inner, whole[-1], *strides, *_rows(dlogits, lead, "dlogits"),
                     inv_temp, clip_low, clip_high, kl_coef, grad_scale)
    _check(binding.load_library().odsgd_policy_loss(d, workspace.data_ptr(), 12 * n if n > 1 else 16, _handle(stream, dev)))
    if given:
        increment_version(dlogits)
    return PolicyLoss(stats, logp, dlogits)


# --------------------------------------------------------------------------- gated feed-forward block

def _gated_inputs(x, w_gate, w_up, activation, dev):
    kind = _need(x, "x", _HALVES, dev)
    weight_type = _need(w_gate, "w_gate", _OR_FLOAT32[x.dtype], dev)
    _need(w_up, "w_up", _SAME[w_gate.dtype], dev)
    if x.dim() < 1:
        raise ValueError("x: need [..., dim]")
    width, dim, gate_stride = _table(w_gate, "w_gate")
    _shape(w_up, w_gate.shape, "w_up")
    up_stride = _table(w_up, "w_up")[2]
    if x.shape[-1] != dim:
        raise ValueError(f"x: last axis {x.shape[-1]}, expected {dim}")
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation: {activation!r}, expected one of {sorted(_ACTIVATIONS)}")
    return kind, weight_type, width, dim, gate_stride, up_stride


def _workspace(need: int, given: Optional[torch.Tensor], like: torch.Tensor, dev: int, stream):
    """(tensor to keep, address, bytes) of a call's workspace; none where none is needed."""
    if given is None:
        if need == 0:
            return None, 0, 0
        given = _new(like, need, torch.uint8, stream)
    elif not given.is_contiguous() or given.get_device() != dev:
        raise ValueError("workspace: need a contiguous tensor on the current device")
    return given, given.data_ptr(), given.nbytes


def gated_ffn(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, *, activation: str = "silu", save: bool = False,
              out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
              stream: Optional[torch.cuda.Stream] = None) -> GatedFfn:
    """h = act(x w_gate^T) * (x w_up^T) for x [..., dim] of bfloat16 or float16 and weights [width, dim] of x's type, or
    float32 (views of a weight arena, rounded to x's type by the call).  `save`: gate and up are kept for gated_ffn_grad.
    activation: "silu" or "gelu" (by the error function)."""
    dev = torch.cuda.current_device()
    kind, weight_type, width, dim, gate_stride, up_stride = _gated_inputs(x, w_gate, w_up, activation, dev)
    lead = x.dim() - 1
    shape = (*x.shape[:-1], width)
    given = out is not None
    if not given:
        out = _new(x, shape, x.dtype, stream)
    else:
        _need(out, "out", _SAME[x.dtype], dev)
        _shape(out, shape, "out")
    gate = up = None
    dense, at, up_at = _dense(shape), 0, 0
    if save:
        gate, up = _new(x, shape, x.dtype, stream), _new(x, shape, x.dtype, stream)
        at, up_at = gate.data_ptr(), up.data_ptr()
    d = _GATED.pack(x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), out.data_ptr(), at, up_at, 0, 0, 0, kind, weight_type, kind,
                    _ACTIVATIONS[activation], 0, *_sizes(shape[:-1]), dim, width, *_rows(x, lead, "x"),
                    *(_rows(out, lead, "out") if given else dense), *dense, *dense, 0, 0, gate_stride, up_stride, 0, 0)
    lib, handle = binding.load_library(), _handle(stream, dev)
    # most calls need no workspace and are done here; one that does has been refused, with nothing written
    if workspace is not None or lib.odsgd_gated_forward(d, 0, 0, handle) != OK:
        need = ctypes.c_size_t()
        _check(lib.odsgd_gated_workspace(d, 0, ctypes.byref(need)))
        workspace, ws_at, ws_bytes = _workspace(need.value, workspace, x, dev, stream)
        _check(lib.odsgd_gated_forward(d, ws_at, ws_bytes, handle))
    if given:
        increment_version(out)
    return GatedFfn(out, gate, up)


def gated_ffn_grad(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, gate: torch.Tensor, up: torch.Tensor, dh: torch.Tensor, *,
                   activation: str = "silu", want_dx: bool = True, want_dw: bool = True, dx: Optional[torch.Tensor] = None,
                   dw_gate: Optional[torch.Tensor] = None, dw_up: Optional[torch.Tensor] = None, accumulate: bool = False,
                   workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> GatedFfnGrad:
    """The gradients of x and of both weights, from dh and what gated_ffn kept.  dw_gate and dw_up may be float32 views of a
    gradient arena (accumulate: added to what is there); new ones are of x's type."""
    dev = torch.cuda.current_device()
    kind, weight_type, width, dim, gate_stride, up_stride = _gated_inputs(x, w_gate, w_up, activation, dev)
    lead = x.dim() - 1
    shape = (*x.shape[:-1], width)
    same = _SAME[x.dtype]
    for t, name in ((gate, "gate"), (up, "up"), (dh, "dh")):
        _need(t, name, same, dev)
        if t.shape != shape:
            _shape(t, shape, name)
    want_dx, want_dw = want_dx or dx is not None, want_dw or dw_gate is not None or dw_up is not None
    if (dw_gate is None) != (dw_up is None):
        raise ValueError("dw_gate and dw_up go together")
    if accumulate and dw_gate is None:
        raise ValueError("accumulate: need dw_gate and dw_up to add to")
    written = [t for t in (dx, dw_gate, dw_up) if t is not None]
    dx_strides, dx_at = (0, 0), 0
    if want_dx:
        if dx is None:
            dx = _new(x, x.shape, x.dtype, stream)
            dx_strides = _dense(x.shape)
        else:
            _need(dx, "dx", same, dev)
            _shape(dx, x.shape, "dx")
            dx_strides = _rows(dx, lead, "dx")
        dx_at = dx.data_ptr()
    dw_type, dg_stride, du_stride, dg_at, du_at = kind, 0, 0, 0, 0
    if want_dw:
        if dw_gate is None:
            dw_gate, dw_up = _new(x, (width, dim), x.dtype, stream), _new(x, (width, dim), x.dtype, stream)
            dg_stride = du_stride = dim
        else:
            dw_type = _need(dw_gate, "dw_gate", _OR_FLOAT32[x.dtype], dev)
            _need(dw_up, "dw_up", _SAME[dw_gate.dtype], dev)
            _shape(dw_gate, (width, dim), "dw_gate")
            _shape(dw_up, (width, dim), "dw_up")
            dg_stride, du_stride = _table(dw_gate, "dw_gate")[2], _table(dw_up, "dw_up")[2]
        dg_at, du_at = dw_gate.data_ptr(), dw_up.data_ptr()
    d = _GATED.pack(x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), dh.data_ptr(), gate.data_ptr(), up.data_ptr(), dx_at, dg_at, du_at,
                    kind, weight_type, dw_type, _ACTIVATIONS[activation], 1 if accumulate else 0, *_sizes(x.shape[:-1]), dim, width,
                    *_rows(x, lead, "x"), *_rows(dh, lead, "dh"), *_rows(gate, lead, "gate"), *_rows(up, lead, "up"), *dx_strides,
                    gate_stride, up_stride, dg_stride, du_stride)
    lib = binding.load_library()
    need = ctypes.c_size_t()
    _check(lib.odsgd_gated_workspace(d, 1, ctypes.byref(need)))
    workspace, ws_at, ws_bytes = _workspace(need.value, workspace, x, dev, stream)
    _check(lib.odsgd_gated_backward(d, ws_at, ws_bytes, _handle(stream, dev)))
    if written:
        increment_version(written)
    return GatedFfnGrad(dx, dw_gate, dw_up)


def stalled_waits() -> int:
    """How many waits inside the kernels of the gated block have given up on the current device since the library was loaded: what a
    program looks at where it waits for the GPU anyway (a checkpoint, a report).  Always 0, unless the GPU was kept from running a
    kernel for seconds: results since the last look are void then.  Waits for the device; not while a stream is being captured."""
    if torch.cuda.is_current_stream_capturing():
        raise RuntimeError("stalled_waits: the current stream is being captured")
    count = ctypes.c_uint()
    _check(binding.load_library().odsgd_stalled_waits(ctypes.byref(count)))
    return count.value


# --------------------------------------------------------------------------- dropout

def dropout(x: torch.Tensor, p: float, seed: int, *, offset: int = 0, counter: Optional[torch.Tensor] = None,
            residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
            stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """residual + dropout(x) in the residual's type (without one: x's), by a mask that follows from seed, offset, shape and p
    alone.  The gradient of x is dropout(grad, p, seed, offset=offset), that of the residual is grad.  `offset`: a number of the call
    (step, layer); `counter`: an int64 tensor of one element that is added to it on the device, for captured graphs."""
    dev = torch.cuda.current_device()
    kind = _need(x, "x", _FLOATS, dev)
    if x.dim() < 1:
        raise ValueError("x: need [..., dim]")
    lead = x.dim() - 1
    r_at, r_strides, dtype = 0, (0, 0), x.dtype
    if residual is not None:
        _need(residual, "residual", _FLOATS, dev)
        _shape(residual, x.shape, "residual")
        r_at, r_strides, dtype = residual.data_ptr(), _rows(residual, lead, "residual"), residual.dtype
    given = out is not None
    if not given:
        out = _new(x, None, dtype, stream)
    else:
        _shape(out, x.shape, "out")
    out_type = _need(out, "out", _FLOATS if residual is None else {dtype: _FLOATS[dtype]}, dev)
    c_at = 0
    if counter is not None:
        _need(counter, "counter", {torch.int64: I64}, dev)
        if counter.numel() != 1:
            raise ValueError("counter: need one element")
        c_at = counter.data_ptr()
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise ValueError("seed and offset must be in [0, 2^64)")
    if x.shape[-1] == 0:
        return out
    d = _DROPOUT.pack(x.data_ptr(), r_at, out.data_ptr(), c_at, kind, out_type, *_sizes(x.shape[:-1]), x.shape[-1],
                      *_rows(x, lead, "x"), *r_strides, *_rows(out, lead, "out"), seed, offset, p)
    _check(binding.load_library().odsgd_dropout(d, _handle(stream, dev)))
    if given:
        increment_version(out)
    return out


# --------------------------------------------------------------------------- drafted tokens

def verify_draft(target: torch.Tensor, draft_tokens: torch.Tensor, uniforms: torch.Tensor, *, draft: Optional[torch.Tensor] = None,
                 inv_temp: float = 1.0, draft_inv_temp: Optional[float] = None, workspace: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> Verified:
    """Drafts accepted against the target's probabilities, and one token more, drawn so that all are distributed as the target is.

    target [batch, drafts + 1, vocab] logits (the last row follows the last draft); draft_tokens [batch, drafts], -1 behind a
    shorter draft; draft [batch, drafts, vocab] the logits that they were drawn from, of the target's type, at draft_inv_temp (default:
    inv_temp), or None where they were not drawn; uniforms [batch, drafts + 1] float32 in [0, 1)."""
    dev = torch.cuda.current_device()
    kind = _need(target, "target", _FLOATS, dev)
    token_type = _need(draft_tokens, "draft_tokens", _INTS, dev)
    _need(uniforms, "uniforms", _FLOAT32, dev)
    if target.dim() != 3:
        raise ValueError("target: need [batch, drafts + 1, vocab]")
    batch, many, vocab = target.shape
    if many < 1:
        raise ValueError("target: need [batch, drafts + 1, vocab]")
    _shape(draft_tokens, (batch, many - 1), "draft_tokens")
    _shape(uniforms, (batch, many), "uniforms")
    at, strides = 0, (0, 0)
    if draft is not None:
        _need(draft, "draft", {target.dtype: kind}, dev)
        _shape(draft, (batch, many - 1, vocab), "draft")
        at, strides = draft.data_ptr(), _rows(draft, 2, "draft")
    accepted, tokens = _new(target, (batch,), torch.int32, stream), _new(target, (batch, many), draft_tokens.dtype, stream)
    logp = _new(target, (batch, many), torch.float32, stream)
    d = _VERIFY.pack(target.data_ptr(), at, draft_tokens.data_ptr(), uniforms.data_ptr(), tokens.data_ptr(), accepted.data_ptr(),
                     logp.data_ptr(), kind, token_type, batch, many - 1, vocab, *_rows(target, 2, "target"), *strides,
                     *_levels(draft_tokens, 2, "draft_tokens"), *_levels(uniforms, 2, "uniforms"), inv_temp,
                     inv_temp if draft_inv_temp is None else draft_inv_temp)
    lib = binding.load_library()
    need = ctypes.c_size_t()
    _check(lib.odsgd_verify_workspace(d, ctypes.byref(need)))
    workspace, ws_at, ws_bytes = _workspace(need.value, workspace, target, dev, stream)
    _check(lib.odsgd_verify_draft(d, ws_at, ws_bytes, _handle(stream, dev)))
    return Verified(accepted, tokens, logp)


# --------------------------------------------------------------------------- gradient norm and clip

class GradSet:
    """A checked list of gradient tensors, one group per worker, whose norms are taken and whose
    elements are scaled together (odsgd_grad_set_*).

    groups   one sequence of contiguous float32 / bfloat16 / float16 tensors per worker
    arenas   one float32 arena per worker that receives the scaled gradients, or None: the tensors
             are scaled in place
    offsets  with arenas: first element of each tensor (the same for every worker, or one list per
             worker)

    The set keeps its tensors alive; they must stay where they are, and calls of one set must not
    overlap on the GPU.  Its table is filled on `stream`: calls on other streams have to be ordered
    behind that.  Like a context it can be closed; it frees its table when dropped, so a graph that recorded its
    calls needs the set for as long as it is replayed.
    """

    def __init__(self, groups: Sequence[Sequence[torch.Tensor]], *, offsets: Optional[Sequence] = None,
                 arenas: Optional[Sequence[torch.Tensor]] = None, stream: Optional[torch.cuda.Stream] = None):
        self._h = ctypes.c_void_p()
        self._lib = binding.load_library()
        self.n_groups = len(groups)
        if self.n_groups == 0:
            raise ValueError("need at least one group of gradient tensors")
        if (arenas is None) != (offsets is None):
            raise ValueError("arenas and offsets go together")
        if arenas is not None:
            if len(arenas) != self.n_groups:
                raise ValueError(f"need {self.n_groups} arenas, got {len(arenas)}")
            if len({a.numel() for a in arenas}) != 1:
                raise ValueError("the arenas differ in length")
        self._keep = ([list(g) for g in groups], list(arenas) if arenas is not None else None)
        # what clip() writes besides the norms, of the views of one tensor (which share its version) one
        written = [t for g in self._keep[0] for t in g] if arenas is None else self._keep[1]
        self._written = list({id(t._base if t._is_view() else t): t for t in written}.values())
        self._dev = dev = torch.cuda.current_device()
        per_group = offsets is not None and len(offsets) > 0 and isinstance(offsets[0], (list, tuple))
        rows = []
        for g, tensors in enumerate(groups):
            offs = None
            if offsets is not None:
                offs = offsets[g] if per_group else offsets
                if len(offs) < len(tensors):
                    raise ValueError(f"group {g}: {len(tensors)} tensors, {len(offs)} offsets")
                if any(o < 0 for o in offs):
                    raise ValueError("negative offset")
            for k, t in enumerate(tensors):
                kind = _need(t, f"groups[{g}][{k}]", _FLOATS, dev)
                if not t.is_contiguous():
                    raise ValueError(f"groups[{g}][{k}]: need a contiguous tensor")
                rows.append(_GRAD_TENSOR.pack(t.data_ptr(), t.numel(), int(offs[k]) if offs is not None else 0, kind, g))
        atab, alen = None, 0
        if arenas is not None:
            for i, a in enumerate(arenas):
                _need(a, f"arenas[{i}]", _FLOAT32, dev)
            atab = binding._ptr_table([binding._dev_ptr(a, f"arenas[{i}]") for i, a in enumerate(arenas)])
            alen = arenas[0].numel()
        _check(self._lib.odsgd_grad_set_create(ctypes.byref(self._h), b"".join(rows), len(rows), self.n_groups, atab, alen,
                                               _handle(stream, dev)))

    def _out(self, out: Optional[torch.Tensor], stream) -> torch.Tensor:
        if not self._h:
            raise ValueError("the gradient set is closed")
        if out is None:
            with torch.cuda.stream(stream):
                return torch.empty(self.n_groups, dtype=torch.float32, device=torch.device("cuda", self._dev))
        _need(out, "out", _FLOAT32, self._dev)
        if out.numel() != self.n_groups or not out.is_contiguous():
            raise ValueError(f"out: need {self.n_groups} contiguous elements")
        return out

    def norm(self, *, out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """The 2-norm of each group over all its tensors (float32); nothing else is written."""
        out = self._out(out, stream)
        _check(self._lib.odsgd_grad_set_norm(self._h, out.data_ptr(), _handle(stream, self._dev)))
        increment_version(out)
        return out

    def clip(self, max_norm: float, *, out: Optional[torch.Tensor] = None,
             stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """Scales each group by min(1, max_norm / norm), into its arena or in place; returns the
        norms of before."""
        out = self._out(out, stream)
        _check(self._lib.odsgd_grad_set_clip(self._h, max_norm, out.data_ptr(), _handle(stream, self._dev)))
        increment_version([*self._written, out])
        return out

    def close(self) -> None:
        if self._h:
            self._lib.odsgd_grad_set_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
