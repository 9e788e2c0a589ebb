"""Language-model operators around the update: argument marshalling for the odsgd_embed_*,
odsgd_token_logprob, odsgd_policy_loss and odsgd_grad_set_* calls of libodsgd.so.

What a worker runs on either side of its model when the parameter set is a language model's:

* `embed_lookup` / `embed_grad`: token rows out of the weight arena, and their gradient into the
  gradient arena (`arena[a:b].view(vocab, dim)` is a table);
* `token_logprob`: the score of each taken token (acting policy, reference policy, evaluation);
* `policy_loss`: the clipped policy loss with a KL term, and its gradient, in one pass;
* `GradSet`: norm and clipping of a list of gradient tensors, laid out into the arenas the server
  reads.

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

# odsgd_embed_desc, odsgd_policy_desc and odsgd_grad_tensor of include/odsgd.h, packed by struct: a call is
# a few microseconds, and filling a ctypes structure would be one of them.
_EMBED = struct.Struct("3P4i10qf4x")
_POLICY = struct.Struct("10P2i17q5f4x")
_GRAD_TENSOR = struct.Struct("PNN2i")


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
    if t.stride(-1) != 1 and t.shape[-1] != 1:
        raise ValueError(f"{name}: the last axis must be contiguous")
    return _levels(t, lead, name)


def _new(like: torch.Tensor, shape, dtype, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    """Contiguous memory of the stream that the work runs on; `shape` None: like's."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return _new(like, shape, dtype, None)
    if shape is None:
        return torch.empty_like(like, dtype=dtype, memory_format=torch.contiguous_format)
    return like.new_empty(shape, dtype=dtype)


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
