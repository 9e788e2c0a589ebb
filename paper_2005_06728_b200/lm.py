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
new tensors unless a buffer is given.  Tensors may be strided in their leading axes (a shifted
view, an expanded value) as long as the last axis is contiguous and the leading ones fold into two
levels.  There is no CPU fallback and no autograd: the gradient calls are the backward pass.
"""
from __future__ import annotations

import ctypes
from typing import List, NamedTuple, Optional, Sequence, Tuple

import torch

from . import binding
from .binding import OK, OdsgdError

F32, BF16, F16, I32, I64 = 0, 1, 2, 3, 4
MAX_TOKENS = 1 << 24

_TYPE = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16, torch.int32: I32, torch.int64: I64}
_FLOATS = (torch.float32, torch.bfloat16, torch.float16)
_INTS = (torch.int32, torch.int64)

_vp, _ci, _i64, _cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float


class _EmbedDesc(ctypes.Structure):
    _fields_ = [
        ("tokens", _vp), ("act", _vp), ("table", _vp),
        ("token_type", _ci), ("act_type", _ci), ("table_type", _ci), ("accumulate", _ci),
        ("n_outer", _i64), ("n_inner", _i64),
        ("token_stride_outer", _i64), ("token_stride_inner", _i64),
        ("act_stride_outer", _i64), ("act_stride_inner", _i64),
        ("vocab", _i64), ("dim", _i64), ("table_stride", _i64), ("padding_token", _i64),
        ("scale", _cf),
    ]


class _PolicyDesc(ctypes.Structure):
    _fields_ = [
        ("logits", _vp), ("labels", _vp), ("old_logp", _vp), ("ref_logp", _vp), ("advantages", _vp), ("weights", _vp),
        ("dlogits", _vp), ("logp", _vp), ("lse", _vp), ("stats", _vp),
        ("type", _ci), ("label_type", _ci),
        ("n_outer", _i64), ("n_inner", _i64), ("vocab", _i64),
        ("logits_stride_outer", _i64), ("logits_stride_inner", _i64),
        ("label_stride_outer", _i64), ("label_stride_inner", _i64),
        ("old_stride_outer", _i64), ("old_stride_inner", _i64),
        ("ref_stride_outer", _i64), ("ref_stride_inner", _i64),
        ("adv_stride_outer", _i64), ("adv_stride_inner", _i64),
        ("weight_stride_outer", _i64), ("weight_stride_inner", _i64),
        ("dlogits_stride_outer", _i64), ("dlogits_stride_inner", _i64),
        ("inv_temp", _cf), ("clip_low", _cf), ("clip_high", _cf), ("kl_coef", _cf), ("grad_scale", _cf),
    ]


class _GradTensor(ctypes.Structure):
    _fields_ = [("data", _vp), ("numel", ctypes.c_size_t), ("offset", ctypes.c_size_t), ("type", _ci), ("group", _ci)]


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


def _need(t: torch.Tensor, name: str, dtypes) -> None:
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in dtypes:
        raise TypeError(f"{name}: need a CUDA tensor of {' / '.join(str(d) for d in dtypes)}")


def _on_device(*tensors: Optional[torch.Tensor]) -> None:
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{dev}")


def _levels(t: torch.Tensor, lead: int, name: str) -> Tuple[int, int, int, int]:
    """(n_outer, n_inner, stride_outer, stride_inner) of the first `lead` axes."""
    if lead == 2:
        s, st = t.shape, t.stride()
        return s[0], s[1], st[0], st[1]
    if lead == 1:
        return 1, t.shape[0], 0, t.stride(0)
    if lead == 0:
        return 1, 1, 0, 0
    shape, stride = list(t.shape[:lead]), list(t.stride()[:lead])
    outer, step = 1, 0  # all but the last leading axis fold into one level
    for n, s in reversed(list(zip(shape[:-1], stride[:-1]))):
        if n == 1:
            continue
        if outer == 1:
            step = s
        elif s != outer * step:
            raise ValueError(f"{name}: its leading axes do not fold into two strided levels (make it contiguous)")
        outer *= n
    return outer, shape[-1], step, stride[-1]


def _last_contiguous(t: torch.Tensor, name: str) -> None:
    if t.dim() == 0 or (t.stride(-1) != 1 and t.shape[-1] != 1):
        raise ValueError(f"{name}: the last axis must be contiguous")


def _same_shape(t: torch.Tensor, shape, name: str) -> None:
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")


def _empty(shape, dtype, device, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    """Memory of the stream that the work runs on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _table(table: torch.Tensor, name: str) -> Tuple[int, int, int]:
    if table.dim() != 2:
        raise ValueError(f"{name}: need [vocab, dim]")
    _last_contiguous(table, name)
    vocab, dim = table.shape
    return vocab, dim, table.stride(0) if vocab > 1 else max(dim, table.stride(0))


# --------------------------------------------------------------------------- embedding

def embed_lookup(tokens: torch.Tensor, table: torch.Tensor, *, scale: float = 1.0, dtype: Optional[torch.dtype] = None,
                 out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """scale * table[tokens], rounded once to `dtype` (default: the table's).  A token outside
    [0, vocab), such as the -1 that pads a ragged batch, gives a row of zeros."""
    _need(tokens, "tokens", _INTS)
    _need(table, "table", _FLOATS)
    vocab, dim, stride = _table(table, "table")
    lead = tokens.dim()
    if out is None:
        out = _empty((*tokens.shape, dim), table.dtype if dtype is None else dtype, tokens.device, stream)
    elif dtype is not None and out.dtype != dtype:
        raise ValueError("out and dtype disagree")
    _need(out, "out", _FLOATS)
    _same_shape(out, torch.Size((*tokens.shape, dim)), "out")
    _last_contiguous(out, "out")
    _on_device(tokens, table, out)
    no, ni, tso, tsi = _levels(tokens, lead, "tokens")
    _, _, aso, asi = _levels(out, lead, "out")
    d = _EmbedDesc(tokens.data_ptr(), out.data_ptr(), table.data_ptr(), _TYPE[tokens.dtype], _TYPE[out.dtype],
                   _TYPE[table.dtype], 0, no, ni, tso, tsi, aso, asi, vocab, dim, stride, -1, scale)
    _check(binding.load_library().odsgd_embed_lookup(ctypes.addressof(d), binding._stream_handle(stream)))
    return out


def embed_grad(tokens: torch.Tensor, grad: torch.Tensor, dtable: torch.Tensor, *, scale: float = 1.0,
               padding_token: Optional[int] = None, accumulate: bool = False, workspace: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """dtable[v] = scale * sum of grad over the positions of token v, zeros where there is none
    (accumulate: added to what is there).  `dtable` is float32, normally a view of the worker's
    gradient arena.  Tokens outside [0, vocab) and `padding_token` contribute nothing."""
    _need(tokens, "tokens", _INTS)
    _need(grad, "grad", _FLOATS)
    _need(dtable, "dtable", (torch.float32,))
    vocab, dim, stride = _table(dtable, "dtable")
    _same_shape(grad, torch.Size((*tokens.shape, dim)), "grad")
    _last_contiguous(grad, "grad")
    _on_device(tokens, grad, dtable, workspace)
    lead = tokens.dim()
    no, ni, tso, tsi = _levels(tokens, lead, "tokens")
    _, _, aso, asi = _levels(grad, lead, "grad")
    d = _EmbedDesc(tokens.data_ptr(), grad.data_ptr(), dtable.data_ptr(), _TYPE[tokens.dtype], _TYPE[grad.dtype], F32,
                   1 if accumulate else 0, no, ni, tso, tsi, aso, asi, vocab, dim, stride,
                   -1 if padding_token is None else padding_token, scale)
    lib = binding.load_library()
    if workspace is None:
        need = ctypes.c_size_t()
        _check(lib.odsgd_embed_grad_workspace(ctypes.addressof(d), ctypes.byref(need)))
        workspace = _empty((max(16, need.value),), torch.uint8, tokens.device, stream)
    _check(lib.odsgd_embed_grad(ctypes.addressof(d), workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                binding._stream_handle(stream)))
    return dtable


def embed_grad_workspace(tokens: torch.Tensor, grad: torch.Tensor, dtable: torch.Tensor) -> int:
    """Bytes of workspace that embed_grad needs for tensors of these shapes and types."""
    no, ni, _, _ = _levels(tokens, tokens.dim(), "tokens")
    d = _EmbedDesc(None, None, None, _TYPE[tokens.dtype], _TYPE[grad.dtype], F32, 0, no, ni, 0, 0, 0, 0,
                   dtable.shape[0], dtable.shape[1], dtable.shape[1], -1, 1.0)
    need = ctypes.c_size_t()
    _check(binding.load_library().odsgd_embed_grad_workspace(ctypes.addressof(d), ctypes.byref(need)))
    return need.value


# --------------------------------------------------------------------------- scores and policy loss

def token_logprob(logits: torch.Tensor, labels: torch.Tensor, *, inv_temp: float = 1.0,
                  stream: Optional[torch.cuda.Stream] = None) -> TokenLogprob:
    """log softmax(inv_temp * logits)[label] and the row's log of summed exponentials, in float32;
    zeros where the label is outside [0, vocab)."""
    _need(logits, "logits", _FLOATS)
    _need(labels, "labels", _INTS)
    _last_contiguous(logits, "logits")
    _same_shape(labels, logits.shape[:-1], "labels")
    _on_device(logits, labels)
    lead = labels.dim()
    no, ni, zso, zsi = _levels(logits, lead, "logits")
    _, _, lso, lsi = _levels(labels, lead, "labels")
    both = _empty((2, *labels.shape), torch.float32, logits.device, stream)
    logp, lse = both.unbind(0)
    d = _PolicyDesc(logits.data_ptr(), labels.data_ptr(), None, None, None, None, None, logp.data_ptr(), lse.data_ptr(),
                    None, _TYPE[logits.dtype], _TYPE[labels.dtype], no, ni, logits.shape[-1], zso, zsi, lso, lsi)
    d.inv_temp = inv_temp
    _check(binding.load_library().odsgd_token_logprob(ctypes.addressof(d), binding._stream_handle(stream)))
    return TokenLogprob(logp, lse)


def policy_loss(logits: torch.Tensor, labels: torch.Tensor, old_logp: torch.Tensor, advantages: torch.Tensor,
                weights: torch.Tensor, *, ref_logp: Optional[torch.Tensor] = None, clip_low: float = 0.2,
                clip_high: float = 0.2, kl_coef: float = 0.0, inv_temp: float = 1.0, grad_scale: float = 1.0,
                dlogits: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> PolicyLoss:
    """The clipped policy loss with a KL term, and its gradient, over rows of logits.

    `old_logp`, `ref_logp`, `advantages` and `weights` are float32 of the labels' shape (expanded
    views welcome); a weight is mask and normalisation in one.  `dlogits` may be `logits` itself.
    """
    _need(logits, "logits", _FLOATS)
    _need(labels, "labels", _INTS)
    _last_contiguous(logits, "logits")
    shape = logits.shape[:-1]
    _same_shape(labels, shape, "labels")
    lead = len(shape)
    vectors = (old_logp, ref_logp, advantages, weights)
    strides: List[int] = []
    for t, name in zip(vectors, ("old_logp", "ref_logp", "advantages", "weights")):
        if t is None:
            strides += (0, 0)
            continue
        _need(t, name, (torch.float32,))
        _same_shape(t, shape, name)
        strides += _levels(t, lead, name)[2:]
    if dlogits is None:
        dlogits = _empty(logits.shape, logits.dtype, logits.device, stream)
    else:
        _need(dlogits, "dlogits", (logits.dtype,))
        _same_shape(dlogits, logits.shape, "dlogits")
        _last_contiguous(dlogits, "dlogits")
    _on_device(logits, labels, *vectors, dlogits)
    no, ni, zso, zsi = _levels(logits, lead, "logits")
    _, _, lso, lsi = _levels(labels, lead, "labels")
    _, _, dso, dsi = _levels(dlogits, lead, "dlogits")
    # one allocation: the four sums, then the rows' scores; and the workspace (12 bytes a row)
    n = no * ni
    out = _empty((4 + n,), torch.float32, logits.device, stream)
    stats, logp = out[:4], out[4:].view(shape)
    work = _empty((max(4, 3 * n),), torch.float32, logits.device, stream)
    d = _PolicyDesc(logits.data_ptr(), labels.data_ptr(), old_logp.data_ptr(),
                    None if ref_logp is None else ref_logp.data_ptr(), advantages.data_ptr(), weights.data_ptr(),
                    dlogits.data_ptr(), logp.data_ptr(), None, stats.data_ptr(), _TYPE[logits.dtype],
                    _TYPE[labels.dtype], no, ni, logits.shape[-1], zso, zsi, lso, lsi, *strides, dso, dsi,
                    inv_temp, clip_low, clip_high, kl_coef, grad_scale)
    _check(binding.load_library().odsgd_policy_loss(ctypes.addressof(d), work.data_ptr(), 4 * work.numel(),
                                                    binding._stream_handle(stream)))
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
    overlap on the GPU.  Like a context it can be closed; it frees its table when dropped.
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
        per_group = offsets is not None and len(offsets) > 0 and isinstance(offsets[0], (list, tuple))
        rows = []
        for g, tensors in enumerate(groups):
            offs = None
            if offsets is not None:
                offs = offsets[g] if per_group else offsets
                if len(offs) < len(tensors):
                    raise ValueError(f"group {g}: {len(tensors)} tensors, {len(offs)} offsets")
            for k, t in enumerate(tensors):
                _need(t, f"groups[{g}][{k}]", _FLOATS)
                if not t.is_contiguous():
                    raise ValueError(f"groups[{g}][{k}]: need a contiguous tensor")
                _on_device(t)
                rows.append((t.data_ptr(), t.numel(), int(offs[k]) if offs is not None else 0, _TYPE[t.dtype], g))
        if any(r[2] < 0 for r in rows):
            raise ValueError("negative offset")
        tab = (_GradTensor * max(1, len(rows)))(*[_GradTensor(*r) for r in rows])
        atab, alen = None, 0
        if arenas is not None:
            atab = binding._ptr_table([binding._dev_ptr(a, f"arenas[{i}]") for i, a in enumerate(arenas)])
            _on_device(*arenas)
            alen = arenas[0].numel()
        self._device = torch.device("cuda", torch.cuda.current_device())
        _check(self._lib.odsgd_grad_set_create(ctypes.byref(self._h), ctypes.addressof(tab), len(rows), self.n_groups, atab, alen,
                                               binding._stream_handle(stream)))

    def _out(self, out: Optional[torch.Tensor], stream) -> torch.Tensor:
        if not self._h:
            raise ValueError("the gradient set is closed")
        if out is None:
            return _empty((self.n_groups,), torch.float32, self._device, stream)
        binding._dev_ptr(out, "out", self.n_groups)
        return out

    def norm(self, *, out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """The 2-norm of each group over all its tensors (float32); nothing else is written."""
        out = self._out(out, stream)
        _check(self._lib.odsgd_grad_set_norm(self._h, out.data_ptr(), binding._stream_handle(stream)))
        return out

    def clip(self, max_norm: float, *, out: Optional[torch.Tensor] = None,
             stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """Scales each group by min(1, max_norm / norm), into its arena or in place; returns the
        norms of before."""
        out = self._out(out, stream)
        _check(self._lib.odsgd_grad_set_clip(self._h, max_norm, out.data_ptr(), binding._stream_handle(stream)))
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
