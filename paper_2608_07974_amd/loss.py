"""Losses over a vocabulary on torch device tensors (include/zl_loss.h).

A teacher's top logits (top_logits); the loss of logits in memory against labels,
such a teacher, or both, and its gradient (logit_loss, logit_loss_bwd); the same
loss of a readout head's logits x w^T, which are never kept, with the gradients
of x and w (head_loss, head_loss_bwd).  torch provides memory and streams; the
kernels are libzl's.

Rows are tokens: every loss is [T] fp32, 0 for a row without label and teacher,
and the backward takes the rows' weights (dloss; 1 / count for a mean).  Logits
are bf16 or fp32 [T, V], rows contiguous, any row stride and alignment; x and w
are bf16 or fp32 [T, d] and [V, d], row strides a multiple of 8.  All tensors are
on one GPU; work goes to its current stream.  Shapes, types and placement are
checked here (the kernels take them on trust), the rest by the library, which
raises zl.ZlError.  As with the layer operators (layer.py), outputs may be given,
autograd does not record these calls and refuses inputs that would be cut off its
graph, and tensors that a call writes count as changed in place.
"""
from collections import namedtuple

import torch

from . import zl
from .layer import _DT, _call, _check_device, _no_graph, _ptr, _rows, _wrote

TopLogits = namedtuple("TopLogits", "ids values rest", defaults=(None,))
TopLogits.__doc__ = """A teacher's top logits per row: ids int32 [T, k], values fp32 [T, k], rest fp32 [T]
(log of the sum of exp(logit / temperature) over the other columns) or None.  An id outside the
vocabulary, or one named before in its row, is absent; a row without ids has no teacher."""


def _logits(name, t):
    """(T, V, row stride) of a matrix of logits."""
    if t.dim() != 2 or t.dtype not in _DT:
        raise TypeError(f"{name} must be a bf16 or fp32 matrix")
    T, V = t.shape
    if t.requires_grad:
        _no_graph(name)
    s0, s1 = t.stride()
    if V > 1 and s1 != 1:
        raise ValueError(f"{name} must have contiguous rows")
    if T > 1 and s0 < V:
        raise ValueError(f"{name} must not overlap itself")
    return T, V, s0 if T > 1 else V


def _dense(name, t, shape, dtype):
    """Address of a contiguous tensor of that shape and type, or 0."""
    if t is None:
        return 0
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {list(shape)}")
    if t.requires_grad:
        _no_graph(name)
    return t.data_ptr()


def _targets(T, labels, teacher, alpha, temperature):
    """The targets as the library takes them, and their tensors."""
    ids, values, rest = teacher if teacher is not None else (None, None, None)
    if labels is None and ids is None:
        raise ValueError("labels, a teacher or both must be there")
    k = 0
    if ids is not None:
        if ids.dim() != 2 or values is None:
            raise ValueError(f"a teacher has ids and values [{T}, k]")
        k = ids.shape[1]
    fields = (_dense("labels", labels, (T,), torch.int32), _dense("ids", ids, (T, k), torch.int32),
              _dense("values", values, (T, k), torch.float32), _dense("rest", rest, (T,), torch.float32),
              k if k < 1 << 31 else 0x7fffffff, alpha, temperature)
    return fields, (labels, ids, values, rest)


_TARGETS = " labels ids values rest"


def top_logits(logits, k, *, temperature=1.0, rest=True, out=None):
    """The k largest of every row as TopLogits, in descending order, equal ones by
    column; with their rest at that temperature, which is None with rest=False.
    out: a TopLogits of tensors that receive them (its rest decides then)."""
    T, V, ld = _logits("logits", logits)
    dev = logits.device
    if out is None:
        out = TopLogits(torch.empty(T, k, dtype=torch.int32, device=dev), torch.empty(T, k, dtype=torch.float32, device=dev),
                        torch.empty(T, dtype=torch.float32, device=dev) if rest else None)
    ids, values, r = out
    pi, pv = _dense("ids", ids, (T, k), torch.int32), _dense("values", values, (T, k), torch.float32)
    pr = _dense("rest", r, (T,), torch.float32)
    _check_device(dev, "ids values rest", ids, values, r)
    _call(zl.zl_top_logits, dev, T, V, logits.data_ptr(), ld, _DT[logits.dtype], k, temperature, pi, pv, pr)
    _wrote((ids, values) if r is None else (ids, values, r))
    return out


def logit_loss(logits, labels=None, teacher=None, *, alpha=0.5, temperature=1.0, loss=None, stats=None):
    """alpha CE(labels) + (1 - alpha) temperature^2 KL(teacher || softmax(logits / temperature)) of
    every row; one of them alone has weight 1.  labels: int32 [T] (not int64), outside [0, V): none; teacher: a
    TopLogits.  Returns (loss [T], stats [T, 4]); the backward takes stats."""
    T, V, ld = _logits("logits", logits)
    dev = logits.device
    fields, held = _targets(T, labels, teacher, alpha, temperature)
    loss = torch.empty(T, dtype=torch.float32, device=dev) if loss is None else loss
    stats = torch.empty(T, 4, dtype=torch.float32, device=dev) if stats is None else stats
    pl, ps = _dense("loss", loss, (T,), torch.float32), _dense("stats", stats, (T, 4), torch.float32)
    _check_device(dev, "loss stats" + _TARGETS, loss, stats, *held)
    _call(zl.zl_logit_loss, dev, T, V, logits.data_ptr(), ld, _DT[logits.dtype], zl.pack_targets(*fields), pl, ps)
    _wrote((loss, stats))
    return loss, stats


def logit_loss_bwd(logits, stats, labels=None, teacher=None, *, alpha=0.5, temperature=1.0, dloss=None, scale=1.0,
                   out=None):
    """Gradient of scale * sum(dloss * loss) with respect to the logits (dloss [T], None: ones), of
    their type.  out may be logits; rows that start at another place in 16 bytes than those of logits
    take longer."""
    T, V, ld = _logits("logits", logits)
    dev = logits.device
    fields, held = _targets(T, labels, teacher, alpha, temperature)
    out = torch.empty(T, V, dtype=logits.dtype, device=dev) if out is None else out
    To, Vo, ldo = _logits("out", out)
    if (To, Vo) != (T, V) or out.dtype != logits.dtype:
        raise ValueError(f"out must be {logits.dtype} of {[T, V]}, not {out.dtype} of {[To, Vo]}")
    ps, pd = _dense("stats", stats, (T, 4), torch.float32), _dense("dloss", dloss, (T,), torch.float32)
    _check_device(dev, "stats dloss out" + _TARGETS, stats, dloss, out, *held)
    _call(zl.zl_logit_loss_backward, dev, T, V, logits.data_ptr(), ld, _DT[logits.dtype], zl.pack_targets(*fields), ps, pd,
          scale, out.data_ptr(), ldo)
    _wrote((out,))
    return out


def _head(x, w):
    """(T, V, d, row strides) of x [T, d] and w [V, d]."""
    if x.dim() != 2 or w.dim() != 2 or x.dtype not in _DT:
        raise TypeError("x and w must be bf16 or fp32 matrices")
    (T, d), V = x.shape, w.shape[0]
    if w.requires_grad and w.is_leaf:  # a parameter, whose gradient the backward gives
        w = w.detach()
    return T, V, d, _rows("x", x, T, d, _DT), _rows("w", w, V, d, (x.dtype,))


def head_workspace(x, w, *, k=0, rest=True, backward=False, need_dx=True, need_dw=False, columns=0):
    """Scratch memory for head_loss or (backward) head_loss_bwd of such x and w: may be used again by
    any call of those sizes that is ordered after the last one.  k: ids per row; rest: whether the
    teacher has one; columns: as in head_loss_bwd."""
    n = zl.zl_head_loss_workspace(x.shape[0], w.shape[0], x.shape[1], _DT[x.dtype], k, rest and k > 0, backward, need_dx,
                                  need_dw, columns)
    return torch.empty(max(n, 1), dtype=torch.uint8, device=x.device)


def _scratch(workspace):
    if workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous uint8 tensor")
    return workspace.data_ptr(), workspace.numel()


def head_loss(x, w, labels=None, teacher=None, *, alpha=0.5, temperature=1.0, loss=None, stats=None, workspace=None):
    """logit_loss of the logits x w^T, which are not kept: x [T, d], w [V, d].  Returns (loss [T],
    stats [T, 4 + k]).  workspace: see head_workspace; made here if None."""
    T, V, d, ldx, ldw = _head(x, w)
    dev = x.device
    fields, held = _targets(T, labels, teacher, alpha, temperature)
    k = fields[4]
    loss = torch.empty(T, dtype=torch.float32, device=dev) if loss is None else loss
    stats = torch.empty(T, 4 + k, dtype=torch.float32, device=dev) if stats is None else stats
    pl, ps = _dense("loss", loss, (T,), torch.float32), _dense("stats", stats, (T, 4 + k), torch.float32)
    if workspace is None:
        workspace = head_workspace(x, w, k=k, rest=held[3] is not None)
    _check_device(dev, "w loss stats workspace" + _TARGETS, w, loss, stats, workspace, *held)
    _call(zl.zl_head_loss, dev,
          zl.pack_head_args(T, V, d, _DT[x.dtype], x.data_ptr(), ldx, w.data_ptr(), ldw, *fields, ps, pl, 0, 0.0, 0, 0, 0, 0,
                            0, 0, 0, 0, *_scratch(workspace)))
    _wrote((loss, stats, workspace))
    return loss, stats


def head_loss_bwd(x, w, stats, labels=None, teacher=None, *, alpha=0.5, temperature=1.0, dloss=None, scale=1.0, dx=None,
                  dw=None, need_dx=True, need_dw=False, accumulate=False, columns=0, workspace=None):
    """Gradients (dx, dw) of scale * sum(dloss * loss) (dloss [T], None: ones).

    dx [T, d] and dw [V, d], bf16 or fp32, are made in x's type where they are needed and not given
    (None otherwise; a dw that is given is needed); accumulate adds dw to what is there (fp32).
    columns: of the vocabulary in one piece, 0: as many as 1 GiB of dL/dlogits holds."""
    T, V, d, ldx, ldw = _head(x, w)
    dev = x.device
    fields, held = _targets(T, labels, teacher, alpha, temperature)
    k = fields[4]
    ps, pd = _dense("stats", stats, (T, 4 + k), torch.float32), _dense("dloss", dloss, (T,), torch.float32)
    if dx is None and need_dx:
        dx = torch.empty(T, d, dtype=x.dtype, device=dev)
    if dw is None and need_dw:
        dw = (torch.zeros if accumulate else torch.empty)(V, d, dtype=x.dtype, device=dev)
    lddx = tdx = lddw = tdw = 0
    if dx is not None:
        lddx, tdx = _rows("dx", dx, T, d, _DT), _DT[dx.dtype]
    if dw is not None:
        lddw, tdw = _rows("dw", dw, V, d, _DT), _DT[dw.dtype]
    if workspace is None:
        workspace = head_workspace(x, w, k=k, rest=held[3] is not None, backward=True, need_dx=dx is not None,
                                   need_dw=dw is not None, columns=columns)
    _check_device(dev, "w stats dloss dx dw workspace" + _TARGETS, w, stats, dloss, dx, dw, workspace, *held)
    _call(zl.zl_head_loss_backward, dev,
          zl.pack_head_args(T, V, d, _DT[x.dtype], x.data_ptr(), ldx, w.data_ptr(), ldw, *fields, ps, 0, pd, scale, columns,
                            _ptr(dx), lddx, tdx, _ptr(dw), lddw, tdw, accumulate, *_scratch(workspace)))
    _wrote([t for t in (dx, dw, workspace) if t is not None])
    return dx, dw
