"""Layer operators on torch device tensors (include/zl_layer.h).

Activations saved in 8 bits (pack, unpack) and their use in the backward
(mlp_act, mlp_act_bwd, wgrad), the norms around a block with gate and residual
scale (block_norm, block_norm_bwd), rotary positions with several axes
(rotary).  torch provides memory and streams; the kernels are libzl's.

Tensors are 2-D [T, columns], rows contiguous (any row stride that is a
multiple of 8), bf16 or fp32, all on one GPU; work goes to that GPU's current
stream.  Shapes, types and placement are checked here (the kernels take them
on trust), the rest by the library, which raises zl.ZlError.  Output tensors
may be given (and are returned); else they are made.  autograd does not record
these calls: a layer calls the backward functions itself.  So in gradient mode a
matrix that requires a gradient is refused, as are weights, biases and gates that
autograd computed (as parameters they may require one); tensors that a call
writes count as changed in place.
"""
from collections import namedtuple

import torch

from . import zl

_DT = {torch.float32: zl.ZL_F32, torch.bfloat16: zl.ZL_BF16}
_KIND = {"swiglu": zl.ZL_MLP_SWIGLU, "gelu": zl.ZL_MLP_GELU}
_NONE = (0, 0, 0, 0)  # no packed matrix
_NO_WB = (None, None)  # no weight and bias
_F32, _U8 = (torch.float32,), torch.uint8


def _up(n, m):
    return (n + m - 1) // m * m


def _ptr(t):
    return 0 if t is None else t.data_ptr()


# The host's share of a small call is most of it: the checks of this file are
# written for the case that passes.
def _check_device(dev, names, *tensors):
    """Every tensor, Packed or None is on the GPU dev; names: theirs, in one text."""
    if dev.type != "cuda":
        raise ValueError(f"tensors must be on a GPU, not {dev}")
    index = dev.index
    for i, t in enumerate(tensors):
        if t is None:
            continue
        if isinstance(t, Packed):
            if t.scales.get_device() != index:
                raise ValueError(f"{names.split()[i]}.scales must be on {dev}, not {t.scales.device}")
            t = t.codes
        if t.get_device() != index:  # (-1 off the GPUs)
            raise ValueError(f"{names.split()[i]} must be on {dev}, not {t.device}")


def _no_graph(name):
    if torch.is_grad_enabled():
        raise ValueError(f"{name} must not require a gradient: autograd does not record this call (use torch.no_grad(), "
                         "an autograd.Function, or detach())")


# Says of tensors (a list or tuple) that a call wrote them, as torch's in-place
# functions do: a graph that saved one of them refuses its backward.
_wrote = getattr(torch._C, "_increment_version", torch.autograd.graph.increment_version)


def _rows(name, t, T, n, dtypes):
    """Row stride of a [T, n] matrix with contiguous rows."""
    if t.requires_grad:
        _no_graph(name)
    if t.dtype in dtypes and t.shape == (T, n):
        s0, s1 = t.stride()
        if s1 == 1 and s0 >= n and T > 1:
            return s0
        if n > 1 and s1 != 1:
            raise ValueError(f"{name} must have contiguous rows")
        if T > 1:
            raise ValueError(f"{name} must not overlap itself")
        return _up(n, 8)
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, not {t.dtype}")
    raise ValueError(f"{name} must be [{T}, {n}], not {list(t.shape)}")


def _vec(name, t, n):
    if t is None:
        return 0
    if t.dtype != torch.float32 or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous fp32 vector of {n}")
    if t.requires_grad and not t.is_leaf:
        _no_graph(name)
    return t.data_ptr()


# torch's own accessor of the current stream's handle, without a Stream object
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)
_one_gpu = None  # whether this process sees one GPU only


def _call(fn, dev, *args):
    """fn(*args, stream) on dev's current stream, with dev current."""
    global _one_gpu
    if _one_gpu is None:
        _one_gpu = torch.cuda.device_count() == 1
    if _one_gpu or torch.cuda.current_device() == dev.index:
        fn(*args, _raw_stream(dev.index))
    else:
        with torch.cuda.device(dev):
            fn(*args, _raw_stream(dev.index))


def _packed_rows(codes, scales, n):
    """Rows of a packed matrix and the row strides of its tensors, whose types, shapes
    and strides are checked."""
    c, s, c16, c32 = codes.shape, scales.shape, n + 15 & -16, n + 31 >> 5
    if codes.dtype is not _U8 or scales.dtype is not _U8 or len(c) != 2 or len(s) != 2:
        raise TypeError("codes and scales must be uint8 matrices")
    (T, W), (Ts, Ws) = c, s
    if W < c16 or Ts != T or Ws < c32:
        raise ValueError(f"codes and scales must be [{T}, >= {c16}] and [{T}, >= {c32}], not [{T}, {W}] and [{Ts}, {Ws}]")
    if codes.is_contiguous() and scales.is_contiguous():
        return (T, W, Ws) if T > 1 else (T, c16, c32)
    (lc, c1), (ls, s1) = codes.stride(), scales.stride()
    if (c1 != 1 and W > 1) or (s1 != 1 and Ws > 1):
        raise ValueError("codes and scales must have contiguous rows")
    if T > 1 and (lc < c16 or ls < c32):
        raise ValueError("codes and scales must not overlap themselves")
    return (T, lc, ls) if T > 1 else (T, c16, c32)


class Packed:
    """A matrix [T, n] in 8 bits: `codes` uint8 [T, >= n rounded up to 16] and
    `scales` uint8 [T, >= ceil(n / 32)], both with contiguous rows.  Every call takes
    the two tensors as they are then."""

    __slots__ = ("codes", "scales", "n")

    def __init__(self, codes, scales, n):
        self.codes, self.scales, self.n = codes, scales, n
        _packed_rows(codes, scales, n)
        if codes.get_device() != scales.get_device():
            raise ValueError(f"codes on {codes.device}, scales on {scales.device}")

    def fields(self):
        """The matrix as the library takes it: pointers and row strides."""
        codes, scales = self.codes, self.scales
        if codes.device != scales.device:
            raise ValueError(f"codes on {codes.device}, scales on {scales.device}")
        return (codes.data_ptr(), scales.data_ptr()) + _packed_rows(codes, scales, self.n)[1:]

    @classmethod
    def empty(cls, T, n, device="cuda"):
        return cls(torch.empty(T, _up(n, 16), dtype=torch.uint8, device=device),
                   torch.empty(T, (n + 31) // 32, dtype=torch.uint8, device=device), n)

    @property
    def shape(self):
        return (self.codes.shape[0], self.n)

    @property
    def device(self):
        return self.codes.device

    def nbytes(self):
        return self.codes.numel() + self.scales.numel()


def _packed(name, p, T, n):
    if p is None:
        return _NONE
    if p.n == n:
        codes, scales = p.codes, p.scales
        rows, lc, ls = _packed_rows(codes, scales, n)
        if rows == T:
            return codes.data_ptr(), scales.data_ptr(), lc, ls
    raise ValueError(f"{name} must be [{T}, {n}], not {list(p.shape)}")


def pack(x, out=None):
    """x in 8 bits."""
    T, n = x.shape
    dev = x.device
    ldx = _rows("x", x, T, n, _DT)
    out = Packed.empty(T, n, dev) if out is None else out
    p = zl.pack_packed(*_packed("out", out, T, n))
    _check_device(dev, "out", out)
    _call(zl.zl_pack, dev, T, n, x.data_ptr(), ldx, _DT[x.dtype], p)
    _wrote((out.codes, out.scales))
    return out


def unpack(p, dtype=torch.bfloat16, out=None):
    """The values of a Packed matrix."""
    codes, scales, n = p.codes, p.scales, p.n
    T, lc, ls = _packed_rows(codes, scales, n)
    dev = codes.device
    out = torch.empty(T, n, dtype=dtype, device=dev) if out is None else out
    ld = _rows("out", out, T, n, _DT)
    _check_device(dev, "scales out", scales, out)
    _call(zl.zl_unpack, dev, T, n, zl.pack_packed(codes.data_ptr(), scales.data_ptr(), lc, ls), out.data_ptr(), ld, _DT[out.dtype])
    _wrote((out,))
    return out


def _ff(h, kind):
    """kind's number and the activation's width."""
    k, nh = _KIND[kind], h.shape[1]
    if k == zl.ZL_MLP_GELU:
        return k, nh
    if nh % 2:
        raise ValueError(f"h must be gate | up, not of {nh} columns")
    return k, nh // 2


def mlp_act(h, kind="swiglu", dtype=None, act=None, packed=None):
    """silu(gate) * up of h = gate | up [T, 2 ff], or gelu(h), h [T, ff].
    packed: a Packed of h's shape that receives h."""
    T, nh = h.shape
    k, ff = _ff(h, kind)
    dev = h.device
    ldh = _rows("h", h, T, nh, _DT)
    act = torch.empty(T, ff, dtype=dtype or h.dtype, device=dev) if act is None else act
    lda = _rows("act", act, T, ff, _DT)
    ps = _packed("packed", packed, T, nh)
    _check_device(dev, "act packed", act, packed)
    _call(zl.zl_mlp_act, dev, zl.pack_mlp_args(T, ff, k, _DT[h.dtype], _DT[act.dtype], h.data_ptr(), ldh, *ps,
                                               act.data_ptr(), lda, 0, 0, 0, 0))
    _wrote((act,) if packed is None else (act, packed.codes, packed.scales))
    return act


def mlp_act_bwd(h, dact, kind="swiglu", dtype=None, dh=None, act=None):
    """Gradient with respect to h (a tensor of dact's type, or its Packed
    copy).  act: a tensor that receives the activation, formed again."""
    T, nh = h.shape
    k, ff = _ff(h, kind)
    dev = dact.device
    ldda = _rows("dact", dact, T, ff, _DT)
    dh = torch.empty(T, nh, dtype=dtype or dact.dtype, device=dev) if dh is None else dh
    lddh = _rows("dh", dh, T, nh, _DT)
    lda = 0 if act is None else _rows("act", act, T, ff, (dh.dtype,))
    if isinstance(h, Packed):
        hp, ldh, ps = 0, 0, _packed("h", h, T, nh)
    else:
        hp, ldh, ps = h.data_ptr(), _rows("h", h, T, nh, (dact.dtype,)), _NONE
    _check_device(dev, "h dh act", h, dh, act)
    _call(zl.zl_mlp_act_backward, dev,
          zl.pack_mlp_args(T, ff, k, _DT[dact.dtype], _DT[dh.dtype], hp, ldh, *ps, _ptr(act), lda, dact.data_ptr(), ldda,
                           dh.data_ptr(), lddh))
    _wrote((dh,) if act is None else (dh, act))
    return dh


NormGrads = namedtuple("NormGrads", "w_post b_post w_pre b_pre gate", defaults=(None,) * 5)
NormGrads.__doc__ = "Gradients of block_norm's parameters (fp32; None = not wanted)."


def _norm_common(d, T, dev, post, pre, gate, gate_rows, stats):
    """Pointers of the weights, biases, the gate, its rows and the statistics,
    everything of them checked."""
    (w0, b0), (w1, b1) = post or _NO_WB, pre or _NO_WB
    gp = 0
    if gate is not None:
        if gate_rows < 1:
            raise ValueError("a gate needs gate_rows >= 1")
        G = -(-T // gate_rows)
        if gate.dtype != torch.float32 or gate.shape != (G, d) or not gate.is_contiguous():
            raise ValueError(f"gate must be a contiguous fp32 [{G}, {d}] tensor")
        if gate.requires_grad and not gate.is_leaf:
            _no_graph("gate")
        gp = gate.data_ptr()
    if stats.dtype != torch.float32 or stats.shape != (T, 4) or not stats.is_contiguous():
        raise ValueError(f"stats must be a contiguous fp32 [{T}, 4] tensor")
    _check_device(dev, "w_post b_post w_pre b_pre gate stats", w0, b0, w1, b1, gate, stats)
    return (_vec("w_post", w0, d), _vec("b_post", b0, d), _vec("w_pre", w1, d), _vec("b_pre", b1, d), gp, gate_rows,
            stats.data_ptr())


def block_norm(x, y, post, pre, *, gate=None, gate_rows=0, scale=1.0, eps=1e-5, layernorm=False, dtype=None,
               xo=None, n=None, stats=None, y_packed=None, n_packed=None):
    """xo = x + scale * gate * Norm(y), n = Norm(xo); returns (xo, n, stats).

    x [T, d] fp32; post, pre: (weight, bias or None) of the norm of y and of
    the norm of xo, or None (without post: y is None, xo is x itself; without
    pre: n is None).  gate [ceil(T / gate_rows), d].  stats [T, 4] is what the
    backward needs besides.  y_packed, n_packed: Packed [T, d] that receive y
    and n.  n has `dtype` (default: y's, or bf16).  xo may be x."""
    T, d = x.shape
    dev = x.device
    ldx = _rows("x", x, T, d, _F32)
    stats = torch.empty(T, 4, dtype=torch.float32, device=dev) if stats is None else stats
    params = _norm_common(d, T, dev, post, pre, gate, gate_rows, stats)
    if (y is None) != (post is None):
        raise ValueError("y and post go together")
    ldy = ldn = 0
    ty, tn = zl.ZL_F32, zl.ZL_BF16
    if y is not None:
        ldy, ty = _rows("y", y, T, d, _DT), _DT[y.dtype]
        xo = torch.empty_strided((T, d), (ldx, 1), dtype=torch.float32, device=dev) if xo is None else xo
        if _rows("xo", xo, T, d, _F32) != ldx:
            raise ValueError("xo must have x's row stride")
    elif xo is not None:
        raise ValueError("xo is x where there is no y")
    if pre is not None:
        n = torch.empty(T, d, dtype=dtype or (torch.bfloat16 if y is None else y.dtype), device=dev) if n is None else n
        ldn, tn = _rows("n", n, T, d, _DT), _DT[n.dtype]
    elif n is not None:
        raise ValueError("n needs pre")
    _check_device(dev, "y xo n y_packed n_packed", y, xo, n, y_packed, n_packed)
    _call(zl.zl_block_norm, dev,
          zl.pack_norm_args(T, d, int(layernorm), ty, tn, eps, scale, *params, x.data_ptr(), _ptr(xo), ldx, _ptr(y), ldy,
                            _ptr(n), ldn, *_packed("y_packed", y_packed, T, d), *_packed("n_packed", n_packed, T, d),
                            0, 0, 0, 0, 0, 0, 0, 0, 0, 0.0, 0, 0, 0))
    wrote = [stats]
    if y is not None:
        wrote.append(xo)
    if pre is not None:
        wrote.append(n)
    for p in (y_packed, n_packed):
        if p is not None:
            wrote += p.codes, p.scales
    _wrote(wrote)
    return (x if y is None else xo), n, stats


def block_norm_bwd(dxo, dn, y, xo, stats, post, pre, *, gate=None, gate_rows=0, scale=1.0, eps=1e-5,
                   layernorm=False, dtype=None, dx=None, dy=None, grads=None, grad_scale=1.0, accumulate=False,
                   workspace=None):
    """Backward of block_norm; returns (dx, dy).

    dxo [T, d] fp32: gradient of xo besides that through n (None = 0); dn
    [T, d]; y: block_norm's, or its Packed copy; xo, stats: block_norm's
    outputs.  dn and y have one type.  dy has `dtype` (default: dn's or y's).
    grads: NormGrads of fp32 tensors that receive (accumulate: are added)
    grad_scale times the parameters' gradients.  dx may be dxo.  workspace:
    fp32, zl.zl_block_norm_workspace elements, made here if None."""
    src = dn if dn is not None else xo if xo is not None else dxo
    if src is None:
        raise ValueError("dxo, dn or xo must be there")
    T, d = src.shape
    dev = src.device
    params = _norm_common(d, T, dev, post, pre, gate, gate_rows, stats)
    if (y is None) != (post is None) or (dn is None) != (pre is None) or (pre is not None and xo is None):
        raise ValueError("y and post, dn, xo and pre go together")
    if pre is None:
        xo = None
    ldx = None
    for t in (dxo, dx, xo):
        if t is not None:
            ld = _rows("dxo, dx and xo", t, T, d, _F32)
            if ldx is not None and ld != ldx:
                raise ValueError("dxo, dx and xo must have one row stride")
            ldx = ld
    if ldx is None:
        ldx = d
    if dx is None:
        dx = torch.empty_strided((T, d), (ldx, 1), dtype=torch.float32, device=dev)
    tin, ldn, ldy, yp, ys = None, 0, 0, 0, _NONE
    if dn is not None:
        ldn, tin = _rows("dn", dn, T, d, _DT), dn.dtype
    if isinstance(y, Packed):
        ys = _packed("y", y, T, d)
    elif y is not None:
        ldy, yp = _rows("y", y, T, d, _DT if tin is None else (tin,)), y.data_ptr()
        tin = y.dtype
    tin = torch.float32 if tin is None else tin
    if post is not None:
        if dy is None:
            dy = torch.empty_strided((T, d), (ldy or d, 1), dtype=dtype or tin, device=dev)
        ld = _rows("dy", dy, T, d, _DT)
        if yp and ld != ldy:
            raise ValueError("dy must have y's row stride")
        ldy = ld
    elif dy is not None:
        raise ValueError("dy needs post")
    gw, gb, gv, gc, gg = grads or NormGrads()
    if gg is not None and (gate is None or gg.shape != gate.shape or gg.dtype != torch.float32 or
                           not gg.is_contiguous()):
        raise ValueError("grads.gate must be a contiguous fp32 tensor like gate")
    if workspace is None:
        workspace = torch.empty(zl.zl_block_norm_workspace(T, d, gate_rows if gate is not None else 0),
                                dtype=torch.float32, device=dev)
    elif workspace.dtype != torch.float32 or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous fp32 tensor")
    _check_device(dev, "dxo y xo dx dy workspace w_post b_post w_pre b_pre gate", dxo, y, xo, dx, dy, workspace, gw, gb,
                  gv, gc, gg)
    _call(zl.zl_block_norm_backward, dev,
          zl.pack_norm_args(T, d, int(layernorm), _DT[tin], zl.ZL_F32 if dy is None else _DT[dy.dtype], eps, scale,
                            *params, 0, _ptr(xo), ldx, yp, ldy, 0, ldn, *ys, *_NONE, _ptr(dxo), _ptr(dn), dx.data_ptr(),
                            _ptr(dy), _vec("grads.w_post", gw, d), _vec("grads.b_post", gb, d),
                            _vec("grads.w_pre", gv, d), _vec("grads.b_pre", gc, d), _ptr(gg), grad_scale,
                            int(accumulate), workspace.data_ptr(), workspace.numel()))
    _wrote([t for t in (dx, dy, gw, gb, gv, gc, gg, workspace) if t is not None])
    return dx, dy


def wgrad(dy, x, out=None, scale=1.0, accumulate=False, workspace=None):
    """dw [n_out, n_in] fp32 = scale * dy^T x (added to `out` with
    accumulate); dy [T, n_out], x a Packed [T, n_in].  workspace: fp32 scratch
    that lets a small dw split the sum over T, each part as large as dw (bf16,
    T = 4096, dw 768 x 768: 21 us with 6 parts, 35 without a workspace)."""
    T, M = dy.shape
    N, dev = x.n, dy.device
    lddy = _rows("dy", dy, T, M, _DT)
    p = zl.pack_packed(*_packed("x", x, T, N))
    if out is None:
        out = (torch.zeros if accumulate else torch.empty)(M, N, dtype=torch.float32, device=dev)
    ld = _rows("out", out, M, N, _F32)
    if workspace is not None and (workspace.dtype != torch.float32 or not workspace.is_contiguous()):
        raise TypeError("workspace must be a contiguous fp32 tensor")
    _check_device(dev, "x out workspace", x, out, workspace)
    _call(zl.zl_wgrad_packed, dev, T, M, N, dy.data_ptr(), lddy, _DT[dy.dtype], p, out.data_ptr(), ld, scale, accumulate,
          _ptr(workspace), 0 if workspace is None else workspace.numel())
    _wrote((out,) if workspace is None else (out, workspace))
    return out


def rotary(x, pos, axis_of, n_heads, head_dim, theta, *, inverse=False, out=None):
    """x [T, >= n_heads * head_dim] with the heads rotated by pos [axes, T]
    (int32, contiguous); returns [T, n_heads * head_dim].  axis_of: bytes (or
    another sequence of integers), the axis of each frequency; 2 len(axis_of)
    columns of a head are rotated, the others copied.  inverse: the gradient's way back.  out may be x."""
    T, W = x.shape[0], n_heads * head_dim
    dev = x.device
    if x.dim() != 2 or x.shape[1] < W:
        raise ValueError(f"x must be [{T}, >= {W}], not {list(x.shape)}")
    ldx, s1 = x.stride()
    if x.dtype not in _DT or (s1 != 1 and W > 1):
        raise TypeError("x must be fp32 or bf16 with contiguous rows")
    if pos.dtype != torch.int32 or pos.dim() != 2 or pos.shape[1] != T or not pos.is_contiguous():
        raise TypeError(f"pos must be a contiguous int32 [axes, {T}] tensor")
    out = torch.empty(T, W, dtype=x.dtype, device=dev) if out is None else out
    if out.dtype != x.dtype or out.dim() != 2 or out.shape[0] != T or out.shape[1] < W or out.stride(1) != 1:
        raise ValueError(f"out must be [{T}, >= {W}] of x's type with contiguous rows")
    if x.requires_grad or out.requires_grad:
        _no_graph("x" if x.requires_grad else "out")
    _check_device(dev, "pos out", pos, out)
    ldx, ldo = (ldx, out.stride(0)) if T > 1 else (W, W)
    _call(zl.zl_rotary, dev, T, n_heads, head_dim, 2 * len(axis_of), x.data_ptr(), ldx, out.data_ptr(), ldo, _DT[x.dtype],
          pos.data_ptr(), pos.shape[0], axis_of, theta, inverse)
    _wrote((out,))
    return out
