"""The layer operators (include/zl_layer.h) in fp64 NumPy: the packed 8-bit
format, the MLP activation, the norms around a block and the rotary positions
with several axes, from their definitions."""
import numpy as np

from . import ops

EMIN, EMAX, TOP = -117, 119, 448.0


# ------------------------------------------------------------ packed format
def e4m3_value(code):
    """Value of an e4m3 byte: sign, 4 bits of exponent (bias 7), 3 of fraction;
    no infinities, S.1111.111 is NaN."""
    c = np.asarray(code).astype(np.int64)
    ex, fr = (c >> 3) & 15, c & 7
    mag = np.where(ex == 0, fr * 2.0 ** -9, (8 + fr) * 2.0 ** (ex - 10.0))
    mag = np.where((c & 127) == 127, np.nan, mag)
    return np.where(c & 128, -mag, mag)


_POS = e4m3_value(np.arange(127))  # 0 .. 448, ascending


def e4m3_code(v):
    """Nearest code of values within +-448, ties to the even code; NaN 127."""
    v = np.asarray(v, np.float64)
    a = np.abs(np.where(np.isnan(v), 0.0, v))
    hi = np.clip(np.searchsorted(_POS, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POS[lo], _POS[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isnan(v), 127, c + 128 * np.signbit(v)).astype(np.uint8)


def pack(x):
    """(codes [T, n], scale bytes [T, ceil(n / 32)]) of x [T, n]."""
    x = np.asarray(x, np.float64)
    T, n = x.shape
    nb = -(-n // 32)
    b = np.zeros((T, nb * 32))
    b[:, :n] = x
    b = b.reshape(T, nb, 32)
    fine = np.isfinite(b)
    top = np.where(fine, np.abs(b), 0.0).max(-1)
    es = np.arange(EMIN, EMAX + 1)
    e = EMIN + np.minimum(np.searchsorted(TOP * 2.0 ** es, top), es.size - 1)  # first that holds top
    v = np.where(fine, np.clip(np.where(fine, b, 0.0) / 2.0 ** e[..., None], -TOP, TOP), np.nan)
    return e4m3_code(v).reshape(T, -1)[:, :n], (e + 127).astype(np.uint8)


def values(codes, scales):
    """What codes [T, n] and scale bytes stand for."""
    s = np.asarray(scales).astype(np.float64)
    s = np.where(s == 255, np.nan, 2.0 ** (s - 127))
    return e4m3_value(codes) * np.repeat(s, 32, 1)[:, : np.asarray(codes).shape[1]]


def packed(x):
    """The values that x has after packing."""
    return values(*pack(x))


# --------------------------------------------------------------- activation
def _sigmoid(z):
    """1 / (1 + exp(-z)) without cancellation at either end."""
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0, e) / (1.0 + e)


def _gate(x, kind):
    """s(z) of a = x s(z) (u), and the derivative of x s(z): silu has z = x, the
    tanh form of gelu z = 2 sqrt(2 / pi) (x + 0.044715 x^3)."""
    if kind == "gelu":
        z, dz = 2 * ops._GELU_C * (x + 0.044715 * x ** 3), 2 * ops._GELU_C * (1 + 3 * 0.044715 * x ** 2)
    else:
        z, dz = x, 1.0
    s = _sigmoid(z)
    return s, s + x * s * _sigmoid(-z) * dz


def mlp_act(h, kind):
    if kind == "gelu":
        return h * _gate(h, kind)[0]
    g, u = np.split(h, 2, -1)
    return g * _gate(g, kind)[0] * u


def mlp_act_bwd(h, da, kind):
    if kind == "gelu":
        return da * _gate(h, kind)[1]
    g, u = np.split(h, 2, -1)
    s, ds = _gate(g, kind)
    return np.concatenate([da * u * ds, da * g * s], -1)


# ------------------------------------------------------- norms around a block
def _norm(v, w, b, eps, ln):
    if ln:
        return ops.layernorm_fwd(v, w, 0.0 if b is None else b, eps)
    return ops.rmsnorm_fwd(v, w, eps)


def _norm_bwd(dy, cache, ln):
    if ln:
        return ops.layernorm_bwd(dy, cache)
    return (*ops.rmsnorm_bwd(dy, cache), None)


def _stats(v, eps, ln):
    mu = v.mean(-1) if ln else np.zeros(v.shape[0])
    return np.stack([mu, 1.0 / np.sqrt(((v - mu[:, None]) ** 2).mean(-1) + eps)], -1)


def block_norm(x, y, post, pre, gate=None, gate_rows=0, scale=1.0, eps=1e-5, ln=False):
    """xo = x + scale gate Norm(y), n = Norm(xo), stats [T, 4]; post, pre:
    (weight, bias or None), or None."""
    T = x.shape[0]
    stats = np.zeros((T, 4))
    xo, n = x, None
    if post is not None:
        p, _ = _norm(y, *post, eps, ln)
        stats[:, :2] = _stats(y, eps, ln)
        xo = x + scale * (p if gate is None else gate[np.arange(T) // gate_rows] * p)
    if pre is not None:
        n, _ = _norm(xo, *pre, eps, ln)
        stats[:, 2:] = _stats(xo, eps, ln)
    return xo, n, stats


def block_norm_bwd(dxo, dn, y, xo, stats, post, pre, gate=None, gate_rows=0, scale=1.0, ln=False):
    """Gradients (a dict) from the saved y (as packed, where it was) and xo and
    the forward's statistics."""
    out = {}
    D = np.zeros_like(dn if dn is not None else dxo) if dxo is None else dxo
    T, d = D.shape
    hat = lambda v, m, r: (v - m[:, None]) * r[:, None]  # noqa: E731
    if pre is not None:
        cache = (hat(xo, stats[:, 2], stats[:, 3]), stats[:, 3:4], pre[0])
        dx, out["w_pre"], out["b_pre"] = _norm_bwd(dn, cache, ln)
        D = D + dx
    out["dx"] = D
    if post is not None:
        yh = hat(y, stats[:, 0], stats[:, 1])
        g = np.ones_like(D) if gate is None else gate[np.arange(T) // gate_rows]
        out["dy"], out["w_post"], out["b_post"] = _norm_bwd(scale * g * D, (yh, stats[:, 1:2], post[0]), ln)
        if gate is not None:
            p = yh * post[0] + (0.0 if post[1] is None else post[1])
            out["gate"] = np.zeros_like(gate)
            np.add.at(out["gate"], np.arange(T) // gate_rows, scale * D * p)
    return out


# ------------------------------------------------------------------- rotary
def rotary(x, pos, axis_of, n_heads, head_dim, theta, inverse=False):
    """x [T, n_heads * head_dim], pos [axes, T], axis_of: the axis of each of
    the rot / 2 frequencies."""
    T, half = x.shape[0], len(axis_of)
    ang = np.stack([pos[a].astype(np.float64) * theta ** (-j / half) for j, a in enumerate(axis_of)], -1)
    v = x.reshape(1, T, n_heads, head_dim)
    r = ops.rope_fwd(v[..., : 2 * half], -ang[None] if inverse else ang[None])
    return np.concatenate([r, v[..., 2 * half:]], -1).reshape(T, -1)
