"""The layer operators on the GPU (include/zl_layer.h, through layer.py)
against the fp64 oracle (oracle/layer.py).

Tolerances, with u = 2^-24 (half a step of fp32) and half a step of bf16,
2^-8 of the value, where the output is bf16:
  packed bytes and unpacked values: equal.
  activation: the exponential's argument rounds to |x| u, the function and the
    reciprocal to 2 u each, six products to u: (2 |x| + 16) u of every term.
    The hardware reciprocal of 2^126 and more is 0, so s(z) is off by up to
    2^-126 there, which its factors multiply.
  norms: a row's sum has at most 32 terms per lane and 10 levels above, so 48 u
    of the sum of magnitudes; the values made of it another 16 u.  256 u of
    the terms' magnitudes holds both norms in a row.
  sums over rows: at most 64 rows in one register, 8 + 5 + 8 levels above, on
    terms that are 128 u off themselves: 256 u of the sum of magnitudes.
  weight gradient: T terms added in any order: T u of the sum of magnitudes;
    and 2e-6 in the norm (independent roundings of T <= 5000).
  rotary: angles to 2^-23 turns times 2 pi and u each for sine, cosine and two
    products: 16 u of |x| + |y|.
"""
import zlib

import numpy as np
import pytest

from oracle import layer as ol
from oracle import ops

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
BF, F32 = "bf16", "f32"


def _L():
    from paper_2608_07974_amd import layer
    return layer


def _dt(name):
    return torch.bfloat16 if name == BF else torch.float32


def _rng(*key):
    return np.random.default_rng([zlib.crc32(k.encode()) if isinstance(k, str) else int(k) for k in key])


def _dev(a, dt=F32, pad=0):
    """A device matrix, in rows `pad` columns longer that hold NaN."""
    a = np.atleast_2d(np.asarray(a, np.float32))
    t = torch.full((a.shape[0], a.shape[1] + pad), float("nan"), dtype=_dt(dt), device="cuda")[:, : a.shape[1]]
    t.copy_(torch.from_numpy(np.ascontiguousarray(a)))
    return t


def _out(T, n, dt=F32, pad=0):
    return torch.full((T, n + pad), float("nan"), dtype=_dt(dt), device="cuda")[:, :n]


def _vec(a):
    return torch.tensor(np.asarray(a, np.float32), device="cuda")


def _np(t):
    return t.detach().double().cpu().numpy()


def _near(got, ref, tol, dt=F32, what=""):
    """|got - ref| <= tol (+ half a bf16 step), elementwise; NaN where ref is."""
    got, ref, tol = np.asarray(got), np.asarray(ref), np.broadcast_to(tol, np.shape(ref))
    if dt == BF:
        tol = tol + (np.abs(ref) + tol) * 2.0 ** -8 + 2.0 ** -134
    nan = np.isnan(ref)
    assert np.array_equal(np.isnan(got), nan), what
    over = np.where(nan, 0.0, np.abs(got - ref) - tol)
    if over.size:
        at = np.unravel_index(over.argmax(), over.shape)
        worst = (what, at, float(got[at]), float(ref[at]), float(tol[at]))
        fine = bool(over[at] <= 0)
        assert fine, worst


def _acts(rng, T, n):
    col = np.exp(rng.standard_normal(n))
    col[:: max(1, n // 3)] *= 30
    return rng.standard_normal((T, n)) * col


def _bytes(p, T, n):
    return p.codes.cpu().numpy()[:, :n], p.scales.cpu().numpy()[:, : -(-n // 32)]


def _same_codes(got, want):
    """Equal bytes (any NaN code is NaN)."""
    g, w = got[0], want[0]
    nan = (w & 127) == 127
    assert np.array_equal((g & 127) == 127, nan)
    assert np.array_equal(g[~nan], w[~nan])
    assert np.array_equal(got[1], want[1])


def _packed(a, pad=0):
    """The oracle's packing of a, on the device; bytes past the row are 0x7f (NaN)."""
    layer = _L()
    c, s = ol.pack(a)
    T, n = c.shape
    codes = torch.full((T, -(-n // 16) * 16 + pad), 0x7f, dtype=torch.uint8, device="cuda")
    scales = torch.full((T, s.shape[1] + pad), 255, dtype=torch.uint8, device="cuda")
    codes[:, :n] = torch.from_numpy(c).cuda()
    scales[:, : s.shape[1]] = torch.from_numpy(s).cuda()
    return layer.Packed(codes, scales, n)


def _empty_packed(T, n, pad=0):
    layer = _L()
    return layer.Packed(torch.full((T, -(-n // 16) * 16 + pad), 0xaa, dtype=torch.uint8, device="cuda"),
                        torch.full((T, -(-n // 32) + pad), 0xaa, dtype=torch.uint8, device="cuda"), n)


def _untouched(p, T, n):
    """Bytes past the rows are as they were."""
    assert (p.codes[:, n:] == 0xaa).all() and (p.scales[:, -(-n // 32):] == 0xaa).all()


# ------------------------------------------------------------------- packed
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("T,n,pad", [(1, 8, 0), (3, 40, 16), (125, 200, 0), (7, 4096, 0), (2050, 72, 16), (1, 8192, 0),
                                     (300, 1032, 32), (4100, 2088, 0)])
def test_pack_and_unpack(dt, T, n, pad):
    layer = _L()
    rng = _rng("pack", T, n)
    x = _acts(rng, T, n) * 2.0 ** rng.integers(-8, 9, (T, 1))
    xt = _dev(x, dt, pad)
    p = layer.pack(xt, out=_empty_packed(T, n, pad))
    want = ol.pack(_np(xt))
    _same_codes(_bytes(p, T, n), want)
    _untouched(p, T, n)
    for odt in (F32, BF):
        back = layer.unpack(p, out=_out(T, n, odt, pad))
        assert np.array_equal(_np(back), ol.values(*want))
        if pad:
            assert torch.isnan(back.as_strided((T, pad), (back.stride(0), 1), n)).all()


@pytest.mark.parametrize("dt", [F32, BF])
def test_pack_special_values(dt):
    """Zeros of both signs, subnormals, the largest values, infinities and NaN
    (alone, in a block of others, and a whole block of them), values at the
    scale's border and halfway between two codes."""
    layer = _L()
    rng = _rng("special")
    x = rng.standard_normal((16, 72))
    x[0] = 0.0
    x[1] = -0.0
    x[2] *= 2.0 ** -130
    x[3] *= 2.0 ** -125
    x[4] = np.where(rng.random(72) < 0.5, 1, -1) * 3.0e38
    x[5, :32] = 448.0
    x[5, 32:64] = 452.0
    x[6, 4], x[6, 40], x[6, 41] = np.inf, -np.inf, np.nan
    x[7, :32] = np.nan
    x[7, 64:] = np.inf
    x[8, 0] = 2.0 ** 127 * 1.75
    x[9] = 2.0 ** -149 if dt == F32 else 2.0 ** -133
    x[10, 0], x[10, 1:32] = 448.0, np.repeat((ol._POS[:-1] + ol._POS[1:]) / 2, 1)[40:71]
    x[11] *= 2.0 ** 120
    xt = _dev(x, dt)
    p = layer.pack(xt)
    with np.errstate(invalid="ignore"):
        want = ol.pack(_np(xt))
    _same_codes(_bytes(p, 16, 72), want)
    for odt in (F32, BF):
        np.testing.assert_array_equal(_np(layer.unpack(p, dtype=_dt(odt))), ol.values(*want))


def test_unpack_every_code_and_scale():
    layer = _L()
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(256, 1)
    scales = torch.arange(256, dtype=torch.uint8, device="cuda")[:, None].repeat(1, 8)
    got = _np(layer.unpack(layer.Packed(codes, scales, 256), dtype=torch.float32))
    with np.errstate(over="ignore"):
        want = ol.values(codes.cpu().numpy(), scales.cpu().numpy()).astype(np.float32)
    np.testing.assert_array_equal(got, want)


# --------------------------------------------------------------- activation
@pytest.mark.parametrize("kind", ["swiglu", "gelu"])
@pytest.mark.parametrize("inp,out", [(BF, BF), (F32, BF), (F32, F32), (BF, F32)])
@pytest.mark.parametrize("T,ff,pad,saved", [(1, 32, 0, True), (5, 96, 16, True), (33, 2080, 0, True), (700, 1056, 16, True),
                                            (3, 40, 16, False), (1500, 2056, 0, False)])
def test_mlp_act(kind, inp, out, T, ff, pad, saved):
    layer = _L()
    rng = _rng("mlp", T, ff)
    nh = 2 * ff if kind == "swiglu" else ff
    h = 2.5 * rng.standard_normal((T, nh))
    h[0, 0], h[0, ff - 1] = -60.0, 60.0
    ht = _dev(h, inp, pad)
    h = _np(ht)
    p = _empty_packed(T, nh, pad) if saved else None
    act = layer.mlp_act(ht, kind, act=_out(T, ff, out, pad), packed=p)
    ref = ol.mlp_act(h, kind)
    x = np.abs(h[:, :ff])
    tiny = 2.0 ** -126 * (1 + x) * (1 + np.abs(h[:, ff:]) if kind == "swiglu" else 1.0)
    _near(_np(act), ref, (2 * (x if kind == "swiglu" else 0.2 * x ** 3 + 2 * x) + 16) * U * np.abs(ref) + tiny, out)
    if saved:
        _same_codes(_bytes(p, T, nh), ol.pack(h))
        _untouched(p, T, nh)


@pytest.mark.parametrize("kind", ["swiglu", "gelu"])
@pytest.mark.parametrize("inp,out", [(BF, BF), (F32, BF), (F32, F32), (BF, F32)])
@pytest.mark.parametrize("T,ff,pad,saved", [(1, 32, 0, True), (5, 96, 16, True), (33, 2080, 0, True), (700, 1056, 16, True),
                                            (3, 40, 16, False), (1500, 2056, 0, False)])
def test_mlp_act_backward(kind, inp, out, T, ff, pad, saved):
    layer = _L()
    rng = _rng("mlpb", T, ff)
    sw = kind == "swiglu"
    nh = 2 * ff if sw else ff
    h = 2.5 * rng.standard_normal((T, nh))
    h[0, 0], h[0, ff - 1] = -60.0, 60.0
    src = _packed(h, pad) if saved else _dev(h, inp, pad)
    h = ol.packed(h) if saved else _np(src)
    da = _dev(rng.standard_normal((T, ff)), inp, pad)
    dh, act = _out(T, nh, out, pad), _out(T, ff, out, pad)
    layer.mlp_act_bwd(src, da, kind, dh=dh, act=act)
    d, x = _np(da), np.abs(h[:, :ff])
    k = ((2 * x if sw else 0.4 * x ** 3 + 4 * x) + 24) * U
    ref = ol.mlp_act(h, kind)
    u = np.abs(h[:, ff:]) if sw else 1.0
    tiny = 2.0 ** -126 * (1 + x) * (1 + u)
    _near(_np(act), ref, k * np.abs(ref) + tiny, out, "act")
    ref = ol.mlp_act_bwd(h, d, kind)
    # the derivative is s (1 + x (1 - s) z'): both terms count where they cancel
    s = ol._gate(h[:, :ff], kind)[0]
    dz = x if sw else x * 1.6 * (1 + 0.135 * x * x)
    slope = s * (1 + dz * (1 - s))
    tiny = tiny * (1 + dz) * (1 + np.abs(d))
    _near(_np(dh)[:, :ff], ref[:, :ff], k * slope * np.abs(d) * u + tiny, out, "dgate")
    if sw:
        _near(_np(dh)[:, ff:], ref[:, ff:], k * np.abs(ref[:, ff:]) + tiny, out, "dup")
    # without the activation
    dh2 = _out(T, nh, out)
    layer.mlp_act_bwd(src, da, kind, dh=dh2)
    assert torch.equal(dh2, dh)
    if pad:
        assert torch.isnan(dh.as_strided((T, pad), (dh.stride(0), 1), nh)).all()


def test_mlp_act_beyond_the_exponential():
    """Inputs whose exponential or cube leaves the range of fp32."""
    layer = _L()
    h = np.zeros((2, 64))
    h[0, :8] = [-1e20, 1e20, -200.0, 200.0, -1e5, 1e5, -3e38, 3e38]
    h[1] = h[0]
    h[:, 32:] = 1.0
    for kind in ("swiglu", "gelu"):
        ht = _dev(h if kind == "swiglu" else h[:, :32])
        act = _np(layer.mlp_act(ht, kind))
        dh = _np(layer.mlp_act_bwd(ht, _dev(np.ones((2, 32))), kind))
        x = h[:, :8]
        assert np.array_equal(act[:, :8], np.maximum(np.float32(x), 0)) and np.array_equal(dh[:, :8], (x > 0) * 1.0)


# ------------------------------------------- large calls against small ones
def _in_rows(T, step=400):
    """Slices of few rows: calls of at most four blocks a CU, one row per thread."""
    return [slice(t, min(T, t + step)) for t in range(0, T, step)]


def _rows_of(p, r):
    return _L().Packed(p.codes[r], p.scales[r], p.n)


def _randn(T, n, dt, seed=7):
    return torch.empty(T, n, dtype=_dt(dt), device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(seed))


def _equal_packed(p, q):
    assert torch.equal(p.codes[:, : p.n], q.codes[:, : p.n]) and torch.equal(p.scales, q.scales)


# Outputs above 32 MB are stored past the caches, inputs above 384 MB are loaded so
# too; many rows go several to a thread.  The same values, bit for bit, as in
# pieces that do neither (those are what the tests above compare with the oracle).
@pytest.mark.parametrize("dt,T", [(BF, 2051), (F32, 2051), (BF, 8195), (F32, 8195), (BF, 49157), (F32, 24579)])
def test_pack_and_unpack_of_many_rows(dt, T):
    layer = _L()
    n = 4104
    x = _randn(T, n, dt)
    p, q = layer.pack(x), layer.Packed.empty(T, n)
    for r in _in_rows(T):
        layer.pack(x[r], out=_rows_of(q, r))
    _equal_packed(p, q)
    del x
    for odt in (BF, F32):
        got = layer.unpack(p, dtype=_dt(odt))
        assert all(torch.equal(got[r], layer.unpack(_rows_of(p, r), dtype=_dt(odt))) for r in _in_rows(T))


@pytest.mark.parametrize("kind,inp,out,T,ff", [
    ("swiglu", BF, BF, 2051, 2080), ("swiglu", F32, BF, 2051, 2080), ("swiglu", BF, F32, 2051, 2080), ("swiglu", F32, F32, 2051, 2080),
    ("gelu", BF, BF, 2051, 2088), ("gelu", F32, F32, 2051, 2088), ("gelu", F32, BF, 2051, 2088),
    ("swiglu", BF, BF, 4099, 2080), ("swiglu", F32, F32, 4099, 2080), ("gelu", BF, BF, 8195, 2088), ("gelu", F32, BF, 8195, 2088),
    ("swiglu", BF, BF, 48403, 2080), ("gelu", F32, BF, 48403, 2088)])
def test_mlp_act_of_many_rows(kind, inp, out, T, ff):
    layer = _L()
    n = (2 if kind == "swiglu" else 1) * ff
    h, da = _randn(T, n, inp), _randn(T, ff, inp, 8)
    for saved in (True, False):
        p, q = (layer.Packed.empty(T, n) if saved else None for _ in range(2))
        act = layer.mlp_act(h, kind, dtype=_dt(out), packed=p)
        again = torch.empty_like(act)
        src = p if saved else h
        dh = layer.mlp_act_bwd(src, da, kind, dtype=_dt(out), act=again)
        for r in _in_rows(T):
            a = layer.mlp_act(h[r], kind, dtype=_dt(out), packed=_rows_of(q, r) if saved else None)
            assert torch.equal(act[r], a)
            b = torch.empty_like(a)
            d = layer.mlp_act_bwd(_rows_of(p, r) if saved else h[r], da[r], kind, dtype=_dt(out), act=b)
            assert torch.equal(dh[r], d) and torch.equal(again[r], b)
        if saved:
            _equal_packed(p, q)


@pytest.mark.parametrize("dt,T,H,hd,rot", [(BF, 4099, 40, 128, 128), (BF, 4099, 40, 128, 96), (BF, 8195, 40, 64, 64), (F32, 4099, 24, 128, 128)])
def test_rotary_of_many_rows(dt, T, H, hd, rot):
    layer = _L()
    x = _randn(T, H * hd + 16, dt)
    pos = torch.randint(0, 100000, (3, T), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(9))
    axes = bytes(i % 3 for i in range(rot // 2))
    got = layer.rotary(x, pos, axes, H, hd, 5e5)
    for r in _in_rows(T):
        assert torch.equal(got[r], layer.rotary(x[r], pos[:, r].contiguous(), axes, H, hd, 5e5))


# -------------------------------------------------------- norms around a block
def _norm_case(rng, T, d, ln, parts, rows, inp):
    x = _acts(rng, T, d) + (0.5 if ln else 0.0)
    y = 2 * rng.standard_normal((T, d)) + 0.25
    vec = lambda at: at + 0.2 * rng.standard_normal(d)  # noqa: E731
    post = (vec(1.0), vec(0.0) if ln else None) if parts != "pre" else None
    pre = (vec(1.0), vec(0.0) if ln else None) if parts != "post" else None
    gate = 0.5 * rng.standard_normal((-(-T // rows), d)) if rows and post else None
    r32 = lambda v: None if v is None else np.float32(v).astype(np.float64)  # noqa: E731
    post, pre = (p and tuple(map(r32, p)) for p in (post, pre))
    return x, y, post, pre, r32(gate)


def _tv(p):
    return None if p is None else tuple(None if v is None else _vec(v) for v in p)


_NORM_CASES = [  # T, d, gate rows, parts, pad
    (1, 8, 0, "both", 0), (1, 4096, 1, "both", 0), (2, 64, 2, "both", 16), (33, 200, 7, "both", 16),
    (33, 768, 1, "both", 0), (5, 8192, 5, "both", 0), (6, 8192, 1, "both", 0), (300, 2048, 150, "both", 0),
    (17, 2056, 17, "both", 0), (2100, 520, 700, "both", 0), (2100, 1000, 3, "both", 0), (2051, 2048, 0, "both", 0),
    (40, 4104, 2, "both", 0), (9, 4096, 0, "post", 0), (50, 1024, 25, "post", 0), (9, 4096, 0, "pre", 0),
    (2048, 512, 0, "pre", 16), (3000, 136, 1000, "both", 0), (700, 8, 64, "both", 0),
    (3, 72, 1000, "both", 0), (1000, 520, 1500, "both", 0), (4500, 64, 5, "both", 0), (520, 8192, 130, "both", 0),
(9000, 72, 4100, "both", 0), (4098, 520, 4097, "both", 0), (4099, 1032, 2049, "both", 0),
    (2111, 2056, 1055, "post", 0), (2100, 2056, 1050, "both", 0)]


@pytest.mark.parametrize("ln", [False, True])
@pytest.mark.parametrize("inp,out", [(BF, BF), (F32, BF), (F32, F32)])
@pytest.mark.parametrize("T,d,rows,parts,pad", _NORM_CASES)
def test_block_norm(ln, inp, out, T, d, rows, parts, pad):
    layer = _L()
    rng = _rng("norm", T, d, rows)
    x, y, post, pre, gate = _norm_case(rng, T, d, ln, parts, rows, inp)
    xt, yt = _dev(x, F32, pad), _dev(y, inp, pad)
    x, y = _np(xt), _np(yt)
    kw = dict(gate_rows=rows, scale=0.75)
    xo, n, stats = ol.block_norm(x, y, post, pre, gate=gate, ln=ln, **kw)
    saved = parts == "both"
    yp, npk = (_empty_packed(T, d, pad) if saved else None for _ in range(2))
    gxo, gn, gst = layer.block_norm(
        xt, yt if post else None, _tv(post), _tv(pre), gate=None if gate is None else _vec(gate), layernorm=ln,
        xo=_out(T, d, F32, pad) if post else None, n=_out(T, d, out, pad) if pre else None, y_packed=yp, n_packed=npk, **kw)
    k = 256 * U
    one = lambda v, w, b, m, r: np.abs(w) * (np.abs(v) + np.abs(v).mean(1, keepdims=True)) * r[:, None] + \
        (0.0 if b is None else np.abs(b))  # noqa: E731
    tx = np.zeros_like(xo)
    if post:
        g = 1.0 if gate is None else np.abs(gate[np.arange(T) // rows])
        tx = k * (np.abs(x) + 0.75 * g * one(y, *post, *stats[:, :2].T))
        _near(_np(gxo), xo, tx, what="xo")
    else:
        assert gxo is xt
    if pre:
        # the error of xo passes through the norm
        tn = k * one(xo, *pre, *stats[:, 2:].T) + np.abs(pre[0]) * stats[:, 3:4] * (tx + tx.mean(1, keepdims=True))
        _near(_np(gn), n, tn, out, "n")
    mag = np.stack([np.abs(y).mean(1), stats[:, 1], np.abs(xo).mean(1) + tx.mean(1) / k, 2 * stats[:, 3]], 1)
    mag[:, 0] *= ln
    mag[:, 2] *= ln
    _near(_np(gst), stats, k * mag, what="stats")
    if saved:
        _same_codes(_bytes(yp, T, d), ol.pack(y))
        _same_codes(_bytes(npk, T, d), ol.pack(_np(gn)))  # of n as it was stored
        _untouched(yp, T, d)
        _untouched(npk, T, d)
    if pad and post:
        assert torch.isnan(gxo.as_strided((T, pad), (gxo.stride(0), 1), d)).all()


@pytest.mark.parametrize("ln", [False, True])
@pytest.mark.parametrize("inp,out,saved", [(BF, BF, True), (F32, BF, False), (F32, F32, True), (BF, F32, False)])
@pytest.mark.parametrize("T,d,rows,parts,pad", _NORM_CASES)
def test_block_norm_backward(ln, inp, out, saved, T, d, rows, parts, pad):
    layer = _L()
    rng = _rng("normb", T, d, rows)
    x, y, post, pre, gate = _norm_case(rng, T, d, ln, parts, rows, inp)
    xo, _, stats = ol.block_norm(x, y, post, pre, gate=gate, gate_rows=rows, scale=0.75, ln=ln)
    xo, stats = np.float32(xo).astype(np.float64), np.float32(stats).astype(np.float64)
    if saved:
        yt = _packed(y, pad)
        y = ol.packed(y)
    else:
        yt = _dev(y, inp, pad)
        y = _np(yt)
    dxo, dn = _dev(rng.standard_normal((T, d)), F32, pad), _dev(rng.standard_normal((T, d)), inp, pad)
    a, b = _np(dxo), _np(dn)
    kw = dict(gate=gate, gate_rows=rows, scale=0.75, ln=ln)
    ref = ol.block_norm_bwd(a, b if pre else None, y, xo, stats, post, pre, **kw)
    old = {n: rng.standard_normal(ref[n].shape).astype(np.float32) for n in ("w_post", "b_post", "w_pre", "b_pre", "gate")
           if ref.get(n) is not None}
    acc = {n: _vec(v) for n, v in old.items()}
    gkw = dict(gate=None if gate is None else _vec(gate), gate_rows=rows, scale=0.75, layernorm=ln)
    args = (dn if pre else None, yt if post else None, _dev(xo, F32, pad) if pre else None, _vec(stats), _tv(post), _tv(pre))
    dy = (_out(T, d, out) if saved else _out(T, d, out, pad)) if post else None
    dx, dy = layer.block_norm_bwd(dxo, *args, dx=_out(T, d, F32, pad), dy=dy, grads=layer.NormGrads(**acc),
                                  grad_scale=0.5, accumulate=True, **gkw)
    # magnitudes of every term
    k = 256 * U
    mean = lambda v: np.abs(v).mean(1, keepdims=True)  # noqa: E731
    tD = np.abs(a)
    if pre:
        xh, g = (xo - stats[:, 2:3]) * stats[:, 3:4], np.abs(b * pre[0])
        tD = tD + stats[:, 3:4] * (g + np.abs(xh) * mean(g * xh) + mean(g))
        xm = (np.abs(xo) + np.abs(stats[:, 2:3])) * stats[:, 3:4]
        tD += stats[:, 3:4] * xm * mean(g * xh)
    _near(_np(dx), ref["dx"], k * tD, what="dx")
    sums = {}
    if pre:
        sums["w_pre"], sums["b_pre"] = np.abs(b) * xm, np.abs(b)
    if post:
        ym = (np.abs(y) + np.abs(stats[:, :1])) * stats[:, 1:2]
        gg = 0.75 * (1.0 if gate is None else np.abs(gate[np.arange(T) // rows]))
        q = gg * np.abs(post[0]) * (tD + np.abs(ref["dx"]))
        _near(_np(dy), ref["dy"], k * stats[:, 1:2] * (q + ym * mean(q * ym) + mean(q)), out, "dy")
        sums["w_post"], sums["b_post"] = gg * tD * ym, gg * tD
        sums["gate"] = 0.75 * tD * (ym * np.abs(post[0]) + (0.0 if post[1] is None else np.abs(post[1])))
    for n, v in old.items():
        if n == "gate":
            t = np.zeros_like(ref["gate"])
            np.add.at(t, np.arange(T) // rows, sums[n])
        else:
            t = sums[n].sum(0)
        want = v + 0.5 * ref[n]
        _near(_np(acc[n]), want, k * (t + np.abs(v)), what=n)
    # written instead of added; in place; no gradient of the residual stream
    new = {n: torch.full_like(t, float("nan")) for n, t in acc.items()}
    dx2, dy2 = layer.block_norm_bwd(dxo, *args, dx=dxo, dtype=_dt(out), grads=layer.NormGrads(**new), **gkw)
    assert torch.equal(dx2, dx) and (dy is None or torch.equal(dy2, dy))
    for n, v in old.items():
        _near(_np(new[n]), ref[n], 2 * k * (sums[n].sum(0) if n != "gate" else t), what=n)
    ref0 = ol.block_norm_bwd(None if pre else np.zeros_like(a), b if pre else None, y, xo, stats, post, pre, **kw)
    dx0, _ = layer.block_norm_bwd(None, *args, **gkw) if pre else (None, None)
    if pre:
        _near(_np(dx0), ref0["dx"], k * tD, what="dx without dxo")


@pytest.mark.parametrize("ln,inp,out,saved", [(False, BF, BF, True), (True, F32, F32, False), (True, BF, F32, False), (False, F32, BF, True)])
@pytest.mark.parametrize("T,d,rows,slots", [(16400, 72, 8195, 4), (8200, 8, 8199, 4), (8195, 1000, 4097, 2), (6150, 2048, 2050, 1)])
def test_block_norm_backward_through_long_gate_rows(ln, inp, out, saved, T, d, rows, slots):
    """Few long gate rows, every one of them gone through by all blocks with 4, 2 and 1
    rows in turn, the last gate row short in some."""
    from paper_2608_07974_amd import zl
    blocks, gates = zl.zl_block_norm_workspace(T, d) // (4 * d), -(-T // rows)
    assert zl.zl_block_norm_workspace(T, d, rows) == (4 + gates * slots) * blocks * d  # what this plan needs
    test_block_norm_backward(ln, inp, out, saved, T, d, rows, "both", 0)


def test_block_norm_rows_of_one_value():
    """Rows without variance (and rows of zeros): 1 / sqrt(eps), no NaN; a NaN
    row stays its own."""
    layer = _L()
    T, d = 4, 96
    x = np.zeros((T, d))
    y = np.zeros((T, d))
    y[1] = 3.0
    y[3, 5] = np.nan
    w = (_vec(np.ones(d)), None)
    for ln in (False, True):
        xo, n, st = layer.block_norm(_dev(x), _dev(y), w, w, layernorm=ln)
        r = ol.block_norm(x[:3], y[:3], (np.ones(d), None), (np.ones(d), None), ln=ln)
        _near(_np(xo)[:3], r[0], 256 * U * (1 + np.abs(r[0])))
        _near(_np(st)[:3], r[2], 256 * U * np.maximum(np.abs(r[2]), 3.0))
        assert torch.isnan(xo[3]).all() and torch.isnan(n[3]).all() and torch.isfinite(n[:3]).all()


def test_block_norm_empty_batch():
    """No rows: sums over nothing are zero where written, kept where added."""
    layer = _L()
    d = 64
    e = torch.empty(0, d, device="cuda")
    w = (torch.ones(d, device="cuda"), None)
    for acc in (False, True):
        g = layer.NormGrads(w_post=torch.ones(d, device="cuda"), w_pre=torch.ones(d, device="cuda"))
        layer.block_norm_bwd(e, e, e, e, torch.empty(0, 4, device="cuda"), w, w, grads=g, accumulate=acc)
        assert (g.w_post == float(acc)).all() and (g.w_pre == float(acc)).all()
    assert layer.block_norm(e, e, w, w)[0].shape == (0, d)
    dw = layer.wgrad(e, layer.Packed.empty(0, 32), out=torch.ones(d, 32, device="cuda"))
    assert (dw == 0).all()
    dw = layer.wgrad(e, layer.Packed.empty(0, 32), out=torch.ones(d, 32, device="cuda"), accumulate=True)
    assert (dw == 1).all()
    p = layer.pack(e)
    assert layer.unpack(p).shape == (0, d) and layer.mlp_act(e, packed=layer.Packed.empty(0, d)).shape == (0, 32)
    assert layer.mlp_act_bwd(p, e[:, :32]).shape == (0, d)
    assert layer.rotary(e, torch.empty(1, 0, dtype=torch.int32, device="cuda"), bytes(8), 4, 16, 1e4).shape == (0, d)


@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("ld", [0, -8, 1 << 62])
def test_wgrad_of_no_tokens(dt, ld):
    """No tokens, no operands, any strides: zeros written, nothing added."""
    from paper_2608_07974_amd import zl
    for acc in (0, 1):
        dw = torch.full((64, 72), 3.0, device="cuda")
        zl.zl_wgrad_packed(0, 64, 72, 0, ld, zl.ZL_BF16 if dt == BF else zl.ZL_F32, zl.zl_packed(0, 0, ld, ld), dw.data_ptr(), 72,
                           accumulate=acc, stream=torch.cuda.current_stream().cuda_stream)
        assert (dw == 3.0 * acc).all()
    e = torch.empty(0, 64, dtype=_dt(dt), device="cuda")
    assert (_L().wgrad(e, _L().Packed.empty(0, 72)) == 0).all()


@pytest.mark.parametrize("T,d", [(1, 64), (3, 64), (5, 1000), (40, 64), (300, 2048), (9, 8192)])
@pytest.mark.parametrize("rows", [(1 << 63) - 1, 1 << 62, 1 << 61])
def test_one_gate_row_for_any_number_of_rows(T, d, rows):
    layer = _L()
    rng = _rng("gate", T, d)
    x, y, post, pre, gate = _norm_case(rng, T, d, True, "both", T, BF)
    xt, yt, gt = _dev(x, F32), _dev(y, BF), _vec(gate)
    got = []
    for n in (T, rows):
        kw = dict(gate=gt, gate_rows=n, scale=0.75, layernorm=True)
        xo, nn, st = layer.block_norm(xt, yt, _tv(post), _tv(pre), **kw)
        g = layer.NormGrads(*(torch.empty(d, device="cuda") for _ in range(4)), torch.empty(1, d, device="cuda"))
        got.append([xo, nn, st, *layer.block_norm_bwd(xt, nn, yt, xo, st, _tv(post), _tv(pre), grads=g, **kw), *g])
    for a, b in zip(*got):
        assert torch.equal(a, b)


# ---------------------------------------------------------- weight gradient
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("T,M,N,pad", [(1, 8, 8, 0), (33, 72, 40, 16), (31, 256, 256, 0), (32, 264, 48, 0), (64, 128, 1000, 0),
                                       (1000, 264, 520, 16), (5000, 64, 64, 0), (4096, 136, 768, 0), (700, 520, 2056, 0),
                                       (257, 2048, 264, 0), (1024, 768, 768, 0), (333, 4096, 3848, 0)])
@pytest.mark.parametrize("ws", [0, 1 << 22])
def test_wgrad(dt, T, M, N, pad, ws):
    layer = _L()
    rng = _rng("wgrad", T, M, N)
    dy = _dev(rng.standard_normal((T, M)), dt, pad)
    x = _acts(rng, T, N)
    p = _packed(x, pad)
    a, b = _np(dy), ol.packed(x)
    ref, mag = a.T @ b, np.abs(a).T @ np.abs(b)
    w = torch.full((ws,), float("nan"), device="cuda") if ws else None
    dw = layer.wgrad(dy, p, out=_out(M, N, F32, pad), workspace=w)
    _near(_np(dw), ref, (T + 8) * U * mag)
    assert np.linalg.norm(_np(dw) - ref) <= 2e-6 * np.linalg.norm(ref)
    again = layer.wgrad(dy, p, out=_out(M, N, F32, pad), workspace=w)
    assert torch.equal(dw, again)
    old = rng.standard_normal((M, N)).astype(np.float32)
    acc = layer.wgrad(dy, p, out=_dev(old, F32, pad), scale=0.25, accumulate=True, workspace=w)
    _near(_np(acc), old + 0.25 * ref, (T + 8) * U * (mag + np.abs(old)))
    if pad:
        assert torch.isnan(dw.as_strided((M, pad), (dw.stride(0), 1), N)).all()


@pytest.mark.parametrize("dt", [F32, BF])
def test_one_row_of_any_stride(dt):
    from paper_2608_07974_amd import zl
    layer = _L()
    rng = _rng("stride")
    dy, x = _dev(rng.standard_normal((1, 136)), dt), _packed(_acts(rng, 1, 264))
    ref, out = layer.wgrad(dy, x), torch.full((136, 264), float("nan"), device="cuda")
    for ld in (1 << 30, 1 << 31, 1 << 62):
        p = zl.zl_packed(x.codes.data_ptr(), x.scales.data_ptr(), ld, ld)
        zl.zl_wgrad_packed(1, 136, 264, dy.data_ptr(), ld, zl.ZL_BF16 if dt == BF else zl.ZL_F32, p, out.data_ptr(), 264,
                           stream=torch.cuda.current_stream().cuda_stream)
        assert torch.equal(out, ref)
        out.fill_(float("nan"))


def test_wgrad_non_finite_stays_in_its_column():
    """A NaN code and an infinite gradient reach their column and row only."""
    layer = _L()
    T, M, N = 100, 136, 264
    rng = _rng("nan")
    dy, x = rng.standard_normal((T, M)), rng.standard_normal((T, N))
    x[40, 100], dy[60, 7] = np.nan, np.inf
    for dt in (F32, BF):
        got = _np(layer.wgrad(_dev(dy, dt), _packed(x)))
        bad = ~np.isfinite(got)
        assert bad[:, 100].all() and bad[7].all() and bad.sum() == M + N - 1


@pytest.mark.parametrize("dt", [F32, BF])
def test_wgrad_takes_every_scale(dt):
    """Scale bytes that packing never writes: 255 is NaN, the smallest and the
    largest stand for what they say (values below the normal range may be
    dropped, as the bf16 products do)."""
    layer = _L()
    T, M, N = 40, 136, 256
    rng = _rng("scales")
    codes = torch.from_numpy(rng.integers(0, 127, (T, N)).astype(np.uint8)).cuda()
    scales = torch.full((T, N // 32), 127, dtype=torch.uint8, device="cuda")
    scales[0, 0], scales[1, 1], scales[2, 2], scales[3, 3] = 255, 1, 0, 240
    dy = np.abs(rng.standard_normal((T, M))) + 0.1
    dyt = _dev(dy, dt)
    got = _np(layer.wgrad(dyt, layer.Packed(codes, scales, N)))
    a, b = _np(dyt), ol.values(codes.cpu().numpy(), scales.cpu().numpy())
    assert np.isnan(got[:, :32]).all() and np.isfinite(got[:, 32:]).all()
    ref, mag = a.T @ b[:, 32:], np.abs(a).T @ np.abs(b[:, 32:])
    _near(got[:, 32:], ref, (T + 8) * U * mag)


def test_wgrad_in_segments_of_tokens():
    """Rows so far apart that 32-bit offsets do not reach the last: the sum
    goes on in further launches (200000 apart) or through 64-bit addresses
    (2^20 apart)."""
    layer = _L()
    rng = _rng("segments")
    for T, ld, M, N, ws in ((5000, 200000, 264, 72, 0), (5000, 200000, 64, 64, 1 << 20), (1100, 1 << 20, 72, 40, 1 << 20)):
        dy = torch.empty(T, ld, dtype=torch.bfloat16, device="cuda")[:, :M]
        dy.copy_(torch.from_numpy(rng.standard_normal((T, M)).astype(np.float32)))
        x = _acts(rng, T, N)
        p = _packed(x)
        a, b = _np(dy), ol.packed(x)
        old = rng.standard_normal((M, N)).astype(np.float32)
        w = torch.empty(ws, device="cuda") if ws else None
        for acc in (False, True):
            got = layer.wgrad(dy, p, out=_dev(old), scale=0.5, accumulate=acc, workspace=w)
            _near(_np(got), acc * old + 0.5 * a.T @ b, (T + 16) * U * (np.abs(a).T @ np.abs(b) + np.abs(old)))
        del dy, got


@pytest.mark.parametrize("dt,M", [(F32, 65536 * 128 + 8), (BF, 65535 * 128 + 72)])
def test_wgrad_of_more_than_65535_tile_rows(dt, M):
    layer = _L()
    rng = _rng("rows", M)
    T, N = 3, 8
    dy = torch.empty(T, M, dtype=_dt(dt), device="cuda")
    dy.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    x = _packed(_acts(rng, T, N))
    dw = layer.wgrad(dy, x, out=torch.full((M, N), float("nan"), device="cuda"))
    v = torch.from_numpy(ol.values(*_bytes(x, T, N))).cuda()
    d = dy.double()
    ref, mag = (sum(a[t][:, None] * b[t] for t in range(T)) for a, b in ((d, v), (d.abs(), v.abs())))
    assert ((dw - ref).abs() <= (T + 8) * U * mag).all()


@pytest.mark.parametrize("ld,T", [(262144, 3100), (524288, 1400), (690000, 1111)])
def test_wgrad_of_wide_bf16_rows_stays_on_bf16_tiles(ld, T):
    """A launch reaches 2^31 bytes, of rows as wide as a large vocabulary a few hundred
    to a few thousand tokens: as many launches as it takes, each what a call of its
    own on narrow rows gives, bit for bit (fp32 tiles add up in another order)."""
    layer = _L()
    rng = _rng("wide", ld)
    M, N = 264, 72
    near = _dev(rng.standard_normal((T, M)), BF)
    dy = torch.empty(T, ld, dtype=torch.bfloat16, device="cuda")[:, :M]
    dy.copy_(near)
    p = _packed(_acts(rng, T, N))
    step = ((2 ** 31 - 1024) // (2 * ld) - 1024) // 32 * 32
    assert 256 <= step < T
    want = torch.zeros(M, N, device="cuda")
    for t in range(0, T, step):
        e = min(T, t + step)
        layer.wgrad(near[t:e], layer.Packed(p.codes[t:e], p.scales[t:e], N), out=want, accumulate=t > 0)
    assert torch.equal(layer.wgrad(dy, p), want)


def test_rows_beyond_32_bit_offsets():
    """Four rows 2^30 bytes and more apart through every other operator."""
    layer = _L()
    rng = _rng("far")
    T, d, far = 4, 72, (1 << 29) + 8

    def wide(a, dt=F32, ld=far):
        t = torch.empty(T, ld, dtype=_dt(dt), device="cuda")[:, : a.shape[1]]
        t.copy_(torch.from_numpy(np.asarray(a, np.float32)))
        return t

    x, y = _acts(rng, T, d), rng.standard_normal((T, d))
    xw, yw = wide(x), wide(y, BF)
    p = layer.Packed(torch.empty(T, 1 << 30, dtype=torch.uint8, device="cuda"), torch.empty(T, 1 << 30, dtype=torch.uint8, device="cuda"), d)
    layer.pack(xw, out=p)
    _same_codes(_bytes(p, T, d), ol.pack(_np(xw)))
    back = layer.unpack(p, out=wide(0 * x))
    assert np.array_equal(_np(back), ol.packed(_np(xw)))
    assert torch.equal(layer.mlp_act(xw, "gelu", act=back), layer.mlp_act(xw.contiguous(), "gelu"))
    assert torch.equal(layer.mlp_act_bwd(xw, xw, "gelu", dh=back), layer.mlp_act_bwd(xw.contiguous(), xw.contiguous(), "gelu"))
    w = (_vec(1 + 0.1 * rng.standard_normal(d)), None)
    near = layer.block_norm(xw.contiguous(), yw.contiguous(), w, w)
    got = layer.block_norm(xw, yw, w, w, n=wide(y, BF))
    assert all(torch.equal(a, b) for a, b in zip(got, near))
    args = lambda f: (f(xw), f(yw), f(yw), f(got[0]), near[2], w, w)  # noqa: E731
    assert all(torch.equal(a, b) for a, b in zip(layer.block_norm_bwd(*args(lambda t: t)), layer.block_norm_bwd(*args(lambda t: t.contiguous()))))
    pos = torch.arange(T, dtype=torch.int32, device="cuda")[None]
    assert torch.equal(layer.rotary(xw, pos, bytes(12), 3, 24, 1e4, out=back), layer.rotary(xw.contiguous(), pos, bytes(12), 3, 24, 1e4))


# ------------------------------------------------------------------- rotary
@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("T,H,hd,rot,axes,pad", [
    (1, 1, 16, 16, 1, 0), (8, 40, 128, 128, 3, 0), (5, 3, 64, 32, 2, 16), (301, 6, 128, 128, 3, 8), (17, 2, 16, 8, 4, 0),
    (4, 3, 6, 4, 2, 0), (9, 2, 256, 256, 16, 0), (33, 5, 32, 2, 1, 3), (2000, 1, 64, 64, 3, 0), (3, 7, 80, 80, 3, 16)])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotary(dt, T, H, hd, rot, axes, pad, inverse):
    layer = _L()
    rng = _rng("rot", T, H, hd, rot)
    x = _dev(rng.standard_normal((T, H * hd + pad)), dt)
    pos = rng.integers(0, 100000, (axes, T)).astype(np.int32)
    pos[:, 0] = [(-1) ** a * (2 ** 31 - 1 - a) for a in range(axes)]
    which = bytes(int(a) for a in rng.integers(0, axes, rot // 2))
    out = _out(T, H * hd, dt, pad)
    pt = torch.from_numpy(pos).cuda()
    got = layer.rotary(x, pt, which, H, hd, 5e5, inverse=inverse, out=out)
    assert got is out
    v = _np(x)[:, : H * hd]
    ref = ol.rotary(v, pos, which, H, hd, 5e5, inverse=inverse)
    m = np.abs(v).reshape(T, H, hd)
    pair = np.concatenate([m[..., : rot // 2] + m[..., rot // 2: rot]] * 2 + [0 * m[..., rot:]], -1).reshape(T, -1)
    # far positions: 64 bits leave pos 2^-53 of a turn, twice (product, frequency), times 2 pi
    far = np.concatenate([np.repeat(np.abs(pos.astype(np.float64)).max(0)[:, None] * 2.0 ** -49, H * hd, 1)])
    _near(_np(got)[:, : H * hd], ref, (16 * U + far) * pair, dt)
    if pad:
        assert torch.isnan(out.as_strided((T, pad), (out.stride(0), 1), H * hd)).all()
    same = layer.rotary(x, pt, which, H, hd, 5e5, inverse=inverse, out=x)  # in place
    assert torch.equal(same[:, : H * hd], out[:, : H * hd])


# ------------------------------------------------------- streams and graphs
def _everything(layer, s):
    """Every operator once, as a backward and forward of small sizes; outputs in a list."""
    p = layer.pack(s["x"], out=s["p"])
    act = layer.mlp_act(s["h"], act=s["act"], packed=s["hp"])
    dh = layer.mlp_act_bwd(s["hp"], s["act"], dh=s["dh"], act=s["act2"])
    layer.block_norm(s["x"], s["y"], s["w"], s["w"], gate=s["gate"], gate_rows=40, xo=s["xo"], n=s["n"], stats=s["st"],
                     y_packed=s["yp"], n_packed=s["np"])
    layer.block_norm_bwd(s["x"], s["y"], s["yp"], s["xo"], s["st"], s["w"], s["w"], gate=s["gate"], gate_rows=40, dx=s["dx"],
                         dy=s["dy"], grads=s["g"], workspace=s["ws"])
    dw = layer.wgrad(s["dy"], s["np"], out=s["dw"], workspace=s["ws2"])
    r = layer.rotary(s["y"], s["pos"], bytes(i % 3 for i in range(32)), 4, 64, 1e4, out=s["r"])
    return [layer.unpack(p, out=s["x2"]), act, dh, s["act2"], s["xo"], s["n"], s["st"], s["dx"], s["dy"], *s["g"], dw, r]


def _some(layer, seed, T=200, d=256):
    from paper_2608_07974_amd import zl
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *sh: torch.randn(*sh, device="cuda", generator=g)  # noqa: E731
    e = lambda *sh: torch.empty(*sh, device="cuda")  # noqa: E731
    P = layer.Packed.empty
    return dict(x=r(T, d), h=r(T, 2 * d), y=r(T, d), gate=r(T // 40, d), w=(r(d), None), p=P(T, d), act=e(T, d), hp=P(T, 2 * d),
                dh=e(T, 2 * d), act2=e(T, d), xo=e(T, d), n=e(T, d), st=e(T, 4), yp=P(T, d), np=P(T, d), dx=e(T, d),
                dy=e(T, d), g=layer.NormGrads(w_post=e(d), w_pre=e(d), gate=e(T // 40, d)),
                ws=e(zl.zl_block_norm_workspace(T, d, 40)), dw=e(d, d), ws2=e(1 << 20), x2=e(T, d), r=e(T, d),
                pos=torch.randint(0, 4096, (3, T), dtype=torch.int32, device="cuda", generator=g))


def test_captured_and_on_another_stream():
    """All operators in a graph, replayed on new inputs between eager work, and
    on a stream of their own: the eager results, bit for bit."""
    layer = _L()
    a, b = _some(layer, 1), _some(layer, 2)
    want_a = [t.clone() for t in _everything(layer, a) if t is not None]
    want_b = [t.clone() for t in _everything(layer, b) if t is not None]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = [t.clone() for t in _everything(layer, a) if t is not None]
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(x, y) for x, y in zip(got, want_a))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = [t for t in _everything(layer, a) if t is not None]
    inputs = lambda s: [s["x"], s["h"], s["y"], s["gate"], s["pos"], s["w"][0]]  # noqa: E731
    keep = [t.clone() for t in inputs(a)]
    for src, want in ((keep, want_a), (inputs(b), want_b), (keep, want_a)):
        for t, v in zip(inputs(a), src):
            t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want))
        again = [t for t in _everything(layer, b) if t is not None]  # eager work between the replays
        assert all(torch.equal(x, y) for x, y in zip(again, want_b))


def test_torchs_default_type_does_not_matter():
    """With bf16 as torch's default type, tensors and scratch that the calls make
    themselves are what they are without: the results, bit for bit."""
    layer = _L()
    s = _some(layer, 5)

    def calls():
        xo, n, st = layer.block_norm(s["x"], s["y"], s["w"], s["w"], gate=s["gate"], gate_rows=40)
        g = layer.NormGrads(*(None if t is None else torch.empty_like(t) for t in s["g"]))
        dxy = layer.block_norm_bwd(s["x"], n, s["y"], xo, st, s["w"], s["w"], gate=s["gate"], gate_rows=40, grads=g)
        return [xo, n, st, *dxy, *(t for t in g if t is not None), layer.wgrad(s["y"], layer.pack(s["x"]))]

    want = calls()
    torch.set_default_dtype(torch.bfloat16)
    try:
        got = calls()
    finally:
        torch.set_default_dtype(torch.float32)
    assert all(a.dtype == b.dtype and torch.equal(a, b) for a, b in zip(got, want))


def test_in_an_autograd_function():
    """A function whose forward and backward are these calls, between operations that
    autograd records."""
    layer = _L()

    class Act(torch.autograd.Function):
        @staticmethod
        def forward(ctx, h):
            ctx.h = layer.Packed.empty(*h.shape)
            return layer.mlp_act(h, packed=ctx.h)

        @staticmethod
        def backward(ctx, da):
            return layer.mlp_act_bwd(ctx.h, da.contiguous())

    x, w = _randn(40, 64, F32), _randn(40, 32, F32, 8)
    leaf = x.clone().requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        layer.mlp_act(leaf * 2.0)
    y = Act.apply(leaf * 2.0)
    (y * w).sum().backward()
    h = _np(x) * 2.0
    _near(_np(y), ol.mlp_act(h, "swiglu"), (2 * np.abs(h[:, :32]) + 16) * U * np.abs(ol.mlp_act(h, "swiglu")) + 2.0 ** -126)
    want = 2.0 * layer.mlp_act_bwd(layer.pack(x * 2.0), w)
    assert torch.equal(leaf.grad, want)


# ------------------------------------------------------------ a whole layer
def test_a_layer_with_packed_activations():
    """One decoder layer with norms around both blocks, gated residuals and
    positions on three axes, its saved activations in 8 bits: forward and
    backward through the operators and the library's products and attention,
    against the oracle that packs the same tensors.  fp32 throughout; values at
    the border of two codes may round either way (one in 2^16 at most, by a
    sixteenth): 2e-3 in the norm."""
    layer = _L()
    from paper_2608_07974_amd import zl
    rng = _rng("layer")
    B, S, Hq, Hkv, hd, ff, eps = 2, 24, 4, 2, 16, 96, 1e-5
    d, T, theta = Hq * hd, B * S, 1e4
    nq = (Hq + 2 * Hkv) * hd
    lens, which = np.array([S, 17]), bytes([0, 1, 2, 0, 1, 2, 0, 0])
    pos = rng.integers(0, 30, (3, T)).astype(np.int32)
    W = {k: 0.15 * rng.standard_normal(s) for k, s in dict(qkv=(nq, d), o=(d, d), up=(2 * ff, d), dn=(d, ff)).items()}
    nw = {k: 1 + 0.1 * rng.standard_normal(d) for k in ("n1", "p1", "n2", "p2")}
    gate = {k: 0.6 + 0.2 * rng.standard_normal((B, d)) for k in ("1", "2")}
    x, dout = rng.standard_normal((T, d)), rng.standard_normal((T, d))
    W, nw, gate = ({k: np.float32(v).astype(np.float64) for k, v in t.items()} for t in (W, nw, gate))
    x, dout = np.float32(x).astype(np.float64), np.float32(dout).astype(np.float64)

    # ---- oracle
    post = lambda k: (nw[k], None)  # noqa: E731
    kw1, kw2 = (dict(gate=gate[k], gate_rows=S, scale=0.8) for k in ("1", "2"))
    _, n1, st0 = ol.block_norm(x, None, None, post("n1"))
    qkv = n1 @ W["qkv"].T
    rot = lambda v, inv=False: np.concatenate([ol.rotary(v[:, : (Hq + Hkv) * hd], pos, which, Hq + Hkv, hd, theta, inv),
                                               v[:, (Hq + Hkv) * hd:]], 1)  # noqa: E731
    qr = rot(qkv).reshape(B, S, Hq + 2 * Hkv, hd)
    q, k, v = qr[:, :, :Hq], qr[:, :, Hq: Hq + Hkv], qr[:, :, Hq + Hkv:]
    o4, cache = ops.attention_fwd(q, k, v, lens)
    o = o4.reshape(T, d)
    y1 = o @ W["o"].T
    x1, n2, st1 = ol.block_norm(x, y1, post("p1"), post("n2"), **kw1)
    h = n2 @ W["up"].T
    y2 = ol.mlp_act(h, "swiglu") @ W["dn"].T
    x2, _, st2 = ol.block_norm(x1, y2, post("p2"), None, **kw2)
    g2 = ol.block_norm_bwd(dout, None, ol.packed(y2), x2, st2, post("p2"), None, **kw2)
    hp = ol.packed(h)
    dh = ol.mlp_act_bwd(hp, g2["dy"] @ W["dn"], "swiglu")
    g1 = ol.block_norm_bwd(g2["dx"], dh @ W["up"], ol.packed(y1), x1, st1, post("p1"), post("n2"), **kw1)
    dq, dk, dv = ops.attention_bwd((g1["dy"] @ W["o"]).reshape(B, S, Hq, hd), cache)
    dqkv = rot(np.concatenate([dq, dk, dv], 2).reshape(T, nq), True)
    g0 = ol.block_norm_bwd(g1["dx"], dqkv @ W["qkv"], None, x, st0, None, post("n1"))
    want = dict(out=x2, dx=g0["dx"], w_dn=g2["dy"].T @ ol.mlp_act(hp, "swiglu"), w_up=dh.T @ ol.packed(n2),
                w_o=g1["dy"].T @ o, w_qkv=dqkv.T @ ol.packed(n1), n1=g0["w_pre"], p1=g1["w_post"], n2=g1["w_pre"],
                p2=g2["w_post"], gate1=g1["gate"], gate2=g2["gate"])

    # ---- the library
    s = torch.cuda.current_stream().cuda_stream

    def mm(a, b, ta=False, tb=False):
        """a (or a^T) times b^T (or b)."""
        M, K = (a.shape[1], a.shape[0]) if ta else a.shape
        N = b.shape[1] if tb else b.shape[0]
        c = torch.empty(M, N, device="cuda")
        zl.zl_kernel_gemm(M, N, K, a.data_ptr(), a.stride(0), not ta, b.data_ptr(), b.stride(0), not tb, c.data_ptr(), N,
                          zl.ZL_F32, s)
        return c

    w = {k: _dev(v) for k, v in W.items()}
    nv = {k: (_vec(v), None) for k, v in nw.items()}
    gt = {k: _vec(v) for k, v in gate.items()}
    P = layer.Packed.empty
    pt, lt = torch.from_numpy(pos).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    kw1, kw2 = (dict(gate=gt[k], gate_rows=S, scale=0.8, eps=eps) for k in ("1", "2"))
    n1p, n2p, y1p, y2p, hpk = P(T, d), P(T, d), P(T, d), P(T, d), P(T, 2 * ff)
    xt = _dev(x)
    _, tn1, ts0 = layer.block_norm(xt, None, None, nv["n1"], dtype=torch.float32, n_packed=n1p)
    tq = mm(tn1, w["qkv"])
    layer.rotary(tq, pt, which, Hq + Hkv, hd, theta, out=tq)
    to, lse = torch.empty(T, d, device="cuda"), torch.empty(B, Hq, S, device="cuda")
    at = lambda t: (t.data_ptr(), t.data_ptr() + Hq * hd * 4, t.data_ptr() + (Hq + Hkv) * hd * 4)  # noqa: E731
    zl.zl_kernel_attention(B, S, Hq, Hkv, hd, *at(tq), nq, lt.data_ptr(), to.data_ptr(), lse.data_ptr(), 0, 0, 0, 0, 0,
                           zl.ZL_F32, 0, s)
    tx1, tn2, ts1 = layer.block_norm(xt, mm(to, w["o"]), nv["p1"], nv["n2"], y_packed=y1p, n_packed=n2p, **kw1)
    ta = layer.mlp_act(mm(tn2, w["up"]), packed=hpk)
    tx2, _, ts2 = layer.block_norm(tx1, mm(ta, w["dn"]), nv["p2"], None, y_packed=y2p, **kw2)
    e = lambda *sh: torch.empty(*sh, device="cuda")  # noqa: E731
    gr2, gr1 = layer.NormGrads(w_post=e(d), gate=e(B, d)), layer.NormGrads(w_post=e(d), w_pre=e(d), gate=e(B, d))
    gr0 = layer.NormGrads(w_pre=e(d))
    tdx, tdy2 = layer.block_norm_bwd(_dev(dout), None, y2p, None, ts2, nv["p2"], None, grads=gr2, **kw2)
    act = e(T, ff)
    tdh = layer.mlp_act_bwd(hpk, mm(tdy2, w["dn"], tb=True), act=act)
    got = dict(out=tx2, w_dn=mm(tdy2, act, ta=True, tb=True), w_up=layer.wgrad(tdh, n2p))
    tdx, tdy1 = layer.block_norm_bwd(tdx, mm(tdh, w["up"], tb=True), y1p, tx1, ts1, nv["p1"], nv["n2"], dx=tdx, grads=gr1, **kw1)
    got["w_o"] = mm(tdy1, to, ta=True, tb=True)
    tdo, tdq, delta = mm(tdy1, w["o"], tb=True), e(T, nq), e(B, Hq, S)
    zl.zl_kernel_attention(B, S, Hq, Hkv, hd, *at(tq), nq, lt.data_ptr(), to.data_ptr(), lse.data_ptr(), tdo.data_ptr(),
                           *at(tdq), delta.data_ptr(), zl.ZL_F32, 1, s)
    layer.rotary(tdq, pt, which, Hq + Hkv, hd, theta, inverse=True, out=tdq)
    got["w_qkv"] = layer.wgrad(tdq, n1p)
    got["dx"], _ = layer.block_norm_bwd(tdx, mm(tdq, w["qkv"], tb=True), None, xt, ts0, None, nv["n1"], dx=tdx, grads=gr0, eps=eps)
    got.update(n1=gr0.w_pre, p1=gr1.w_post, n2=gr1.w_pre, p2=gr2.w_post, gate1=gr1.gate, gate2=gr2.gate)
    assert set(got) == set(want)
    for key in want:
        err = np.linalg.norm(_np(got[key]) - want[key]) / np.linalg.norm(want[key])
        assert err < 2e-3, (key, err)
    assert np.linalg.norm(_np(tx2) - x2) <= 1e-5 * np.linalg.norm(x2)  # nothing packed on the way forward
