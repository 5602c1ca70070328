"""The losses over a vocabulary on the GPU (include/zl_loss.h, through loss.py)
against the fp64 oracle (oracle/loss.py).

Tolerances, with u = 2^-24 (half a step of fp32), M the largest finite magnitude among
a row's logits and teacher's values (over the temperature where that is below 1) and
its rests:
  log-sums: a term's exponent is a difference (u) times a constant (u), so the term
    is off by (2 a + 4) u at distance a below the maximum, which over the terms'
    weights makes at most (2 log V + 4) u < 32 u; V / 256 terms one after the other,
    rescales and 16 levels of sums: (V / 256 + 120) u in all, and 2 u of the value.
  loss: two log-sums, their differences and k products: LOG = (V / 256 + 200) (1 + M) u
    of each term's weight.
  gradient of the logits: q = exp(z - lse) carries the log-sum's error, its own exponent's
    and 8 u: 2 LOG of (q + target), and half a step of bf16, 2^-8 of the value, where
    the output is bf16.
  logits formed by the head: d products added in any order: ez = (d + 8) u sum |x w|;
    log-sums shift by at most ez, terms by 2 ez / tau.
  dx, dw: the error of dL/dz (with bf16 its rounding, 2^-8 of the value) through the
    other factor's magnitudes, and the sum's own (n + 64) u for n terms.
"""
import zlib

import numpy as np
import pytest

from oracle import loss as ol

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
BF, F32 = "bf16", "f32"


def _L():
    from paper_2608_07974_amd import loss
    return loss


def _dt(name):
    return torch.bfloat16 if name == BF else torch.float32


def _rng(*key):
    return np.random.default_rng([zlib.crc32(k.encode()) if isinstance(k, str) else int(k) for k in key])


def _np(t):
    return t.detach().double().cpu().numpy()


def _dev(a, dt=F32, pad=0, skip=0):
    """A device matrix that starts `skip` elements into rows `pad` longer, which hold NaN;
    and its values as stored."""
    a = np.atleast_2d(np.asarray(a, np.float64))
    t = torch.full((a.shape[0], skip + a.shape[1] + pad), float("nan"), dtype=_dt(dt), device="cuda")
    t = t[:, skip: skip + a.shape[1]]
    t.copy_(torch.from_numpy(a.astype(np.float32)))
    return t


def _f32(a):
    return None if a is None else torch.tensor(np.asarray(a, np.float32), device="cuda")


def _i32(a):
    return None if a is None else torch.tensor(np.asarray(a, np.int32), device="cuda")


def _near(got, ref, tol, dt=F32, what=""):
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    # fp32 has no value below 2^-149 and the exponential none below 2^-126: each of two
    # terms (factors at most 1) may vanish there
    tol = np.broadcast_to(tol, ref.shape) + 2.0 ** -125
    if dt == BF:
        tol = tol + (np.abs(ref) + tol) * 2.0 ** -8
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), what
    inf = ~fine & ~np.isnan(ref)
    assert np.array_equal(got[inf], ref[inf]), what
    over = np.where(fine, np.abs(np.where(fine, got, 0) - np.where(fine, ref, 0)) - tol, 0.0)
    if over.size:
        at = np.unravel_index(over.argmax(), over.shape)
        worst = (what, at, float(got[at]), float(ref[at]), float(tol[at]))
        assert bool(over[at] <= 0), worst


def _untouched(t):
    """Nothing was written around the columns of t."""
    base = t._base if t._base is not None else t
    base = base.clone()
    lo = t.storage_offset() % base.stride(0)
    base[:, lo: lo + t.shape[1]] = float("nan")
    assert bool(torch.isnan(base.float()).all())


def _targets(rng, z, k, rest, hard, tau, near=0.9):
    """Labels and a teacher near logits z with what real ones have: ignored labels, rows
    without a teacher, absent and repeated ids, ids at the vocabulary's ends, the label
    among the ids."""
    T, V = z.shape
    y = ids = values = r = None
    if hard:
        y = rng.integers(0, V, T)
        y[::7] = -100
        if T > 2:
            y[2] = V  # outside as well
    if k:
        t = near * np.where(np.isfinite(z), z, -5.0) + rng.standard_normal(z.shape)
        ids, values, r = ol.top_logits(t, k, tau)
        if T > 3 and not rest:
            ids[3, k // 2:] = -1
        if T > 4:
            ids[4] = -1
        if T > 5 and k > 2:
            ids[5, 1] = ids[5, 0]
            ids[5, 2] = V + 3
        if T > 6 and k > 1 and hard:
            if y[6] not in ids[6]:
                ids[6, 1] = y[6]
            else:
                y[6] = ids[6, 1]
        if T > 8 and k > 1:
            ids[8, :2] = [V - 1, 0] if V > 1 else ids[8, :2]
        values = values.astype(np.float32).astype(np.float64)
        r = r.astype(np.float32).astype(np.float64) if rest else None
    return y, ids, values, r


def _mag(z, values, rest, tau):
    fin = lambda a: np.abs(np.where(np.isfinite(a), a, 0.0))  # noqa: E731
    z = np.where(np.abs(z) > 1e30, 0.0, z)  # the type's lowest values: terms of weight 0
    m = fin(z).max(1) / min(1.0, tau)
    if values is not None:
        m = np.maximum(m, fin(values).max(1) / min(1.0, tau))
    return m if rest is None else np.maximum(m, fin(rest))


def _spread(z, y, ids, values, rest, alpha, tau):
    """(a q1 + b tau (qt + target)) of every logit: what relative errors of dL/dz apply to."""
    a, b = ol.weights(y, ids, alpha)
    out = np.zeros(z.shape)
    for t in range(z.shape[0]):
        if y is not None and 0 <= y[t] < z.shape[1]:
            out[t] += a * np.exp(z[t] - ol.lse(z[t]))
            out[t, y[t]] += a
        row = None if ids is None else ol.teacher_row(z.shape[1], ids[t], values[t], None if rest is None else rest[t], tau)
        if row is not None:
            q = np.exp(z[t] / tau - ol.lse(z[t] / tau))
            out[t] += b * tau * 2 * q
            out[t, row[0]] += b * tau * row[1]
            if rest is not None:
                other = np.ones(z.shape[1], bool)
                other[row[0]] = False
                if q[other].sum() > 0:
                    out[t, other] += b * tau * row[2] * q[other] / q[other].sum()
    return out


def _teacher(ids, values, rest):
    return None if ids is None else _L().TopLogits(_i32(ids), _f32(values), _f32(rest))


# ------------------------------------------------------------- loss of logits
# V below a group, of one group, odd, of several steps; row starts of every alignment
SIZES = [(1, 1, 1), (3, 2, 1), (9, 7, 3), (2, 8, 8), (12, 64, 5), (11, 255, 16), (9, 1000, 256), (5, 4099, 33)]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("hard,soft,rest,tau", [(1, 0, 0, 1.0), (0, 1, 0, 1.0), (0, 1, 1, 2.0), (1, 1, 0, 1.0), (1, 1, 0, 2.0),
                                                (1, 1, 1, 1.0), (1, 1, 1, 0.5)])
@pytest.mark.parametrize("T,V,k", SIZES)
def test_logit_loss(T, V, k, hard, soft, rest, tau, dt):
    rng = _rng("logit", T, V, k, hard, soft, rest, int(tau * 2), dt)
    for skip, pad in ((0, 0), (1, 0), (3, 4)):
        zd = _dev(rng.standard_normal((T, V)) * 3, dt, pad, skip)
        z = _np(zd)
        y, ids, values, r = _targets(rng, z, k if soft else 0, rest, hard, tau)
        kw = dict(labels=_i32(y), teacher=_teacher(ids, values, r), alpha=0.3, temperature=tau)
        loss, stats = _L().logit_loss(zd, **kw)
        g = rng.standard_normal(T)
        g = g.astype(np.float32).astype(np.float64)
        out = _dev(np.zeros((T, V)), dt, pad, skip)
        dz = _L().logit_loss_bwd(zd, stats, dloss=_f32(g), scale=0.5, out=out, **kw)
        ref, rs, rdz = ol.loss(z, y, ids, values, r, 0.3, tau)
        log = (V / 256 + 200) * (1 + _mag(z, values, r, tau)) * U
        a, b = ol.weights(y, ids, 0.3)
        _near(_np(loss), ref, (a + b * tau * tau) * 2 * log, what="loss")
        _near(_np(stats), rs, log[:, None], what="stats")
        f = 0.5 * np.abs(g)[:, None]
        _near(_np(dz), 0.5 * g[:, None] * rdz, f * _spread(z, y, ids, values, r, 0.3, tau) * 2 * log[:, None], dt, "dz")
        _untouched(zd)
        _untouched(dz)
        none = np.zeros(T, bool)
        for t in range(T):
            none[t] = (y is None or not 0 <= y[t] < V) and \
                (ids is None or ol.teacher_row(V, ids[t], values[t], None if r is None else r[t], tau) is None)
        assert not np.any(_np(dz)[none]) and not np.any(_np(loss)[none])


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("rest", [False, True])
def test_logit_loss_large_vocabulary(dt, rest):
    """Every step of the streaming loop, more groups than the test of named columns has
    bits for, and other output alignment than the input's."""
    V = 300001
    rng = _rng("large", dt, rest)
    zd = _dev(rng.standard_normal((3, V)) * 3, dt, 0, 5)
    z = _np(zd)
    y, ids, values, r = _targets(rng, z, 100, rest, True, 2.0)
    kw = dict(labels=_i32(y), teacher=_teacher(ids, values, r), temperature=2.0)
    loss, stats = _L().logit_loss(zd, **kw)
    out = _dev(np.zeros((3, V)), dt, 2, 2)
    dz = _L().logit_loss_bwd(zd, stats, out=out, **kw)
    ref, rs, rdz = ol.loss(z, y, ids, values, r, 0.5, 2.0)
    log = (V / 256 + 200) * (1 + _mag(z, values, r, 2.0)) * U
    _near(_np(loss), ref, 5 * log, what="loss")
    _near(_np(stats), rs, log[:, None], what="stats")
    _near(_np(dz), rdz, _spread(z, y, ids, values, r, 0.5, 2.0) * 2 * log[:, None], dt, "dz")
    _untouched(dz)


@pytest.mark.parametrize("dt", [BF, F32])
def test_logit_loss_in_place_and_repeatable(dt):
    rng = _rng("place", dt)
    z = _dev(rng.standard_normal((40, 5003)) * 3, dt)
    y, ids, values, r = _targets(rng, _np(z), 64, True, True, 2.0)
    kw = dict(labels=_i32(y), teacher=_teacher(ids, values, r), temperature=2.0)
    a, b = _L().logit_loss(z, **kw), _L().logit_loss(z, **kw)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    apart = _L().logit_loss_bwd(z, a[1], **kw)
    same = z.clone()
    assert _L().logit_loss_bwd(same, a[1], out=same, **kw) is same
    assert torch.equal(same, apart)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("rest", [False, True])
def test_logit_loss_masked_logits(dt, rest):
    """Columns at -inf and at the type's lowest value, rows far from 0, a student as sure as
    the type allows; rows without targets may hold anything."""
    low = torch.finfo(_dt(dt)).min
    V, k = 515, 4
    rng = _rng("mask", dt, rest)
    z = rng.standard_normal((8, V))
    z[0, 5:] = -np.inf      # five columns left
    z[1, ::2] = low
    z[2] += 3000.0          # an offset that exp cannot take
    z[3] -= 3000.0
    z[4, 7] = 200.0         # sure of a column the teacher names
    z[5] = low              # every column masked alike
    z[6] = np.nan
    z[7] = np.inf
    zd = _dev(z, dt)
    z = _np(zd)
    ids = np.tile(np.array([0, 1, 3, 7], np.int32), (8, 1))
    values = np.tile(np.array([2.0, 1.0, 0.5, -np.inf]), (8, 1))
    values[4, 3] = 1.0
    ids[6:] = -1
    values[6:] = np.nan     # no one reads them
    y = np.array([3, 1, 2, 3, 7, 9, -1, V], np.int32)
    r = np.full(8, -1.0) if rest else None
    kw = dict(labels=_i32(y), teacher=_teacher(ids, values, r))
    loss, stats = _L().logit_loss(zd, **kw)
    dz = _L().logit_loss_bwd(zd, stats, **kw)
    with np.errstate(invalid="ignore", divide="ignore"):
        ref, rs, rdz = ol.loss(np.where(np.isfinite(z) | (z == -np.inf), z, 0.0), y, ids, values, r)
    with np.errstate(invalid="ignore"):
        log = (V / 256 + 200) * (1 + _mag(z, np.nan_to_num(values, neginf=0.0), r, 1.0)) * U
    # row 5: logits of magnitude 2^127, whose log-sum's log V is below half a step
    log[5] = np.abs(low) * 2 * U
    # row 1: the teacher names a masked column, whose logit enters the loss as p z, not
    # through an exponential: p is off by 4 u, the product and the sum over ids by u each
    _near(_np(loss), ref, 3 * log + 8 * U * np.abs(ref), what="loss")
    _near(_np(stats), rs, log[:, None], what="stats")
    with np.errstate(invalid="ignore"):
        s = _spread(np.where(np.isfinite(z) | (z == -np.inf), z, 0.0), y, ids, np.nan_to_num(values, neginf=-np.inf), r,
                    0.5, 1.0)
    keep = np.array([0, 1, 2, 3, 4, 6, 7])
    _near(_np(dz)[keep], rdz[keep], s[keep] * 2 * log[keep, None], dt, "dz")
    assert bool(torch.isfinite(dz[5].float()).all())
    assert not _np(dz)[6:].any() and not _np(loss)[6:].any() and not _np(stats)[6:].any()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("tau", [2.0, 4.0, 10.0, 0.5])
@pytest.mark.parametrize("T,V,head", [(6, 8192, 2048), (6, 30000, 16384), (2100, 4000, 1024), (6, 1500, 512)])
def test_logit_loss_of_a_masked_head(T, V, head, tau, rest, dt):
    """A row's first columns, as many as a block looks at for a reference, are all at -inf and
    the others far from 0, where exp(z) or its square leaves fp32 and exp(z / tau) does not."""
    rng = _rng("masked head", T, V, int(tau * 2), rest, dt)
    far = np.array([-90.0, -100.0, -130.0, -200.0, -700.0, 120.0])
    z = rng.standard_normal((6, V)) + far[:, None]
    z[:, :head] = -np.inf
    zd = torch.zeros(T, V, dtype=_dt(dt), device="cuda")
    zd[:6] = _dev(z, dt)
    z = _np(zd[:6])
    y = rng.integers(head, V, T)
    ids = rng.permuted(np.tile(np.arange(head, V), (T, 1)), axis=1)[:, :5]
    ids[1, 2] = y[1]
    values = rng.standard_normal((T, 5)).astype(np.float32).astype(np.float64)
    r = rng.standard_normal(T).astype(np.float32).astype(np.float64) if rest else None
    kw = dict(labels=_i32(y), teacher=_teacher(ids, values, r), alpha=0.3, temperature=tau)
    loss, stats = _L().logit_loss(zd, **kw)
    dz = _L().logit_loss_bwd(zd, stats, **kw)
    six = (z, y[:6], ids[:6], values[:6], r[:6] if rest else None, 0.3, tau)
    ref, rs, rdz = ol.loss(*six)
    log = (V / 256 + 200) * (1 + _mag(z, values[:6], six[4], tau)) * U
    _near(_np(loss[:6]), ref, (0.3 + 0.7 * tau * tau) * 2 * log, what="loss")
    _near(_np(stats[:6]), rs, log[:, None], what="stats")
    _near(_np(dz[:6]), rdz, _spread(*six) * 2 * log[:, None], dt, "dz")


def _label_parts(z, y):
    """CE and 1 - q_y of every row from what the other columns weigh beside the label: both
    to 64 bits of their own, however sure the label."""
    x = np.array([ol.lse(np.delete(z[t], y[t])) - z[t, y[t]] for t in range(len(y))])
    ce = np.logaddexp(0, x)
    return ce, np.where(np.isfinite(x), np.exp(np.where(np.isfinite(x), x, 0) - ce), 0.0)


def _sure_rows(rng, V, rows=9):
    """Logits of magnitude 20 to 200 whose label stands 5 to 50 above the others, or below them."""
    z = rng.standard_normal((rows, V))
    y = rng.integers(0, V, rows)
    y[0], y[1] = 0, V - 1
    at = np.array([20.0, 40.0, 100.0, 200.0, -50.0, 60.0, 30.0, -120.0, 24.0])
    gap = np.array([12.0, 24.0, 20.0, 30.0, 16.0, 50.0, -8.0, 18.0, 5.0])
    z += (at - gap)[:, None]
    z[np.arange(rows), y] = at
    return z, y


# the teacher's part of the loss has weight 0, its sums are formed all the same
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("soft,rest,tau", [(0, 0, 1.0), (1, 0, 1.0), (1, 1, 1.0), (1, 0, 2.0), (1, 1, 2.0), (1, 1, 3.0),
                                           (1, 0, 0.5)])
@pytest.mark.parametrize("T,V", [(9, 300), (9, 50001), (2100, 3000), (9, 2)])
def test_logit_loss_of_sure_labels(T, V, soft, rest, tau, dt):
    """CE and the label's gradient have the digits of what the other columns weigh: their terms'
    exponents (2 a + 4 u at distance a), their sum, the distance to the label."""
    rng = _rng("sure", T, V, soft, rest, int(tau * 2), dt)
    z9, y9 = _sure_rows(rng, V)
    zd, y = torch.zeros(T, V, dtype=_dt(dt), device="cuda"), np.full(T, -1)
    zd[:9], y[:9] = _dev(z9, dt), y9
    z = _np(zd[:9])
    kw = dict(labels=_i32(y), alpha=1.0, temperature=tau)
    k = min(3, V)
    if soft:
        ids = rng.permuted(np.tile(np.arange(V), (9, 1)), axis=1)[:, :k]
        ids[2, 1], ids[3, 0] = y9[2], y9[3]
        ids[4] = -1
        ids = np.concatenate([ids, np.full((T - 9, k), -1)])
        kw["teacher"] = _teacher(ids, rng.standard_normal((T, k)), rng.standard_normal(T) if rest else None)
    ce, off = _label_parts(z, y9)
    gap = np.abs(z[np.arange(9), y9] - np.array([np.delete(z[t], y9[t]).max() for t in range(9)]))
    tol = (V / 256 + 200 + 4 * gap) * U
    loss, stats = _L().logit_loss(zd, **kw)
    _near(_np(loss)[:9], ce, tol * ce, what="loss")
    g = rng.uniform(0.5, 1.5, T).astype(np.float32).astype(np.float64)
    dz = _L().logit_loss_bwd(zd, stats, dloss=_f32(g), **kw)
    same = zd.clone()
    assert torch.equal(_L().logit_loss_bwd(same, stats, dloss=_f32(g), out=same, **kw), dz)
    dz = _np(dz)[:9]
    q = np.exp(z - np.array([ol.lse(r) for r in z])[:, None])
    q[np.arange(9), y9] = -off
    # q carries the log-sum's rounding
    rel = 2 * (tol + (V / 256 + 200) * U + 4 * U * np.abs(z).max(1))[:, None]
    _near(dz, g[:9, None] * q, rel * g[:9, None] * np.abs(q), dt, "dz")


@pytest.mark.parametrize("alpha", [0.0, 1.0])
@pytest.mark.parametrize("tau", [1.0, 2.0, 3.0])
def test_alpha_at_its_ends(alpha, tau):
    """One term has weight 0, also in rows that have no other."""
    rng = _rng("alpha", int(alpha), int(tau))
    zd = _dev(rng.standard_normal((12, 300)) * 3)
    z = _np(zd)
    y, ids, values, r = _targets(rng, z, 6, True, True, tau)
    kw = dict(labels=_i32(y), teacher=_teacher(ids, values, r), alpha=alpha, temperature=tau)
    loss, stats = _L().logit_loss(zd, **kw)
    dz = _L().logit_loss_bwd(zd, stats, **kw)
    ref, _, rdz = ol.loss(z, y, ids, values, r, alpha, tau)
    log = (300 / 256 + 200) * (1 + _mag(z, values, r, tau)) * U
    _near(_np(loss), ref, 2 * tau * tau * log)
    _near(_np(dz), rdz, _spread(z, y, ids, values, r, alpha, tau) * 2 * log[:, None])
    w = _dev(np.eye(300, 304))  # logits are x's columns
    x = torch.zeros(12, 304, device="cuda")
    x[:, :300] = zd
    hl, hs = _L().head_loss(x, w, **kw)
    dx, _ = _L().head_loss_bwd(x, w, hs, **kw)
    _near(_np(hl), ref, 2 * tau * tau * log)
    _near(_np(dx)[:, :300], rdz, _spread(z, y, ids, values, r, alpha, tau) * 2 * log[:, None])


@pytest.mark.parametrize("tau", [1.0, 2.0, 3.0])
def test_a_term_of_weight_0_may_be_infinite(tau):
    """alpha 1 beside a teacher whose divergence is infinite (its rest has no column, or an id is
    masked), alpha 0 beside a masked label."""
    z = np.array([[1.0, -2.0, 0.5], [1.0, -2.0, -np.inf], [1.0, 0.0, -1.0]])
    zd = _dev(z)
    ids, values, rest = np.array([[0, 1, 2]] * 3), np.ones((3, 3)), np.array([0.0, -np.inf, -np.inf])
    none = np.full((3, 3), -1)
    y = np.array([1, 0, 2])
    kw = dict(teacher=_teacher(ids, values, rest), alpha=1.0, temperature=tau)
    loss, stats = _L().logit_loss(zd, _i32(y), **kw)
    want = ol.loss(z, y, none, values, None, 1.0)
    _near(_np(loss), want[0], 1e-5)  # (3 columns of magnitude 2: a few u)
    _near(_np(_L().logit_loss_bwd(zd, stats, _i32(y), **kw)), want[2], 1e-5)
    y[:] = 2
    kw = dict(teacher=_teacher(ids[:, :2], values[:, :2], None), alpha=0.0, temperature=tau)
    loss, stats = _L().logit_loss(zd, _i32(y), **kw)
    want = ol.loss(z, None, ids[:, :2], values[:, :2], None, tau=tau)
    _near(_np(loss), want[0], 1e-4)  # (tau^2 times that)
    _near(_np(_L().logit_loss_bwd(zd, stats, _i32(y), **kw)), want[2], 1e-4)
    x, w = torch.ones(2, 8, device="cuda"), torch.zeros(3, 8, device="cuda")
    w[:, 0] = zd[0]
    x[:, 1:] = 0.0
    kw = dict(teacher=_teacher(ids[:2], values[:2], np.zeros(2)), alpha=1.0, temperature=tau)
    loss, stats = _L().head_loss(x, w, _i32(y[:2]), **kw)
    want = ol.loss(np.stack([z[0]] * 2), y[:2])
    _near(_np(loss), want[0], 1e-5)
    dx, _ = _L().head_loss_bwd(x, w, stats, _i32(y[:2]), **kw)
    _near(_np(dx), want[2] @ _np(w), 1e-4)


def test_teacher_that_weighs_nothing_is_none():
    z = _dev(np.ones((3, 20)))
    ids, values = np.array([[1, 2]] * 3), np.array([[-np.inf, -np.inf], [1.0, -np.inf], [-np.inf, -np.inf]])
    rest = np.array([-np.inf, -np.inf, 0.5])
    for r in (None, rest):
        loss, stats = _L().logit_loss(z, None, _teacher(ids, values, r))
        dz = _L().logit_loss_bwd(z, stats, None, _teacher(ids, values, r))
        ref, rs, rdz = ol.loss(_np(z), None, ids, values, r)
        _near(_np(loss), ref, 1e-5)
        _near(_np(stats), rs, 1e-5)
        _near(_np(dz), rdz, 1e-5)
        assert not _np(dz)[0].any()


@pytest.mark.parametrize("tau", [0.1, 1.0, 2.0, 3.0])
@pytest.mark.parametrize("rest", [False, True])
def test_teacher_that_weighs_nothing_beside_labels(rest, tau):
    """The labels' loss alone, also where the ids' logits are such that exp(z / tau) of them
    leaves fp32, the label's among them."""
    V, k, T = 300, 3, 7
    rng = _rng("nothing", rest, int(tau * 10))
    z = rng.standard_normal((T, V)) * 3
    ids = np.tile(np.array([4, 90, 299]), (T, 1))
    z[1:, 4] = [9.0, 50.0, 100.0, 700.0, 100.0, 100.0]
    z[2:, 90] = 120.0
    y = np.array([1, 4, 4, 90, 2, 4, -1])
    values, r = np.full((T, k), -np.inf), np.full(T, -np.inf) if rest else None
    values[5] = [1.0, 2.0, -np.inf]  # one row has a teacher
    kw = dict(labels=_i32(y), teacher=_teacher(ids, values, r), alpha=0.3, temperature=tau)
    zd = _dev(z)
    z = _np(zd)
    ref, rs, rdz = ol.loss(z, y, ids, values, r, 0.3, tau)
    log = (V / 256 + 200) * (1 + _mag(z, np.nan_to_num(values, neginf=0.0), r, tau)) * U
    tol = _spread(z, y, ids, values, r, 0.3, tau) * 2 * log[:, None]
    loss, stats = _L().logit_loss(zd, **kw)
    _near(_np(loss), ref, (0.3 + 0.7 * tau * tau) * 2 * log, what="loss")
    _near(_np(stats), rs, log[:, None], what="stats")
    _near(_np(_L().logit_loss_bwd(zd, stats, **kw)), rdz, tol, what="dz")
    # the head of the same logits: each is one product with 1 and zeros
    w, x = torch.eye(V, 304, device="cuda"), torch.zeros(T, 304, device="cuda")
    x[:, :V] = zd
    loss, stats = _L().head_loss(x, w, **kw)
    _near(_np(loss), ref, (0.3 + 0.7 * tau * tau) * 2 * log, what="head's loss")
    dx, _ = _L().head_loss_bwd(x, w, stats, **kw)
    _near(_np(dx)[:, :V], rdz, tol, what="dx")


def test_nan_is_seen():
    """A NaN in a row that counts reaches its loss."""
    z = np.zeros((2, 300))
    z[0, 250] = np.nan
    zd = _dev(z)
    y = _i32([3, 3])
    loss, stats = _L().logit_loss(zd, y)
    assert torch.isnan(loss).tolist() == [True, False]
    values = _f32([[1.0, np.nan], [1.0, 0.0]])
    loss, _ = _L().logit_loss(_dev(np.zeros((2, 300))), None, _L().TopLogits(_i32([[1, 2]] * 2), values))
    assert torch.isnan(loss).tolist() == [True, False]


def test_empty_batch():
    L = _L()
    z = torch.empty(0, 50, device="cuda")
    y = torch.empty(0, dtype=torch.int32, device="cuda")
    loss, stats = L.logit_loss(z, y)
    assert loss.shape == (0,) and L.logit_loss_bwd(z, stats, y).shape == (0, 50)
    assert L.top_logits(z, 3).ids.shape == (0, 3)
    x, w = torch.empty(0, 16, device="cuda"), torch.ones(50, 16, device="cuda")
    loss, stats = L.head_loss(x, w, y)
    dw = torch.full((50, 16), 7.0, device="cuda")
    dx, _ = L.head_loss_bwd(x, w, stats, y, dw=dw, accumulate=True)
    assert dx.shape == (0, 16) and bool((dw == 7).all())
    L.head_loss_bwd(x, w, stats, y, dw=dw)
    assert not bool(dw.any())


def test_empty_batch_of_a_frozen_head():
    """An empty dx has no address, and there is no dw."""
    L = _L()
    x, w = torch.ones(3, 16, device="cuda"), torch.ones(50, 16, device="cuda")
    y = _i32([1, 2, 3])
    _, stats = L.head_loss(x, w, y)
    for empty in (torch.empty(0, 16, device="cuda"), x[0:0]):
        dx, dw = L.head_loss_bwd(empty, w, stats[0:0], y[0:0])
        assert dx.shape == (0, 16) and dw is None
    top = L.TopLogits(_i32([[1, 2]] * 3), _f32([[1.0, 2.0]] * 3))
    _, stats = L.head_loss(x[0:0], w, None, L.TopLogits(top.ids[0:0], top.values[0:0]))
    assert L.head_loss_bwd(x[0:0], w, stats, None, L.TopLogits(top.ids[0:0], top.values[0:0]))[0].shape == (0, 16)


# --------------------------------------------------------------- top logits
def _check_top(x, k, tau=1.0):
    got = _L().top_logits(x, k, temperature=tau)
    ids, values, rest = ol.top_logits(_np(x), k, tau)
    assert np.array_equal(got.ids.cpu().numpy(), ids)
    assert np.array_equal(np.nan_to_num(_np(got.values), nan=9e99), np.nan_to_num(values, nan=9e99))
    V = x.shape[1]
    fin = np.where(np.isfinite(rest), np.abs(rest), 0.0)
    _near(_np(got.rest), rest, (V / 512 + 160) * U + 4 * U * fin, what="rest")
    return got


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V,k", [(1, 1), (2, 1), (2, 2), (9, 4), (64, 64), (255, 255), (256, 256), (1000, 5), (1024, 256),
                                 (4097, 64), (50257, 1), (128256, 256)])
def test_top_logits(V, k, dt):
    for skip in (0, 1, 6):
        rng = _rng("top", V, k, dt, skip)
        x = _dev(rng.standard_normal((4, V)) * 3, dt, 3, skip)
        _check_top(x, k, 2.0)
        _untouched(x)


@pytest.mark.parametrize("dt", [BF, F32])
def test_top_logits_of_equal_columns(dt):
    """Ties go to the lower column, also where more columns are equal than the list holds."""
    rng = _rng("ties", dt)
    x = np.zeros((9, 20011))
    x[1] = -np.inf
    x[2] = rng.integers(0, 3, 20011)
    x[3, rng.integers(0, 20011, 30)] = 1.0
    x[4] = np.where(rng.random(20011) < 0.5, 0.0, -0.0)
    x[5] = -np.inf
    x[5, [19999, 7]] = [1.0, 2.0]
    x[6] = np.nan
    x[7] = rng.standard_normal(20011)
    x[7, ::40] = np.nan
    x[8] = torch.finfo(_dt(dt)).min
    for k in (1, 50, 256):
        _check_top(_dev(x, dt), k)
    y = np.full((2, 700), np.inf)
    y[1, :690] = 5.0
    _check_top(_dev(y, dt), 8)


def test_top_logits_one_strand():
    """All the large columns in one thread's strand: the bound is far below them."""
    x = np.arange(40000, dtype=np.float64)[None] * -1e-3
    x[0, 8 * 512 * np.arange(9)] = 50 + np.arange(9)
    _check_top(_dev(x), 9)
    _check_top(_dev(-np.arange(30000, dtype=np.float64)[None]), 200)
    _check_top(_dev(np.arange(30000, dtype=np.float64)[None]), 200)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("k", [5, 64, 256])
@pytest.mark.parametrize("T", [64, 600])
def test_top_logits_repeatable(T, k, dt):
    # rising rows, whose list is cut many times, and plain ones
    L = _L()
    g = torch.Generator(device="cuda").manual_seed(T + k)
    z = torch.randn(T, 40003, generator=g, device="cuda")
    z[::2] += torch.linspace(0, 8, 40003, device="cuda")
    z = z.to(_dt(dt))
    a = L.top_logits(z, k, temperature=2.0)
    for _ in range(10):
        b = L.top_logits(z, k, temperature=2.0)
        assert torch.equal(a.ids, b.ids) and torch.equal(a.values, b.values)
        assert torch.equal(a.rest, b.rest)


def _check_top_rows(x, k, rows, tau=2.0):
    """Some rows of a batch whose size decides the kernel's form."""
    got = _L().top_logits(x, k, temperature=tau)
    ids, values, rest = ol.top_logits(_np(x[rows]), k, tau)
    assert np.array_equal(got.ids[rows].cpu().numpy(), ids)
    assert np.array_equal(_np(got.values[rows]), values)
    _near(_np(got.rest[rows]), rest, (x.shape[1] / 512 + 160) * U + 4 * U * np.abs(rest), what="rest")


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("k", [5, 150, 256])
@pytest.mark.parametrize("T,V,step", [(600, 70001, 8192), (4, 300001, 32768), (600, 1000, 100)])
def test_top_logits_of_ties_that_grow(T, V, step, k, dt):
    """Equal columns nearly fill the list in the first round and more come in every later one
    (step: columns of a round of fp32; a round of bf16 has twice as many)."""
    rng = _rng("grow", T, V, k, dt)
    x = _dev(np.zeros((T, V)), dt, 3, 1)
    x.copy_(torch.randn(T, V, generator=torch.Generator(device="cuda").manual_seed(k), device="cuda"))
    step *= 2 if dt == BF else 1
    cap = 512 if k <= 64 else 1024
    rows = [0, 1, T // 2, T - 1]
    for r, fill in zip(rows, (0.8, 0.9, 0.97, 0.99)):
        x[r, torch.from_numpy(rng.permutation(step)[: int(cap * fill)] % V).cuda()] = 9.0
        for at in range(step, V, step):
            n = min(V - at, step)
            x[r, at + torch.from_numpy(rng.permutation(n)[: 100]).cuda()] = 9.0
    _check_top_rows(x, k, rows)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("k", [5, 64, 256])
@pytest.mark.parametrize("skip", [0, 3])
def test_top_logits_of_many_rows(skip, k, dt):
    """Rows of many rounds whose list is cut between them, in the form for many rows."""
    T, V = 600, 40003
    x = torch.full((T, V + 5), float("nan"), dtype=_dt(dt), device="cuda")[:, skip: skip + V]
    z = torch.randn(T, V, generator=torch.Generator(device="cuda").manual_seed(k + skip), device="cuda")
    z[::2] += torch.linspace(0, 8, V, device="cuda")
    x.copy_(z)
    _check_top_rows(x, k, [0, 1, 2, 3, 298, 299, 598, 599])


def test_top_logits_without_rest():
    x = _dev(_rng("norest").standard_normal((3, 500)))
    a, b = _L().top_logits(x, 7, rest=False), _L().top_logits(x, 7)
    assert a.rest is None and torch.equal(a.ids, b.ids) and torch.equal(a.values, b.values)


# ------------------------------------------------------------- loss of a head
def _head_case(T, V, d, k, rest, hard, tau, dt, seed=0, pad=0):
    rng = _rng("head", T, V, d, k, rest, hard, int(tau * 2), dt, seed)
    x, w = _dev(rng.standard_normal((T, d)), dt, pad), _dev(rng.standard_normal((V, d)) * 2.5 / np.sqrt(d), dt, pad)
    xn, wn = _np(x), _np(w)
    y, ids, values, r = _targets(rng, xn @ wn.T, k, rest, hard, tau)
    return rng, x, w, xn, wn, y, ids, values, r


def _check_head(case, tau, dt, alpha=0.3, columns=0, gdt=None, accumulate=False, need_dx=True, dloss=True):
    rng, x, w, xn, wn, y, ids, values, r = case
    T, V, d = xn.shape[0], wn.shape[0], xn.shape[1]
    kw = dict(labels=_i32(y), teacher=_teacher(ids, values, r), alpha=alpha, temperature=tau)
    loss, stats = _L().head_loss(x, w, **kw)
    g = rng.uniform(0.5, 1.5, T) * np.where(rng.random(T) < 0.2, -1, 1) if dloss else np.ones(T)
    g = g.astype(np.float32).astype(np.float64)
    ref, rs, rdx, rdw = ol.head(xn, wn, y, ids, values, r, alpha, tau, g)
    z = xn @ wn.T
    ez = (d + 8) * U * (np.abs(xn) @ np.abs(wn).T).max(1)
    log = (V / 256 + 200) * (1 + _mag(z, values, r, tau)) * U + 4 * ez / min(1.0, tau)
    a, b = ol.weights(y, ids, alpha)
    _near(_np(loss), ref, (a + b * tau * tau) * 2 * log, what="loss")
    _near(_np(stats), rs, log[:, None], what="stats")
    gdt = gdt or dt
    pad = 8 if x.stride(0) > d else 0
    dx = _dev(np.zeros((T, d)), gdt, pad) if need_dx else None
    dw0 = rng.standard_normal((V, d)).astype(np.float32).astype(np.float64)
    dw = _dev(dw0, gdt, pad)
    _L().head_loss_bwd(x, w, stats, dloss=_f32(g) if dloss else None, scale=0.25, dx=dx, dw=dw, need_dx=need_dx,
                       accumulate=accumulate, columns=columns, **kw)
    dz = ol.loss(z, y, ids, values, r, alpha, tau)[2] * g[:, None]
    err = np.abs(g)[:, None] * _spread(z, y, ids, values, r, alpha, tau) * 2 * log[:, None]
    if dt == BF:
        err = err + 2.0 ** -8 * (np.abs(dz) + err)
    tx = 0.25 * (err @ np.abs(wn) + (V + 64) * U * (np.abs(dz) @ np.abs(wn)))
    tw = 0.25 * (err.T @ np.abs(xn) + (T + 64) * U * (np.abs(dz).T @ np.abs(xn)))
    if need_dx:
        _near(_np(dx), 0.25 * rdx, tx + 1e-30, gdt, "dx")
        if pad:
            _untouched(dx)
    base = dw0 if accumulate else 0.0
    _near(_np(dw), 0.25 * rdw + base, tw + 2 * U * np.abs(base) + 1e-30, gdt, "dw")
    if pad:
        _untouched(dw)
    return loss, stats, dx, dw


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("hard,k,rest,tau", [(1, 0, 0, 1.0), (0, 5, 0, 1.0), (0, 5, 1, 2.0), (1, 5, 0, 1.0), (1, 5, 0, 2.0),
                                             (1, 5, 1, 0.5)])
@pytest.mark.parametrize("T,V,d", [(1, 9, 8), (9, 100, 24), (130, 257, 64), (33, 1031, 136)])
def test_head_loss(T, V, d, hard, k, rest, tau, dt):
    _check_head(_head_case(T, V, d, k, rest, hard, tau, dt), tau, dt)


@pytest.mark.parametrize("dt", [BF, F32])
def test_head_loss_in_pieces(dt):
    """Several pieces, the last of one column more than a whole number of them, fp32
    gradients added up, strided operands."""
    case = _head_case(70, 513, 40, 17, True, 1, 2.0, dt, pad=8)
    _check_head(case, 2.0, dt, columns=256, gdt=F32, accumulate=True)
    _check_head(case, 2.0, dt, columns=200, gdt=BF)
    _check_head(case, 2.0, dt, need_dx=False, dloss=False)


@pytest.mark.parametrize("hard,k,rest", [(1, 0, 0), (1, 256, 1)])
def test_head_loss_large_tiles(hard, k, rest):
    """Sizes that take 256 x 256 tiles, with ragged edges."""
    from paper_2608_07974_amd import zl  # noqa: F401
    _check_head(_head_case(1000, 16421, 72, k, rest, hard, 1.0 if not k else 2.0, BF), 1.0 if not k else 2.0, BF)


@pytest.mark.parametrize("T,V,dt", [(300, 4209, BF), (3, 33001, BF), (130, 4209, F32), (1100, 4001, F32), (20, 17001, F32)])
@pytest.mark.parametrize("hard,k,rest,tau", [(1, 0, 0, 1.0), (0, 33, 0, 1.0), (0, 200, 1, 2.0), (1, 9, 0, 2.0)])
def test_head_loss_more_tiles(T, V, dt, hard, k, rest, tau):
    """Sizes beyond the smallest tiles, of every tile in between, strided operands."""
    _check_head(_head_case(T, V, 40, k, rest, hard, tau, dt, pad=8), tau, dt)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("d", [8, 56, 64, 72, 256, 264, 1000])
def test_head_loss_few_tiles_any_width(d, dt):
    """A sum over d split over the waves, parts of it empty or cut."""
    _check_head(_head_case(34, 70, d, 5, True, 1, 2.0, dt, pad=8), 2.0, dt)


@pytest.mark.parametrize("dt", [BF, F32])
def test_head_loss_many_rows_few_columns(dt):
    """Few tiles of a long sum: the weight's gradient is split over the rows."""
    _check_head(_head_case(4200, 70, 48, 3, True, 1, 2.0, dt), 2.0, dt)


@pytest.mark.parametrize("dt", [BF, F32])
def test_head_loss_rows_without_targets_may_hold_anything(dt):
    rng, x, w, xn, wn, y, ids, values, r = case = _head_case(40, 90, 32, 4, True, 1, 2.0, dt)
    y[:] = np.where(np.arange(40) % 3 == 0, -100, np.arange(40) % 90)
    ids[np.arange(40) % 3 == 0] = -1
    values[np.arange(40) % 3 == 0] = np.nan
    want = _check_head((rng, x, w, xn, wn, y, ids, np.nan_to_num(values), r), 2.0, dt, dloss=False)
    bad = x.clone()
    bad[::3] = float("nan")
    bad[3] = float("inf")
    kw = dict(labels=_i32(y), teacher=_teacher(ids, values, r), alpha=0.3, temperature=2.0)
    loss, stats = _L().head_loss(bad, w, **kw)
    assert torch.equal(loss, want[0]) and torch.equal(stats[:, :4], want[1][:, :4])
    dx, dw = _L().head_loss_bwd(bad, w, stats, scale=0.25, need_dw=True, **kw)
    assert torch.equal(dx, want[2]) and torch.equal(dw, want[3])
    assert not bool(dx[::3].any())


@pytest.mark.parametrize("T,V,dt", [(300, 4209, BF), (1000, 16421, BF), (130, 4209, F32), (1100, 4001, F32), (20, 17001, F32)])
def test_head_loss_rows_without_targets_in_every_tile(T, V, dt):
    L = _L()
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, 40, generator=g, device="cuda").to(_dt(dt))
    w = (torch.randn(V, 40, generator=g, device="cuda") / 3).to(_dt(dt))
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    top = L.top_logits(x.float() @ w.float().t(), 7, temperature=2.0)
    y[::3] = -100
    top.ids[::3] = -1
    kw = dict(labels=y, teacher=top, temperature=2.0)
    bad = x.clone()
    bad[::3] = float("nan")
    bad[3] = float("inf")
    (a, sa), (b, sb) = L.head_loss(x, w, **kw), L.head_loss(bad, w, **kw)
    assert torch.equal(a, b) and torch.equal(sa, sb)
    p, q = L.head_loss_bwd(x, w, sa, need_dw=True, **kw), L.head_loss_bwd(bad, w, sb, need_dw=True, **kw)
    assert torch.equal(p[0], q[0]) and torch.equal(p[1], q[1]) and not bool(q[0][::3].any())


@pytest.mark.parametrize("T,V,dt", [(9, 300, BF), (9, 300, F32), (300, 4209, BF), (9, 40000, BF), (1000, 16421, BF), (130, 4209, F32),
                                    (1100, 4001, F32), (20, 17001, F32)])
@pytest.mark.parametrize("soft,rest,tau", [(0, 0, 1.0), (1, 0, 1.0), (1, 1, 1.0), (1, 0, 2.0), (1, 1, 3.0)])
def test_head_loss_of_sure_labels(T, V, dt, soft, rest, tau):
    """As of logits, whose sums are exact here: multiples of 1 / 64 below 256, of which three
    products are not 0."""
    rng = _rng("sure head", T, V, dt, soft, rest, int(tau))
    at = np.array([20.0, 40.0, 100.0, 180.0, -50.0, 60.0, 30.0, -120.0, 24.0])
    gap = np.array([12.0, 24.0, 20.0, 30.0, 16.0, 50.0, -8.0, 18.0, 5.0])
    y9 = rng.permutation(V)[:9]
    y9[0], y9[1] = 0, V - 1
    w = np.zeros((V, 16))
    w[:, 0], w[:, 1] = 1.0, np.clip(np.round(rng.standard_normal(V) * 64), -255, 255) / 64
    w[y9, 2 + np.arange(9)] = gap
    x = np.zeros((T, 16))
    r = np.arange(T) % 9
    x[:, 0], x[:, 1], x[np.arange(T), 2 + r] = (at - gap)[r], 1.0, 1.0
    y = y9[r]
    z = x[:9] @ w.T
    kw = dict(labels=_i32(y), alpha=1.0, temperature=tau)
    if soft:
        ids = rng.permuted(np.tile(np.arange(V), (T, 1)), axis=1)[:, :3] if T < 99 else rng.integers(0, V, (T, 3))
        ids[2::9, 1], ids[3::9, 0] = y9[2], y9[3]
        ids[4::9] = -1
        kw["teacher"] = _teacher(ids, rng.standard_normal((T, 3)), rng.standard_normal(T) if rest else None)
    loss, stats = _L().head_loss(_dev(x, dt), _dev(w, dt), **kw)
    ce, _ = _label_parts(z, y9)
    far = np.abs(z[np.arange(9), y9] - np.array([np.delete(z[t], y9[t]).max() for t in range(9)]))
    _near(_np(loss), ce[r], ((V / 256 + 200 + 4 * far) * U * ce)[r], what="loss")
    assert np.array_equal(_np(stats)[:, 3], z[r, y])
    # no label's gradient has the wrong sign
    assert bool((stats[:, 0] >= stats[:, 3]).all())


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("gdt", [BF, F32])
@pytest.mark.parametrize("T,V,d,columns", [(5, 40, 24, 0), (300, 4209, 40, 0), (300, 4209, 40, 1024), (40, 30000, 64, 0),
                                           (1000, 16421, 72, 0)])
def test_head_loss_rows_without_targets_of_a_broken_head(T, V, d, columns, gdt, dt):
    """Their dx is 0 also where it is the weight that is infinite or NaN, and they add nothing to
    dw, in one piece or several, with and without splits of the sum."""
    L = _L()
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, d, generator=g, device="cuda").to(_dt(dt))
    w = (torch.randn(V, d, generator=g, device="cuda") / 4).to(_dt(dt))
    w[V // 2] = float("inf")
    w[V - 1, 3] = float("nan")
    y = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    some = y.clone()
    some[T // 2] = 3
    for labels in (y, some):
        loss, stats = L.head_loss(x, w, labels)
        dx, dw = torch.full((T, d), 7.0, dtype=_dt(gdt), device="cuda"), torch.full((V, d), 7.0, dtype=_dt(gdt), device="cuda")
        L.head_loss_bwd(x, w, stats, labels, dx=dx, dw=dw, columns=columns)
        dead = labels < 0
        assert not bool(loss[dead].any()) and not bool(dx[dead].any())
        if labels is y:
            assert not bool(dw.any())
        else:
            assert bool(torch.isnan(loss[T // 2])) and bool(torch.isnan(dx[T // 2]).any())


@pytest.mark.parametrize("dt", [BF, F32])
def test_head_loss_weights_do_not_round(dt):
    """A label's weight is no part of the bf16 operand: with no teacher in any row alpha only
    scales the result."""
    L = _L()
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w = torch.randn(70, 64, generator=g, device="cuda").to(_dt(dt)), torch.randn(130, 64, generator=g, device="cuda").to(_dt(dt))
    y = torch.randint(0, 130, (70,), generator=g, device="cuda", dtype=torch.int32)
    none = L.TopLogits(torch.full((70, 3), -1, dtype=torch.int32, device="cuda"), torch.zeros(70, 3, device="cuda"))
    out = []
    for kw, scale in ((dict(teacher=none, alpha=0.3), 1.0), (dict(), 0.3)):
        dx, dw = torch.empty(70, 64, device="cuda"), torch.empty(130, 64, device="cuda")
        _, stats = L.head_loss(x, w, y, **kw)
        out.append(L.head_loss_bwd(x, w, stats, y, dx=dx, dw=dw, scale=scale, **kw))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T,V,k", [(70, 130, 0), (70, 130, 3), (1500, 130, 3), (5000, 130, 0), (5000, 130, 3)])
@pytest.mark.parametrize("big", [3e38, float("inf"), float("nan")])
def test_head_loss_weights_of_rows_without_targets(T, V, k, big, dt):
    """They may be anything: the other rows' gradients are what they are beside weights of 0."""
    L = _L()
    g = torch.Generator(device="cuda").manual_seed(T + k)
    x = torch.randn(T, 64, generator=g, device="cuda").to(_dt(dt))
    w = (torch.randn(V, 64, generator=g, device="cuda") / 4).to(_dt(dt))
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    y[1::2] = -1
    kw = dict(labels=y)
    if k:
        top = L.top_logits(x.float() @ w.float().t(), k)
        top.ids[::3] = -1
        kw.update(teacher=top)
    dead = torch.zeros(T, dtype=torch.bool, device="cuda")
    dead[1::2] = True
    if k:
        dead[1::2] = top.ids[1::2, 0] < 0
    dloss = (torch.rand(T, generator=g, device="cuda") + 0.5) / T
    dloss[dead] = 0.0
    _, stats = L.head_loss(x, w, **kw)
    want = L.head_loss_bwd(x, w, stats, dloss=dloss, need_dw=True, **kw)
    assert bool(want[0].any())
    got = L.head_loss_bwd(x, w, stats, dloss=torch.where(dead, big, dloss), need_dw=True, **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_head_loss_is_the_loss_of_its_logits():
    """The two operators agree on logits that fp32 holds exactly."""
    rng = _rng("same")
    x, w = rng.integers(-4, 5, (50, 32)) / 4.0, rng.integers(-4, 5, (300, 32)) / 8.0
    z = x @ w.T
    y, ids, values, r = _targets(rng, z, 9, True, True, 2.0)
    kw = dict(labels=_i32(y), teacher=_teacher(ids, values, r), temperature=2.0)
    for dt in (BF, F32):
        loss, stats = _L().head_loss(_dev(x, dt), _dev(w, dt), **kw)
        want, ws = _L().logit_loss(_dev(z), **kw)
        _near(_np(loss), _np(want), 1e-5)  # two sums of 300 terms: 2 (300 / 256 + 200) (1 + 8) u * 2.5 < 6e-4 at most
        _near(_np(stats[:, :4]), _np(ws), 1e-5)


# ------------------------------------------------------------ large offsets
def test_rows_beyond_32_bit_offsets():
    """The last rows of 5 GB of logits give what they give alone."""
    L = _L()
    T, V = 20001, 130000
    z = torch.empty(T, V, dtype=torch.bfloat16, device="cuda")
    for i in range(0, T, 2000):
        z[i: i + 2000] = torch.randn(min(2000, T - i), V, device="cuda") * 2
    y = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    top = L.top_logits(z, 5)
    kw = dict(labels=y, teacher=top)
    loss, stats = L.logit_loss(z, **kw)
    tail = slice(T - 3, T)
    part = dict(labels=y[tail], teacher=L.TopLogits(*[t[tail].contiguous() for t in top]))
    alone = z[tail].clone()
    for a, b in zip(L.top_logits(alone, 5), top):
        assert torch.allclose(a, b[tail], rtol=0, atol=1e-5)  # (rows few or many are summed in other orders)
    l2, s2 = L.logit_loss(alone, **part)
    # two orders of 130000 positive terms: (130000 / 256 + 120) u of the log-sum each
    assert torch.allclose(l2, loss[tail], rtol=0, atol=1e-3)
    want = L.logit_loss_bwd(alone, s2, **part).float()
    got = L.logit_loss_bwd(z, stats, out=z, **kw)[tail].float()
    assert torch.allclose(got, want, rtol=2.0 ** -7, atol=1e-6)


def test_head_beyond_32_bit_offsets():
    """A weight of 5 GB and its gradient; a weight whose rows lie 4 MB apart."""
    L = _L()
    T, V, d = 4, 300000, 8192
    w = torch.empty(V, d, dtype=torch.bfloat16, device="cuda")
    for i in range(0, V, 50000):
        w[i: i + 50000] = torch.randn(50000, d, device="cuda") / 40
    x = torch.randn(T, d, device="cuda").bfloat16()
    y = _i32([V - 1, 5, V - 2, 100])
    z = torch.cat([x.float() @ w[i: i + 50000].float().t() for i in range(0, V, 50000)], 1)
    loss, stats = L.head_loss(x, w, y)
    want, ws = L.logit_loss(z, y)
    # logits of spread 2 to 8000 u sum |x w|, 1e-3
    assert torch.allclose(loss, want, rtol=0, atol=5e-3)
    dx, dw = L.head_loss_bwd(x, w, stats, y, need_dw=True)
    dz = L.logit_loss_bwd(z, ws, y)
    for v in (0, 5, 100, 262143, 262144, V - 2, V - 1):
        ref = dz[:, v] @ x.float()
        assert (dw[v].float() - ref).norm() <= 2e-2 * ref.norm() + 1e-8, v
    ref = sum(dz[:, i: i + 50000] @ w[i: i + 50000].float() for i in range(0, V, 50000))
    assert (dx.float() - ref).norm() <= 2e-2 * ref.norm()
    del w, dw, z, dz
    far = torch.zeros(600, (1 << 21) - 8, dtype=torch.bfloat16, device="cuda")[:, :64]
    near = torch.randn(600, 64, device="cuda").bfloat16()
    far.copy_(near)
    x = torch.randn(40, 64, device="cuda").bfloat16()
    y = torch.randint(0, 600, (40,), device="cuda", dtype=torch.int32)
    a, b = L.head_loss(x, far, y), L.head_loss(x, near, y)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    q = L.head_loss_bwd(x, near, b[1], y, need_dw=True, columns=256)
    p = L.head_loss_bwd(x, far, a[1], y, need_dw=True, columns=256)
    assert torch.equal(p[0], q[0]) and torch.equal(p[1], q[1])
    # pieces as wide as the offsets reach, with more scratch memory and so other splits of a
    # sum of 600 terms: 2 (600 + 64) u of sum |dz w| (at most 2 max |w|, 8) and a bf16 step
    p = L.head_loss_bwd(x, far, a[1], y, need_dw=True)
    for m, n in zip(p, q):
        assert torch.allclose(m.float(), n.float(), rtol=2.0 ** -7, atol=1e-3)


@pytest.mark.parametrize("T,dt", [(300, BF), (1000, BF), (130, F32), (20, F32)])
def test_head_of_rows_far_apart(T, dt):
    """A weight whose rows lie 4 or 8 MB apart, in every tile; the same sums as one of close rows."""
    L = _L()
    V = 4209 if T > 20 else 3001
    far = torch.empty(V, (1 << 21) - 8, dtype=_dt(dt), device="cuda")[:, :64]
    near = (torch.randn(V, 64, device="cuda") / 4).to(_dt(dt))
    far.copy_(near)
    x = torch.randn(T, 64, device="cuda").to(_dt(dt))
    y = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    a, b = L.head_loss(x, far, y), L.head_loss(x, near, y)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    p, q = (L.head_loss_bwd(x, m, a[1], y, need_dw=True, columns=256) for m in (far, near))
    assert torch.equal(p[0], q[0]) and torch.equal(p[1], q[1])


# ------------------------------------------------------- as a program uses them
def test_teacher_to_student_step():
    """A teacher's logits to its top ones, the student's loss through its head, a step down
    the gradient: the loss falls by the step times the gradient's square (first order),
    checked against the oracle's own loss before and after."""
    L = _L()
    rng = _rng("step")
    T, V, d, tau = 64, 700, 48, 2.0
    teacher_z = _dev(rng.standard_normal((T, V)) * 2, F32)
    x, w = _dev(rng.standard_normal((T, d)), F32), _dev(rng.standard_normal((V, d)) / 7, F32)
    y = _i32(rng.integers(0, V, T))
    top = L.top_logits(teacher_z, 20, temperature=tau)
    ids, values, rest = ol.top_logits(_np(teacher_z), 20, tau)
    kw = dict(labels=y, teacher=top, temperature=tau)
    n = torch.full((T,), 1.0 / T, device="cuda")
    loss, stats = L.head_loss(x, w, **kw)
    dx, dw = L.head_loss_bwd(x, w, stats, dloss=n, need_dw=True, **kw)
    _, _, rdx, rdw = ol.head(_np(x), _np(w), y.cpu().numpy(), ids, values, rest, 0.5, tau, np.full(T, 1.0 / T))
    # 1e-5 of the norm: fp32 sums of 700 and 64 terms, see above
    assert np.linalg.norm(_np(dx) - rdx) < 1e-5 * np.linalg.norm(rdx)
    assert np.linalg.norm(_np(dw) - rdw) < 1e-5 * np.linalg.norm(rdw)
    # the derivative along the gradient by a central difference of the oracle's loss: the
    # quadratic term cancels, h^3 leaves 1e-4 of it at this step
    h = 1e-2
    f = lambda s: ol.loss((_np(x) + s * rdx) @ (_np(w) + s * rdw).T, y.cpu().numpy(), ids, values, rest,  # noqa: E731
                          0.5, tau, grad=False)[0].mean()
    slope = (f(h) - f(-h)) / (2 * h)
    got = (_np(dx) * rdx).sum() + (_np(dw) * rdw).sum()
    assert abs(got - slope) < 1e-3 * abs(slope)


def test_block_to_head():
    """Norm, head loss and back through the norm, with the layer operators."""
    from paper_2608_07974_amd import layer
    L = _L()
    rng = _rng("block")
    T, V, d = 33, 200, 64
    h = _dev(rng.standard_normal((T, d)), F32)
    g = _f32(rng.uniform(0.5, 1.5, d))
    w = _dev(rng.standard_normal((V, d)) / 8, F32)
    y = _i32(rng.integers(0, V, T))
    n_out = torch.full((T,), 1.0 / T, device="cuda")
    _, n, stats = layer.block_norm(h, None, None, (g, None), dtype=torch.float32)
    loss, s = L.head_loss(n, w, y)
    dn, _ = L.head_loss_bwd(n, w, s, y, dloss=n_out)
    dh, _ = layer.block_norm_bwd(None, dn, None, h, stats, None, (g, None))
    ht = torch.tensor(_np(h), requires_grad=True)
    nt = ht * torch.rsqrt(ht.square().mean(-1, keepdim=True) + 1e-5) * torch.tensor(_np(g))
    lt = torch.nn.functional.cross_entropy(nt @ torch.tensor(_np(w)).t(), y.cpu().long())
    lt.backward()
    assert abs(float(loss.mean()) - float(lt.detach())) < 1e-5
    assert np.linalg.norm(_np(dh) - ht.grad.numpy()) < 1e-5 * np.linalg.norm(ht.grad.numpy())


@pytest.mark.parametrize("dt", [BF, F32])
def test_captured_and_replayed(dt):
    """One graph of the whole chain, replayed on new inputs with eager work in between."""
    L = _L()
    T, V, d, k, tau = 96, 1003, 64, 12, 2.0
    rng = _rng("graph", dt)
    x, w = _dev(rng.standard_normal((T, d)), dt), _dev(rng.standard_normal((V, d)) / 5, dt)
    tz = _dev(rng.standard_normal((T, V)) * 2, dt)
    zz = _dev(rng.standard_normal((T, V)) * 2, dt)
    y = _i32(rng.integers(0, V, T))
    dw = torch.zeros(V, d, device="cuda")
    ws, wb = L.head_workspace(x, w, k=k), L.head_workspace(x, w, k=k, backward=True, need_dw=True)

    def step():
        top = L.top_logits(tz, k, temperature=tau)
        kw = dict(labels=y, teacher=top, temperature=tau)
        loss, stats = L.head_loss(x, w, workspace=ws, **kw)
        dx, _ = L.head_loss_bwd(x, w, stats, dw=dw, workspace=wb, **kw)
        l2, s2 = L.logit_loss(zz, **kw)
        return [*top, loss, stats, dx, dw, l2, L.logit_loss_bwd(zz, s2, **kw)]

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for i in range(3):
        r = _rng("replay", i)
        x.copy_(torch.from_numpy(r.standard_normal((T, d)).astype(np.float32)))
        tz.copy_(torch.from_numpy(r.standard_normal((T, V)).astype(np.float32)))
        y.copy_(torch.from_numpy(r.integers(-3, V, T).astype(np.int32)))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), i


def test_two_streams_with_workspaces_of_their_own():
    L = _L()
    rng = _rng("streams")
    x, w = _dev(rng.standard_normal((200, 64)), BF), _dev(rng.standard_normal((3000, 64)) / 8, BF)
    y = _i32(rng.integers(0, 3000, 200))
    loss, stats = L.head_loss(x, w, y)
    want = L.head_loss_bwd(x, w, stats, y, need_dw=True)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        with torch.cuda.stream(s):
            l, st = L.head_loss(x, w, y)
            got.append((l, *L.head_loss_bwd(x, w, st, y, need_dw=True)))
    torch.cuda.synchronize()
    for l, dx, dw in got:
        assert torch.equal(l, loss) and torch.equal(dx, want[0]) and torch.equal(dw, want[1])


def test_autograd_is_told():
    """Outputs count as changed in place; matrices on the graph are refused; a head that is
    a parameter is not."""
    L = _L()
    x = torch.randn(5, 16, device="cuda")
    w = torch.nn.Parameter(torch.randn(30, 16, device="cuda"))
    y = _i32([1, 2, 3, 4, 5])
    loss, stats = L.head_loss(x, w, y)
    v = loss._version
    L.head_loss(x, w, y, loss=loss, stats=stats)
    assert loss._version > v
    _, dw = L.head_loss_bwd(x, w, stats, y, need_dw=True)
    assert dw.shape == w.shape
    with pytest.raises(ValueError, match="gradient"):
        L.head_loss(x.requires_grad_(), w, y)
    with pytest.raises(ValueError, match="gradient"):
        L.logit_loss(torch.randn(5, 9, device="cuda", requires_grad=True), y)
    with torch.no_grad():
        L.head_loss(x, w, y)


def test_refused_on_the_host():
    """Placement and shapes that the kernels would take on trust."""
    L = _L()
    z, y = torch.zeros(4, 10, device="cuda"), _i32([1, 2, 3, 4])
    top = L.TopLogits(_i32([[1, 2]] * 4), _f32([[1.0, 2.0]] * 4))
    for kw in (dict(labels=y.cpu()), dict(teacher=top._replace(ids=top.ids.cpu())), dict(labels=y, loss=torch.zeros(4)),
               dict(labels=y[:3]), dict(labels=y.long()), dict(teacher=top._replace(values=top.values[:, :1])),
               dict(teacher=top._replace(rest=torch.zeros(3, device="cuda"))), dict(),
               dict(labels=y, stats=torch.zeros(4, 5, device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            L.logit_loss(z, **kw)
    with pytest.raises((ValueError, TypeError)):
        L.logit_loss_bwd(z, torch.zeros(4, 4, device="cuda"), y, out=torch.zeros(4, 9, device="cuda"))
    x, w = torch.zeros(4, 16, device="cuda"), torch.zeros(10, 16, device="cuda")
    for args in ((x, w.bfloat16(), y), (x, w[:, :8], y), (x.cpu(), w, y), (x, w.cpu(), y)):
        with pytest.raises((ValueError, TypeError)):
            L.head_loss(*args)
    with pytest.raises(ValueError):
        L.head_loss(x, w, y, workspace=torch.empty(1 << 20, dtype=torch.uint8))
