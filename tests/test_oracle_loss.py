"""Pins of the fp64 losses over a vocabulary (oracle/loss.py): closed forms, torch's
fp64 routines, finite differences, brute force."""
import numpy as np
import pytest

from oracle import loss as ol

torch = pytest.importorskip("torch")


def _case(T=6, V=23, k=5, seed=0, rest=True):
    r = np.random.RandomState(seed)
    z = r.randn(T, V) * 2
    labels = r.randint(0, V, T).astype(np.int32)
    labels[1] = -100
    ids = np.stack([r.permutation(V)[:k] for _ in range(T)]).astype(np.int32)
    values = r.randn(T, k) * 2
    return z, labels, ids, values, r.randn(T) if rest else None


def test_labels_are_torchs_cross_entropy():
    z, y, *_ = _case()
    got = ol.loss(z, y)[0]
    ref = torch.nn.functional.cross_entropy(torch.tensor(z), torch.tensor(y).long(), reduction="none").numpy()
    assert np.allclose(got, ref, rtol=0, atol=1e-13) and got[1] == 0


@pytest.mark.parametrize("tau", [1.0, 2.0, 0.5])
def test_cut_off_teacher_is_torchs_kl(tau):
    z, _, ids, values, _ = _case()
    got = ol.loss(z, None, ids, values, tau=tau)[0]
    for t in range(z.shape[0]):
        p = torch.softmax(torch.tensor(values[t]) / tau, 0)
        full = torch.zeros(z.shape[1], dtype=torch.float64)
        full[ids[t].astype(int)] = p
        logq = torch.log_softmax(torch.tensor(z[t]) / tau, 0)
        ref = tau ** 2 * torch.nn.functional.kl_div(logq, full, reduction="sum").item()
        assert abs(got[t] - ref) < 1e-12


def test_whole_vocabulary_with_an_empty_rest_is_the_full_kl():
    """k = V: the teacher's whole distribution, whatever form it comes in."""
    z, _, _, _, _ = _case(V=9)
    r = np.random.RandomState(3)
    t = r.randn(6, 9)
    ids, values, rest = ol.top_logits(t, 9, 2.0)
    assert np.all(rest == -np.inf)
    p = np.exp(t / 2) / np.exp(t / 2).sum(1, keepdims=True)
    logq = z / 2 - np.log(np.exp(z / 2).sum(1, keepdims=True))
    ref = 4 * (p * (np.log(p) - logq)).sum(1)
    for u in (None, rest):
        assert np.allclose(ol.loss(z, None, ids, values, u, tau=2.0)[0], ref, atol=1e-12)


def test_rest_is_one_outcome_more():
    """Against the distributions written out with the other columns in one bucket."""
    z, _, ids, values, rest = _case()
    got = ol.loss(z, None, ids, values, rest, tau=2.0)[0]
    for t in range(z.shape[0]):
        u = np.append(values[t] / 2, rest[t])
        p = np.exp(u) / np.exp(u).sum()
        q = np.exp(z[t] / 2) / np.exp(z[t] / 2).sum()
        q = np.append(q[ids[t]], q.sum() - q[ids[t]].sum())
        assert abs(got[t] - 4 * (p * np.log(p / q)).sum()) < 1e-12


def test_teacher_that_is_the_student_costs_nothing():
    z, *_ = _case()
    ids, values, rest = ol.top_logits(z, 4, 2.0)
    out, _, dz = ol.loss(z, None, ids, values, rest, tau=2.0)
    assert np.allclose(out, 0, atol=1e-13) and np.allclose(dz, 0, atol=1e-13)


@pytest.mark.parametrize("hard,soft,rest", [(1, 0, 0), (0, 1, 0), (0, 1, 1), (1, 1, 0), (1, 1, 1)])
@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_gradient_is_the_difference(hard, soft, rest, tau):
    z, y, ids, values, r = _case(rest=bool(rest))
    ids[2, 1] = ids[2, 0]   # named twice
    ids[3, 2] = -1          # absent
    ids[4] = -1             # no teacher
    ids[0, 0] = y[0]        # the label among the ids
    kw = dict(labels=y if hard else None, alpha=0.3, tau=tau)
    if soft:
        kw.update(ids=ids, values=values, rest=r)
    _, _, dz = ol.loss(z, **kw)
    h = 1e-5
    for t in range(z.shape[0]):
        for v in range(z.shape[1]):
            zp, zm = z.copy(), z.copy()
            zp[t, v] += h
            zm[t, v] -= h
            ref = (ol.loss(zp, grad=False, **kw)[0][t] - ol.loss(zm, grad=False, **kw)[0][t]) / (2 * h)
            assert abs(dz[t, v] - ref) < 1e-8  # h^2 / 6 times third derivatives below 10
    if hard and not soft:
        assert np.allclose(dz.sum(1), 0, atol=1e-14)


def test_head_gradient_is_the_difference():
    r = np.random.RandomState(1)
    x, w = r.randn(4, 8), r.randn(23, 8) / 3
    z, y, ids, values, rest = _case(T=4)
    kw = dict(labels=y, ids=ids, values=values, rest=rest, alpha=0.4, tau=2.0)
    g = r.rand(4)
    _, stats, dx, dw = ol.head(x, w, dloss=g, **kw)
    f = lambda a, b: (g * ol.loss(a @ b.T, grad=False, **kw)[0]).sum()  # noqa: E731
    h = 1e-5
    for m, d in ((x, dx), (w, dw)):
        for i in np.ndindex(m.shape):
            old = m[i]
            m[i] = old + h
            up = f(x, w)
            m[i] = old - h
            dn = f(x, w)
            m[i] = old
            assert abs(d[i] - (up - dn) / (2 * h)) < 1e-7
    assert np.allclose(stats[:, 4:], np.take_along_axis(x @ w.T, ids, 1))


def test_top_logits_by_brute_force():
    r = np.random.RandomState(5)
    x = np.round(r.randn(7, 40) * 2)  # many ties
    x[2, 5] = np.nan
    x[3, :] = -np.inf
    x[4, 3] = 0.0
    x[4, 2] = -0.0
    ids, values, rest = ol.top_logits(x, 6)
    for t in range(7):
        key = lambda i: (-np.inf if np.isnan(x[t, i]) else -x[t, i], i)  # noqa: E731
        nan = [i for i in range(40) if np.isnan(x[t, i])]
        order = nan + sorted((i for i in range(40) if i not in nan), key=key)
        assert list(ids[t]) == order[:6]
        others = [x[t, i] for i in order[6:]]
        ref = np.log(np.exp(others).sum()) if t != 3 else -np.inf
        assert rest[t] == ref or abs(rest[t] - ref) < 1e-12
