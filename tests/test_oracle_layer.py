"""Pins of the layer operators' oracle: the packed format against its
definition by search, every gradient against central differences."""
import numpy as np
import pytest

from oracle import layer as ol
from oracle import ops


def test_e4m3_codes_are_the_nearest_values():
    vals = ol.e4m3_value(np.arange(256))
    assert vals[126] == 448 and vals[1] == 2.0 ** -9 and vals[8] == 2.0 ** -6 and np.isnan(vals[127])
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.uniform(-448, 448, 500), rng.uniform(-0.03, 0.03, 500), vals[np.isfinite(vals)],
                        (vals[:126] + vals[1:127]) / 2])
    fin = vals[np.isfinite(vals)]
    for x, c in zip(v, ol.e4m3_code(v)):
        assert abs(vals[c] - x) == np.abs(fin - x).min()
    assert np.all(ol.e4m3_code((vals[:126] + vals[1:127]) / 2) % 2 == 0)  # between two codes: the even one


def test_pack_takes_the_smallest_scale():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((40, 72)) * 2.0 ** rng.integers(-140, 120, (40, 1))
    x[0] = 0
    x[1, :32] = 448.0
    x[2, :32] = np.nextafter(448.0, 1e9)
    c, s = ol.pack(x)
    top = np.abs(np.pad(x, ((0, 0), (0, 24))).reshape(40, 3, 32)).max(-1)
    e = s.astype(int) - 127
    assert np.all(top <= 448 * 2.0 ** e) and np.all((e == -117) | (top > 448 * 2.0 ** (e - 1)))
    assert e[1, 0] == 0 and e[2, 0] == 1
    # half a step: 2^-4 of the value, or 2^-10 of the scale below 2^-6 of it
    err = np.abs(ol.values(c, s) - x)
    assert np.all(err <= np.maximum(np.abs(x) / 16, 2.0 ** -10 * 2.0 ** np.repeat(e, 32, 1)[:, :72]))


def test_pack_keeps_non_finite_apart():
    x = np.ones((1, 40))
    x[0, 3], x[0, 5], x[0, 7] = np.inf, np.nan, -np.inf
    v = ol.packed(x)
    assert np.isnan(v[0, [3, 5, 7]]).all() and np.delete(v, [3, 5, 7], 1).tolist() == [[1.0] * 37]
    big = np.full((1, 8), float(np.finfo(np.float32).max))
    assert ol.packed(big).tolist() == [[448 * 2.0 ** 119] * 8]


def _fd(f, v, h=1e-6):
    g = np.zeros_like(v)
    for i in np.ndindex(v.shape):
        old = v[i]
        v[i] = old + h
        a = f()
        v[i] = old - h
        b = f()
        v[i] = old
        g[i] = (a - b) / (2 * h)
    return g


@pytest.mark.parametrize("kind", ["swiglu", "gelu"])
def test_mlp_gradient(kind):
    rng = np.random.default_rng(2)
    h, da = rng.standard_normal((3, 8)) * 2, rng.standard_normal((3, 4 if kind == "swiglu" else 8))
    fd = _fd(lambda: np.sum(da * ol.mlp_act(h, kind)), h)
    np.testing.assert_allclose(ol.mlp_act_bwd(h, da, kind), fd, rtol=1e-6, atol=1e-8)
    same = ops.gelu_fwd(h) if kind == "gelu" else ops.swiglu_fwd(h[:, :4], h[:, 4:])
    np.testing.assert_allclose(ol.mlp_act(h, kind), same, rtol=1e-12, atol=1e-14)  # 1 + tanh cancels to 2^-53 there


@pytest.mark.parametrize("ln", [False, True])
@pytest.mark.parametrize("parts", ["both", "post", "pre"])
@pytest.mark.parametrize("rows", [0, 1, 3, 5])
def test_block_norm_gradients(ln, parts, rows):
    rng = np.random.default_rng(3)
    T, d = 5, 6
    x, y, dxo, dn = (rng.standard_normal((T, d)) for _ in range(4))
    vec = lambda: rng.standard_normal(d)  # noqa: E731
    post = (vec(), vec() if ln else None) if parts != "pre" else None
    pre = (vec(), vec() if ln else None) if parts != "post" else None
    gate = rng.standard_normal((-(-T // rows), d)) if rows and post else None
    kw = dict(gate=gate, gate_rows=rows, scale=0.7, ln=ln)

    def loss():
        xo, n, _ = ol.block_norm(x, y, post, pre, **kw)
        return np.sum(dxo * xo) + (0.0 if n is None else np.sum(dn * n))

    xo, _, stats = ol.block_norm(x, y, post, pre, **kw)
    g = ol.block_norm_bwd(dxo, None if pre is None else dn, y, xo, stats, post, pre, **kw)
    want = {"dx": x, "dy": y if post else None, "gate": gate, "w_post": post and post[0], "b_post": post and post[1],
            "w_pre": pre and pre[0], "b_pre": pre and pre[1]}
    for k, v in want.items():
        if v is None:
            assert g.get(k) is None
        else:
            np.testing.assert_allclose(g[k], _fd(loss, v), rtol=2e-6, atol=1e-7, err_msg=k)


def test_rotary_is_a_rotation_by_the_axis_positions():
    rng = np.random.default_rng(4)
    T, H, hd = 4, 2, 8
    x, pos = rng.standard_normal((T, H * hd)), rng.integers(0, 50, (2, T))
    out = ol.rotary(x, pos, [0, 1, 0], H, hd, 1e4)
    np.testing.assert_allclose(ol.rotary(out, pos, [0, 1, 0], H, hd, 1e4, inverse=True), x, atol=1e-13)
    z, w = x.reshape(T, H, hd), out.reshape(T, H, hd)
    for j, a in enumerate([0, 1, 0]):
        turn = np.exp(1j * pos[a] * 1e4 ** (-2 * j / 6))[:, None]
        np.testing.assert_allclose(w[..., j] + 1j * w[..., j + 3], (z[..., j] + 1j * z[..., j + 3]) * turn, atol=1e-12)
    np.testing.assert_array_equal(w[..., 6:], z[..., 6:])
