"""Refusals of the losses over a vocabulary (include/zl_loss.h): every call here is
turned down on the host, before anything is launched (no GPU)."""
import ctypes

import pytest

from paper_2608_07974_amd import zl

torch = pytest.importorskip("torch")
from paper_2608_07974_amd import loss as L  # noqa: E402

A = 1 << 20  # an address that is never used: 256-byte aligned
INV, UNS, WS = zl.ZL_ERR_INVALID_ARG, zl.ZL_ERR_UNSUPPORTED, zl.ZL_ERR_WORKSPACE
BIG = 1 << 45


def _refused(status, fn, *args, **kw):
    with pytest.raises(zl.ZlError) as ei:
        fn(*args, **kw)
    assert ei.value.status == status, ei.value
    return str(ei.value)


def _t(**kw):
    a = dict(labels=A, ids=A, values=A, rest=A, k=4, alpha=0.5, temperature=1.0)
    a.update(kw)
    return zl.zl_targets(**a)


BAD_TARGETS = [dict(labels=0, ids=0, values=0, rest=0, k=0), dict(k=0), dict(k=-1), dict(ids=0), dict(values=0),
               dict(ids=0, values=0, rest=0, k=3), dict(ids=0, values=0, k=0), dict(alpha=-0.1), dict(alpha=1.5),
               dict(alpha=float("nan")), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("inf")),
               dict(temperature=float("nan")), dict(temperature=1e-45), dict(labels=A + 2), dict(ids=A + 1),
               dict(values=A + 2), dict(rest=A + 3)]


@pytest.mark.parametrize("kw", [dict(T=-1), dict(V=0), dict(V=-5), dict(dtype=2), dict(dtype=-1), dict(x=0), dict(x=A + 1),
                                dict(ld=99), dict(k=0), dict(k=101), dict(k=-1), dict(ids=0), dict(values=0),
                                dict(ids=A + 2), dict(values=A + 1), dict(rest=A + 2), dict(tau=0.0),
                                dict(tau=float("nan")), dict(tau=float("inf")), dict(tau=1e-45)])
def test_top_logits_refuses(kw):
    a = dict(T=4, V=100, x=A, ld=100, dtype=zl.ZL_BF16, k=8, tau=1.0, ids=A, values=A, rest=A)
    a.update(kw)
    _refused(INV, zl.zl_top_logits, a["T"], a["V"], a["x"], a["ld"], a["dtype"], a["k"], a["tau"], a["ids"], a["values"],
             a["rest"])


@pytest.mark.parametrize("kw", [dict(T=(1 << 21) + 1), dict(T=BIG), dict(V=(1 << 30) + 1, ld=1 << 31),
                                dict(V=1 << 33, ld=1 << 34), dict(k=257, V=300, ld=300)])
def test_top_logits_limits(kw):
    a = dict(T=4, V=100, ld=100, k=8)
    a.update(kw)
    _refused(UNS, zl.zl_top_logits, a["T"], a["V"], A, a["ld"], zl.ZL_F32, a["k"], 1.0, A, A, A)


@pytest.mark.parametrize("kw", BAD_TARGETS)
def test_targets_refused(kw):
    t = _t(**kw)
    _refused(INV, zl.zl_logit_loss, 4, 100, A, 100, zl.ZL_F32, t, A, A)
    _refused(INV, zl.zl_logit_loss_backward, 4, 100, A, 100, zl.ZL_F32, t, A, A, 1.0, A, 100)
    _refused(INV, zl.zl_head_loss, _head(targets=t))
    _refused(INV, zl.zl_head_loss_backward, _head(True, targets=t))


@pytest.mark.parametrize("tau", [2.0 ** -61, 4e-39, 2.0 ** 61, 1e38])
def test_temperatures_refused(tau):
    # log2(e) / tau or tau^2 leaves fp32
    t = _t(temperature=tau)
    for said in (_refused(INV, zl.zl_top_logits, 4, 100, A, 100, zl.ZL_F32, 8, tau, A, A, A),
                 _refused(INV, zl.zl_logit_loss, 4, 100, A, 100, zl.ZL_F32, t, A, A),
                 _refused(INV, zl.zl_logit_loss_backward, 4, 100, A, 100, zl.ZL_F32, t, A, A, 1.0, A, 100),
                 _refused(INV, zl.zl_head_loss, _head(targets=t)), _refused(INV, zl.zl_head_loss_backward, _head(True, targets=t))):
        assert "temperature" in said


@pytest.mark.parametrize("kw", [dict(T=-1), dict(V=0), dict(z=0), dict(z=A + 2), dict(ld=99), dict(dtype=7), dict(loss=0),
                                dict(stats=0), dict(stats=A + 8), dict(loss=A + 2)])
def test_logit_loss_refuses(kw):
    a = dict(T=4, V=100, z=A, ld=100, dtype=zl.ZL_F32, loss=A, stats=A)
    a.update(kw)
    _refused(INV, zl.zl_logit_loss, a["T"], a["V"], a["z"], a["ld"], a["dtype"], _t(), a["loss"], a["stats"])


@pytest.mark.parametrize("kw", [dict(T=-1), dict(V=0), dict(z=0), dict(ld=99), dict(dtype=7), dict(stats=0), dict(stats=A + 4),
                                dict(dloss=A + 2), dict(dz=0), dict(dz=A + 1), dict(ldo=99), dict(ldo=128)])
def test_logit_loss_backward_refuses(kw):
    """(ldo 128: dz is z, with another stride)"""
    a = dict(T=4, V=100, z=A, ld=100, dtype=zl.ZL_F32, stats=A, dloss=A, dz=A, ldo=100)
    a.update(kw)
    _refused(INV, zl.zl_logit_loss_backward, a["T"], a["V"], a["z"], a["ld"], a["dtype"], _t(), a["stats"], a["dloss"], 1.0,
             a["dz"], a["ldo"])


def test_logit_loss_limits():
    for T, V, t in (((1 << 21) + 1, 100, _t()), (4, (1 << 30) + 1, _t()), (4, 1 << 40, _t()), (4, 1000, _t(k=257))):
        _refused(UNS, zl.zl_logit_loss, T, V, A, 1 << 41, zl.ZL_F32, t, A, A)
        _refused(UNS, zl.zl_logit_loss_backward, T, V, A, 1 << 41, zl.ZL_F32, t, A, A, 1.0, A, 1 << 41)


def _head(back=False, **kw):
    a = dict(T=4, V=100, d=64, dtype=zl.ZL_BF16, x=A, ldx=64, w=A, ldw=64, targets=_t(), stats=A, workspace=A,
             workspace_bytes=1 << 40)
    if back:
        a.update(dloss=A, scale=1.0, dx=A, lddx=64, dx_dtype=zl.ZL_BF16, dw=A, lddw=64, dw_dtype=zl.ZL_F32, accumulate=1)
    else:
        a.update(loss=A)
    a.update(kw)
    return zl.zl_head_args(**a)


BAD_HEAD = [dict(T=-1), dict(V=0), dict(d=0), dict(d=-8), dict(d=60), dict(dtype=2), dict(x=0), dict(w=0), dict(x=A + 8),
            dict(w=A + 8), dict(ldx=56), dict(ldx=68), dict(ldw=56), dict(ldw=68), dict(stats=0), dict(stats=A + 2)]


@pytest.mark.parametrize("kw", BAD_HEAD + [dict(loss=0), dict(loss=A + 1)])
def test_head_loss_refuses(kw):
    _refused(INV, zl.zl_head_loss, _head(**kw))


@pytest.mark.parametrize("kw", BAD_HEAD + [dict(dx=0, dw=0), dict(dloss=A + 2), dict(columns=-1), dict(dx_dtype=2),
                                           dict(dw_dtype=-1), dict(dx=A + 8), dict(dw=A + 8), dict(lddx=56), dict(lddx=68),
                                           dict(lddw=56), dict(lddw=68)])
def test_head_loss_backward_refuses(kw):
    _refused(INV, zl.zl_head_loss_backward, _head(True, **kw))


@pytest.mark.parametrize("kw", [dict(dx=0, dw=0), dict(dx=0, dw=0, x=0, stats=0, dloss=0, workspace=0, workspace_bytes=0),
                                dict(dx=0, dw=0, targets=_t(labels=0, ids=0, values=0, rest=0, k=0))])
def test_head_loss_backward_of_nothing_is_not_invalid(kw):
    """No rows, no dw: nothing to do, as of empty tensors, which have no addresses."""
    try:
        zl.zl_head_loss_backward(_head(True, T=0, accumulate=0, **kw))
    except zl.ZlError as e:
        assert e.status == zl.ZL_ERR_HIP, e  # (a machine without a GPU)


def test_head_loss_limits():
    for kw in (dict(T=(1 << 21) + 1), dict(V=(1 << 30) + 1), dict(d=65544, ldx=65544, ldw=65544), dict(ldx=1 << 21),
               dict(ldw=1 << 21), dict(targets=_t(k=257))):
        _refused(UNS, zl.zl_head_loss, _head(**kw))
        _refused(UNS, zl.zl_head_loss_backward, _head(True, **kw))
    assert "2^36" in _refused(UNS, zl.zl_head_loss, _head(T=1 << 20, V=(1 << 16) + 1))
    assert "accumulation" in _refused(UNS, zl.zl_head_loss_backward, _head(True, dw_dtype=zl.ZL_BF16))
    wide = dict(T=1 << 18, d=4096, ldx=4096, ldw=4096, lddx=4096, lddw=4096)
    assert "2^30" in _refused(UNS, zl.zl_head_loss_backward, _head(True, **wide))


def test_head_loss_backward_beyond_a_launch():
    # a thread per eight elements: 2^32 of them are one launch too many
    rows = dict(T=1 << 21, d=16384, ldx=16384, ldw=16384, lddx=16384, lddw=16384)
    assert "2^35" in _refused(UNS, zl.zl_head_loss_backward, _head(True, **rows, dw=0))
    wide = dict(V=1 << 30, d=64, ldx=64, ldw=64, lddx=64, lddw=64)
    assert "2^35" in _refused(UNS, zl.zl_head_loss_backward, _head(True, **wide))
    assert "2^35" in _refused(UNS, zl.zl_head_loss_backward, _head(True, **wide, T=0))


def test_head_loss_workspace():
    for back in (False, True):
        fn = zl.zl_head_loss_backward if back else zl.zl_head_loss
        need = zl.zl_head_loss_workspace(4, 100, 64, zl.ZL_BF16, 4, True, back, True, True)
        assert 0 < need < 1 << 23
        _refused(WS, fn, _head(back, workspace=0))
        _refused(WS, fn, _head(back, workspace_bytes=need - 1))
        _refused(WS, fn, _head(back, workspace=A + 128))
    assert zl.zl_head_loss_workspace(0, 100, 64, zl.ZL_BF16) == 0
    # smaller pieces need less, and none is larger than 1 GiB of dL/dz
    a = [zl.zl_head_loss_workspace(16384, 128256, 4096, zl.ZL_BF16, backward=True, columns=c) for c in (256, 8192, 0, 1 << 20)]
    assert a[0] < a[1] < a[2] == a[3]
    assert zl.zl_head_loss_workspace(1 << 21, 1 << 30, 8, zl.ZL_F32, 256, True, True) < 1 << 40
    for kw in (dict(T=-1), dict(V=0), dict(d=4), dict(dtype=3), dict(k=-1), dict(columns=-1)):
        b = dict(T=4, V=100, d=64, dtype=zl.ZL_BF16, k=0, columns=0)
        b.update(kw)
        _refused(INV, zl.zl_head_loss_workspace, b["T"], b["V"], b["d"], b["dtype"], b["k"], columns=b["columns"])
    for kw in (dict(T=1 << 40), dict(V=1 << 31), dict(d=1 << 20), dict(k=1000)):
        b = dict(T=4, V=100, d=64, k=0)
        b.update(kw)
        _refused(UNS, zl.zl_head_loss_workspace, b["T"], b["V"], b["d"], zl.ZL_BF16, b["k"])


def test_head_loss_workspace_of_labels_alone():
    """One partial sum per row and column block: 8 bytes, where a teacher may take a pair."""
    for T, V, d, width in ((16384, 128256, 4096, 128), (1, 128256, 4096, 64), (4, 100, 64, 32)):
        n = zl.zl_head_loss_workspace(T, V, d, zl.ZL_BF16)
        sums = T * -(-V // width) * 8
        assert sums <= n <= sums + 4 * T + 512, (T, V)
        assert zl.zl_head_loss_workspace(T, V, d, zl.ZL_BF16, k=1) >= n + sums


def test_null_argument_structures():
    lib = zl.load()
    assert lib.zl_logit_loss(4, 100, A, 100, 0, None, A, A, None) == INV
    assert lib.zl_logit_loss_backward(4, 100, A, 100, 0, None, A, A, 1.0, A, 100, None) == INV
    assert lib.zl_head_loss(None, None) == INV
    assert lib.zl_head_loss_backward(None, None) == INV
    assert lib.zl_head_loss_workspace(4, 100, 64, 0, 0, 0, 0, 1, 0, 0, None) == INV


def test_argument_structures_as_bytes():
    """The two ways to give them are the same bytes."""
    t = _t()
    assert bytes(t)[:44] == zl.pack_targets(A, A, A, A, 4, 0.5, 1.0)[:44]
    assert len(zl.pack_targets(A, A, A, A, 4, 0.5, 1.0)) == ctypes.sizeof(zl.zl_targets)
    h = _head(True, loss=A + 64, columns=512)
    p = zl.pack_head_args(4, 100, 64, zl.ZL_BF16, A, 64, A, 64, A, A, A, A, 4, 0.5, 1.0, A, A + 64, A, 1.0, 512, A, 64,
                          zl.ZL_BF16, A, 64, zl.ZL_F32, 1, A, 1 << 40)
    assert len(p) == ctypes.sizeof(h)
    back = zl.zl_head_args.from_buffer_copy(p)
    for name, _ in zl.zl_head_args._fields_:
        if name != "targets":
            assert getattr(back, name) == getattr(h, name), name


def test_torch_functions_refuse_host_tensors():
    z, y = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        L.logit_loss(z, y)
    with pytest.raises(ValueError, match="GPU"):
        L.top_logits(z, 2)
    with pytest.raises(ValueError, match="GPU"):
        L.head_loss(torch.zeros(4, 16), torch.zeros(10, 16), y)


@pytest.mark.parametrize("fn", [
    lambda z, y: L.logit_loss(z),                                     # no targets
    lambda z, y: L.logit_loss(z, y[:3]),                              # short labels
    lambda z, y: L.logit_loss(z, y.long()),                           # labels' type
    lambda z, y: L.logit_loss(z.double(), y),                         # logits' type
    lambda z, y: L.logit_loss(z[0], y),                               # not a matrix
    lambda z, y: L.logit_loss(z.t(), y),                              # columns apart
    lambda z, y: L.logit_loss(z[:1].expand(4, 10), y),                # rows on one another
    lambda z, y: L.logit_loss(z, y, L.TopLogits(y[:, None], None)),   # values missing
    lambda z, y: L.logit_loss(z, y, L.TopLogits(y[:, None], torch.zeros(4, 2))),
    lambda z, y: L.logit_loss_bwd(z, torch.zeros(4, 5), y),           # stats' shape
    lambda z, y: L.logit_loss_bwd(z, torch.zeros(4, 4), y, dloss=torch.zeros(3)),
    lambda z, y: L.logit_loss_bwd(z, torch.zeros(4, 4), y, out=torch.zeros(4, 10).bfloat16()),
    lambda z, y: L.top_logits(z, 2, out=L.TopLogits(torch.zeros(4, 3, dtype=torch.int32), torch.zeros(4, 2))),
    lambda z, y: L.head_loss(z[:, :8], torch.zeros(5, 16), y),        # widths differ
    lambda z, y: L.head_loss(z[:, :8], torch.zeros(5, 8).bfloat16(), y),
    lambda z, y: L.head_loss_bwd(z[:, :8], torch.zeros(5, 8), torch.zeros(4, 3), y),
])
def test_torch_functions_refuse(fn):
    with pytest.raises((ValueError, TypeError)):
        fn(torch.zeros(4, 10), torch.zeros(4, dtype=torch.int32))
