"""Refusals of the layer operators (include/zl_layer.h): every call here is
turned down on the host, before anything is launched (no GPU)."""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest

from paper_2608_07974_amd import zl

torch = pytest.importorskip("torch")
from paper_2608_07974_amd import layer  # noqa: E402

A = 1 << 20  # an address that is never used: 16-byte aligned
INV, UNS, WS = zl.ZL_ERR_INVALID_ARG, zl.ZL_ERR_UNSUPPORTED, zl.ZL_ERR_WORKSPACE


def _refused(status, fn, *args, **kw):
    with pytest.raises(zl.ZlError) as ei:
        fn(*args, **kw)
    assert ei.value.status == status, ei.value
    return str(ei.value)


def _pk(n=64, codes=A, scales=A, ldc=None, lds=None):
    return zl.zl_packed(codes, scales, n if ldc is None else ldc, -(-n // 32) if lds is None else lds)


@pytest.mark.parametrize("kw", [dict(T=-1), dict(n=0), dict(n=60), dict(n=-8), dict(x=0), dict(x=A + 8), dict(ldx=56),
                                dict(ldx=68), dict(dtype=2), dict(p=_pk(codes=0)), dict(p=_pk(scales=0)),
                                dict(p=_pk(codes=A + 8)), dict(p=_pk(ldc=72)), dict(p=_pk(ldc=48)),
                                dict(p=_pk(lds=1))])
def test_pack_refuses(kw):
    a = dict(T=4, n=64, x=A, ldx=64, dtype=zl.ZL_BF16, p=_pk())
    a.update(kw)
    _refused(INV, zl.zl_pack, a["T"], a["n"], a["x"], a["ldx"], a["dtype"], a["p"])
    _refused(INV, zl.zl_unpack, a["T"], a["n"], a["p"], a["x"], a["ldx"], a["dtype"])


def test_null_argument_structures():
    lib = zl.load()
    assert lib.zl_pack(4, 64, A, 64, zl.ZL_F32, None, None) == INV
    assert lib.zl_unpack(4, 64, None, A, 64, zl.ZL_F32, None) == INV
    for f in (lib.zl_mlp_act, lib.zl_mlp_act_backward, lib.zl_block_norm, lib.zl_block_norm_backward):
        assert f(None, None) == INV
    assert lib.zl_block_norm_workspace(4, 64, 0, None) == INV
    assert lib.zl_wgrad_packed(4, 8, 8, A, 8, zl.ZL_F32, None, 1.0, 0, A, 8, None, 0, None) == INV


def _mlp(back, **kw):
    a = dict(T=4, ff=64, kind=zl.ZL_MLP_SWIGLU, in_dtype=zl.ZL_BF16, out_dtype=zl.ZL_BF16, h=A, ldh=128,
             packed=zl.zl_packed(), a=A, lda=64)
    if back:
        a.update(da=A, ldda=64, dh=A, lddh=128)
    a.update(kw)
    return zl.zl_mlp_args(**a)


@pytest.mark.parametrize("kw", [dict(T=-1), dict(ff=60), dict(ff=0), dict(kind=2), dict(in_dtype=2), dict(out_dtype=-1),
                                dict(h=0), dict(h=A + 2), dict(ldh=120), dict(a=A + 8), dict(lda=56),
                                dict(packed=_pk(64))])
@pytest.mark.parametrize("back", [False, True])
def test_mlp_refuses(back, kw):
    _refused(INV, zl.zl_mlp_act_backward if back else zl.zl_mlp_act, _mlp(back, **kw))


def test_mlp_refuses_more():
    _refused(INV, zl.zl_mlp_act, _mlp(False, a=0))
    for kw in (dict(da=0), dict(dh=0), dict(ldda=56), dict(lddh=64), dict(packed=_pk(128))):  # the last: h as well
        _refused(INV, zl.zl_mlp_act_backward, _mlp(True, **kw))
    for back in (False, True):  # 8-bit blocks that both halves would share
        kw = dict(ff=40, ldh=80, packed=_pk(80), h=0 if back else A)
        _refused(UNS, zl.zl_mlp_act_backward if back else zl.zl_mlp_act, _mlp(back, **kw))


def test_more_columns_than_numbers_of_32_bits():
    n = (1 << 30) + 32
    p, io = _pk(n), dict(ldh=n, lda=n)
    _refused(UNS, zl.zl_pack, 1, n, A, n, zl.ZL_BF16, p)
    _refused(UNS, zl.zl_unpack, 1, n, p, A, n, zl.ZL_BF16)
    _refused(UNS, zl.zl_wgrad_packed, 1, n, 64, A, n, zl.ZL_BF16, _pk(), A, 64)
    _refused(UNS, zl.zl_wgrad_packed, 1, 64, n, A, 64, zl.ZL_BF16, p, A, n)
    for back in (False, True):
        fn, bw = (zl.zl_mlp_act_backward, dict(ldda=n, lddh=n)) if back else (zl.zl_mlp_act, {})
        _refused(UNS, fn, _mlp(back, T=1, ff=n, kind=zl.ZL_MLP_GELU, **io, **bw))
        _refused(UNS, fn, _mlp(back, T=1, ff=n // 2, **io, **bw))


def _norm(back, **kw):
    a = dict(T=4, d=64, layernorm=0, in_dtype=zl.ZL_BF16, out_dtype=zl.ZL_BF16, eps=1e-5, scale=1.0, w_post=A, w_pre=A,
             gate=A, gate_rows=4, stats=A, xo=A, ldx=64, y=A, ldy=64, ldn=64)
    if back:
        a.update(dn=A, dx=A, dy=A, dw_post=A, dw_pre=A, dgate=A, grad_scale=1.0, workspace=A, workspace_elems=1 << 30)
    else:
        a.update(x=A, n=A)
    a.update(kw)
    return zl.zl_norm_args(**a)


@pytest.mark.parametrize("kw", [dict(T=-1), dict(d=60), dict(d=0), dict(in_dtype=3), dict(out_dtype=3), dict(eps=0.0),
                                dict(eps=float("nan")), dict(eps=float("inf")), dict(w_post=0, w_pre=0),
                                dict(w_post=A + 4), dict(b_post=A), dict(b_pre=A), dict(gate_rows=0),
                                dict(gate_rows=-3), dict(gate=A + 4), dict(w_post=0), dict(stats=0), dict(stats=A + 8),
                                dict(xo=0), dict(ldx=60), dict(ldx=56), dict(y=0), dict(y=A + 2), dict(ldy=8),
                                dict(ldn=8), dict(y_packed=_pk(32))])
@pytest.mark.parametrize("back", [False, True])
def test_block_norm_refuses(back, kw):
    _refused(INV, zl.zl_block_norm_backward if back else zl.zl_block_norm, _norm(back, **kw))


def test_block_norm_refuses_more():
    for kw in (dict(x=0), dict(n=0), dict(n_packed=_pk(32)), dict(w_pre=0, n_packed=_pk())):
        _refused(INV, zl.zl_block_norm, _norm(False, **kw))
    for kw in (dict(dx=0), dict(dn=0), dict(dy=0), dict(db_post=A), dict(db_pre=A), dict(gate=0), dict(dgate=A + 4),
               dict(w_pre=0), dict(dxo=A + 4), dict(y_packed=_pk())):
        _refused(INV, zl.zl_block_norm_backward, _norm(True, **kw))
    for back in (False, True):
        kw = dict(d=8200, ldx=8200, ldy=8200, ldn=8200)
        _refused(UNS, zl.zl_block_norm_backward if back else zl.zl_block_norm, _norm(back, **kw))
    need = zl.zl_block_norm_workspace(4, 64, 4)
    for kw in (dict(workspace=0), dict(workspace=A + 4), dict(workspace_elems=need - 1)):
        _refused(WS, zl.zl_block_norm_backward, _norm(True, **kw))


def test_block_norm_workspace_is_bounded():
    """Four partial rows per block and some of the gate's, of a number of blocks
    that does not grow with the rows."""
    for T in (0, 1, 5, 255, 256, 4096, 16384, 1000000):
        for d in (8, 768, 4096, 8192):
            for rows in (0, 1, 7, 64, 1000, 5000, T, 2 * T + 1):
                part = zl.zl_block_norm_workspace(T, d, rows) // d
                assert 4 * min(T, 1) <= part <= min(10 * T, 45000), (T, d, rows)
    for args in ((-1, 64, 0), (4, 60, 0), (4, 64, -1)):
        _refused(INV, zl.zl_block_norm_workspace, *args)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), INV), (dict(T=1 << 31), UNS), (dict(M=60), INV), (dict(N=0), INV), (dict(dy=0), INV), (dict(dy=A + 4), INV),
    (dict(lddy=56), INV), (dict(dtype=5), INV), (dict(p=_pk(32)), INV), (dict(p=_pk(codes=A + 8)), INV), (dict(dw=0), INV),
    (dict(dw=A + 4), INV), (dict(lddw=56), INV), (dict(ws=A + 4), INV)])
def test_wgrad_refuses(kw, status):
    a = dict(T=4, M=64, N=64, dy=A, lddy=64, dtype=zl.ZL_BF16, p=_pk(), dw=A, lddw=64, ws=0)
    a.update(kw)
    _refused(status, zl.zl_wgrad_packed, a["T"], a["M"], a["N"], a["dy"], a["lddy"], a["dtype"], a["p"], a["dw"], a["lddw"],
             workspace=a["ws"], workspace_elems=1000)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), INV), (dict(H=0), INV), (dict(hd=7), INV), (dict(hd=0), INV), (dict(hd=258, rot=16), UNS), (dict(rot=3), INV),
    (dict(rot=0), INV), (dict(rot=18), INV), (dict(axes=bytes([0, 1, 2, 0, 1, 2, 3, 0])), INV), (dict(na=0), INV),
    (dict(na=17), INV), (dict(theta=1.0), INV), (dict(theta=float("nan")), INV), (dict(theta=float("inf")), INV),
    (dict(x=0), INV), (dict(out=0), INV), (dict(pos=0), INV), (dict(pos=A + 2), INV), (dict(x=A + 1), INV),
    (dict(ldx=60), INV), (dict(ldo=63), INV), (dict(ldo=72), INV), (dict(dtype=9), INV), (dict(H=1 << 22, ldx=1 << 30), UNS)])
def test_rotary_refuses(kw, status):
    a = dict(T=4, H=4, hd=16, rot=16, x=A, ldx=64, out=A, ldo=64, dtype=zl.ZL_BF16, pos=A, na=3,
             axes=bytes([0, 1, 2, 0, 1, 2, 0, 0]), theta=1e4)
    a.update(kw)
    if len(a["axes"]) < a["rot"] // 2:
        a["axes"] = bytes(a["rot"] // 2)
    _refused(status, zl.zl_rotary, a["T"], a["H"], a["hd"], a["rot"], a["x"], a["ldx"], a["out"], a["ldo"], a["dtype"],
             a["pos"], a["na"], a["axes"], a["theta"])


def test_rotary_needs_every_axis_number():
    with pytest.raises(ValueError, match="axis numbers"):
        zl.zl_rotary(4, 4, 16, 16, A, 64, A, 64, zl.ZL_BF16, A, 3, bytes(7), 1e4)
    assert zl.load().zl_rotary(4, 4, 16, 16, A, 64, A, 64, zl.ZL_BF16, A, 3, None, 1e4, 0, None) == INV


def test_structures_match_the_header():
    """Sizes that the C compiler gives the argument structures."""
    assert ctypes.sizeof(zl.zl_packed) == 32
    assert ctypes.sizeof(zl.zl_mlp_args) == 8 + 16 + 16 + 32 + 3 * 16
    assert ctypes.sizeof(zl.zl_norm_args) == 8 + 24 + 6 * 8 + 8 + 7 * 8 + 64 + 9 * 8 + 8 + 16


def test_packed_bytes_are_the_structures():
    """The one-step byte forms of the argument structures hold the same bytes as
    the structures filled field by field."""
    def values(cls, at):
        out = []
        for _, ty in cls._fields_:
            if ty is zl.zl_packed:
                v, sub = values(ty, at)
                out += sub
                at = v
            else:
                at += 1
                out.append(at + 0.5 if ty is ctypes.c_float else at)
        return at, out

    def filled(cls, vals):
        args = []
        for _, ty in cls._fields_:
            args.append(filled(ty, vals) if ty is zl.zl_packed else vals.pop(0))
        return cls(*args)

    for cls, pack in ((zl.zl_packed, zl.pack_packed), (zl.zl_mlp_args, zl.pack_mlp_args), (zl.zl_norm_args, zl.pack_norm_args)):
        vals = values(cls, 100)[1]
        assert pack(*vals) == bytes(filled(cls, list(vals)))
    # and the library reads them
    _refused(INV, zl.zl_pack, 4, 64, A, 64, zl.ZL_F32, zl.pack_packed(0, A, 64, 2))
    _refused(INV, zl.zl_pack, 4, 64, A, 64, zl.ZL_F32, zl.pack_packed(A, A, 72, 2))
    _refused(UNS, zl.zl_mlp_act, zl.pack_mlp_args(4, 40, 0, 1, 1, A, 80, A, A, 80, 3, A, 40, 0, 0, 0, 0))


def test_torch_layer_refuses_host_tensors_and_bad_shapes():
    """The torch functions check what the library cannot see: placement,
    shapes, types, overlapping rows."""
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError, match="GPU"):
        layer.pack(x, out=layer.Packed.empty(4, 64, "cpu"))
    with pytest.raises(ValueError, match="out must be on"):
        layer._check_device(torch.device("cuda", 0), "x out", None, x)
    with pytest.raises(ValueError):
        layer.pack(x, out=layer.Packed.empty(3, 64, "cpu"))
    with pytest.raises(TypeError):
        layer.pack(x.half())
    with pytest.raises(ValueError, match="contiguous rows"):
        layer.pack(torch.zeros(64, 4).t())
    with pytest.raises(ValueError, match="overlap"):
        layer.pack(torch.zeros(1, 64).expand(4, 64))
    with pytest.raises(ValueError):  # the last code row would be read past its end
        layer.Packed(torch.zeros(4, 72, dtype=torch.uint8), torch.zeros(4, 3, dtype=torch.uint8), 72)
    with pytest.raises(TypeError):
        layer.Packed(x, torch.zeros(4, 2, dtype=torch.uint8), 64)
    with pytest.raises(ValueError):
        layer.mlp_act(torch.zeros(4, 65))
    with pytest.raises(KeyError):
        layer.mlp_act(x, "relu")
    with pytest.raises(ValueError):
        layer.mlp_act_bwd(x, torch.zeros(4, 64))
    with pytest.raises(TypeError):  # h and its gradient of two types
        layer.mlp_act_bwd(x, torch.zeros(4, 32, dtype=torch.bfloat16))
    w = torch.ones(64)
    for kw in (dict(y=None), dict(post=None), dict(post=(torch.ones(63), None)), dict(gate=torch.ones(3, 64), gate_rows=2),
               dict(gate=torch.ones(2, 64)), dict(stats=torch.zeros(4, 3)), dict(xo=torch.zeros(4, 72)[:, :64]),
               dict(n=torch.zeros(4, 64), pre=None)):
        a = dict(y=x, post=(w, None), pre=(w, None))
        a.update(kw)
        with pytest.raises(ValueError):
            layer.block_norm(x, **a)
    st = torch.zeros(4, 4)
    for kw in (dict(dn=None), dict(y=None), dict(xo=None), dict(dy=torch.zeros(4, 72)[:, :64]),
               dict(grads=layer.NormGrads(gate=torch.zeros(1, 64))), dict(grads=layer.NormGrads(w_pre=torch.zeros(63))),
               dict(dxo=torch.zeros(4, 72)[:, :64])):
        a = dict(dxo=x, dn=x, y=x, xo=x, stats=st, post=(w, None), pre=(w, None))
        a.update(kw)
        with pytest.raises(ValueError):
            layer.block_norm_bwd(**a)
    with pytest.raises(ValueError):
        layer.wgrad(torch.zeros(3, 8), layer.Packed.empty(4, 64, "cpu"))
    with pytest.raises(TypeError):
        layer.rotary(x, torch.zeros(3, 4), bytes(8), 4, 16, 1e4)
    with pytest.raises(TypeError):
        layer.rotary(x, torch.zeros(3, 5, dtype=torch.int32), bytes(8), 4, 16, 1e4)
    with pytest.raises(ValueError):
        layer.rotary(x, torch.zeros(3, 4, dtype=torch.int32), bytes(8), 5, 16, 1e4)


@pytest.fixture
def on_host(monkeypatch):
    """The torch functions up to the library's call, on host tensors; returns the
    list of calls (the library's function and its arguments)."""
    calls = []
    monkeypatch.setattr(layer, "_check_device", lambda *a: None)
    monkeypatch.setattr(layer, "_call", lambda fn, dev, *args: calls.append((fn, args)))
    return calls


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float16, torch.float64])
def test_tensors_made_here_have_types_of_their_own(on_host, monkeypatch, default):
    """Whatever torch's default type: the workspace has the bytes of the floats that
    the library is told of, statistics and gradients are fp32."""
    made, empty = [], torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: made.append(empty(*a, **kw)) or made[-1])
    f32 = dict(dtype=torch.float32)
    x, w = torch.zeros(512, 256, **f32), (torch.ones(256, **f32), None)
    torch.set_default_dtype(default)
    try:
        _, n, stats = layer.block_norm(x, x, w, w)
        dx, dy = layer.block_norm_bwd(x, x, x, x, stats, w, w)
        dws = [layer.wgrad(x, layer.Packed.empty(512, 64, "cpu"), accumulate=a) for a in (False, True)]
        others = [layer.pack(x).codes, layer.unpack(layer.Packed.empty(4, 64, "cpu")), layer.mlp_act(x), layer.mlp_act_bwd(x, x[:, :128])]
    finally:
        torch.set_default_dtype(torch.float32)
    assert all(t.dtype == torch.float32 for t in (n, stats, dx, dy, *dws))
    assert [t.dtype for t in others] == [torch.uint8, torch.bfloat16, torch.float32, torch.float32]
    fn, (args,) = on_host[1]
    args = zl.zl_norm_args.from_buffer_copy(args)
    ws, = (t for t in made if t.data_ptr() == args.workspace)
    need = zl.zl_block_norm_workspace(512, 256)
    assert fn is zl.zl_block_norm_backward and args.workspace_elems >= need > 0
    assert ws.numel() * ws.element_size() >= 4 * args.workspace_elems


@pytest.mark.parametrize("dtype", ["ZL_F32", "ZL_BF16"])
@pytest.mark.parametrize("ld", [0, -8, 1 << 62])
def test_wgrad_of_no_tokens_reads_no_stride(dtype, ld):
    """T = 0: operands and strides may be anything.  In a process of its own that
    sees no GPU, where the launch is what fails."""
    code = f"""
from paper_2608_07974_amd import zl
try:
    zl.zl_wgrad_packed(0, 64, 64, 0, {ld}, zl.{dtype}, zl.zl_packed(0, 0, {ld}, {ld}), {A}, 64)
except zl.ZlError as e:
    print("status", e.status)
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, env=dict(os.environ, HIP_VISIBLE_DEVICES="-1"),
                       capture_output=True, text=True, timeout=120)
    assert (r.returncode, r.stdout.split()) == (0, ["status", str(zl.ZL_ERR_HIP)]), (r.returncode, r.stdout, r.stderr)


def test_packed_follows_its_tensors():
    """Tensors of a Packed that are replaced, resized or given other strides: the
    call takes them as they are then, or refuses them."""
    u8 = dict(dtype=torch.uint8)
    new = lambda: layer.Packed(torch.zeros(4, 64, **u8), torch.zeros(4, 2, **u8), 64)  # noqa: E731
    p = new()
    wide = torch.zeros(4, 160, **u8)
    p.codes, p.scales = wide[:, 32:96], torch.zeros(4, 8, **u8)[:, 3:5]
    assert p.fields() == (wide.data_ptr() + 32, p.scales.data_ptr(), 160, 8)
    assert layer._packed("p", p, 4, 64) == p.fields()
    p = new()
    p.codes.resize_(4, 80)
    p.scales.set_(torch.zeros(4, 5, **u8))
    assert p.fields()[2:] == (80, 5)

    def refused(change, error=ValueError, match=None):
        p = new()
        change(p)
        with pytest.raises(error, match=match):
            p.fields()

    refused(lambda p: setattr(p, "codes", torch.zeros(4, 48, **u8)))
    refused(lambda p: setattr(p, "codes", torch.zeros(3, 64, **u8)))
    refused(lambda p: setattr(p, "codes", torch.zeros(64, 4, **u8).t()), match="contiguous rows")
    refused(lambda p: setattr(p, "codes", torch.zeros(1, 64, **u8).expand(4, 64)), match="overlap")
    refused(lambda p: setattr(p, "codes", torch.zeros(4, 64)), TypeError)
    refused(lambda p: setattr(p, "codes", torch.zeros(4, 4, 64, **u8)), TypeError)
    refused(lambda p: setattr(p, "scales", torch.zeros(4, 1, **u8)))
    refused(lambda p: setattr(p, "scales", torch.zeros(4, 2, device="meta", **u8)), match="scales on meta")
    refused(lambda p: setattr(p, "n", 72))
    refused(lambda p: p.codes.resize_(4, 32))
    refused(lambda p: p.codes.resize_(0), TypeError)
    refused(lambda p: p.scales.resize_(2, 2))
    refused(lambda p: p.codes.t_())
    class On:  # stands for a tensor on GPU 1 or 2
        def __init__(self, index):
            self.index = self.device = index

        def get_device(self):
            return self.index

    dev = torch.device("cuda", 1)
    for codes, scales, bad in ((1, 1, None), (1, 2, "out.scales"), (2, 1, "out"), (2, 2, "out.scales")):
        p = new()
        p.codes, p.scales = On(codes), On(scales)
        if bad is None:
            layer._check_device(dev, "x out", None, p)
        else:
            with pytest.raises(ValueError, match=f"{bad} must be on"):
                layer._check_device(dev, "x out", None, p)
    p = type("Own", (layer.Packed,), {})(torch.zeros(4, 64, **u8), torch.zeros(4, 2, **u8), 64)
    with pytest.raises(ValueError, match="out.scales must be on"):  # a class of the user's
        layer._check_device(dev, "x out", None, p)
    with pytest.raises(ValueError):
        p = new()
        p.codes.resize_(3, 64)
        p.scales.resize_(3, 2)
        layer._packed("p", p, 4, 64)


@pytest.mark.parametrize("make", [bytes, list, tuple, bytearray, lambda a: memoryview(bytes(a)), np.array, torch.tensor,
                                  lambda a: np.array(a, np.int32), lambda a: np.array(a, np.uint8),
                                  lambda a: np.array([a, a]).T[:, 0], lambda a: torch.tensor(a, dtype=torch.uint8)])
def test_rotary_takes_axis_numbers_one_by_one(monkeypatch, make):
    """Axis numbers in any sequence of integers: their values, not their memory."""
    axes, seen = [0, 1, 2, 0, 1, 2, 2, 1], []

    class Lib:
        @staticmethod
        def zl_rotary(*a):
            seen.append(a[11])
            return zl.ZL_OK

    monkeypatch.setattr(zl, "load", lambda: Lib)
    monkeypatch.setattr(layer, "_check_device", lambda *a: None)
    monkeypatch.setattr(layer, "_call", lambda fn, dev, *args: fn(*args, 0))
    zl.zl_rotary(4, 4, 16, 16, A, 64, A, 64, zl.ZL_BF16, A, 3, make(axes), 1e4)
    layer.rotary(torch.zeros(4, 64), torch.zeros(3, 4, dtype=torch.int32), make(axes), 4, 16, 1e4)
    assert seen == [bytes(axes)] * 2


@pytest.mark.parametrize("axes", [[0.0] * 8, np.zeros(8), np.zeros((8, 2), np.int64), [0] * 7 + [256], [0] * 7 + [-1], "01201201",
                                  torch.zeros(8), [0] * 7, np.zeros(7, np.int64), torch.tensor([3])])
def test_rotary_refuses_other_axis_numbers(axes):
    with pytest.raises((TypeError, ValueError)):
        zl.zl_rotary(4, 4, 16, 16, A, 64, A, 64, zl.ZL_BF16, A, 3, axes, 1e4)


def test_numbers_of_more_than_32_bits(monkeypatch):
    """Sizes whose lower 32 bits alone would pass are refused."""
    n = (1 << 32) + 64
    wide = _pk(n)
    _refused(UNS, zl.zl_pack, 1, n, A, n, zl.ZL_BF16, wide)
    _refused(UNS, zl.zl_unpack, 1, n, wide, A, n, zl.ZL_BF16)
    _refused(UNS, zl.zl_wgrad_packed, 1, n, 64, A, n, zl.ZL_BF16, _pk(), A, 64)
    _refused(UNS, zl.zl_wgrad_packed, 1, 64, n, A, 64, zl.ZL_BF16, wide, A, n)
    _refused(INV, zl.zl_pack, 1, -n, A, n, zl.ZL_BF16, wide)
    _refused(INV, zl.zl_pack, 1, 64 - (1 << 32), A, n, zl.ZL_BF16, wide)
    ok = dict(T=4, n_heads=4, head_dim=16, rot=16, x=A, ldx=1 << 40, out=A, ldo=1 << 40, dtype=zl.ZL_BF16, pos=A, n_axes=3,
              axis_of=bytes(8), theta=1e4)
    for key in ("n_heads", "head_dim", "rot", "n_axes"):
        with pytest.raises((zl.ZlError, ValueError)) as e:
            zl.zl_rotary(**{**ok, key: (1 << 32) + ok[key]})
        assert getattr(e.value, "status", INV) in (INV, UNS)
    assert zl.zl_block_norm_workspace(4, n) > zl.zl_block_norm_workspace(4, 1 << 20)
    monkeypatch.setattr(layer, "_check_device", lambda *a: None)
    monkeypatch.setattr(layer, "_raw_stream", lambda i: 0)
    monkeypatch.setattr(layer, "_one_gpu", True)
    x = torch.empty(1, n, dtype=torch.bfloat16, device="meta")
    _refused(UNS, layer.pack, x)
    _refused(UNS, layer.unpack, layer.Packed.empty(1, n, "meta"))


def test_wgrad_of_more_than_65535_tile_rows():
    """No limit on rows besides columns and threads: with no GPU the launch fails for
    the lack of one.  In a process of its own that sees none."""
    code = f"""
from paper_2608_07974_amd import zl
for M in (65536 * 128 + 8, 1 << 30):
    try:
        zl.zl_wgrad_packed(3, M, 8, {A}, M, zl.ZL_F32, zl.zl_packed({A}, {A}, 16, 1), {A}, 8)
    except zl.ZlError as e:
        print(e)
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, env=dict(os.environ, HIP_VISIBLE_DEVICES="-1"),
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.count("no ROCm-capable device") == 2, (r.returncode, r.stdout, r.stderr)


def _calls():
    """Every torch function with tensors for each argument: name -> (function, fixed
    arguments, tensor arguments, the ones it writes)."""
    z = lambda *sh: torch.zeros(*sh)  # noqa: E731
    w, v = (torch.ones(64), torch.zeros(64)), (torch.ones(64), torch.zeros(64))
    P = lambda n: layer.Packed.empty(4, n, "cpu")  # noqa: E731
    norm = dict(gate_rows=4, layernorm=True)
    return dict(
        pack=(layer.pack, {}, dict(x=z(4, 64), out=P(64)), ["out"]),
        unpack=(layer.unpack, dict(p=P(64)), dict(out=z(4, 64)), ["out"]),
        mlp_act=(layer.mlp_act, {}, dict(h=z(4, 64), act=z(4, 32), packed=P(64)), ["act", "packed"]),
        mlp_act_bwd=(layer.mlp_act_bwd, {}, dict(h=z(4, 64), dact=z(4, 32), dh=z(4, 64), act=z(4, 32)), ["dh", "act"]),
        block_norm=(layer.block_norm, dict(post=w, pre=v, **norm),
                    dict(x=z(4, 64), y=z(4, 64), gate=z(1, 64), xo=z(4, 64), n=z(4, 64), stats=z(4, 4), y_packed=P(64), n_packed=P(64)),
                    ["xo", "n", "stats", "y_packed", "n_packed"]),
        block_norm_bwd=(layer.block_norm_bwd, dict(post=w, pre=v, grads=layer.NormGrads(*(z(64) for _ in range(4)), z(1, 64)), **norm),
                        dict(dxo=z(4, 64), dn=z(4, 64), y=z(4, 64), xo=z(4, 64), stats=z(4, 4), gate=z(1, 64), dx=z(4, 64),
                             dy=z(4, 64), workspace=z(1 << 16)), ["dx", "dy", "workspace"]),
        wgrad=(layer.wgrad, dict(x=P(64)), dict(dy=z(4, 64), out=z(64, 64), workspace=z(1 << 16)), ["out", "workspace"]),
        rotary=(layer.rotary, dict(pos=torch.zeros(1, 4, dtype=torch.int32), axis_of=bytes(8), n_heads=4, head_dim=16, theta=1e4),
                dict(x=z(4, 64), out=z(4, 64)), ["out"]))


@pytest.mark.parametrize("name", list(_calls()))
def test_autograd_is_not_passed_by(on_host, name):
    """No graph is made here: in gradient mode a matrix that requires a gradient is
    refused; weights, biases and gates may be parameters, not results.  Tensors that
    a call writes count as changed."""
    fn, fixed, tensors, written = _calls()[name]
    fn(**fixed, **tensors)
    assert len(on_host) == 1
    for key, t in tensors.items():
        if isinstance(t, layer.Packed) or key in ("stats", "workspace"):
            continue
        leaf = t.clone().requires_grad_()
        for bad in [leaf * 1.0] + ([] if key == "gate" else [leaf]):
            with pytest.raises(ValueError, match=f"{key}.* gradient"):
                fn(**fixed, **{**tensors, key: bad})
            with torch.no_grad():
                fn(**fixed, **{**tensors, key: bad})
    for key in ("post", "pre"):
        if key in fixed:
            par = tuple(t.clone().requires_grad_() for t in fixed[key])
            fn(**{**fixed, key: par}, **{**tensors, "gate": tensors["gate"].clone().requires_grad_()})
            with pytest.raises(ValueError, match="gradient"):
                fn(**{**fixed, key: (par[0] * 1.0, par[1])}, **tensors)
            with pytest.raises(ValueError, match="gradient"):
                fn(**{**fixed, key: (par[0], par[1] * 1.0)}, **tensors)
    # a graph that saved what is written next finds out
    for key in written:
        for t in (tensors[key].codes, tensors[key].scales) if isinstance(tensors[key], layer.Packed) else (tensors[key],):
            leaf = torch.ones(t.shape, requires_grad=True)
            out = (leaf * t).sum()
            fn(**fixed, **tensors)
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                out.backward()
    for t in fixed.get("grads", ()):
        leaf = torch.ones(t.shape, requires_grad=True)
        out = (leaf * t).sum()
        fn(**fixed, **tensors)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            out.backward()
    with torch.inference_mode():
        fn(**fixed, **tensors)


@pytest.mark.parametrize("ld", [0, -8, 3, 1 << 62])
def test_empty_batches_have_no_memory(ld):
    """T = 0: no pointers, any strides, nothing launched (the weight gradient, which
    writes zeros, aside)."""
    none = zl.zl_packed(0, 0, ld, ld)
    for dt in (zl.ZL_F32, zl.ZL_BF16):
        zl.zl_pack(0, 64, 0, ld, dt, none)
        zl.zl_unpack(0, 64, none, 0, ld, dt)
        zl.zl_rotary(0, 4, 16, 16, 0, ld, 0, ld + 8, dt, 0, 3, bytes(8), 1e4)
        zl.zl_rotary(0, 4, 16, 8, A + 1, ld, A + 1, ld + 8, dt, A + 1, 1, bytes(4), 1e4, 1)
        io = dict(T=0, in_dtype=dt, out_dtype=dt)
        zl.zl_mlp_act(zl.zl_mlp_args(ff=64, ldh=ld, lda=ld, packed=none, **io))
        zl.zl_mlp_act_backward(zl.zl_mlp_args(ff=64, ldh=ld, ldda=ld, lddh=ld, packed=none, **io))
        zl.zl_block_norm(zl.zl_norm_args(d=64, eps=1e-5, w_post=A, w_pre=A, ldx=ld, ldy=ld, ldn=ld, **io))
        zl.zl_block_norm_backward(zl.zl_norm_args(d=64, eps=1e-5, w_post=A, w_pre=A, ldx=ld, ldy=ld, ldn=ld, **io))
