"""The layer operators (include/zl_layer.h): their plain forms, and cases to
measure them by.

A case is a dict of plain values.  `op` names the operator:
  pack      a saved activation to 8 bits and back: layer.pack, layer.unpack
  mlp       the MLP activation, forward (writes the packed pre-activations) or
            backward (reads them): layer.mlp_act, layer.mlp_act_bwd
  norm      norm after a block, gate, scaled residual and norm before the next
            block, forward or backward: layer.block_norm, layer.block_norm_bwd
  wgrad     a weight gradient from a packed activation: layer.wgrad
  rotary    rotary positions with several axes: layer.rotary
The widths are those of workload/configs.py, or generic ones.

Packed values: e4m3 codes with one power of two per 32 columns of a row, the
smallest 2^e (e in [-117, 119]) that brings the block's finite values within
448.
"""
import math

import torch

own = False

EPS = 1e-5
THETA = 5e5


def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


# ------------------------------------------------------------------- cases
def listed():
    named = [
        # The readout norm's input of the tiny fp32 chunk, a width that ends inside a block.
        ("pack_tiny_f32", dict(op="pack", T=125, n=200, dtype="f32")),
        # A layer's normalised input over a whole micro-batch of the 8B chunk.
        ("pack_8b", dict(op="pack", T=16384, n=4096, dtype="bf16")),
        # SwiGLU of the 8B chunk: gate and up in, the activation and the saved copy out.
        ("mlp_fwd_8b", dict(op="mlp", back=False, kind="swiglu", T=16384, ff=14336, inp="bf16", dtype="bf16")),
        # Its backward from the saved copy, with the activation formed again.
        ("mlp_bwd_8b", dict(op="mlp", back=True, kind="swiglu", T=16384, ff=14336, inp="bf16", dtype="bf16")),
        # A short batch of a small GELU model, after a product with an fp32 result.
        ("mlp_bwd_gelu_odd", dict(op="mlp", back=True, kind="gelu", T=509, ff=2056, inp="f32", dtype="bf16")),
        # One new token of an 8B layer.
        ("norm_fwd_token", dict(op="norm", back=False, ln=False, B=1, S=1, d=4096, gate="shared", scale=0.5,
                                save=False, inp="bf16", dtype="bf16")),
        # LayerNorm with biases over a small model's batch of odd length, both copies saved.
        ("norm_fwd_ln_odd", dict(op="norm", back=False, ln=True, B=8, S=511, d=768, gate="none", scale=1.0,
                                 save=True, inp="f32", dtype="f32")),
        # The backward at full length with a gate per sequence, from the saved copy.
        ("norm_bwd_8b", dict(op="norm", back=True, ln=False, B=4, S=4096, d=4096, gate="sequence", scale=0.25,
                             save=True, inp="bf16", dtype="bf16")),
        # Few output tiles and a long sum: an output projection of a small model.
        ("wgrad_gpt2", dict(op="wgrad", T=4096, out=768, inner=768, dtype="bf16")),
        # The gate projection of the 8B chunk.
        ("wgrad_8b", dict(op="wgrad", T=16384, out=14336, inner=4096, dtype="bf16")),
        # Eight new tokens, positions in time, height and width.
        ("rotary_tokens", dict(op="rotary", T=8, heads=40, hd=128, rot=128, axes=3, mixed=True, far=100000,
                               inverse=False, dtype="bf16")),
        # The queries and keys of a whole micro-batch of the 8B chunk.
        ("rotary_8b", dict(op="rotary", T=16384, heads=40, hd=128, rot=128, axes=3, mixed=False, far=16384,
                           inverse=False, dtype="bf16")),
    ]
    return [dict(c, name=n) for n, c in named]


def _log(rng, lo, hi, step=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(step, v // step * step)


def draw(rng):
    op = rng.choice(["pack", "mlp", "mlp", "norm", "norm", "wgrad", "rotary"])
    inp, dtype = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
    if op == "pack":
        n = _log(rng, 8, 8192, 8)
        return dict(op=op, T=_log(rng, 1, min(16384, (1 << 25) // n)), n=n, dtype=dtype)
    if op == "mlp":
        kind = rng.choice(["swiglu", "swiglu", "gelu"])
        ff = _log(rng, 32, 14336, 32 if kind == "swiglu" else 8)
        return dict(op=op, back=rng.random() < 0.5, kind=kind, T=_log(rng, 1, min(16384, (1 << 26) // ff)), ff=ff,
                    inp=inp, dtype=dtype)
    if op == "norm":
        d = _log(rng, 64, 8192, 8)
        B = rng.choice([1, 2, 3, 8])
        return dict(op=op, back=rng.random() < 0.5, ln=rng.random() < 0.4, B=B,
                    S=_log(rng, 1, max(1, min(16384, (1 << 25) // d) // B)), d=d,
                    gate=rng.choice(["none", "shared", "sequence", "token"]), scale=rng.choice([1.0, 0.5, 0.125]),
                    save=rng.random() < 0.6, inp=inp, dtype=dtype)
    if op == "wgrad":
        most = 1 << (33 if dtype == "f32" else 38)
        out, inner = _log(rng, 64, 8192, 8), _log(rng, 64, 8192, 8)
        return dict(op=op, T=_log(rng, 1, max(1, min(16384, most // (out * inner)))), out=out, inner=inner, dtype=dtype)
    hd = rng.choice([16, 32, 64, 128])
    heads = rng.choice([1, 4, 16, 24, 40])
    return dict(op=op, T=_log(rng, 1, 16384), heads=heads, hd=hd, rot=rng.choice([hd, hd, hd // 2]),
                axes=rng.choice([1, 2, 3, 4]), mixed=rng.random() < 0.5, far=rng.choice([4096, 100000, 1000000]),
                inverse=rng.random() < 0.4, dtype=dtype)


# ------------------------------------------------------------------ inputs
def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed(1000003 * int(seed) + salt)


def _randn(shape, g, dtype=torch.float32, scale=1.0):
    return torch.empty(shape, device="cuda").normal_(0.0, scale, generator=g).to(dtype)


def _act(T, n, g, dtype):
    """Activations: columns of unlike size, a few of them far larger."""
    col = torch.empty(n, device="cuda").normal_(0.0, 0.5, generator=g).exp_()
    col[:: max(1, n // 5)] *= 20.0
    x = torch.empty(T, n, device="cuda").normal_(0.0, 1.0, generator=g)
    return x.mul_(col).to(dtype)


def _empty_packed(T, n):
    return (torch.empty(T, (n + 15) // 16 * 16, dtype=torch.uint8, device="cuda"),
            torch.empty(T, (n + 31) // 32, dtype=torch.uint8, device="cuda"))


def _packed(x):
    """Buffers of 8-bit codes and scales that hold x."""
    T, n = x.shape
    codes, scales = _empty_packed(T, n)
    codes.zero_()
    c, s = _plain_pack(x)
    codes[:, :n] = c.view(torch.uint8)
    scales.copy_(s.view(torch.uint8))
    return codes, scales


def _axes(c):
    """The axis of each of the rot / 2 frequencies: in turn, or in
    sections of even length."""
    half, A = c["rot"] // 2, c["axes"]
    return bytes(i % A if c["mixed"] else i * A // half for i in range(half))


def prepare(case, seed):
    c = case
    g = _gen(seed, 5)
    st = dict(c=c)
    if c["op"] == "pack":
        T, n = c["T"], c["n"]
        st.update(x=_act(T, n, g, _dt(c["dtype"])), buf=_empty_packed(T, n),
                  out=torch.empty(T, n, dtype=_dt(c["dtype"]), device="cuda"))
    elif c["op"] == "mlp":
        T, ff = c["T"], c["ff"]
        nh = (2 if c["kind"] == "swiglu" else 1) * ff
        h = _randn((T, nh), g, scale=1.5).to(_dt(c["inp"]))
        act = torch.empty(T, ff, dtype=_dt(c["dtype"]), device="cuda")
        if c["back"]:
            st.update(h=_packed(h), dact=_randn((T, ff), g, _dt(c["inp"])), act=act,
                      dh=torch.empty(T, nh, dtype=_dt(c["dtype"]), device="cuda"))
        else:
            st.update(h=h, act=act, buf=_empty_packed(T, nh))
    elif c["op"] == "norm":
        T, d = c["B"] * c["S"], c["d"]
        x = _act(T, d, g, torch.float32)
        y = _randn((T, d), g, _dt(c["inp"]), 2.0)
        vec = lambda at: at + _randn((d,), g, scale=0.1)  # noqa: E731
        post, pre = (vec(1.0), vec(0.0) if c["ln"] else None), (vec(1.0), vec(0.0) if c["ln"] else None)
        rows = {"none": 0, "shared": max(T, 1), "sequence": c["S"], "token": 1}[c["gate"]]
        G = 0 if not rows else T // rows
        gate = _randn((G, d), g, scale=0.5) if G else None
        st.update(x=x, y=y, post=post, pre=pre, gate=gate, rows=rows)
        if c["back"]:
            xo, n, stats = _plain_norm(c, x, y, post, pre, gate, rows)[:3]
            st.update(xo=xo, stats=stats, dxo=_randn((T, d), g), dn=_randn((T, d), g, _dt(c["inp"])),
                      dx=torch.empty(T, d, device="cuda"), dy=torch.empty(T, d, dtype=_dt(c["dtype"]), device="cuda"),
                      grads=[torch.empty(d, device="cuda") if k in ("w", "v") or c["ln"] else None
                             for k in ("w", "b", "v", "c")] +
                            [torch.empty(G, d, device="cuda") if G else None])
            st["saved"] = _packed(y) if c["save"] else y
            del st["x"], st["y"]
        else:
            st.update(xo=torch.empty(T, d, device="cuda"), n=torch.empty(T, d, dtype=_dt(c["dtype"]), device="cuda"),
                      stats=torch.empty(T, 4, device="cuda"))
            st["bufs"] = (_empty_packed(T, d), _empty_packed(T, d)) if c["save"] else None
    elif c["op"] == "wgrad":
        T = c["T"]
        dt = _dt(c["dtype"])
        st.update(dy=_randn((T, c["out"]), g, dt, 0.1), x=_packed(_act(T, c["inner"], g, dt)),
                  dw=torch.empty(c["out"], c["inner"], device="cuda"),
                  ws=torch.empty(1 << 24, device="cuda"))
    else:
        T, W = c["T"], c["heads"] * c["hd"]
        # queries and keys lie in rows that also hold the values
        st.update(x=_randn((T, W + 2 * c["hd"]), g, _dt(c["dtype"])), axes=_axes(c),
                  pos=torch.randint(0, c["far"], (c["axes"], T), dtype=torch.int32, device="cuda", generator=g),
                  out=torch.empty(T, W, dtype=_dt(c["dtype"]), device="cuda"))
    return st


# ------------------------------------------------------------- plain forms
def _blocks(x):
    T, n = x.shape
    return torch.nn.functional.pad(x, (0, -n % 32)).view(T, -1, 32)


def _plain_pack(x):
    """(codes as e4m3, scales as powers of two) of x."""
    T, n = x.shape
    b = _blocks(x.float())
    fine = torch.isfinite(b)
    amax = torch.where(fine, b.abs(), 0.0).amax(-1)
    m, e = torch.frexp(amax)  # amax = m 2^e, m in [0.5, 1)
    e = torch.where(amax > 0, e.int() - 9 + (m > 0.875), -117).clamp(-117, 119)
    v = torch.ldexp(b, -e[..., None]).clamp(-448.0, 448.0)
    v = torch.where(fine, v, float("nan")).view(T, -1)[:, :n]
    return v.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _values(codes, scales, n):
    """The fp32 values of 8-bit buffers."""
    v = _blocks(codes[:, :n].contiguous().view(torch.float8_e4m3fn).float())
    return torch.ldexp(v, scales.int()[..., None] - 127).view(codes.shape[0], -1)[:, :n]


def _plain_mlp(c, h, dact=None):
    """The activation of h (fp32), and the gradient with respect to h."""
    if c["kind"] == "swiglu":
        g, u = h.chunk(2, -1)
        s = torch.sigmoid(g)
        a = g * s * u
        return a, None if dact is None else torch.cat([dact * u * s * (1 + g * (1 - s)), dact * g * s], -1)
    k = 2.0 * math.sqrt(2.0 / math.pi)
    s = torch.sigmoid(k * (h + 0.044715 * h * h * h))
    return h * s, None if dact is None else dact * (s + h * s * (1 - s) * k * (1 + 3 * 0.044715 * h * h))


def _norm(c, v):
    mu = v.mean(-1, keepdim=True) if c["ln"] else torch.zeros_like(v[:, :1])
    r = torch.rsqrt((v - mu).square().mean(-1, keepdim=True) + EPS)
    return (v - mu) * r, mu, r


def _affine(v, wb):
    return v * wb[0] if wb[1] is None else v * wb[0] + wb[1]


def _rows(gate, rows, T):
    return gate.repeat_interleave(rows, 0)[:T]


def _plain_norm(c, x, y, post, pre, gate, rows):
    T = x.shape[0]
    yh, m0, r0 = _norm(c, y.float())
    p = c["scale"] * _affine(yh, post)
    xo = x + (p if gate is None else p * _rows(gate, rows, T))
    xh, m1, r1 = _norm(c, xo)
    n = _affine(xh, pre).to(_dt(c["dtype"]))
    return xo, n, torch.cat([m0, r0, m1, r1], -1)


def _norm_bwd(c, dy, vh, r):
    m = (dy * vh).mean(-1, keepdim=True)
    return r * (dy - vh * m - (dy.mean(-1, keepdim=True) if c["ln"] else 0.0))


def _plain_norm_bwd(c, dxo, dn, y, xo, stats, post, pre, gate, rows):
    T, d = xo.shape
    m0, r0, m1, r1 = stats.unbind(-1)
    yh, xh = (y - m0[:, None]) * r0[:, None], (xo - m1[:, None]) * r1[:, None]
    dx = dxo + _norm_bwd(c, dn * pre[0], xh, r1[:, None])
    dp = c["scale"] * dx if gate is None else c["scale"] * dx * _rows(gate, rows, T)
    dy = _norm_bwd(c, dp * post[0], yh, r0[:, None])
    dg = None if gate is None else (c["scale"] * dx * _affine(yh, post)).view(gate.shape[0], rows, d).sum(1)
    ln = c["ln"]
    return (dx, dy.to(_dt(c["dtype"])), (dp * yh).sum(0), dp.sum(0) if ln else None, (dn * xh).sum(0),
            dn.sum(0) if ln else None, dg)


def _angles(c, st_pos, axes):
    half = c["rot"] // 2
    f = THETA ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    which = torch.tensor(list(axes), device="cuda")
    a = st_pos[which].double().t() * f  # [T, half]
    return -a if c["inverse"] else a


def _plain_rotary(c, x, pos, axes):
    T, half = x.shape[0], c["rot"] // 2
    a = _angles(c, pos, axes)
    co, si = a.cos().float()[:, None], a.sin().float()[:, None]
    v = x[:, : c["heads"] * c["hd"]].float().view(T, c["heads"], c["hd"])
    p, q, rest = v[..., :half], v[..., half: 2 * half], v[..., 2 * half:]
    return torch.cat([p * co - q * si, q * co + p * si, rest], -1).view(T, -1).to(x.dtype)


# --------------------------------------------------------------------- run
def _eight(buf, n):
    """8-bit buffers as the numbers that they hold: codes and scales."""
    return [buf[0][:, :n].view(torch.float8_e4m3fn), buf[1].view(torch.float8_e8m0fnu)]


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(st):
    c = st["c"]
    dt = _dt(c["dtype"])
    if c["op"] == "pack":
        codes, scales = _plain_pack(st["x"])
        return _values(codes.view(torch.uint8), scales.view(torch.uint8), c["n"]).to(dt)
    if c["op"] == "mlp":
        if not c["back"]:
            return [_plain_mlp(c, st["h"].float())[0].to(dt)] + list(_plain_pack(st["h"]))
        h = _values(*st["h"], (2 if c["kind"] == "swiglu" else 1) * c["ff"])
        act, dh = _plain_mlp(c, h, st["dact"].float())
        return dh.to(dt), act.to(dt)
    if c["op"] == "norm":
        if not c["back"]:
            xo, n, stats = _plain_norm(c, st["x"], st["y"], st["post"], st["pre"], st["gate"], st["rows"])
            return [xo, n, stats] + (list(_plain_pack(st["y"])) + list(_plain_pack(n)) if c["save"] else [])
        y = _values(*st["saved"], c["d"]) if c["save"] else st["saved"].float()
        return _plain_norm_bwd(c, st["dxo"], st["dn"].float(), y, st["xo"], st["stats"], st["post"], st["pre"],
                               st["gate"], st["rows"])
    if c["op"] == "wgrad":
        return st["dy"].float().t() @ _values(*st["x"], c["inner"])
    return _plain_rotary(c, st["x"], st["pos"], st["axes"])


def _run_own(st):
    from paper_2608_07974_amd import layer
    c = st["c"]
    if c["op"] == "pack":
        p = layer.pack(st["x"], out=layer.Packed(*st["buf"], c["n"]))
        return layer.unpack(p, out=st["out"])
    if c["op"] == "mlp":
        n = (2 if c["kind"] == "swiglu" else 1) * c["ff"]
        if not c["back"]:
            act = layer.mlp_act(st["h"], c["kind"], act=st["act"], packed=layer.Packed(*st["buf"], n))
            return [act] + _eight(st["buf"], n)
        dh = layer.mlp_act_bwd(layer.Packed(*st["h"], n), st["dact"], c["kind"], dh=st["dh"], act=st["act"])
        return dh, st["act"]
    if c["op"] == "norm":
        kw = dict(layernorm=c["ln"], eps=EPS, scale=c["scale"], gate=st["gate"], gate_rows=st["rows"])
        if not c["back"]:
            yp, np_ = [layer.Packed(*b, c["d"]) for b in st["bufs"]] if c["save"] else (None, None)
            layer.block_norm(st["x"], st["y"], st["post"], st["pre"], xo=st["xo"], n=st["n"], stats=st["stats"],
                             y_packed=yp, n_packed=np_, **kw)
            return [st["xo"], st["n"], st["stats"]] + \
                (_eight(st["bufs"][0], c["d"]) + _eight(st["bufs"][1], c["d"]) if c["save"] else [])
        y = layer.Packed(*st["saved"], c["d"]) if c["save"] else st["saved"]
        layer.block_norm_bwd(st["dxo"], st["dn"], y, st["xo"], st["stats"], st["post"], st["pre"], dx=st["dx"],
                             dy=st["dy"], grads=layer.NormGrads(*st["grads"]), **kw)
        return (st["dx"], st["dy"], *st["grads"])
    if c["op"] == "wgrad":
        return layer.wgrad(st["dy"], layer.Packed(*st["x"], c["inner"]), out=st["dw"], workspace=st["ws"])
    return layer.rotary(st["x"], st["pos"], st["axes"], c["heads"], c["hd"], THETA, inverse=c["inverse"],
                        out=st["out"])


# -------------------------------------------------------------------- work
def work(case):
    c = case
    sz = {"f32": 4, "bf16": 2}
    pk = lambda T, n: T * (n + (n + 31) // 32)  # noqa: E731
    if c["op"] == "pack":
        T, n = c["T"], c["n"]
        return {"bytes": 2 * (T * n * sz[c["dtype"]] + pk(T, n)), "flops": 4 * T * n}
    if c["op"] == "mlp":
        T, ff, two = c["T"], c["ff"], 2 if c["kind"] == "swiglu" else 1
        i, o = sz[c["inp"]], sz[c["dtype"]]
        b = pk(T, two * ff) + (T * ff * (i + two * o + o) if c["back"] else T * ff * (two * i + o))
        return {"bytes": b, "flops": (25 if c["back"] else 12) * T * ff}
    if c["op"] == "norm":
        T, d = c["B"] * c["S"], c["d"]
        i, o = sz[c["inp"]], sz[c["dtype"]]
        G = {"none": 0, "shared": 1, "sequence": c["B"], "token": T}[c["gate"]]
        vecs = (4 if c["ln"] else 2) * d * 4
        if c["back"]:
            b = T * d * (4 + i + 4 + 4 + o) + (pk(T, d) if c["save"] else T * d * i) + 16 * T + 2 * vecs + 2 * G * d * 4
            return {"bytes": b, "flops": 30 * T * d}
        b = T * d * (4 + i + 4 + o) + (2 * pk(T, d) if c["save"] else 0) + 16 * T + vecs + G * d * 4
        return {"bytes": b, "flops": 14 * T * d}
    if c["op"] == "wgrad":
        T, M, N = c["T"], c["out"], c["inner"]
        return {"bytes": T * M * sz[c["dtype"]] + pk(T, N) + 4 * M * N, "flops": 2 * T * M * N}
    T, W = c["T"], c["heads"] * c["hd"]
    return {"bytes": 2 * T * W * sz[c["dtype"]] + 4 * c["axes"] * T,
            "flops": 3 * T * c["heads"] * c["rot"]}


# ------------------------------------------------------------------- exact
def _grid(v):
    """Values rounded to e4m3 (nearest, ties to even), |v| at most 448."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -20))).clamp_min(-6.0) - 3.0)
    return torch.round(v / step) * step


def _exact_pack(x):
    """(codes, scales) of x in 64 bits: the smallest power of two that brings
    the block within 448, by trial around its logarithm."""
    T, n = x.shape
    b = torch.zeros(T, (n + 31) // 32 * 32, dtype=torch.float64, device=x.device)
    b[:, :n] = x
    b = b.view(T, -1, 32)
    top = b.abs().max(-1).values
    e = torch.floor(torch.log2(top.clamp_min(1e-300) / 448.0)) - 1.0
    for _ in range(3):
        e = torch.where(top > 448.0 * torch.exp2(e), e + 1.0, e)
    s = torch.exp2(e.clamp(-117.0, 119.0))
    v = (b / s[..., None]).clamp(-448.0, 448.0)
    return _grid(v).view(T, -1)[:, :n], s


def _exact_values(codes, scales, n):
    """Codes decoded bit by bit: sign, 4 exponent bits, 3 fraction bits."""
    u = codes[:, :n].long()
    ex, fr = u // 8 % 16, u % 8
    mag = torch.where(ex > 0, (8.0 + fr.double()) * torch.exp2(ex.double() - 10.0), fr.double() * 2.0 ** -9)
    s = torch.exp2(scales.double() - 127.0)
    return torch.where(u >= 128, -mag, mag) * s.repeat_interleave(32, 1)[:, :n]


def exact(case, seed):
    c = case
    st = prepare(case, seed)
    if c["op"] == "pack":
        codes, s = _exact_pack(st["x"].double())
        return codes * s.repeat_interleave(32, 1)[:, : c["n"]]
    if c["op"] == "mlp":
        ff, two = c["ff"], c["kind"] == "swiglu"
        h = _exact_values(*st["h"], 2 * ff if two else ff) if c["back"] else st["h"].double()
        g = h[:, :ff]
        t = 1.0 if two else 2.0 * math.sqrt(2.0 / math.pi)
        z = g if two else t * (g + 0.044715 * g ** 3)
        s = 1.0 / (1.0 + torch.exp(-z))
        slope = s + g * s * (1.0 - s) * (1.0 if two else t * (1.0 + 0.134145 * g ** 2))  # of g s(z(g))
        u = h[:, ff:] if two else None
        act = g * s * u if two else g * s
        if not c["back"]:
            return [act] + list(_exact_pack(h))
        da = st["dact"].double()
        return (torch.cat([da * u * slope, da * g * s], 1) if two else da * slope), act
    if c["op"] == "norm":
        ln, k, T, d = c["ln"], c["scale"], c["B"] * c["S"], c["d"]
        w, b = st["post"][0].double(), st["post"][1].double() if ln else 0.0
        v, e = st["pre"][0].double(), st["pre"][1].double() if ln else 0.0
        gate = st["gate"].double()[torch.arange(T, device="cuda") // st["rows"]] if st["gate"] is not None else 1.0
        if not c["back"]:
            y = st["y"].double()
            m0 = y.sum(1, keepdim=True) / d if ln else torch.zeros(T, 1, dtype=torch.float64, device="cuda")
            r0 = (((y - m0) ** 2).sum(1, keepdim=True) / d + EPS) ** -0.5
            xo = st["x"].double() + k * gate * ((y - m0) * r0 * w + b)
            m1 = xo.sum(1, keepdim=True) / d if ln else torch.zeros_like(m0)
            r1 = (((xo - m1) ** 2).sum(1, keepdim=True) / d + EPS) ** -0.5
            n = (xo - m1) * r1 * v + e
            out = [xo, n, torch.cat([m0, r0, m1, r1], 1)]
            # the copy of n: values at the border of two codes go either way by the last
            # bit of n, so 64 bits name no one result
            return out + (list(_exact_pack(y)) + [None, None] if c["save"] else [])
        y = _exact_values(*st["saved"], d) if c["save"] else st["saved"].double()
        m0, r0, m1, r1 = (t[:, None] for t in st["stats"].double().unbind(1))
        yh, xh = (y - m0) * r0, (st["xo"].double() - m1) * r1
        dn = st["dn"].double()

        def back(a, h, r):
            cut = h * ((a * h).sum(1, keepdim=True) / d)
            return r * (a - cut - a.sum(1, keepdim=True) / d) if ln else r * (a - cut)

        D = st["dxo"].double() + back(dn * v, xh, r1)
        dp = k * gate * D
        dg = None
        if st["gate"] is not None:
            dg = torch.zeros(st["gate"].shape, dtype=torch.float64, device="cuda")
            dg.index_add_(0, torch.arange(T, device="cuda") // st["rows"], k * D * (yh * w + b))
        return (D, back(dp * w, yh, r0), (dp * yh).sum(0), dp.sum(0) if ln else None, (dn * xh).sum(0),
                dn.sum(0) if ln else None, dg)
    if c["op"] == "wgrad":
        return torch.matmul(st["dy"].double().t().contiguous(), _exact_values(*st["x"], c["inner"]))
    T, half = c["T"], c["rot"] // 2
    v = st["x"][:, : c["heads"] * c["hd"]].double().reshape(T, c["heads"], c["hd"])
    out = v.clone()
    sign = -1.0 if c["inverse"] else 1.0
    for j in range(half):
        t = sign * st["pos"][st["axes"][j]].double()[:, None] * THETA ** (-2.0 * j / c["rot"])
        out[..., j] = v[..., j] * t.cos() - v[..., j + half] * t.sin()
        out[..., j + half] = v[..., j + half] * t.cos() + v[..., j] * t.sin()
    return out.reshape(T, -1)
