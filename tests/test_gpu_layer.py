"""The layer operators (include/sc_layer.h) against plain float64 forms.

Tolerances count roundings (u = 2^-24 of float32, half a step of the storage type at the end):
  rotary    a cosine or sine is off by 2^-27 of a turn (4.7e-8), the series' 4e-9 and its roundings (3 u): 2.4e-7 = 4 u;
            a rotated pair by amplitude * (|a| + |b|) * (4 u + 2 u), and by what its inputs are off.  A normalised
            value: sums of d values in chains of at most 20 additions, the deviation from the mean, the factor and the
            product: 50 u (1 + |hat| + max|x| / sigma).  Weight gradients: sums over rows in chains of at most 256.
  ffn       on small integers every product and sum is exact and the results are equal to those of a form that rounds
            where the header says.  On random values a result has two roundings to bf16 behind it (h, dg or du, and its
            own), each of 2^-8 of the value at most and, spread evenly over a step, 2^-8 / sqrt(3) of it in the mean
            square: sqrt(2 / 3) 2^-8 = 0.0032 of the result's 2-norm, 0.0035 with what float32 sums, activations
            (3e-5 at most) and the 24 bits of what is saved (2^-16) add.  A value by itself: 2^-8 of the sum of the
            products' magnitudes, twice, more than float32 sums of up to 4096 products add.
  dropout   masks are equal; x * scale, the FMA with the residual and the store round once each.
"""
import math

import numpy as np
import pytest
import torch

import paper_2310_07109_amd as sc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": (torch.float32, sc.SC_F32, 2.0 ** -24), "bf16": (torch.bfloat16, sc.SC_BF16, 2.0 ** -8)}


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def lens_of(spec, B, n):
    if spec is None:
        return None, torch.full((B,), n)
    L = torch.tensor([spec[b % len(spec)] for b in range(B)], dtype=torch.int32)
    return L.to(DEV), L.clamp(0, n).long()


def valid_mask(L, n):
    return torch.arange(n)[None, :] < L[:, None]


def assert_close(got, want, tol, what):
    got = got.double().cpu()
    assert got.shape == want.shape, what
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst " \
        f"{float(((got - want).abs() / tol.clamp(min=1e-300))[bad].max()):.3g} times the tolerance"


# ---------------------------------------------------------------- rotary ----
def rotate64(x, angle, amplitude, R, layout):
    """x [B, n, H, d] rotated by angle [B, n, R / 2], in float64; and |a| + |b| of every rotated dimension."""
    c, s = angle.cos()[:, :, None], angle.sin()[:, :, None]
    i = torch.arange(R // 2)
    ia, ib = (i, i + R // 2) if layout == sc.SC_ROTARY_HALF else (2 * i, 2 * i + 1)
    out, mag = x.clone(), torch.zeros_like(x)
    a, b = x[..., ia], x[..., ib]
    out[..., ia], out[..., ib] = amplitude * (a * c - b * s), amplitude * (a * s + b * c)
    mag[..., ia] = mag[..., ib] = abs(amplitude) * (a.abs() + b.abs())
    return out, mag


def head_norm64(x, kind, eps):
    """(hat, 1 / sigma, error of hat)"""
    v = x - x.mean(-1, keepdim=True) if kind == sc.SC_NORM_LAYER else x
    inv = (v.pow(2).mean(-1, keepdim=True) + eps).rsqrt()
    hat = v * inv
    return hat, inv, 50 * U * (1 + hat.abs() + x.abs().amax(-1, keepdim=True) * inv)


def rotary_forward64(x, w, angle, amplitude, R, layout, norm, kind, eps):
    err = torch.zeros_like(x)
    if norm:
        hat, _, e = head_norm64(x, kind, eps)
        w = torch.ones(x.shape[-1], dtype=torch.float64) if w is None else w.double()
        x, err = hat * w, (e + 2 * U * hat.abs()) * w.abs()
    out, mag = rotate64(x, angle, amplitude, R, layout)
    _, emag = rotate64(err, angle, amplitude, R, layout)
    return out, torch.where(mag > 0, emag + 6 * U * mag, err)


def rotary_case(B, n, Hq, Hk, d, R, dtype, norm, layout, kind=sc.SC_NORM_RMS, lens=None, fused=True, weights=True,
                pos=None, amplitude=1.0, seed=0, backward=False):
    g = gen(seed)
    dt, code, half = TYPES[dtype]
    W = (Hq + 2 * Hk) * d
    pad = 16 if fused else 0
    rows = (torch.randn((B, n, W + pad), generator=g) * torch.exp(0.5 * torch.randn(W + pad, generator=g))).to(dt)
    L_dev, L = lens_of(lens, B, n)
    m = valid_mask(L, n)
    rows[~m] = float("nan")
    freq, _ = sc.sc_rotary_frequencies(R) if R else (None, 1.0)
    if pos is None:
        p = torch.arange(n).expand(B, n)
    else:
        p = torch.randint(-pos, pos, (B, n), generator=g)
    angle = p.double()[..., None] * (freq if R else torch.zeros(0, dtype=torch.float64))
    cut = (0, Hq * d, (Hq + Hk) * d, W)
    dev = rows.to(DEV)
    parts = [dev[..., cut[i]:cut[i + 1]].unflatten(-1, (-1, d)) for i in range(3)]
    host = [rows[..., cut[i]:cut[i + 1]].unflatten(-1, (-1, d)).double() for i in range(3)]
    host = [torch.where(m[..., None, None], t, 0.0) for t in host]
    if not fused:
        parts = [t.contiguous() for t in parts]
    qw, kw = ((1 + 0.2 * torch.randn(d, generator=g)) if norm and weights else None for _ in range(2))
    D = sc.RotaryDesc(B, n, Hq, Hk, d=d, rot_dim=R, valid_len=L_dev, layout=layout, norm=norm, kind=kind, eps=1e-5,
                      amplitude=amplitude, dtype=code)
    args = dict(q_w=None if qw is None else qw.to(DEV), k_w=None if kw is None else kw.to(DEV),
                positions=None if pos is None else p.to(torch.int32).to(DEV))
    if not backward:
        outs = sc.sc_rotary(D, freq, *parts, **args)
        for i, (nm, w) in enumerate((("q", qw), ("k", kw))):
            want, tol = rotary_forward64(host[i], w, angle, amplitude, R, layout, norm, kind, 1e-5)
            mm = m[..., None, None]
            assert_close(outs[i], torch.where(mm, want, 0.0), torch.where(mm, tol + half * want.abs(), 0.0), nm)
        assert torch.equal(outs[2].double().cpu(), host[2])
        return
    go = [torch.randn((B, n, h, d), generator=g).to(dt) for h in (Hq, Hk, Hk)]
    for t in go:
        t[~m] = float("nan")
    grads = torch.full_like(dev, 7.0)
    gp = [grads[..., cut[i]:cut[i + 1]].unflatten(-1, (-1, d)) for i in range(3)]
    if not fused:
        gp = [torch.empty_like(t) for t in parts]
    dw = dict(dq_w=torch.empty(d, device=DEV), dk_w=torch.empty(d, device=DEV)) if norm else {}
    out = sc.sc_rotary_backward(D, freq, *[t.to(DEV) for t in go], q=parts[0], k=parts[1],
                                grads=dict(dq=gp[0], dk=gp[1], dv=gp[2], **dw), **args)
    if fused:
        assert bool((grads[..., W:] == 7).all())  # only its own parts are written
    mm = m[..., None, None]
    for i, (nm, w) in enumerate((("dq", qw), ("dk", kw))):
        gr = torch.where(mm, go[i].double(), 0.0)
        du, mag = rotate64(gr, -angle, amplitude, R, layout)
        e = 6 * U * mag
        if norm:
            hat, inv, eh = head_norm64(host[i], kind, 1e-5)
            ww = torch.ones(d, dtype=torch.float64) if w is None else w.double()
            dwant, dmag = (du * hat).sum((0, 1, 2)), (du.abs() * hat.abs()).sum((0, 1, 2))
            dtol = (e * hat.abs() + du.abs() * torch.where(mm, eh, 0.0)).sum((0, 1, 2)) + 256 * U * dmag
            assert_close(out["dq_w" if i == 0 else "dk_w"], dwant, dtol, nm + "_w")
            gw, e = du * ww, (e + U * du.abs()) * ww.abs()
            gh = (gw * hat).mean(-1, keepdim=True)
            gs = gw.mean(-1, keepdim=True) if kind == sc.SC_NORM_LAYER else torch.zeros_like(gh)
            want = inv * (gw - hat * gh - gs)
            ah, ag = (gw * hat).abs().mean(-1, keepdim=True), gw.abs().mean(-1, keepdim=True)
            egh = (e * hat.abs() + gw.abs() * eh).mean(-1, keepdim=True) + 25 * U * ah
            tol = inv * (e + eh * gh.abs() + hat.abs() * egh + e.mean(-1, keepdim=True) + 25 * U * ag +
                         4 * U * (gw.abs() + hat.abs() * ah + ag)) + 30 * U * want.abs()
        else:
            want, tol = du, torch.where(mag > 0, e, 0.0)
        assert_close(out[nm], torch.where(mm, want, 0.0), torch.where(mm, tol + half * want.abs(), 0.0), nm)
    assert torch.equal(out["dv"].double().cpu(), torch.where(mm, go[2].double(), 0.0))


HALF, INTER = sc.SC_ROTARY_HALF, sc.SC_ROTARY_INTERLEAVED
ROTARY = [  # B, n, Hq, Hk, d, R, dtype, norm, layout, kind
    (1, 1, 8, 8, 64, 64, "bf16", True, HALF, sc.SC_NORM_RMS), (1, 1, 1, 1, 2, 2, "f32", True, INTER, sc.SC_NORM_RMS),
    (2, 33, 12, 4, 64, 64, "bf16", False, HALF, 0), (3, 17, 5, 5, 80, 40, "f32", True, INTER, sc.SC_NORM_LAYER),
    (2, 40, 3, 1, 128, 64, "bf16", True, HALF, sc.SC_NORM_LAYER), (1, 9, 2, 2, 256, 256, "bf16", True, HALF, 1),
    (2, 31, 4, 2, 96, 32, "f32", True, HALF, 1), (2, 31, 4, 2, 66, 6, "bf16", True, HALF, 0),
    (2, 31, 3, 3, 72, 72, "bf16", True, INTER, 1), (1, 50, 3, 3, 64, 0, "bf16", True, HALF, 1),
    (1, 50, 3, 3, 18, 10, "f32", False, INTER, 0), (7, 700, 2, 1, 64, 48, "f32", True, HALF, 0),
]


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("B,n,Hq,Hk,d,R,dtype,norm,layout,kind", ROTARY)
def test_rotary(B, n, Hq, Hk, d, R, dtype, norm, layout, kind, backward):
    for i, (lens, fused, weights, pos, amp) in enumerate((
            (None, True, True, None, 1.0), ((n, 0, (n + 1) // 2), False, True, 2 ** 31 - 1, 0.75),
            ((1, n), True, False, 5000, 1.0))):
        rotary_case(B, n, Hq, Hk, d, R, dtype, norm, layout, kind, lens=lens, fused=fused, weights=weights, pos=pos,
                    amplitude=amp, seed=i, backward=backward)


def test_rotary_large_grid_and_offsets():
    """More tokens than workgroups, and fused rows whose byte offsets pass 32 bits."""
    rotary_case(9, 2048, 2, 1, 64, 64, "bf16", True, HALF, lens=(2048, 5, 0, 1999), backward=False)
    rotary_case(9, 2048, 2, 1, 64, 64, "bf16", True, HALF, lens=(2048, 5, 0, 1999), backward=True)
    B, n, step = 1, 1 << 15, 1 << 17  # 8 GiB between the first token and the last
    rows = torch.empty(B * n * step, dtype=torch.bfloat16, device=DEV)
    q = rows.as_strided((B, n, 2, 64), (n * step, step, 64, 1))
    q.copy_(torch.randn((B, n, 2, 64), generator=gen(1)).to(torch.bfloat16))
    freq, _ = sc.sc_rotary_frequencies(64)
    D = sc.RotaryDesc(B, n, 2, 1)
    out = sc.sc_rotary(D, freq, q)[0]
    assert torch.equal(out, sc.sc_rotary(D, freq, q.contiguous())[0])
    g = torch.randn((B, n, 2, 64), generator=gen(2)).to(torch.bfloat16).to(DEV)
    sc.sc_rotary_backward(D, freq, g, grads=dict(dq=q))
    assert torch.equal(q.contiguous(), sc.sc_rotary_backward(D, freq, g)["dq"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotary_inverse_in_place_and_parts(dtype):
    """Backward without norms turns back what forward turned; in place; q alone, k alone, v alone."""
    dt, code, half = TYPES[dtype]
    B, n, H = 2, 37, 3
    q = torch.randn((B, n, H, 64), generator=gen(3)).to(dt).to(DEV)
    freq, _ = sc.sc_rotary_frequencies(64, scaling=sc.SC_ROTARY_BANDS, factor=4.0, length=512)
    d = sc.RotaryDesc(B, n, H, H, dtype=code)
    out, k_out, v_out = sc.sc_rotary(d, freq, q)
    assert k_out is None and v_out is None
    assert torch.equal(sc.sc_rotary(d, freq, None, k=q)[1], out)
    assert torch.equal(sc.sc_rotary(d, freq, None, None, q)[2], q)
    back = sc.sc_rotary_backward(d, freq, out)["dq"]
    pair = q.double().abs() + q.double().abs().roll(32, -1)
    assert_close(back, q.double().cpu(), (3 * (12 * U + 2 * half) * pair).cpu(), "turned back")
    buf = q.clone()
    assert sc.sc_rotary(d, freq, buf, q_out=buf)[0].data_ptr() == buf.data_ptr() and torch.equal(buf, out)
    sc.sc_rotary_backward(d, freq, buf, grads=dict(dq=buf))
    assert torch.equal(buf, back)


def test_rotary_gradients_by_differences():
    """Central differences of the float32 forward along random directions, within their own error."""
    B, n, H, d = 2, 5, 2, 16
    g = gen(9)
    x = torch.randn((B, n, H, d), generator=g)
    w = 1 + 0.2 * torch.randn(d, generator=g)
    freq, _ = sc.sc_rotary_frequencies(d)
    for kind in (sc.SC_NORM_LAYER, sc.SC_NORM_RMS):
        D = sc.RotaryDesc(B, n, H, H, d=d, norm=True, kind=kind, eps=1e-5, dtype=sc.SC_F32)
        go = torch.randn((B, n, H, d), generator=g)
        out = sc.sc_rotary_backward(D, freq, go.to(DEV), q=x.to(DEV), q_w=w.to(DEV))

        def loss(x, w):
            return float((sc.sc_rotary(D, freq, x.to(DEV), q_w=w.to(DEV))[0].double().cpu() * go.double()).sum())
        h = 2.0 ** -7
        for _ in range(4):
            vx, vw = torch.randn(x.shape, generator=g), torch.randn(d, generator=g)
            num = (loss(x + h * vx, w + h * vw) - loss(x - h * vx, w - h * vw)) / (2 * h)
            ana = float((out["dq"].double().cpu() * vx).sum() + (out["dq_w"].double().cpu() * vw).sum())
            # third derivatives of a normalised head grow with the step's size against its deviation (about 1 here)
            scale = float((go.abs() * (1 + vx.abs()).pow(3)).sum())
            assert abs(num - ana) <= h * h * scale + 64 * U * scale / h, (num, ana)


# ------------------------------------------------------------------- ffn ----
def bf(t):
    return t.to(torch.bfloat16).double()


def ffn_ints(B, n, D, F, lens, seed):
    """Inputs of small integers, few of them not 0, so that every sum is an integer far below 2^24."""
    g = gen(seed)
    L_dev, L = lens_of(lens, B, n)
    m = valid_mask(L, n)

    def sparse(*shape, keep):
        return (torch.randint(-2, 3, shape, generator=g) * (torch.rand(shape, generator=g) < keep)).to(torch.bfloat16)
    x, dy = sparse(B, n, D, keep=0.5), sparse(B, n, D, keep=0.5)
    wg, wu, wd = sparse(D, F, keep=min(1.0, 8 / D)), sparse(D, F, keep=min(1.0, 8 / D)), sparse(F, D, keep=min(1.0, 8 / F))
    x[~m], dy[~m] = float("nan"), float("nan")
    return L_dev, m, x, wg, wu, wd, dy


def ffn_ints_check(B, n, D, F, lens, seed=0):
    L_dev, m, x, wg, wu, wd, dy = ffn_ints(B, n, D, F, lens, seed)
    d = sc.FfnDesc(B, n, D, F, valid_len=L_dev, act=sc.SC_ACT_NONE)
    dev = [t.to(DEV) for t in (x, wg, wu, wd)]
    y, saved = sc.sc_gated_ffn(d, *dev, saved=True)
    y2, none = sc.sc_gated_ffn(d, *dev)
    assert none is None and torch.equal(y, y2)
    out = sc.sc_gated_ffn_backward(d, *dev, saved, dy.to(DEV))
    xs, ds = x[m].double().to(DEV), dy[m].double().to(DEV)
    wg, wu, wd = (t.double().to(DEV) for t in (wg, wu, wd))
    g, u = xs @ wg, xs @ wu
    h = bf(g * u)
    dh = ds @ wd.t()
    dg, du = bf(dh * u), bf(dh * g)

    def rows(v):
        t = torch.zeros((B, n, D), dtype=torch.float64, device=DEV)
        t[m.to(DEV)] = bf(v)
        return t
    want = dict(y=rows(h @ wd), dx=rows(dg @ wg.t() + du @ wu.t()), dwg=bf(xs.t() @ dg), dwu=bf(xs.t() @ du),
                dwd=bf(h.t() @ ds))
    assert max(float(v.abs().max()) for v in (h.t() @ ds, xs.t() @ dg, xs.t() @ du)) < 2 ** 24
    for nm, v in want.items():
        got = (y if nm == "y" else out[nm]).double()
        assert torch.equal(got, v), f"{nm}: {int((got != v).sum())} of {v.numel()} differ"


@pytest.mark.parametrize("B,n,D,F,lens", [
    (1, 1, 64, 64, None), (1, 1, 8, 8, None), (1, 1, 1, 1, None), (1, 1, 768, 2048, (1,)), (1, 5, 33, 47, None),
    (2, 3, 100, 70, (3, 0)), (2, 9, 64, 136, (0, 0)), (16, 8, 768, 2304, (8, 4, 5, 1)), (1, 40, 96, 1000, None),
    (3, 501, 500, 1111, (300, 501, 0)), (1, 300, 264, 520, None), (5, 129, 72, 328, (129, 128, 1, 64, 65)),
    (1, 2000, 1024, 512, None), (4, 1100, 512, 1536, (1100, 7, 900)), (2, 2048, 1000, 1032, (2048, 1991))])
def test_ffn_exact_on_integers(B, n, D, F, lens):
    ffn_ints_check(B, n, D, F, lens)


def test_ffn_many_tiles():
    """Several tiles a workgroup in every product, padding between them."""
    ffn_ints_check(16, 1024, 1024, 2816, (1024, 1000, 513, 0))


def act64(act, g):
    """act(g) and its slope."""
    if act == sc.SC_ACT_SILU:
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    if act == sc.SC_ACT_GELU:
        p = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    return g, torch.ones_like(g)


@pytest.mark.parametrize("act", [sc.SC_ACT_NONE, sc.SC_ACT_GELU, sc.SC_ACT_SILU])
@pytest.mark.parametrize("B,n,D,F,lens", [(1, 1, 512, 768, None), (3, 11, 200, 333, (11, 0, 4)),
                                          (2, 700, 264, 512, (700, 333)), (1, 3000, 512, 1024, None)])
def test_ffn_values_and_gradients(B, n, D, F, lens, act):
    g_ = gen(D + act)
    L_dev, L = lens_of(lens, B, n)
    m = valid_mask(L, n)
    x = torch.randn((B, n, D), generator=g_).to(torch.bfloat16)
    wg, wu = ((torch.randn((D, F), generator=g_) * 2 / math.sqrt(D)).to(torch.bfloat16) for _ in range(2))
    wd = (torch.randn((F, D), generator=g_) / math.sqrt(F)).to(torch.bfloat16)
    dy = torch.randn((B, n, D), generator=g_).to(torch.bfloat16)
    d = sc.FfnDesc(B, n, D, F, valid_len=L_dev, act=act)
    dev = [t.to(DEV) for t in (x, wg, wu, wd)]
    y, saved = sc.sc_gated_ffn(d, *dev, saved=True)
    out = sc.sc_gated_ffn_backward(d, *dev, saved, dy.to(DEV))
    xs, ds = x[m].double(), dy[m].double()
    wg, wu, wd = (t.double() for t in (wg, wu, wd))
    g, u = xs @ wg, xs @ wu
    a, slope = act64(act, g)
    h, dh = a * u, ds @ wd.t()
    dg, du = dh * u * slope, dh * a
    A = torch.abs
    want = dict(y=(h @ wd, A(h) @ A(wd)), dx=(dg @ wg.t() + du @ wu.t(), A(dg) @ A(wg).t() + A(du) @ A(wu).t()),
                dwg=(xs.t() @ dg, A(xs).t() @ A(dg)), dwu=(xs.t() @ du, A(xs).t() @ A(du)),
                dwd=(h.t() @ ds, A(h).t() @ A(ds)))
    for nm, (v, mag) in want.items():
        got = (y if nm == "y" else out[nm]).double().cpu()
        if nm in ("y", "dx"):
            assert not got[~m].any(), nm
            got = got[m]
        assert float((got - v).norm()) <= 0.0035 * float(v.norm()), nm
        assert_close(got, v, 2 * 2.0 ** -8 * mag, nm)


def test_ffn_gradients_by_differences():
    """The loss along a direction, in float64 on the rounded inputs, against the gradients' product with it."""
    B, n, D, F = 2, 30, 40, 56
    g = gen(4)
    x = torch.randn((B, n, D), generator=g).to(torch.bfloat16)
    w = [(torch.randn(s, generator=g) / math.sqrt(s[0])).to(torch.bfloat16) for s in ((D, F), (D, F), (F, D))]
    dy = torch.randn((B, n, D), generator=g).to(torch.bfloat16)
    for act in (sc.SC_ACT_GELU, sc.SC_ACT_SILU):
        d = sc.FfnDesc(B, n, D, F, act=act)
        dev = [t.to(DEV) for t in (x, *w)]
        _, saved = sc.sc_gated_ffn(d, *dev, saved=True)
        out = sc.sc_gated_ffn_backward(d, *dev, saved, dy.to(DEV))

        def loss(p):
            return float(((act64(act, p[0] @ p[1])[0] * (p[0] @ p[2])) @ p[3] * dy.double()).sum())
        leaves = [t.double() for t in (x, *w)]
        for i, nm in enumerate(("dx", "dwg", "dwu", "dwd")):
            v = torch.randn(leaves[i].shape, generator=g, dtype=torch.float64)
            h = 1e-4
            num = (loss([t + h * v if j == i else t for j, t in enumerate(leaves)]) -
                   loss([t - h * v if j == i else t for j, t in enumerate(leaves)])) / (2 * h)
            ana = float((out[nm].double().cpu() * v).sum())
            # errors of 0.0035 of the gradient's norm in a direction that does not know them: 5 of their deviations
            assert abs(num - ana) <= 5 * 0.0035 * float(out[nm].double().norm()), (nm, num, ana)


def test_ffn_infinities_and_nans_stay_in_their_rows():
    B, n, D, F = 1, 140, 64, 72
    g = gen(6)
    x = torch.randn((B, n, D), generator=g).to(torch.bfloat16)
    w = [(torch.randn(s, generator=g) / math.sqrt(s[0])).to(torch.bfloat16).to(DEV) for s in ((D, F), (D, F), (F, D))]
    d = sc.FfnDesc(B, n, D, F)
    clean = sc.sc_gated_ffn(d, x.to(DEV), *w)[0]
    x[0, 7, 3], x[0, 130, 0] = float("nan"), float("inf")
    y = sc.sc_gated_ffn(d, x.to(DEV), *w)[0]
    assert y[0, 7].isnan().all() and not y[0, 130].isfinite().any()
    keep = [i for i in range(n) if i not in (7, 130)]
    assert torch.equal(y[0, keep], clean[0, keep])


@pytest.mark.parametrize("names", [("dx",), ("dwg",), ("dwu",), ("dwd",), ("dx", "dwd"), ("dwg", "dwu")])
@pytest.mark.parametrize("B,n,D,F", [(2, 20, 24, 40), (1, 1500, 264, 136)])
def test_ffn_backward_parts(B, n, D, F, names):
    """Only the gradients asked for, the same as all of them; backward twice from what was saved once."""
    L_dev, m, x, wg, wu, wd, dy = ffn_ints(B, n, D, F, (n, n - 3), 1)
    x, dy = (torch.nan_to_num(t) for t in (x, dy))
    d = sc.FfnDesc(B, n, D, F, valid_len=L_dev)
    dev = [t.to(DEV) for t in (x, wg, wu, wd)]
    _, saved = sc.sc_gated_ffn(d, *dev, saved=True)
    keep = saved.clone()
    full = sc.sc_gated_ffn_backward(d, *dev, saved, dy.to(DEV))
    part = sc.sc_gated_ffn_backward(d, *dev, saved, dy.to(DEV), grads={k: torch.full_like(full[k], 9) for k in names})
    for k, v in part.items():
        assert (v is None) == (k not in names)
        assert v is None or torch.equal(v, full[k])
    assert torch.equal(saved, keep)


# --------------------------------------------------------------- dropout ----
def philox(counter, key):
    """Philox4x32-10 of uint32 arrays."""
    c = [np.asarray(v, dtype=np.uint64) for v in counter]
    k = [int(v) for v in key]
    lo = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), q & lo, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p & lo]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def keep_mask(B, n, D, p, seed, site):
    G = (D + 7) // 8
    z = np.zeros((B, n, G), dtype=np.uint64)
    seed %= 1 << 64
    w = philox((z + np.arange(G, dtype=np.uint64), z + np.arange(n, dtype=np.uint64)[:, None],
                z + np.arange(B, dtype=np.uint64)[:, None, None], z + np.uint64(site % (1 << 32))),
               (seed & 0xFFFFFFFF, seed >> 32))
    r = np.stack([h for v in w for h in (v & np.uint64(0xFFFF), v >> np.uint64(16))], -1).reshape(B, n, -1)[..., :D]
    return torch.from_numpy(r.astype(np.int64) >= round(p * 65536))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,n,D,lens,p,site", [
    (1, 1, 1, None, 0.5, 0), (1, 1, 512, None, 0.1, 3), (2, 3, 7, (0, 2), 0.3, -1), (3, 17, 33, (17, 0, 5), 0.999, 99),
    (2, 5, 1111, None, 0.0, 1), (5, 300, 768, (300, 11, 299), 0.25, 2), (1, 20000, 96, (19999,), 0.1, 2 ** 31 - 1),
    (9000, 2, 9, (2, 1), 0.5, 4)])
def test_dropout(B, n, D, lens, p, site, dtype):
    dt, code, half = TYPES[dtype]
    g = gen(D)
    L_dev, L = lens_of(lens, B, n)
    m = valid_mask(L, n)[..., None]
    x, res = torch.randn((B, n, D), generator=g).to(dt), torch.randn((B, n, D), generator=g).to(dt)
    x, res = torch.where(m, x, torch.nan).to(dt), torch.where(m, res, torch.nan).to(dt)
    for seed in (-3, 0x123456789ABCDEF):
        s = torch.tensor([seed], device=DEV)
        keep = keep_mask(B, n, D, p, seed, site)
        d = sc.DropoutDesc(B, n, D, p, valid_len=L_dev, site=site, res_scale=0.81, dtype=code)
        t = round(p * 65536)
        dropped = torch.where(keep & m, x.double() * (65536 / (65536 - t)), 0.0)
        out = sc.sc_dropout(d, x.to(DEV), s)
        assert_close(out, dropped, (2 * U + half) * dropped.abs(), "no residual")
        want = torch.where(m, 0.81 * res.double() + dropped, 0.0)
        got = sc.sc_dropout(d, x.to(DEV), s, residual=res.to(DEV))
        # 0.81 itself is rounded to float32
        tol = torch.where(m, 2 * U * (dropped.abs() + res.double().abs()) + (U + half) * want.abs(), 0.0)
        assert_close(got, want, tol, "residual")
        for into in ("x", "residual"):
            a, b = x.to(DEV), res.to(DEV)
            sc.sc_dropout(d, a, s, residual=b, out=a if into == "x" else b)
            assert torch.equal(a if into == "x" else b, got)


def test_dropout_mask_is_a_function_of_the_token():
    """Neither n, D, dtype nor the lengths change a token's mask; seeds and sites do; a dropped infinity is 0."""
    s = torch.tensor([77], device=DEV)
    big = sc.sc_dropout(sc.DropoutDesc(3, 50, 640, 0.5), torch.ones((3, 50, 640), dtype=torch.bfloat16, device=DEV), s)
    small = sc.sc_dropout(sc.DropoutDesc(2, 9, 100, 0.5, dtype=sc.SC_F32), torch.ones((2, 9, 100), device=DEV), s)
    assert torch.equal(small, big[:2, :9, :100].float())
    assert abs(float((big != 0).float().mean()) - 0.5) < 6 * 0.5 / math.sqrt(big.numel())
    x = torch.full((2, 9, 100), float("inf"), device=DEV)
    out = sc.sc_dropout(sc.DropoutDesc(2, 9, 100, 0.5, dtype=sc.SC_F32), x, s)
    assert torch.equal(out == 0, small == 0) and torch.equal(out.isinf(), small != 0)
    other = sc.sc_dropout(sc.DropoutDesc(2, 9, 100, 0.5, dtype=sc.SC_F32, site=1), torch.ones_like(x), s)
    again = sc.sc_dropout(sc.DropoutDesc(2, 9, 100, 0.5, dtype=sc.SC_F32), torch.ones_like(x), s + 1)
    assert not torch.equal(other, small) and not torch.equal(again, small)


# ------------------------------------------------------- far from small ----
def test_rotary_frequencies_of_any_size():
    """Frequencies beyond a turn, negative and tiny ones, at the far ends of 32-bit positions; the angles from integers."""
    from fractions import Fraction
    # 1 / (2 pi) to 100 bits beyond what a double holds
    inv = Fraction(15915494309189533576888376337251436203445964574046, 10 ** 50)
    f = torch.tensor([1.0, -1.0, 300.25, -12345.678, 1e-9, -1e-9, 3.0, 0.0], dtype=torch.float64)
    pos = torch.tensor([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1048577, 77]], dtype=torch.int32)
    n = pos.shape[1]
    turns = torch.tensor([[float(Fraction(float(v)) * inv * int(p) % 1) for v in f] for p in pos[0]], dtype=torch.float64)
    x = torch.randn((1, n, 1, 16), generator=gen(8))
    out = sc.sc_rotary(sc.RotaryDesc(1, n, 1, 1, d=16, dtype=sc.SC_F32), f, x.to(DEV), positions=pos.to(DEV))[0]
    want, mag = rotate64(x.double(), (turns * 2 * math.pi)[None], 1.0, 16, HALF)
    assert_close(out, want, 6 * U * mag, "far")


def test_dropout_offsets_past_32_bits():
    """An array of 5.2 GB in place: its last rows, past 2^31 elements and 2^32 bytes."""
    n, D = 40000, 65544
    x = torch.full((1, n, D), 1.0, dtype=torch.bfloat16, device=DEV)
    sc.sc_dropout(sc.DropoutDesc(1, n, D, 0.5), x, torch.tensor([5], device=DEV), out=x)
    cols = np.arange(D // 8, dtype=np.uint64)
    for j in (0, 32767, 39999):
        w = philox((cols, 0 * cols + np.uint64(j), 0 * cols, 0 * cols), (5, 0))
        r = np.stack([h for v in w for h in (v & np.uint64(0xFFFF), v >> np.uint64(16))], -1).reshape(-1).astype(np.int64)
        assert torch.equal(x[0, j].cpu().float(), torch.from_numpy(r >= 32768).float() * 2)


def test_ffn_offsets_next_to_32_bits():
    """Rows of h that end 70 KB below 4 GiB, and what is kept beside them past 12 GB."""
    torch.cuda.empty_cache()
    ffn_ints_check(1, 32760, 40, 65544, (32760,), seed=3)


def test_ffn_poisoned_outputs_and_workspaces():
    """Nothing that a call writes has to hold anything before, NaNs included, in whole and ragged batches."""
    for B, n, D, F, lens in ((2, 100, 64, 96, (100, 31)), (3, 77, 50, 33, None), (1, 300, 128, 256, (300,))):
        L_dev, m, x, wg, wu, wd, dy = ffn_ints(B, n, D, F, lens, 2)
        d = sc.FfnDesc(B, n, D, F, valid_len=L_dev)
        dev = [t.to(DEV) for t in (x, wg, wu, wd)]
        for save in (False, True):
            y, s = sc.sc_gated_ffn(d, *dev, saved=save)
            y2 = torch.full_like(y, float("nan"))
            work = torch.full((sc.sc_gated_ffn_workspace_size(d, save),), 255, dtype=torch.uint8, device=DEV)
            s2 = torch.full((sc.sc_gated_ffn_saved_size(d),), 255, dtype=torch.uint8, device=DEV) if save else False
            sc.sc_gated_ffn(d, *dev, y=y2, saved=s2, workspace=work)
            assert torch.equal(y, y2)
        out = sc.sc_gated_ffn_backward(d, *dev, s, dy.to(DEV))
        work = torch.full((sc.sc_gated_ffn_backward_workspace_size(d),), 255, dtype=torch.uint8, device=DEV)
        got = sc.sc_gated_ffn_backward(d, *dev, s2, dy.to(DEV), workspace=work,
                                       grads={k: torch.full_like(v, float("nan")) for k, v in out.items()})
        for k in out:
            assert torch.equal(out[k], got[k]), k


def test_many_sequences():
    """As many sequences as the packed rows' table holds, most of them empty; without lengths, more."""
    ffn_ints_check(8192, 2, 16, 24, (0, 2, 0, 1, 0))
    ffn_ints_check(9000, 1, 16, 24, None)
    rotary_case(9000, 2, 1, 1, 16, 16, "bf16", True, HALF, lens=(2, 0, 1))
    rotary_case(9000, 2, 1, 1, 16, 16, "bf16", True, HALF, lens=(2, 0, 1), backward=True)


# ----------------------------------------------- graphs, streams, layers ----
def layer_inputs(B, n, H, F, seed):
    g = gen(seed)
    D = 64 * H
    bf16 = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16)  # noqa: E731
    w = dict(qkv=(torch.randn((D, 3 * D), generator=g) / math.sqrt(D)).to(torch.bfloat16),
             o=(torch.randn((D, D), generator=g) / math.sqrt(D)).to(torch.bfloat16),
             wg=(torch.randn((D, F), generator=g) / math.sqrt(D)).to(torch.bfloat16),
             wu=(torch.randn((D, F), generator=g) / math.sqrt(D)).to(torch.bfloat16),
             wd=(torch.randn((F, D), generator=g) / math.sqrt(F)).to(torch.bfloat16),
             q_w=1 + 0.1 * torch.randn(64, generator=g), k_w=1 + 0.1 * torch.randn(64, generator=g))
    return bf16(B, n, D), bf16(B, n, D), w


class Layer:
    """A training step of one encoder layer on the framework's operators."""

    def __init__(self, B, n, H, F, valid_len, seed_dev, theta=None):
        self.B, self.n, self.H, self.D, self.L, self.seed = B, n, H, 64 * H, valid_len, seed_dev
        self.theta, self.temp = (1.0 / n if theta is None else theta), 0.5 / n
        self.freq, _ = sc.sc_rotary_frequencies(64)
        self.rot = sc.RotaryDesc(B, n, H, H, valid_len=valid_len, norm=True, eps=1e-5)
        self.att = sc.Desc(B, n, H, 32, valid_len)
        self.nd = sc.NormDesc(B, n, self.D, valid_len=valid_len, kind=sc.SC_NORM_RMS)
        self.fd = sc.FfnDesc(B, n, self.D, F, valid_len=valid_len)
        self.drops = [sc.DropoutDesc(B, n, self.D, 0.2, valid_len=valid_len, site=s) for s in range(2)]

    def step(self, x, dout, w):
        B, n, H, D = self.B, self.n, self.H, self.D
        heads = lambda t: [t[..., i * D:(i + 1) * D].unflatten(-1, (H, 64)) for i in range(3)]  # noqa: E731
        y0 = sc.sc_block_norm(self.nd, x, r=False)[1]
        qkv = (y0.view(B * n, D) @ w["qkv"]).view(B, n, 3 * D)
        hw = dict(q_w=w["q_w"], k_w=w["k_w"])
        q, k, v = sc.sc_rotary(self.rot, self.freq, *heads(qkv), **hw)
        o, lse, sp, _ = sc.sc_window_attention(self.att, q, k, v)
        mask, y = sc.sc_ltp_soft_mask(self.att, sc.sc_ltp_score(self.att, sp), self.theta, self.temp, o)
        t1 = (y.view(B * n, D) @ w["o"]).view(B, n, D)
        r1 = sc.sc_dropout(self.drops[0], t1, self.seed, residual=x)
        y1 = sc.sc_block_norm(self.nd, r1, r=False)[1]
        fw = (w["wg"], w["wu"], w["wd"])
        t2, saved = sc.sc_gated_ffn(self.fd, y1, *fw, saved=True)
        out = sc.sc_dropout(self.drops[1], t2, self.seed, residual=r1)
        g = sc.sc_gated_ffn_backward(self.fd, y1, *fw, saved, sc.sc_dropout(self.drops[1], dout, self.seed))
        dr1 = sc.sc_block_norm_backward(self.nd, r1, dr=dout, dy=g["dx"])["dx"]
        dt1 = sc.sc_dropout(self.drops[0], dr1, self.seed)
        dy = (dt1.view(B * n, D) @ w["o"].t()).view(B, n, H, 64)
        dq, dk, dv, dth = sc.sc_ltp_soft_backward(self.att, q, k, v, o, lse, mask, self.temp, dy)
        dqkv = torch.zeros_like(qkv)
        hg = sc.sc_rotary_backward(self.rot, self.freq, dq, dk, dv, *heads(qkv)[:2], **hw, grads=dict(
            zip(("dq", "dk", "dv", "dq_w", "dk_w"), (*heads(dqkv), torch.empty_like(w["q_w"]), torch.empty_like(w["k_w"])))))
        dy0 = (dqkv.view(B * n, 3 * D) @ w["qkv"].t()).view(B, n, D)
        dx = sc.sc_block_norm_backward(self.nd, x, dr=dr1, dy=dy0)["dx"]
        return dict(out=out, dx=dx, wg=g["dwg"], wu=g["dwu"], wd=g["dwd"], q_w=hg["dq_w"], k_w=hg["dk_w"])

    def reference(self, x, dout, w, lens, seed):
        """The same step by float64 autograd."""
        B, n, H, D = self.B, self.n, self.H, self.D
        leaf = {k: t.double().requires_grad_() for k, t in dict(w, x=x).items()}
        m = valid_mask(lens, n)[..., None].double()
        rms = lambda t: t * (t.pow(2).mean(-1, keepdim=True) + 1e-5).rsqrt()  # noqa: E731
        qkv = rms(leaf["x"]) @ leaf["qkv"]
        angle = torch.arange(n).double()[None, :, None] * self.freq
        q, k, v = (qkv[..., i * D:(i + 1) * D].unflatten(-1, (H, 64)) for i in range(3))
        q, k = (rotate64_graph(rms(t) * leaf[nm], angle) for t, nm in ((q, "q_w"), (k, "k_w")))
        s = torch.matmul(q.transpose(1, 2), k.permute(0, 2, 3, 1)) * 0.125
        i = torch.arange(n)
        on = ((i[:, None] - i[None]).abs() <= 16)[None, None] & (m[:, None, None, :, 0] > 0)
        p = torch.softmax(s.masked_fill(~on, -1e30), -1) * m[:, None]
        o = torch.matmul(p, v.transpose(1, 2)).transpose(1, 2)
        score = p.sum((1, 2)) / (H * lens.double()[:, None])
        gate = torch.sigmoid((score - self.theta) / self.temp) * m[..., 0]
        t1 = (o * gate[..., None, None]).flatten(-2) @ leaf["o"]
        keep = [keep_mask(B, n, D, 0.2, seed, site) * (65536 / (65536 - round(0.2 * 65536))) for site in range(2)]
        r1 = leaf["x"] + keep[0] * t1
        y1 = rms(r1)
        a, _ = act64(sc.SC_ACT_SILU, y1 @ leaf["wg"])
        out = (r1 + keep[1] * ((a * (y1 @ leaf["wu"])) @ leaf["wd"])) * m
        out.backward(dout.double())
        return dict(out=out.detach(), dx=leaf["x"].grad, **{nm: leaf[nm].grad for nm in ("wg", "wu", "wd", "q_w", "k_w")})


def rotate64_graph(x, angle):
    c, s = angle.cos()[:, :, None], angle.sin()[:, :, None]
    a, b = x[..., :32], x[..., 32:]
    return torch.cat([a * c - b * s, a * s + b * c], -1)


def test_layer_training_step():
    """The operators together, against float64 autograd: about thirty roundings to bf16 of 2^-8 / sqrt(3) each lie
    behind a gradient, which norms and softmax pass on at most doubled: 2 sqrt(30) 0.0023 = 0.025 of its 2-norm."""
    B, n, H, F, seed = 3, 90, 2, 168, 1234567
    lens = torch.tensor([90, 41, 64])
    x, dout, w = layer_inputs(B, n, H, F, 5)
    m = valid_mask(lens, n)
    dout[~m] = 0
    layer = Layer(B, n, H, F, lens.to(torch.int32).to(DEV), torch.tensor([seed], device=DEV))
    got = layer.step(x.to(DEV), dout.to(DEV), {k: t.to(DEV) for k, t in w.items()})
    want = layer.reference(x, dout, w, lens, seed)
    for nm, v in want.items():
        rel = float((got[nm].double().cpu() - v).norm() / v.norm())
        assert rel <= 0.025, (nm, rel)


def test_layer_step_in_a_graph():
    """A captured training step, replayed with other inputs, lengths and seeds and eager steps between the replays."""
    B, n, H, F = 2, 150, 2, 200
    x, dout, w = layer_inputs(B, n, H, F, 6)
    w = {k: t.to(DEV) for k, t in w.items()}
    x, dout = x.to(DEV), dout.to(DEV)
    L, seed = torch.tensor([150, 77], dtype=torch.int32, device=DEV), torch.tensor([1], device=DEV)
    layer = Layer(B, n, H, F, L, seed)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        layer.step(x, dout, w)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = layer.step(x, dout, w)
    torch.cuda.synchronize()
    for i, lens in enumerate(([150, 77], [1, 150], [0, 0], [150, 150], [64, 33])):
        x.copy_(torch.randn(x.shape, generator=gen(i)).to(torch.bfloat16))
        dout.copy_(torch.randn(x.shape, generator=gen(i + 50)).to(torch.bfloat16))
        L.copy_(torch.tensor(lens, dtype=torch.int32))
        seed.fill_(i * 7919 - 3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        first = {k: v.clone() for k, v in out.items()}
        eager = layer.step(x, dout, w)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, v in eager.items():
            assert torch.equal(first[k], v) and torch.equal(out[k], v), (k, lens)


def test_two_streams_at_once():
    """Calls on two streams with their own outputs and workspaces, and one workspace for two graphs replayed in turn."""
    B, n, D, F = 2, 300, 128, 256
    g = gen(11)
    xs = [torch.randn((B, n, D), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2)]
    w = [(torch.randn(s, generator=g) / math.sqrt(s[0])).to(torch.bfloat16).to(DEV) for s in ((D, F), (D, F), (F, D))]
    L = torch.tensor([300, 123], dtype=torch.int32, device=DEV)
    d = sc.FfnDesc(B, n, D, F, valid_len=L)
    want = []
    for x in xs:
        y, s = sc.sc_gated_ffn(d, x, *w, saved=True)
        want.append((y, sc.sc_gated_ffn_backward(d, x, *w, s, x)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i, st in enumerate(streams):
            y, s = sc.sc_gated_ffn(d, xs[i], *w, saved=True, stream=st)
            got[i].append((y, s, sc.sc_gated_ffn_backward(d, xs[i], *w, s, xs[i], stream=st)))
    torch.cuda.synchronize()
    for i in range(2):
        for y, _, gr in got[i]:
            assert torch.equal(y, want[i][0]) and all(torch.equal(gr[k], want[i][1][k]) for k in gr)
    work = torch.empty(sc.sc_gated_ffn_workspace_size(d), dtype=torch.uint8, device=DEV)
    ys, graphs = [torch.empty_like(x) for x in xs], []
    with torch.cuda.stream(streams[0]):
        for x, y in zip(xs, ys):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=streams[0]):
                sc.sc_gated_ffn(d, x, *w, y=y, workspace=work)
        for _ in range(3):
            for gr in graphs:
                gr.replay()
    torch.cuda.synchronize()
    for y, (ref, _) in zip(ys, want):
        assert float((y.double() - ref.double()).norm()) <= 0.0035 * float(ref.double().norm())


def test_debug_library_refuses_bad_lengths():
    """The debug build reports lengths out of range; the release build clamps them."""
    import ctypes
    import os
    if not os.path.exists(sc.debug_lib_path()):
        pytest.skip("libsc_debug.so not built")
    L = torch.tensor([5, 9], dtype=torch.int32, device=DEV)
    x = torch.ones((2, 8, 16), dtype=torch.bfloat16, device=DEV)
    seed, out = torch.tensor([1], device=DEV), torch.empty_like(x)
    d = sc.DropoutDesc(2, 8, 16, 0.0, valid_len=L)
    for lib, want in ((sc.load(), 0), (sc.load_debug(), -1)):
        assert lib.sc_dropout(ctypes.byref(d.c()), x.data_ptr(), seed.data_ptr(), None, out.data_ptr(), None) == want
    torch.cuda.synchronize()
    assert torch.equal(out[1], x[1]) and not out[0, 5:].any()


def off_by_one(t):
    """The same values one element past an aligned address."""
    buf = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)
    buf[1:] = t.reshape(-1)
    return buf[1:].view(t.shape)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_any_element_address(dtype):
    """Tensors aligned to their elements alone give what aligned ones give; the feed-forward block refuses them."""
    dt, code, _ = TYPES[dtype]
    g = gen(12)
    for D in (64, 37):
        x, r = (torch.randn((2, 9, D), generator=g).to(dt).to(DEV) for _ in range(2))
        d, s = sc.DropoutDesc(2, 9, D, 0.3, dtype=code), torch.tensor([9], device=DEV)
        want = sc.sc_dropout(d, x, s, residual=r)
        assert torch.equal(sc.sc_dropout(d, off_by_one(x), s, residual=off_by_one(r), out=off_by_one(x)), want)
    q = torch.randn((2, 9, 3, 64), generator=g).to(dt).to(DEV)
    w = torch.rand(64, generator=g).to(DEV)
    freq, _ = sc.sc_rotary_frequencies(64)
    d = sc.RotaryDesc(2, 9, 3, 3, norm=True, dtype=code)
    a, b = sc.sc_rotary(d, freq, q, q, q_w=w)[:2], sc.sc_rotary(d, freq, off_by_one(q), q, q_w=off_by_one(w))[:2]
    for u, v in zip(a, b):
        assert_close(u, v.double().cpu(), (4 * TYPES[dtype][2] * v.double().abs() + 64 * U).cpu(), "unaligned")
    if dtype == "bf16":
        f = sc.FfnDesc(2, 9, 64, 64)
        x, m = q[:, :, 0].contiguous(), torch.zeros((64, 64), dtype=dt, device=DEV)
        with pytest.raises(sc.ScError) as e:
            sc.sc_gated_ffn(f, off_by_one(x), m, m, m)
        assert e.value.status == -1


def test_rotary_default_gradients_and_strides():
    """Gradients allocated by the call, laid out as strided inputs; strides that are not a token's run are refused."""
    B, n, H = 2, 11, 2
    rows = torch.randn((B, n, 3 * H * 64 + 8), generator=gen(13)).to(torch.bfloat16).to(DEV)
    q, k, v = (rows[..., i * 128:(i + 1) * 128].unflatten(-1, (H, 64)) for i in range(3))
    go = [torch.randn((B, n, H, 64), generator=gen(i)).to(torch.bfloat16).to(DEV) for i in range(3)]
    freq, _ = sc.sc_rotary_frequencies(64)
    d = sc.RotaryDesc(B, n, H, H, norm=True)
    w = dict(q_w=torch.rand(64, device=DEV), k_w=torch.rand(64, device=DEV))
    a = sc.sc_rotary_backward(d, freq, *go, q=q, k=k, **w)
    b = sc.sc_rotary_backward(d, freq, *go, q=q.contiguous(), k=k.contiguous(), **w)
    assert all(torch.equal(a[nm], b[nm]) for nm in ("dq", "dk", "dv", "dq_w", "dk_w"))
    only = sc.sc_rotary_backward(d, freq, go[0], q=q)
    assert torch.equal(only["dq"], sc.sc_rotary_backward(d, freq, go[0], q=q.contiguous())["dq"]) and only["dk"] is None
    for bad in (rows[..., :128].unflatten(-1, (64, H)).transpose(-1, -2), rows[:, ::1, :128].unflatten(-1, (H, 64)).flip(1)[:, :, :, ::2],
                q.transpose(0, 1).contiguous().transpose(0, 1)):
        with pytest.raises(ValueError):
            sc.sc_rotary(d, freq, bad)


@pytest.mark.parametrize("backward", [False, True])
def test_rotary_many_heads(backward):
    rotary_case(1, 5, 100, 1, 64, 64, "bf16", True, HALF, backward=backward)
    rotary_case(2, 3, 2, 40, 256, 128, "f32", True, INTER, kind=sc.SC_NORM_LAYER, lens=(3, 2), backward=backward)


@pytest.mark.parametrize("T", [1, 15, 16, 17, 32, 33, 64, 65, 127, 128, 129])
def test_ffn_few_rows_exact(T):
    """Around the borders of the few rows' kernels, widths that end inside their blocks and chunks."""
    ffn_ints_check(1, T, 72, 104, None, seed=T)
    ffn_ints_check(1, T, 1000, 2056, (T,), seed=T)


@pytest.mark.parametrize("B,n,D,F,lens", [
    (1, 1024, 768, 2304, None), (2, 1024, 1024, 2816, (1024, 700)), (2, 1024, 4096, 512, (1000, 1024)),
    (1, 5000, 80, 64, None), (8, 2048, 768, 2048, (2048, 2048, 5, 0, 1999)), (8, 2048, 768, 2048, (0, 3, 0, 0))])
def test_ffn_joined_products(B, n, D, F, lens):
    """Backward products that share a launch, with as many tiles as the sizes say, fewer and none; a gradient asked for
    alone, in launches of its own, is the same."""
    ffn_ints_check(B, n, D, F, lens)
    L_dev, m, x, wg, wu, wd, dy = (t.to(DEV) if t is not None else None for t in ffn_ints(B, n, D, F, lens, 1))
    d = sc.FfnDesc(B, n, D, F, valid_len=L_dev)
    _, saved = sc.sc_gated_ffn(d, x, wg, wu, wd, saved=True)
    out = sc.sc_gated_ffn_backward(d, x, wg, wu, wd, saved, dy)
    for nm, v in out.items():
        alone = sc.sc_gated_ffn_backward(d, x, wg, wu, wd, saved, dy, grads={nm: torch.empty_like(v)})[nm]
        assert torch.equal(alone, v), nm


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("B,n,Hq,Hk,d,R,dtype,layout", [
    (2, 40, 4, 4, 80, 40, "bf16", HALF), (2, 40, 4, 2, 80, 40, "f32", HALF), (1, 50, 3, 3, 24, 8, "bf16", HALF),
    (1, 50, 3, 1, 88, 24, "f32", INTER), (1, 50, 3, 3, 40, 40, "bf16", INTER), (2, 30, 2, 2, 76, 20, "bf16", HALF)])
def test_rotary_vectors_of_four_pairs(B, n, Hq, Hk, d, R, dtype, layout, backward):
    """Halves that end inside a lane's eight pairs."""
    rotary_case(B, n, Hq, Hk, d, R, dtype, True, layout, sc.SC_NORM_RMS, lens=(n, n - 3), backward=backward)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("Hq,Hk", [(2, 2), (3, 1)])
def test_rotary_many_padded_sequences(Hq, Hk, backward):
    """Several rounds of tiles, most of them padding."""
    rotary_case(40, 512, Hq, Hk, 64, 32, "bf16", True, HALF, sc.SC_NORM_RMS, lens=[(37 * i) % 300 for i in range(40)],
                backward=backward)


# ------------------------------------------------------ activations everywhere ----
@pytest.mark.parametrize("act", [sc.SC_ACT_NONE, sc.SC_ACT_GELU, sc.SC_ACT_SILU])
@pytest.mark.parametrize("B,n,D,F,lens", [
    (1, 1, 512, 776, None), (1, 17, 520, 768, (17,)), (2, 20, 504, 1032, (20, 9)), (16, 8, 768, 2304, (8, 4, 5, 1)),
    (1, 129, 512, 768, None), (3, 501, 512, 1024, (501, 7, 0)), (1, 1500, 504, 1024, None),
    (2, 2048, 512, 4096, (2048, 1999)), (1, 2048, 512, 4096, None)])
def test_ffn_activations(B, n, D, F, lens, act):
    """Every activation with and without what is kept, from one row to tiles of every kind; a form with gate and up
    exchanged, or with another activation, is beyond the tolerance of the norm, which is the module's.

    A value's tolerance: two roundings to bf16 behind it, (1 + 2^-8)^2 - 1 of the products' magnitudes at most, and 2^-13
    for the activation's 3e-5, the kept factors' 2^-15 and float32 products.  To that the float32 sums add, where they
    cancel (g of 1.5e-6 from 512 products of magnitude 28): K additions of partial sums that are never above the sum A
    of the magnitudes are off by K u A.  So g, u and dh are off by e = D u A; act(g) by 1.13 e_g + 1e-6 and its slope by
    0.8 e_g + 2e-6 (the largest slopes of the activations and of their slopes, and their own errors next to 0), which
    the products pass on to h, dg and du, and the last sums to the results, with K u of their own magnitudes."""
    g_ = gen(B + D + act)
    L_dev, L = lens_of(lens, B, n)
    m = valid_mask(L, n).to(DEV)
    x, dy = (torch.randn((B, n, D), generator=g_).to(torch.bfloat16).to(DEV) for _ in range(2))
    w = [(torch.randn(s, generator=g_) * k / math.sqrt(s[0])).to(torch.bfloat16).to(DEV)
         for s, k in (((D, F), 2), ((D, F), 2), ((F, D), 1))]
    d = sc.FfnDesc(B, n, D, F, valid_len=L_dev, act=act)
    y, _ = sc.sc_gated_ffn(d, x, *w)
    y_kept, saved = sc.sc_gated_ffn(d, x, *w, saved=True)
    out = sc.sc_gated_ffn_backward(d, x, *w, saved, dy)
    xs, ds = x[m].double(), dy[m].double()
    wg, wu, wd = (t.double() for t in w)
    g, u = xs @ wg, xs @ wu
    a, slope = act64(act, g)
    h, dh = a * u, ds @ wd.t()
    dg, du = dh * u * slope, dh * a
    A = torch.abs
    eg, eu, edh = D * U * (A(xs) @ A(wg)), D * U * (A(xs) @ A(wu)), D * U * (A(ds) @ A(wd).t())
    ea, es = 1.13 * eg + 1e-6, 0.8 * eg + 2e-6
    eh, edu = ea * A(u) + A(a) * eu, A(a) * edh + A(dh) * ea
    edg = A(u * slope) * edh + A(dh) * (A(slope) * eu + A(u) * es)
    R = xs.shape[0]

    def wide(v, e, right, K):
        return (2 * 2.0 ** -8 + 2.0 ** -13 + K * U) * (A(v) @ A(right)) + 1.01 * (e @ A(right))
    want = dict(y=(h @ wd, wide(h, eh, wd, F)),
                dx=(dg @ wg.t() + du @ wu.t(), wide(dg, edg, wg.t(), 2 * F) + wide(du, edu, wu.t(), 2 * F)),
                dwg=(xs.t() @ dg, wide(dg.t(), edg.t(), xs, R).t()), dwu=(xs.t() @ du, wide(du.t(), edu.t(), xs, R).t()),
                dwd=(h.t() @ ds, wide(h.t(), eh.t(), ds, R)))
    want["y_kept"] = want["y"]
    for nm, (v, tol) in want.items():
        got = dict(out, y=y, y_kept=y_kept)[nm].double()
        if nm in ("y", "y_kept", "dx"):
            assert not got[~m].any(), nm
            got = got[m]
        assert float((got - v).norm()) <= 0.0035 * float(v.norm()), nm
        assert_close(got, v.cpu(), tol.cpu(), nm)
    for other, (gate, up) in ((act, (u, g)), ((act + 1) % 3, (g, u))):
        wrong = (act64(other, gate)[0] * up) @ wd
        if other != act or act != sc.SC_ACT_NONE:  # without an activation the product is symmetric
            assert float((wrong - want["y"][0]).norm()) > 0.01 * float(wrong.norm())


@pytest.mark.parametrize("T,F,row", [(1, 8, 0), (300, 8, 7), (1500, 1000, 1400), (4096, 4096, 4000)])
def test_ffn_kept_factors_are_rounded(T, F, row):
    """What is kept of g and u is rounded to the nearest of 24 bits, not cut: 3 * 2^-17 beside a tie of bf16 at 1 to 2,
    more than half of the 2^-15 between neighbours, stays on its side, for either sign and either even neighbour."""
    D = 8
    x = torch.tensor([1, 2.0 ** -7, 2.0 ** -8, 3 * 2.0 ** -17, 0, 0, 0, 0])
    cols = [[s, s * odd, s, s * side, 0, 0, 0, 0] for s in (1, -1) for odd in (0, 1) for side in (1, -1)]
    wu = torch.tensor(cols).t().float().repeat(1, F // 8)
    wg = wu.roll(3, 1)
    wd, dy = torch.zeros((F, D)), torch.zeros((1, T, D))
    wd[:, 0], dy[0, row, 0] = 1, 1  # dh = 1 in one row
    dev = [t.to(torch.bfloat16).to(DEV) for t in (x.expand(1, T, D), wg, wu, wd)]
    d = sc.FfnDesc(1, T, D, F, act=sc.SC_ACT_NONE)
    _, saved = sc.sc_gated_ffn(d, *dev, saved=True)
    out = sc.sc_gated_ffn_backward(d, *dev, saved, dy.to(torch.bfloat16).to(DEV))
    for nm, w in (("dwg", wu), ("dwu", wg)):
        want = (x @ w).to(torch.bfloat16)  # exact in float32
        assert torch.equal(out[nm][0].cpu(), want), nm


@pytest.mark.parametrize("Hq,Hk,pad,which", [(4, 2, 0, "qkv"), (4, 2, 8, "qkv"), (3, 3, 0, "qk"), (2, 2, 0, "kv"),
                                            (2, 2, 16, "q")])
def test_rotary_default_gradients_share_rows(Hq, Hk, pad, which):
    """Gradients that the call allocates for parts of fused rows lie side by side in one array of such rows, no larger
    than what it is the gradient of; parts of rows of different widths, or too wide for one row, in rows of their own."""
    B, n, d = 3, 21, 64
    W = (Hq + 2 * Hk) * d + pad
    rows = torch.randn((B, n, W), generator=gen(21)).to(torch.bfloat16).to(DEV)
    cut = (0, Hq * d, (Hq + Hk) * d, (Hq + 2 * Hk) * d)
    parts = [rows[..., cut[i]:cut[i + 1]].unflatten(-1, (-1, d)) for i in range(3)]
    go = [torch.randn((B, n, h, d), generator=gen(h)).to(torch.bfloat16).to(DEV) if nm in which else None
          for nm, h in zip("qkv", (Hq, Hk, Hk))]
    freq, _ = sc.sc_rotary_frequencies(d)
    D = sc.RotaryDesc(B, n, Hq, Hk, norm=True)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    out = sc.sc_rotary_backward(D, freq, *go, q=parts[0], k=parts[1])
    size = (B * n * W * 2 + 511) // 512 * 512  # the allocator's granularity
    assert torch.cuda.memory_allocated() - before <= size
    want = sc.sc_rotary_backward(D, freq, *go, q=parts[0].contiguous(), k=parts[1].contiguous())
    have = [nm for nm in ("dq", "dk", "dv") if out[nm] is not None]
    assert have == ["d" + nm for nm in which]
    for nm in have:
        assert torch.equal(out[nm], want[nm])
        assert out[nm].untyped_storage().data_ptr() == out[have[0]].untyped_storage().data_ptr()
    if which == "qkv":  # together they are the gradient of the fused rows
        fused = out["dq"].as_strided((B, n, W), (n * W, W, 1))
        assert torch.equal(fused[..., :W - pad], torch.cat([want[nm].flatten(-2) for nm in have], -1))
    # rows of other widths
    k2 = torch.randn((B, n, Hk * d + 8), generator=gen(22)).to(torch.bfloat16).to(DEV)[..., :Hk * d].unflatten(-1, (-1, d))
    a = sc.sc_rotary_backward(D, freq, *go, q=parts[0], k=k2)
    b = sc.sc_rotary_backward(D, freq, *go, q=parts[0].contiguous(), k=k2.contiguous())
    assert all(torch.equal(a[nm], b[nm]) for nm in have)
    # rows that hold one part and no second one
    q2 = torch.randn((2, B, n, Hk * d + 8), generator=gen(23)).to(torch.bfloat16).to(DEV)[..., :Hk * d].unflatten(-1, (-1, d))
    E, g2 = sc.RotaryDesc(B, n, Hk, Hk, norm=True), torch.randn((3, B, n, Hk, d), generator=gen(24)).to(torch.bfloat16).to(DEV)
    a = sc.sc_rotary_backward(E, freq, *g2, q=q2[0], k=q2[1])
    b = sc.sc_rotary_backward(E, freq, *g2, q=q2[0].contiguous(), k=q2[1].contiguous())
    assert all(torch.equal(a[nm], b[nm]) for nm in ("dq", "dk", "dv"))
    assert a["dq"].untyped_storage().data_ptr() != a["dk"].untyped_storage().data_ptr()


@pytest.mark.parametrize("act", [sc.SC_ACT_GELU, sc.SC_ACT_SILU])
@pytest.mark.parametrize("B,n,D,F", [(2, 16, 256, 520), (2, 64, 256, 520), (2, 65, 256, 520), (2, 700, 500, 1111),
                                     (2, 1024, 512, 4096)])
def test_ffn_rows_by_themselves(B, n, D, F, act):
    """A row's bits depend neither on other rows, NaNs and infinities among them, nor on the lengths; beyond 128 rows, nor
    on whether anything is kept."""
    g = gen(n)
    x = torch.randn((B, n, D), generator=g).to(torch.bfloat16).to(DEV)
    w = [(torch.randn(s, generator=g) / math.sqrt(s[0])).to(torch.bfloat16).to(DEV) for s in ((D, F), (D, F), (F, D))]
    other = torch.randn((B, n, D), generator=g).to(torch.bfloat16).to(DEV)
    other[:, 1::4], other[:, 3::8] = float("nan"), float("inf")
    other[:, ::2] = x[:, ::2]
    L = torch.tensor([n, n // 2], dtype=torch.int32, device=DEV)
    ys = {}
    for kept in (False, True):
        y = ys[kept] = sc.sc_gated_ffn(sc.FfnDesc(B, n, D, F, act=act), x, *w, saved=kept)[0]
        assert bool(y.isfinite().all())
        assert torch.equal(sc.sc_gated_ffn(sc.FfnDesc(B, n, D, F, act=act), other, *w, saved=kept)[0][:, ::2], y[:, ::2])
        r = sc.sc_gated_ffn(sc.FfnDesc(B, n, D, F, act=act, valid_len=L), x, *w, saved=kept)[0]
        assert torch.equal(r[0], y[0]) and torch.equal(r[1, :n // 2], y[1, :n // 2]) and not r[1, n // 2:].any()
    if B * n > 128:
        assert torch.equal(ys[False], ys[True])
    else:  # rounded once more, from sums and an h that differ in a rounding
        a, b = ys[False].double(), ys[True].double()
        assert float((a - b).norm()) <= 2 * 0.0035 * float(b.norm())


@pytest.mark.parametrize("B,n,Hq,Hk", [(5, 1, 2, 2), (1, 1, 2, 1), (1, 9, 1, 1), (6, 1, 1, 1)])
def test_rotary_default_gradients_of_few_tokens(B, n, Hq, Hk):
    """One token, one sequence, one head: sizes whose strides say nothing."""
    W = (Hq + 2 * Hk) * 64
    rows = torch.randn((B, n, W), generator=gen(31)).to(torch.bfloat16).to(DEV)
    q, k, _ = (t.unflatten(-1, (-1, 64)) for t in rows.split((Hq * 64, Hk * 64, Hk * 64), -1))
    go = [torch.randn((B, n, h, 64), generator=gen(h)).to(torch.bfloat16).to(DEV) for h in (Hq, Hk, Hk)]
    freq, _ = sc.sc_rotary_frequencies(64)
    D = sc.RotaryDesc(B, n, Hq, Hk, norm=True)
    w = dict(q_w=torch.rand(64, generator=gen(32)).to(DEV), k_w=torch.rand(64, generator=gen(33)).to(DEV))
    a = sc.sc_rotary_backward(D, freq, *go, q=q, k=k, **w)
    b = sc.sc_rotary_backward(D, freq, *go, q=q.contiguous().clone(), k=k.contiguous().clone(), **w)
    assert all(torch.equal(a[nm], b[nm]) for nm in b)
