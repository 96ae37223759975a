"""ctypes binding of the layer operators of libsc.so (include/sc_layer.h; argument marshalling only)."""
from __future__ import annotations

import ctypes

from ._binding import (SC_ACT_SILU, SC_BF16, SC_NORM_RMS, SC_ROTARY_HALF, SC_ROTARY_PLAIN, _check, _DropoutDesc,
                       _FfnDesc, _on_stream, _RotaryDesc, _tensor, load)
from ._block import _Call, _float_type


def sc_rotary_frequencies(rot_dim, base=10000.0, scaling=SC_ROTARY_PLAIN, factor=1.0, length=0.0, fast=32.0, slow=1.0):
    """(freq, amplitude): the angle per position of each pair, a float64 tensor [rot_dim / 2] on the host, and the factor
    on the rotated dimensions."""
    import torch
    freq = torch.empty(max(int(rot_dim) // 2, 0), dtype=torch.float64)
    amplitude = ctypes.c_float()
    _check(load().sc_rotary_frequencies(int(rot_dim), float(base), int(scaling), float(factor), float(length),
                                        float(fast), float(slow), freq.data_ptr(), ctypes.byref(amplitude)),
           "sc_rotary_frequencies")
    return freq, amplitude.value


class RotaryDesc:
    """Geometry and form of the rotation of queries and keys (mirrors sc_rotary_desc, whose strides are those of the
    tensors given).  valid_len: int32 device tensor [B] or None; rot_dim: None for all of d."""

    def __init__(self, B, n, Hq, Hk, d=64, rot_dim=None, valid_len=None, layout=SC_ROTARY_HALF, norm=False,
                 kind=SC_NORM_RMS, eps=1e-6, amplitude=1.0, dtype=SC_BF16):
        self.B, self.n, self.Hq, self.Hk, self.d = int(B), int(n), int(Hq), int(Hk), int(d)
        self.rot_dim = self.d if rot_dim is None else int(rot_dim)
        self.valid_len = valid_len
        self.layout, self.norm, self.kind = int(layout), int(bool(norm)), int(kind)
        self.eps, self.amplitude, self.dtype = float(eps), float(amplitude), int(dtype)

    def c(self, strides=(0, 0, 0)) -> _RotaryDesc:
        return _RotaryDesc(self.B, self.n, self.Hq, self.Hk, self.d,
                           None if self.valid_len is None else self.valid_len.data_ptr(), self.rot_dim, self.layout,
                           self.norm, self.kind, self.eps, self.amplitude, self.dtype, *strides)

    def heads(self, part):
        return self.Hk if part else self.Hq


def _freq(desc, freq):
    """Address of the frequencies."""
    import torch
    if desc.rot_dim == 0:
        return None
    if not isinstance(freq, torch.Tensor):
        raise TypeError(f"freq: expected a torch.Tensor, got {type(freq).__name__}")
    if freq.device.type != "cpu" or freq.dtype != torch.float64 or freq.shape != (desc.rot_dim // 2,) or \
            not freq.is_contiguous():
        raise ValueError(f"freq: expected a float64 tensor [{desc.rot_dim // 2}] on the host")
    return freq.data_ptr()


def _heads(call, desc, t, name, part, dt):
    """(address, elements between tokens) of the heads of one part, [B, n, heads, d], dense or in wider rows."""
    H, d = desc.heads(part), desc.d
    row = H * d
    if t is None:
        return None, row
    shape = (desc.B, desc.n, H, d)
    try:
        if t.dtype is dt and t.shape == shape and t.get_device() == call.device:
            if t.is_contiguous():
                return t.data_ptr(), row
            s = t.stride()
            # a token's heads are one run, the tokens evenly spaced (a stride of one token or sequence is not used)
            step = s[1] if desc.n > 1 else s[0] if desc.B > 1 else row
            if s[3] == 1 and (H == 1 or s[2] == d) and step >= row and (desc.B == 1 or s[0] == desc.n * step):
                return t.data_ptr(), step
            raise ValueError(f"{name}: heads of a token have to be contiguous and tokens evenly spaced, got strides {s}")
    except AttributeError:
        pass
    _tensor(t, name, dt, shape)
    raise ValueError(f"{name}: on {t.device}, the call's stream on device {call.device}")


def _default_heads(desc, call, outer, steps, dt):
    """New gradients of the parts whose `outer` are given, steps[part] elements between tokens (None: any).  Parts of
    rows wider than themselves lie side by side in rows of one array, q, k, v, as far as they fit."""
    outs, rows, wide, at = [], None, 0, 0
    for part, (g, step) in enumerate(zip(outer, steps)):
        shape = (desc.B, desc.n, desc.heads(part), desc.d)
        row = shape[2] * desc.d
        fits = rows is not None and step in (None, wide) and at + row <= wide
        if g is None:
            outs.append(None)
        elif step == row or (step is None and not fits):
            outs.append(call.new(dt, shape))
        else:
            if not fits:
                rows, wide, at = call.new(dt, (desc.B * desc.n * step,)), step, 0
            outs.append(rows.as_strided(shape, (desc.n * wide, wide, desc.d, 1), at))
            at += row
    return outs


def _rotary_common(desc, call, q_w, k_w, positions):
    import torch
    call.lengths(desc.valid_len, desc.B)
    vec, f32 = (desc.d,), torch.float32
    return (call.opt(q_w, "q_w", f32, vec), call.opt(k_w, "k_w", f32, vec),
            call.opt(positions, "positions", torch.int32, (desc.B, desc.n)))


@_on_stream
def sc_rotary(desc: RotaryDesc, freq, q, k=None, v=None, q_w=None, k_w=None, positions=None, q_out=None, k_out=None,
              v_out=None, stream=None):
    """Norms and rotates the heads of q and k and copies v, [B, n, heads, d] each, dense or parts of fused rows.  Returns
    (q_out, k_out, v_out), dense; absent ones are None.  q may be None as k and v."""
    L = load()
    call = _Call(stream, q if q is not None else k if k is not None else v)
    dt = _float_type(desc.dtype, "dtype")
    small = _rotary_common(desc, call, q_w, k_w, positions)
    ins, strides, outs, ptrs = [], [], [], []
    for part, (t, o, nm) in enumerate(((q, q_out, "q"), (k, k_out, "k"), (v, v_out, "v"))):
        p, step = _heads(call, desc, t, nm, part, dt)
        ins.append(p)
        strides.append(step)
        shape = (desc.B, desc.n, desc.heads(part), desc.d)
        if t is not None and o is None:
            o = call.new(dt, shape)
        outs.append(o)
        ptrs.append(call.opt(o, nm + "_out", dt, shape))
    _check(L.sc_rotary(ctypes.byref(desc.c(strides)), _freq(desc, freq), *ins, *small, *ptrs, call.stream), "sc_rotary")
    return tuple(outs)


def sc_rotary_backward_workspace_size(desc: RotaryDesc) -> int:
    return load().sc_rotary_backward_workspace_size(ctypes.byref(desc.c()))


@_on_stream
def sc_rotary_backward(desc: RotaryDesc, freq, dq_out=None, dk_out=None, dv_out=None, q=None, k=None, q_w=None,
                       k_w=None, positions=None, grads=None, workspace=None, stream=None):
    """Gradients of sc_rotary from those of its outputs.  Returns a dict of dq, dk, dv, dq_w and dk_w, None for what is
    absent: a weight that was not given has no gradient.

    q, k: the forward's inputs, with desc.norm only.  grads: optional dict of preallocated outputs, of which dq, dk, dv
    may be parts of fused rows laid out as q, k, v; only those it names are computed.  Without, dq, dk and dv are dense,
    or, where q and k are parts of fused rows, lie side by side in rows of that width of one array."""
    import torch
    L = load()
    dt, f32 = _float_type(desc.dtype, "dtype"), torch.float32
    outer = (dq_out, dk_out, dv_out)
    call = _Call(stream, next((t for t in outer if t is not None), None))
    small = _rotary_common(desc, call, q_w, k_w, positions)
    names = ("dq", "dk", "dv")
    if grads is not None:
        unknown = set(grads) - {*names, "dq_w", "dk_w"}
        if unknown:
            raise ValueError(f"grads: unknown outputs {sorted(unknown)}")
    out = {}
    strides, gptr, optr, iptr = [], [], [], []
    outs = outer if grads is None else [grads.get(nm) for nm in names]
    ins = [_heads(call, desc, x, "qkv"[part], part, dt) if desc.norm and x is not None and outs[part] is not None
           else (None, None) for part, x in enumerate((q, k, None))]
    if grads is None:
        outs = _default_heads(desc, call, outer, [s for _, s in ins], dt)
    for part, (g, nm, o, (px, sx)) in enumerate(zip(outer, names, outs, ins)):
        shape = (desc.B, desc.n, desc.heads(part), desc.d)
        if o is not None and g is None:
            raise ValueError(f"{nm}: needs {nm}_out")
        po, step = _heads(call, desc, o, nm, part, dt)
        if px is not None and sx != step:
            raise ValueError(f"{nm}: {step} elements between tokens, {sx} in {'qkv'[part]}")
        out[nm] = o
        iptr.append(px)
        strides.append(step)
        optr.append(po)
        gptr.append(call.opt(g, nm + "_out", dt, shape) if o is not None else None)
    wptr = []
    for nm, w, need in (("dq_w", q_w, out["dq"]), ("dk_w", k_w, out["dk"])):
        o = torch.empty_like(w) if grads is None and w is not None and need is not None else (grads or {}).get(nm)
        out[nm] = o
        wptr.append(call.opt(o, nm, f32, (desc.d,)))
    cd = ctypes.byref(desc.c(strides))
    need = L.sc_rotary_backward_workspace_size(cd) if any(p is not None for p in wptr) else 0
    work, wsb, keep = call.workspace(workspace, need)
    _check(L.sc_rotary_backward(cd, _freq(desc, freq), *gptr, *iptr[:2], *small, *optr, *wptr, work, wsb, call.stream),
           "sc_rotary_backward")
    return out


class FfnDesc:
    """Geometry of a gated feed-forward block (mirrors sc_ffn_desc).  valid_len: int32 device tensor [B] or None."""

    def __init__(self, B, n, D, F, valid_len=None, act=SC_ACT_SILU, dtype=SC_BF16):
        self.B, self.n, self.D, self.F = int(B), int(n), int(D), int(F)
        self.valid_len = valid_len
        self.act, self.dtype = int(act), int(dtype)

    def c(self) -> _FfnDesc:
        return _FfnDesc(self.B, self.n, self.D, self.F, None if self.valid_len is None else self.valid_len.data_ptr(),
                        self.act, self.dtype)


def sc_gated_ffn_workspace_size(desc: FfnDesc, save: bool = False) -> int:
    return load().sc_gated_ffn_workspace_size(ctypes.byref(desc.c()), int(bool(save)))


def sc_gated_ffn_saved_size(desc: FfnDesc) -> int:
    return load().sc_gated_ffn_saved_size(ctypes.byref(desc.c()))


def sc_gated_ffn_backward_workspace_size(desc: FfnDesc) -> int:
    return load().sc_gated_ffn_backward_workspace_size(ctypes.byref(desc.c()))


def _ffn_inputs(call, desc, x, wg, wu, wd):
    dt = _float_type(desc.dtype, "dtype")
    D, F = desc.D, desc.F
    call.lengths(desc.valid_len, desc.B)
    return dt, (call.ptr(x, "x", dt, (desc.B, desc.n, D)), call.ptr(wg, "wg", dt, (D, F)),
                call.ptr(wu, "wu", dt, (D, F)), call.ptr(wd, "wd", dt, (F, D)))


def _saved(call, t, need):
    import torch
    p = call.ptr(t, "saved", torch.uint8, t.shape if isinstance(t, torch.Tensor) else ())
    if t.numel() < need:
        raise ValueError(f"saved: {t.numel()} bytes, {need} needed")
    return p


@_on_stream
def sc_gated_ffn(desc: FfnDesc, x, wg, wu, wd, y=None, saved=False, workspace=None, stream=None):
    """y [B, n, D] = (act(x Wg) * (x Wu)) Wd; wg, wu [D, F], wd [F, D].  Returns (y, saved): saved is a uint8 tensor for
    sc_gated_ffn_backward (True: allocate, or a preallocated one), None without."""
    import torch
    L = load()
    call = _Call(stream, x)
    dt, ins = _ffn_inputs(call, desc, x, wg, wu, wd)
    cd = ctypes.byref(desc.c())
    y = torch.empty_like(x) if y is None else y
    ps = None
    if saved is True:
        saved = call.new(torch.uint8, (L.sc_gated_ffn_saved_size(cd),))
        ps = saved.data_ptr()
    elif saved is False or saved is None:
        saved = None
    else:
        ps = _saved(call, saved, L.sc_gated_ffn_saved_size(cd))
    work, wsb, keep = call.workspace(workspace, L.sc_gated_ffn_workspace_size(cd, int(saved is not None)))
    _check(L.sc_gated_ffn(cd, *ins, call.ptr(y, "y", dt, x.shape), ps, work, wsb, call.stream), "sc_gated_ffn")
    return y, saved


@_on_stream
def sc_gated_ffn_backward(desc: FfnDesc, x, wg, wu, wd, saved, dy, grads=None, workspace=None, stream=None):
    """Gradients of sc_gated_ffn from dy = dL/dy and what its forward saved.  Returns a dict of dx, dwg, dwu and dwd.

    grads: optional dict of preallocated outputs; only those it names are computed."""
    L = load()
    call = _Call(stream, x)
    dt, ins = _ffn_inputs(call, desc, x, wg, wu, wd)
    cd = ctypes.byref(desc.c())
    ps = _saved(call, saved, L.sc_gated_ffn_saved_size(cd))
    pdy = call.ptr(dy, "dy", dt, x.shape)
    names = ("dx", "dwg", "dwu", "dwd")
    if grads is not None and set(grads) - set(names):
        raise ValueError(f"grads: unknown outputs {sorted(set(grads) - set(names))}")
    out, outs = {}, []
    for nm, src in zip(names, (x, wg, wu, wd)):
        out[nm] = call.new(dt, src.shape) if grads is None else grads.get(nm)
        outs.append(call.opt(out[nm], nm, dt, src.shape))
    work, wsb, keep = call.workspace(workspace, L.sc_gated_ffn_backward_workspace_size(cd))
    _check(L.sc_gated_ffn_backward(cd, *ins, ps, pdy, *outs, work, wsb, call.stream), "sc_gated_ffn_backward")
    return out


class DropoutDesc:
    """Geometry and rate of a dropout (mirrors sc_dropout_desc).  valid_len: int32 device tensor [B] or None."""

    def __init__(self, B, n, D, p, valid_len=None, site=0, res_scale=1.0, dtype=SC_BF16):
        self.B, self.n, self.D, self.p = int(B), int(n), int(D), float(p)
        self.valid_len = valid_len
        self.site, self.res_scale, self.dtype = int(site), float(res_scale), int(dtype)

    def c(self) -> _DropoutDesc:
        return _DropoutDesc(self.B, self.n, self.D, None if self.valid_len is None else self.valid_len.data_ptr(),
                            self.p, self.res_scale, self.site, self.dtype)


@_on_stream
def sc_dropout(desc: DropoutDesc, x, seed, residual=None, out=None, stream=None):
    """out [B, n, D] = res_scale residual + mask x / (1 - p); seed: int64 device tensor [1].  The gradient of x is the
    same call on the gradient of out, without the residual.  out may be x or residual."""
    import torch
    L = load()
    call = _Call(stream, x)
    shape, dt = (desc.B, desc.n, desc.D), _float_type(desc.dtype, "dtype")
    call.lengths(desc.valid_len, desc.B)
    px, ps = call.ptr(x, "x", dt, shape), call.ptr(seed, "seed", torch.int64, (1,))
    pr = call.opt(residual, "residual", dt, shape)
    out = torch.empty_like(x) if out is None else out
    _check(L.sc_dropout(ctypes.byref(desc.c()), px, ps, pr, call.ptr(out, "out", dt, shape), call.stream), "sc_dropout")
    return out
