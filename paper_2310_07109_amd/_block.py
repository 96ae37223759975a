"""ctypes binding of the block operators of libsc.so (include/sc_block.h; argument marshalling only)."""
from __future__ import annotations

import ctypes

from ._binding import (SC_ACT_NONE, SC_BF16, SC_F32, SC_GATE_CHANNEL, SC_GATE_NONE, SC_GATE_SEQUENCE, SC_I8,
                       SC_NORM_LAYER, _check, _I8Weight, _LayerI8, _LinearDesc, _min_bytes, _NormDesc, _on_stream,
                       _opt, _ptr, _stream, _tensor, _ws, load)


class _Call:
    """Checks the tensors of one call and gives their addresses.  The checks are _tensor's, and that every tensor lies
    on the device of the call's stream; the common case is settled by comparisons alone, since the smallest calls cost
    less on the GPU than their marshalling does on the host (a norm of one row: 18 us a call with _tensor for each, 12
    so, 4 of it the launch)."""

    def __init__(self, stream, x):
        import torch
        if not (isinstance(x, torch.Tensor) and x.is_cuda):
            _tensor(x, "x")  # raises
        self.device = torch.cuda.current_device() if stream is None else stream.device_index
        self.stream = torch._C._cuda_getCurrentRawStream(self.device) if stream is None else stream.cuda_stream

    def ptr(self, t, name, dtype, shape):
        """Address of a required tensor."""
        try:
            if t.dtype is dtype and t.shape == shape and t.get_device() == self.device and t.is_contiguous():
                return t.data_ptr()
        except AttributeError:
            pass
        _tensor(t, name, dtype, shape)
        raise ValueError(f"{name}: on {t.device}, the call's stream on device {self.device}")

    def opt(self, t, name, dtype, shape):
        """Address of an optional tensor."""
        return None if t is None else self.ptr(t, name, dtype, shape)

    def lengths(self, valid_len, B):
        import torch
        return None if valid_len is None else self.ptr(valid_len, "valid_len", torch.int32, (B,))

    def workspace(self, t, nbytes):
        """(address, bytes, tensor) of the given workspace or of a new one; the tensor is kept by the caller until the
        call is enqueued."""
        import torch
        if t is None:
            if nbytes == 0:
                return None, 0, None
            t = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            return t.data_ptr(), nbytes, t
        _tensor(t, "workspace")
        return self.ptr(t, "workspace", t.dtype, t.shape), t.numel() * t.element_size(), t

    def new(self, dtype, shape):
        import torch
        return torch.empty(shape, dtype=dtype, device=self.device)


def _float_type(code, what):
    import torch
    if code not in (SC_F32, SC_BF16):
        raise ValueError(f"{what}: expected SC_F32 or SC_BF16, got {code}")
    return torch.float32 if code == SC_F32 else torch.bfloat16


def _code(t, name):
    import torch
    if t.dtype == torch.float32:
        return SC_F32
    if t.dtype == torch.bfloat16:
        return SC_BF16
    raise TypeError(f"{name}: expected torch.float32 or torch.bfloat16, got {t.dtype}")


def sc_i8_pitch(K: int) -> int:
    """Bytes of a row of K 8-bit values."""
    return load().sc_i8_pitch(int(K))


@_on_stream
def sc_quantize_rows_i8(x, valid_len=None, xq=None, scale=None, stream=None):
    """8-bit rows of x [B, n, K] (float32 or bf16).  Returns (xq int8 [B, n, pitch], scale float32 [B, n])."""
    import torch
    L = load()
    call = _Call(stream, x)
    code = _code(x, "x")
    B, n, K = x.shape
    shape = (B, n, L.sc_i8_pitch(K))
    xq = call.new(torch.int8, shape) if xq is None else xq
    scale = call.new(torch.float32, (B, n)) if scale is None else scale
    _check(L.sc_quantize_rows_i8(B, n, K, call.lengths(valid_len, B), code, call.ptr(x, "x", x.dtype, x.shape),
                                 call.ptr(xq, "xq", torch.int8, shape),
                                 call.ptr(scale, "scale", torch.float32, (B, n)), call.stream), "sc_quantize_rows_i8")
    return xq, scale


@_on_stream
def sc_quantize_weight_i8(w, wq=None, scale=None, stream=None):
    """8-bit weights of w [K, N] (float32 or bf16).  Returns (wq int8 [N, pitch(K)], scale float32 [N])."""
    import torch
    L = load()
    call = _Call(stream, w)
    code = _code(w, "w")
    K, N = w.shape
    shape = (N, L.sc_i8_pitch(K))
    wq = call.new(torch.int8, shape) if wq is None else wq
    scale = call.new(torch.float32, (N,)) if scale is None else scale
    _check(L.sc_quantize_weight_i8(K, N, code, call.ptr(w, "w", w.dtype, w.shape),
                                   call.ptr(wq, "wq", torch.int8, shape),
                                   call.ptr(scale, "scale", torch.float32, (N,)), call.stream),
           "sc_quantize_weight_i8")
    return wq, scale


class LinearDesc:
    """Geometry and types of an 8-bit product (mirrors sc_linear_desc).  valid_len: int32 device tensor [B] or
    None."""

    def __init__(self, B, n, K, N, valid_len=None, x_dtype=SC_BF16, out_dtype=SC_BF16, act=SC_ACT_NONE):
        self.B, self.n, self.K, self.N = int(B), int(n), int(K), int(N)
        self.valid_len = valid_len
        self.x_dtype, self.out_dtype, self.act = int(x_dtype), int(out_dtype), int(act)

    def c(self) -> _LinearDesc:
        return _LinearDesc(self.B, self.n, self.K, self.N,
                           None if self.valid_len is None else self.valid_len.data_ptr(), self.x_dtype,
                           self.out_dtype, self.act)


def sc_linear_i8_workspace_size(desc: LinearDesc) -> int:
    return load().sc_linear_i8_workspace_size(ctypes.byref(desc.c()))


@_on_stream
def sc_linear_i8(desc: LinearDesc, x, wq, w_scale, bias=None, x_scale=None, out=None, workspace=None, stream=None):
    """out [B, n, N] = act(x . W + bias).  x: [B, n, K] float, or 8-bit rows [B, n, pitch(K)] with x_scale [B, n];
    wq, w_scale: as sc_quantize_weight_i8 returns them."""
    import torch
    L = load()
    call = _Call(stream, x)
    B, n, K, N = desc.B, desc.n, desc.K, desc.N
    pitch = L.sc_i8_pitch(K)
    if desc.x_dtype == SC_I8:
        px = call.ptr(x, "x", torch.int8, (B, n, pitch))
        ps = call.ptr(x_scale, "x_scale", torch.float32, (B, n))
    else:
        px, ps = call.ptr(x, "x", _float_type(desc.x_dtype, "x_dtype"), (B, n, K)), None
        if x_scale is not None:
            raise ValueError("x_scale: only with 8-bit rows")
    pw = call.ptr(wq, "wq", torch.int8, (N, pitch))
    pws = call.ptr(w_scale, "w_scale", torch.float32, (N,))
    pb = call.opt(bias, "bias", torch.float32, (N,))
    call.lengths(desc.valid_len, B)
    dt = _float_type(desc.out_dtype, "out_dtype")
    out = call.new(dt, (B, n, N)) if out is None else out
    po = call.ptr(out, "out", dt, (B, n, N))
    cd = ctypes.byref(desc.c())
    work, wsb, keep = call.workspace(workspace, L.sc_linear_i8_workspace_size(cd))
    _check(L.sc_linear_i8(cd, px, ps, pw, pws, pb, po, work, wsb, call.stream), "sc_linear_i8")
    return out


class NormDesc:
    """Geometry and form of the norms around a block (mirrors sc_norm_desc).  valid_len: int32 device tensor [B]
    or None."""

    def __init__(self, B, n, D, valid_len=None, kind=SC_NORM_LAYER, post=False, pre=True, gate=SC_GATE_NONE, eps=1e-5,
                 res_scale=1.0, dtype=SC_BF16):
        self.B, self.n, self.D = int(B), int(n), int(D)
        self.valid_len = valid_len
        self.kind, self.post, self.pre, self.gate = int(kind), int(bool(post)), int(bool(pre)), int(gate)
        self.eps, self.res_scale, self.dtype = float(eps), float(res_scale), int(dtype)

    def c(self) -> _NormDesc:
        return _NormDesc(self.B, self.n, self.D, None if self.valid_len is None else self.valid_len.data_ptr(),
                         self.kind, self.post, self.pre, self.gate, self.eps, self.res_scale, self.dtype)

    def gate_form(self):
        """(shape, dtype) of the gate."""
        import torch
        if self.gate == SC_GATE_CHANNEL:
            return (self.D,), torch.float32
        return ((self.B, self.D) if self.gate == SC_GATE_SEQUENCE else (self.B, self.n, self.D)), \
            _float_type(self.dtype, "dtype")


def _norm_inputs(stream, desc, x, t, gate, post_w, post_b, pre_w, pre_b):
    """(call, shape, dtype, addresses) of what both directions read."""
    import torch
    shape, dt = (desc.B, desc.n, desc.D), _float_type(desc.dtype, "dtype")
    call = _Call(stream, x)
    call.lengths(desc.valid_len, desc.B)
    gs, gt = desc.gate_form() if gate is not None else (None, None)
    vec, f32 = (desc.D,), torch.float32
    return call, shape, dt, (call.ptr(x, "x", dt, shape), call.opt(t, "t", dt, shape), call.opt(gate, "gate", gt, gs),
                       call.opt(post_w, "post_w", f32, vec), call.opt(post_b, "post_b", f32, vec),
                       call.opt(pre_w, "pre_w", f32, vec), call.opt(pre_b, "pre_b", f32, vec))


@_on_stream
def sc_block_norm(desc: NormDesc, x, t=None, gate=None, post_w=None, post_b=None, pre_w=None, pre_b=None, r=True,
                  y=True, quantized=False, stream=None):
    """r = res_scale x + gate post(t), y = pre(r).  Returns (r, y, yq, yscale); absent outputs are None.

    r / y: True (allocate), False (skip) or a preallocated tensor (r may be x); quantized: True, False or (yq,
    yscale).  Without desc.pre, y is skipped."""
    import torch
    L = load()
    call, shape, dt, ins = _norm_inputs(stream, desc, x, t, gate, post_w, post_b, pre_w, pre_b)
    r = _opt(r, lambda: torch.empty_like(x))
    y = _opt(y, lambda: torch.empty_like(x)) if desc.pre or y is not True else None
    yq = ys = pq = ps = None
    if quantized:
        qshape = (desc.B, desc.n, L.sc_i8_pitch(desc.D))
        yq, ys = (call.new(torch.int8, qshape), call.new(torch.float32, shape[:2])) if quantized is True else quantized
        pq, ps = call.ptr(yq, "yq", torch.int8, qshape), call.ptr(ys, "yscale", torch.float32, shape[:2])
    _check(L.sc_block_norm(ctypes.byref(desc.c()), *ins, call.opt(r, "r", dt, shape), call.opt(y, "y", dt, shape), pq,
                           ps, call.stream), "sc_block_norm")
    return r, y, yq, ys


def sc_block_norm_backward_workspace_size(desc: NormDesc) -> int:
    return load().sc_block_norm_backward_workspace_size(ctypes.byref(desc.c()))


@_on_stream
def sc_block_norm_backward(desc: NormDesc, x, t=None, gate=None, post_w=None, post_b=None, pre_w=None, pre_b=None,
                           dr=None, dy=None, grads=None, workspace=None, stream=None):
    """Gradients of sc_block_norm from dr = dL/dr and dy = dL/dy.  Returns a dict of dx, dt, dgate, dpost_w,
    dpost_b, dpre_w and dpre_b, None for what is absent: a weight that was not given has no gradient.

    grads: optional dict of preallocated outputs; only those it names are computed."""
    import torch
    L = load()
    call, shape, dt, ins = _norm_inputs(stream, desc, x, t, gate, post_w, post_b, pre_w, pre_b)
    pr, py = call.opt(dr, "dr", dt, shape), call.opt(dy, "dy", dt, shape)
    gs, gt = desc.gate_form() if gate is not None else (None, None)
    vec, f32 = (desc.D,), torch.float32
    forms = (("dx", x, dt, shape), ("dt", t, dt, shape), ("dgate", gate, gt, gs), ("dpost_w", post_w, f32, vec),
             ("dpost_b", post_b, f32, vec), ("dpre_w", pre_w, f32, vec), ("dpre_b", pre_b, f32, vec))
    out, outs = {}, []
    if grads is not None:
        unknown = set(grads) - {f[0] for f in forms}
        if unknown:
            raise ValueError(f"grads: unknown outputs {sorted(unknown)}")
        if gate is None and grads.get("dgate") is not None:
            raise ValueError("dgate: there is no gate")
    for nm, src, ty, s in forms:
        if grads is not None:
            g = grads.get(nm)
            outs.append(call.opt(g, nm, ty, s))
        elif src is None:
            g = None
            outs.append(None)
        else:
            g = torch.empty_like(src)  # of that type and shape
            outs.append(g.data_ptr())
        out[nm] = g
    cd = ctypes.byref(desc.c())
    work, wsb, keep = call.workspace(workspace, L.sc_block_norm_backward_workspace_size(cd))
    _check(L.sc_block_norm_backward(cd, *ins, pr, py, *outs, work, wsb, call.stream), "sc_block_norm_backward")
    return out


class LayerI8:
    """One layer of sc_encoder_stack_i8 (mirrors sc_layer_i8).  qkv, o, w1, w2: (wq, scale) or (wq, scale, bias) with
    wq, scale as sc_quantize_weight_i8 returns them; the rest float32 [D] or None."""

    def __init__(self, qkv, o, w1, w2, gate1=None, ln1_w=None, ln1_b=None, gate2=None, ln2_w=None, ln2_b=None):
        self.products = {nm: tuple(w) + (None,) * (3 - len(w)) for nm, w in
                         (("qkv", qkv), ("o", o), ("w1", w1), ("w2", w2))}
        self.vectors = dict(gate1=gate1, ln1_w=ln1_w, ln1_b=ln1_b, gate2=gate2, ln2_w=ln2_w, ln2_b=ln2_b)

    def tensors(self):
        return [t for w in self.products.values() for t in w] + list(self.vectors.values())

    def check(self, where, D, F):
        import torch
        L = load()
        for nm, K, N in (("qkv", D, 3 * D), ("o", D, D), ("w1", D, F), ("w2", F, D)):
            wq, scale, bias = self.products[nm]
            _tensor(wq, f"{where}.{nm}", torch.int8, (N, L.sc_i8_pitch(K)))
            _tensor(scale, f"{where}.{nm} scale", torch.float32, (N,))
            if bias is not None:
                _tensor(bias, f"{where}.{nm} bias", torch.float32, (N,))
        for nm, t in self.vectors.items():
            if t is not None:
                _tensor(t, f"{where}.{nm}", torch.float32, (D,))

    def c(self) -> _LayerI8:
        addr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        return _LayerI8(*(_I8Weight(*map(addr, w)) for w in self.products.values()), *map(addr, self.vectors.values()))


def sc_encoder_stack_i8_workspace_size(desc, n_layers: int, ffn_dim: int) -> int:
    return load().sc_encoder_stack_i8_workspace_size(ctypes.byref(desc.c()), int(n_layers), int(ffn_dim))


@_on_stream
def sc_encoder_stack_i8(desc, x_in, layers, ffn_dim, thresholds, windows=None, keep_global=True, ln_eps=1e-5,
                        res_scale=1.0, x_out=None, workspace=None, stream=None):
    """The encoder stack on 8-bit products (layers: a list of LayerI8).  Returns (x_out, final_len, orig_idx,
    kept_per_layer)."""
    import torch
    L = load()
    cd = desc.c()
    nl, B, n, D, F = len(layers), desc.B, desc.n, desc.H * desc.d, int(ffn_dim)
    _tensor(x_in, "x_in", torch.bfloat16, (B, n, D))
    if x_out is not None:
        _tensor(x_out, "x_out", torch.bfloat16, (B, n, D))
    if len(thresholds) != nl or (windows is not None and len(windows) != nl):
        raise ValueError("thresholds and windows: one per layer")
    for i, y in enumerate(layers):
        y.check(f"layers[{i}]", D, F)
    call = _Call(stream, x_in)
    call.lengths(desc.valid_len, B)
    call.opt(desc.global_pos, "global_pos", torch.int32, (B, desc.G))
    for t in (x_in, x_out, workspace, *(t for y in layers for t in y.tensors())):
        call.opt(t, "argument", t if t is None else t.dtype, t if t is None else t.shape)
    dev = x_in.device
    x_out = torch.empty_like(x_in) if x_out is None else x_out
    i32 = dict(dtype=torch.int32, device=dev)
    final_len, orig, kpl = torch.empty((B,), **i32), torch.empty((B, n), **i32), torch.empty((nl, B), **i32)
    th = (ctypes.c_float * nl)(*[float(t) for t in thresholds])
    win = None if windows is None else (ctypes.c_int32 * nl)(*[int(w) for w in windows])
    wsb = L.sc_encoder_stack_i8_workspace_size(ctypes.byref(cd), nl, F)
    ws = _ws(wsb, dev) if workspace is None else _min_bytes(_tensor(workspace, "workspace"), "workspace", wsb)
    _check(L.sc_encoder_stack_i8(ctypes.byref(cd), nl, win, _ptr(x_in), (_LayerI8 * nl)(*(y.c() for y in layers)), F,
                                 th, int(bool(keep_global)), ctypes.c_float(ln_eps), ctypes.c_float(res_scale),
                                 _ptr(x_out), _ptr(final_len), _ptr(orig), _ptr(kpl), _ptr(ws), wsb,
                                 _stream(stream)), "sc_encoder_stack_i8")
    return x_out, final_len, orig, kpl
