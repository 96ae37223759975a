"""Host-side checks of the block operators (include/sc_block.h), without a GPU: exported symbols, sizes, and the
refusal of invalid arguments before anything reaches the device (the addresses are never dereferenced)."""
import ctypes
import os
import re

import pytest
import torch

import paper_2310_07109_amd as sc
from paper_2310_07109_amd import _binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "sc_block.h")

pytestmark = pytest.mark.skipif(not os.path.exists(sc.lib_path()), reason="libsc.so not built")


class Addr:
    """Stands in for a device tensor: only an address."""

    def __init__(self, addr):
        self.addr = addr

    def data_ptr(self):
        return self.addr


A = [0x100000000 * (i + 1) for i in range(24)]  # disjoint fake device buffers


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(sc_[a-z0-9_]+)\s*\(", text)))


def test_exports_and_signatures():
    L = sc.load()
    assert set(declared()) >= {"sc_i8_pitch", "sc_quantize_rows_i8", "sc_quantize_weight_i8", "sc_linear_i8",
                               "sc_block_norm", "sc_block_norm_backward"}
    for name in declared():
        assert getattr(L, name).argtypes is not None, name
    if os.path.exists(sc.debug_lib_path()):
        for name in declared():
            assert hasattr(sc.load_debug(), name), name


def test_pitch():
    assert [sc.sc_i8_pitch(k) for k in (-1, 0, 1, 127, 128, 129, 4096)] == [0, 0, 128, 128, 128, 256, 4096]


@pytest.mark.parametrize("lib", ["release", "debug"])
def test_linear_refusals(lib):
    if lib == "debug" and not os.path.exists(sc.debug_lib_path()):
        pytest.skip("libsc_debug.so not built")
    L = sc.load() if lib == "release" else sc.load_debug()

    def call(x=A[0], xs=None, wq=A[1], ws=A[2], bias=None, out=A[3], work=A[4], wb=1 << 30, **kw):
        a = dict(B=2, n=800, K=100, N=64)
        a.update(kw)
        return L.sc_linear_i8(ctypes.byref(sc.LinearDesc(**a).c()), x, xs, wq, ws, bias, out, work, wb, None)

    for bad in (dict(B=0), dict(n=0), dict(K=0), dict(N=0), dict(x_dtype=3), dict(x_dtype=-1), dict(out_dtype=2),
                dict(act=2), dict(x=None), dict(wq=None), dict(ws=None), dict(out=None),
                dict(xs=A[5]),                                  # a scale with float rows
                dict(x_dtype=sc.SC_I8),                         # 8-bit rows without one
                dict(x_dtype=sc.SC_I8, xs=A[5], x=A[0] + 8),    # 8-bit rows not 16-byte aligned
                dict(wq=A[1] + 8),
                dict(out=A[0] + 64), dict(out=A[1]), dict(out=A[2]), dict(out=A[4] + 256), dict(work=A[0]),
                dict(bias=A[3] + 4)):
        assert call(**bad) == B.SC_EINVAL, bad
    for big in (dict(K=131073), dict(B=1 << 16, n=1 << 15), dict(B=1 << 13, n=1 << 13, K=4096), dict(N=1 << 25, K=129),
                dict(B=8193, n=1, valid_len=Addr(A[6]))):
        assert call(**big) == B.SC_EUNSUPPORTED, big
    need = sc.sc_linear_i8_workspace_size(sc.LinearDesc(2, 800, 100, 64))
    assert need >= 1600 * 128 + 1600 * 4
    assert call(work=None) == B.SC_EWORKSPACE
    assert call(wb=need - 1) == B.SC_EWORKSPACE
    assert sc.sc_linear_i8_workspace_size(sc.LinearDesc(2, 800, 100, 64, x_dtype=sc.SC_I8)) == 0
    assert sc.sc_linear_i8_workspace_size(sc.LinearDesc(0, 800, 100, 64)) == 0
    assert L.sc_linear_i8(None, A[0], None, A[1], A[2], None, A[3], A[4], 1 << 30, None) == B.SC_EINVAL


def test_quantize_refusals():
    L = sc.load()

    def rows(B_=2, n=8, K=100, dt=sc.SC_BF16, x=A[0], q=A[1], s=A[2], length=None):
        return L.sc_quantize_rows_i8(B_, n, K, length, dt, x, q, s, None)

    for bad in (dict(B_=0), dict(n=0), dict(K=0), dict(dt=2), dict(x=None), dict(q=None), dict(s=None),
                dict(q=A[1] + 4), dict(q=A[0]), dict(s=A[0] + 8), dict(s=A[1] + 128), dict(length=A[1])):
        assert rows(**bad) == B.SC_EINVAL, bad
    assert rows(B_=1 << 16, n=1 << 15) == B.SC_EUNSUPPORTED

    def weight(K=100, N=64, dt=sc.SC_F32, w=A[0], q=A[1], s=A[2]):
        return L.sc_quantize_weight_i8(K, N, dt, w, q, s, None)

    for bad in (dict(K=0), dict(N=0), dict(dt=2), dict(w=None), dict(q=None), dict(s=None), dict(q=A[1] + 8),
                dict(q=A[0]), dict(s=A[0]), dict(s=A[1])):
        assert weight(**bad) == B.SC_EINVAL, bad
    assert weight(N=1 << 25, K=129) == B.SC_EUNSUPPORTED


def norm_desc(**kw):
    a = dict(B=2, n=8, D=64)
    a.update(kw)
    return sc.NormDesc(**a)


@pytest.mark.parametrize("lib", ["release", "debug"])
def test_norm_refusals(lib):
    if lib == "debug" and not os.path.exists(sc.debug_lib_path()):
        pytest.skip("libsc_debug.so not built")
    L = sc.load() if lib == "release" else sc.load_debug()

    def call(x=A[0], t=A[1], gate=None, w=(None, None, None, None), r=A[2], y=A[3], yq=None, ys=None, patch=None, **kw):
        c = norm_desc(**kw).c()
        for k, v in (patch or {}).items():
            setattr(c, k, v)
        return L.sc_block_norm(ctypes.byref(c), x, t, gate, *w, r, y, yq, ys, None)

    for bad in (dict(B=0), dict(n=0), dict(D=0), dict(kind=2), dict(patch=dict(post=2)), dict(patch=dict(pre=-1)),
                dict(gate=A[5]), dict(patch=dict(gate_mode=4), gate=A[5]), dict(patch=dict(gate_mode=1)),
                dict(eps=0.0), dict(eps=float("nan")), dict(res_scale=float("inf")), dict(dtype=2), dict(x=None),
                dict(t=None, post=True), dict(t=None, patch=dict(gate_mode=1), gate=A[5]),
                dict(w=(A[6], None, None, None)),               # a weight of the absent norm
                dict(pre=False, y=None, w=(None, None, A[6], None)), dict(pre=False), dict(r=None, y=None),
                dict(yq=A[7]), dict(ys=A[7]), dict(yq=A[7] + 8, ys=A[8]), dict(pre=False, y=None, yq=A[7], ys=A[8]),
                dict(r=A[0] + 64), dict(r=A[1]), dict(y=A[0]), dict(y=A[2] + 16), dict(yq=A[3], ys=A[8]),
                dict(yq=A[7], ys=A[7] + 64), dict(y=A[6], w=(None, None, A[6], None))):
        assert call(**bad) == B.SC_EINVAL, bad
    assert call(D=4097) == B.SC_EUNSUPPORTED
    assert call(B=1 << 16, n=1 << 15) == B.SC_EUNSUPPORTED
    assert L.sc_block_norm(None, A[0], A[1], None, None, None, None, None, A[2], A[3], None, None, None) == B.SC_EINVAL


def test_norm_backward_refusals():
    L = sc.load()

    def call(x=A[0], t=A[1], gate=None, w=(None, None, None, None), dr=A[2], dy=A[3], dx=A[4], dt=A[5], dgate=None,
             dw=(None, None, None, None), work=A[6], wb=1 << 30, patch=None, **kw):
        c = norm_desc(**kw).c()
        for k, v in (patch or {}).items():
            setattr(c, k, v)
        return L.sc_block_norm_backward(ctypes.byref(c), x, t, gate, *w, dr, dy, dx, dt, dgate, *dw, work, wb, None)

    for bad in (dict(dr=None, dy=None), dict(pre=False), dict(dx=None, dt=None), dict(t=None), dict(dgate=A[7]),
                dict(dw=(A[7], None, None, None)), dict(dw=(None, A[7], None, None)),
                dict(pre=False, dy=None, dw=(None, None, A[7], None)), dict(dx=A[0]), dict(dx=A[1]), dict(dx=A[3]),
                dict(dt=A[2]), dict(dt=A[4]), dict(dx=A[2] + 16), dict(work=A[0]), dict(work=A[4]),
                dict(work=A[6] + 4), dict(dw=(None, None, A[7], A[7]))):
        assert call(**bad) == B.SC_EINVAL, bad
    need = sc.sc_block_norm_backward_workspace_size(norm_desc())
    assert need > 0 and sc.sc_block_norm_backward_workspace_size(norm_desc(D=4097)) == 0
    assert call(work=None) == B.SC_EWORKSPACE
    assert call(wb=need - 1) == B.SC_EWORKSPACE
    assert call(D=4097) == B.SC_EUNSUPPORTED


def test_backward_workspace_covers_every_plan():
    """Records of every block for each gate form: never less than 5 sums per block of a row, nor than what a gate by
    sequence adds per sequence."""
    for Bn in ((1, 1), (3, 501), (300, 2), (700, 1), (64, 1024)):
        for gate in range(4):
            d = sc.NormDesc(*Bn, 96, gate=gate)
            blocks = min(512, (Bn[0] * Bn[1] + 3) // 4)
            least = 5 * blocks + (Bn[0] if gate == sc.SC_GATE_SEQUENCE else 0)
            assert sc.sc_block_norm_backward_workspace_size(d) >= 4 * 96 * least


def test_binding_refuses_host_and_wrong_tensors():
    x = torch.zeros((2, 8, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU tensor"):
        sc.sc_block_norm(norm_desc(), x, x)
    with pytest.raises(ValueError, match="GPU tensor"):
        sc.sc_quantize_rows_i8(x)
    with pytest.raises(TypeError, match="torch.Tensor"):
        sc.sc_linear_i8(sc.LinearDesc(2, 8, 64, 64), [1.0], x, x)
    with pytest.raises(ValueError, match="SC_F32 or SC_BF16"):
        sc.sc_block_norm(norm_desc(dtype=sc.SC_I8), x, x)


def stack_desc(**kw):
    a = dict(B=2, n=256, H=2, window=64, valid_len=Addr(A[0]))
    a.update(kw)
    return sc.Desc(**a)


def layer_i8(**kw):
    w = (A[2], A[3], None)
    parts = dict(qkv=w, o=w, w1=w, w2=w)
    parts.update(kw)
    return B._LayerI8(*(B._I8Weight(*parts[k]) for k in ("qkv", "o", "w1", "w2")), *([None] * 6))


def test_stack_i8_refusals():
    L = sc.load()
    th = (ctypes.c_float * 1)(0.0)

    def call(x=A[1], layer=None, layers=True, F=64, th=th, eps=1e-5, scale=1.0, out=A[4], fl=A[5], work=A[6], wb=1 << 32,
             nl=1, windows=None, **kw):
        arr = (B._LayerI8 * 1)(layer or layer_i8()) if layers else None
        return L.sc_encoder_stack_i8(ctypes.byref(stack_desc(**kw).c()), nl, windows, x, arr, F, th, 1,
                                     ctypes.c_float(eps), ctypes.c_float(scale), out, fl, None, None, work, wb, None)

    for bad in (dict(nl=0), dict(F=0), dict(x=None), dict(layers=False), dict(th=None), dict(out=None), dict(fl=None),
                dict(eps=0.0), dict(scale=float("nan")), dict(layer=layer_i8(w2=(None, A[3], None))),
                dict(layer=layer_i8(o=(A[2], None, None))), dict(layer=layer_i8(qkv=(A[2] + 8, A[3], None))),
                dict(windows=(ctypes.c_int32 * 1)(-1)), dict(out=A[1] + 64), dict(work=A[4]), dict(valid_len=None)):
        assert call(**bad) == B.SC_EINVAL, bad
    for big in (dict(dtype=sc.SC_F32), dict(causal=True), dict(B=8193, n=16), dict(H=33), dict(F=131073),
                dict(B=64, n=16384, F=8192)):
        assert call(**big) == B.SC_EUNSUPPORTED, big
    need = sc.sc_encoder_stack_i8_workspace_size(stack_desc(), 1, 64)
    assert need > 0 and sc.sc_encoder_stack_i8_workspace_size(stack_desc(), 1, 0) == 0
    assert call(work=None) == B.SC_EWORKSPACE
    assert call(wb=need - 1) == B.SC_EWORKSPACE


def test_workspace_alignment_and_long_rows_refused():
    """Workspaces that 8-bit rows lie in start at 16 bytes; rows whose byte offsets pass 32 bits are not quantised."""
    L = sc.load()
    d = sc.LinearDesc(2, 800, 100, 64)
    for off, want in ((4, B.SC_EINVAL), (8, B.SC_EINVAL)):
        assert L.sc_linear_i8(ctypes.byref(d.c()), A[0], None, A[1], A[2], None, A[3], A[4] + off, 1 << 30,
                              None) == want, off
        arr = (B._LayerI8 * 1)(layer_i8())
        assert L.sc_encoder_stack_i8(ctypes.byref(stack_desc().c()), 1, None, A[1], arr, 64, (ctypes.c_float * 1)(0.0),
                                     1, ctypes.c_float(1e-5), ctypes.c_float(1.0), A[4], A[5], None, None, A[6] + off,
                                     1 << 32, None) == want, off
    for K in (1 << 29, (1 << 31) - 129):
        for dt in (sc.SC_F32, sc.SC_BF16):
            assert L.sc_quantize_rows_i8(1, 1, K, None, dt, A[0], A[8], A[16], None) == B.SC_EUNSUPPORTED, (K, dt)


@pytest.mark.parametrize("x_dtype,n,K,N,one_launch", [
    (sc.SC_BF16, 128, 768, 2304, True), (sc.SC_BF16, 128, 2304, 768, True), (sc.SC_BF16, 192, 2304, 768, False),
    (sc.SC_BF16, 64, 767, 768, True), (sc.SC_BF16, 96, 767, 768, False),        # an element a load
    (sc.SC_BF16, 64, 2303, 768, True), (sc.SC_BF16, 96, 2303, 768, False), (sc.SC_BF16, 32, 4095, 4096, False),
    (sc.SC_F32, 48, 1023, 4096, True), (sc.SC_F32, 64, 1023, 4096, False),
    (sc.SC_F32, 64, 4095, 1024, True), (sc.SC_F32, 96, 4095, 1024, False)])
def test_rows_quantised_in_the_products_launch(x_dtype, n, K, N, one_launch):
    """Where every workgroup quantises its rows for itself no rows are kept in a workspace: as long as that is faster for
    rows of the type and length."""
    assert (sc.sc_linear_i8_workspace_size(sc.LinearDesc(1, n, K, N, x_dtype=x_dtype)) == 0) == one_launch


@pytest.mark.parametrize("K", [1 << 29, (1 << 31) - 129, (1 << 31) - 128, (1 << 31) - 1])
def test_quantisation_refuses_long_rows_alike(K):
    """K >= 2^29 is unsupported, of rows and of weights, up to the largest int32; invalid arguments come first."""
    L = sc.load()
    far = [i << 44 for i in range(1, 5)]  # disjoint whatever K
    for dt in (sc.SC_F32, sc.SC_BF16):
        assert L.sc_quantize_rows_i8(1, 1, K, None, dt, far[0], far[1], far[2], None) == B.SC_EUNSUPPORTED
        assert L.sc_quantize_weight_i8(K, 1, dt, far[0], far[1], far[2], None) == B.SC_EUNSUPPORTED
    assert L.sc_quantize_rows_i8(1, 1, K, None, 7, far[0], far[1], far[2], None) == B.SC_EINVAL
    assert L.sc_quantize_weight_i8(K, 1, sc.SC_F32, None, far[1], far[2], None) == B.SC_EINVAL


def test_stream_given_by_position(monkeypatch):
    """A wrapper allocates its outputs and workspaces on the stream that it is given, however it is given."""
    import contextlib
    current = [None]

    @contextlib.contextmanager
    def on(stream):
        before, current[0] = current[0], stream
        yield
        current[0] = before
    monkeypatch.setattr(torch.cuda, "stream", on)

    @B._on_stream
    def wrapper(x, out=None, stream=None):
        return x, out, stream, current[0]
    assert wrapper(1, 2, "s") == (1, 2, "s", "s") == wrapper(1, 2, stream="s")
    assert wrapper(1, stream=None) == (1, None, None, None) == wrapper(1, None, None)
    assert current[0] is None
