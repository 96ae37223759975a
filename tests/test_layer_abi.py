"""Host-side checks of the layer operators (include/sc_layer.h), without a GPU: exported symbols, sizes, frequencies,
the generator's known answers, and the refusal of invalid arguments before anything reaches the device (the addresses
are never dereferenced)."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

import paper_2310_07109_amd as sc
from paper_2310_07109_amd import _binding as B
from test_block_abi import A, Addr
from test_gpu_layer import philox

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "sc_layer.h")

pytestmark = pytest.mark.skipif(not os.path.exists(sc.lib_path()), reason="libsc.so not built")


def libs():
    yield sc.load()
    if os.path.exists(sc.debug_lib_path()):
        yield sc.load_debug()


def test_exports_and_signatures():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(sc_[a-z0-9_]+)\s*\(", text)))
    assert set(names) >= {"sc_rotary", "sc_rotary_backward", "sc_gated_ffn", "sc_gated_ffn_backward", "sc_dropout"}
    for name in names:
        args = re.search(rf"\b{name}\s*\(([^)]*)\)", text).group(1).count(",") + 1
        for L in libs():
            assert len(getattr(L, name).argtypes) == args, name


def test_philox_known_answers():
    """The vectors published with the generator."""
    ones = 0xFFFFFFFF
    for counter, key, want in (
            ((0, 0, 0, 0), (0, 0), "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
            ((ones,) * 4, (ones,) * 2, "408f276d 41c83b0e a20bc7c6 6d5451fd"),
            ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
             "d16cfe09 94fdcceb 5001e420 24126ea1")):
        assert " ".join(f"{int(v):08x}" for v in philox(counter, key)) == want


def test_frequencies():
    f, a = sc.sc_rotary_frequencies(64, base=10000.0)
    i = torch.arange(32, dtype=torch.float64)
    assert a == 1.0 and torch.allclose(f, 10000.0 ** (-2 * i / 64), rtol=1e-14, atol=0)
    assert torch.equal(sc.sc_rotary_frequencies(64, scaling=sc.SC_ROTARY_LINEAR, factor=4.0)[0], f / 4)
    base = 10000.0 * 4.0 ** (64 / 62)
    assert torch.allclose(sc.sc_rotary_frequencies(64, scaling=sc.SC_ROTARY_BASE, factor=4.0)[0],
                          base ** (-2 * i / 64), rtol=1e-13, atol=0)
    assert torch.equal(sc.sc_rotary_frequencies(2, scaling=sc.SC_ROTARY_BASE, factor=4.0)[0], torch.ones(1).double())
    g, a = sc.sc_rotary_frequencies(64, scaling=sc.SC_ROTARY_BANDS, factor=4.0, length=2048, fast=32, slow=1)
    turns = f * 2048 / (2 * math.pi)
    keep = ((turns - 1) / 31).clamp(0, 1)
    assert torch.allclose(g, f * keep + f / 4 * (1 - keep), rtol=1e-13, atol=0)
    assert abs(a - (0.1 * math.log(4) + 1)) < 1e-7 and bool((g[turns > 32] == f[turns > 32]).all())
    for bad in (dict(rot_dim=3), dict(rot_dim=0), dict(base=1.0), dict(base=math.nan), dict(scaling=4),
                dict(scaling=1, factor=0.5), dict(scaling=2, factor=math.inf), dict(scaling=3, factor=2.0),
                dict(scaling=3, factor=2.0, length=8, fast=1.0, slow=1.0), dict(scaling=3, factor=2.0, length=8, slow=-1.0)):
        with pytest.raises(sc.ScError) as e:
            sc.sc_rotary_frequencies(**{"rot_dim": 64, **bad})
        assert e.value.status == B.SC_EINVAL, bad
    with pytest.raises(sc.ScError) as e:
        sc.sc_rotary_frequencies(258)
    assert e.value.status == B.SC_EUNSUPPORTED


FREQ = torch.ones(32, dtype=torch.float64)


def rotary_desc(strides=(256, 128, 128), **kw):
    return sc.RotaryDesc(**{**dict(B=2, n=8, Hq=4, Hk=2), **kw}).c(strides)


@pytest.mark.parametrize("i", [0, 1])
def test_rotary_refusals(i):
    L = list(libs())
    if i >= len(L):
        pytest.skip("libsc_debug.so not built")
    L = L[i]

    def call(freq=FREQ, q=A[0], k=A[1], v=A[2], qw=None, kw_=None, pos=None, qo=A[3], ko=A[4], vo=A[5], patch=None, **kw):
        c = rotary_desc(**kw)
        for name, val in (patch or {}).items():
            setattr(c, name, val)
        return L.sc_rotary(ctypes.byref(c), None if freq is None else freq.data_ptr(), q, k, v, qw, kw_, pos, qo, ko, vo,
                           None)

    inf, nan, far = (torch.full((32,), v, dtype=torch.float64) for v in (math.inf, math.nan, -2.0 ** 20))
    for bad in (dict(B=0), dict(n=0), dict(Hq=-1), dict(d=63), dict(d=0), dict(rot_dim=66), dict(rot_dim=-2),
                dict(rot_dim=3), dict(layout=2), dict(patch=dict(norm=2)), dict(norm=True, kind=2),
                dict(norm=True, eps=0.0), dict(amplitude=math.inf), dict(dtype=2), dict(freq=None), dict(freq=inf),
                dict(freq=nan), dict(freq=far),
                dict(q=None, k=None, v=None, qo=None, ko=None, vo=None), dict(qo=None), dict(q=None), dict(ko=None),
                dict(qw=A[6]), dict(kw_=A[6]), dict(strides=(255, 128, 128)), dict(strides=(256, 128, 127)), dict(Hq=0),
                dict(qo=A[1]), dict(qo=A[0] + 128), dict(ko=A[3] + 64), dict(pos=A[3]),
                dict(strides=(512, 128, 128), qo=A[0])):                # in place needs dense rows
        assert call(**bad) == B.SC_EINVAL, bad
    if i == 0:  # the debug build reads the lengths first
        assert call(vo=A[6], valid_len=Addr(A[6])) == B.SC_EINVAL
    assert call(d=258, rot_dim=64, strides=(4 * 258, 2 * 258, 2 * 258)) == B.SC_EUNSUPPORTED
    assert call(B=1 << 16, n=1 << 15) == B.SC_EUNSUPPORTED
    assert call(Hq=1 << 15, strides=(64 << 15, 128, 128)) == B.SC_EUNSUPPORTED


def test_rotary_backward_refusals():
    L = sc.load()
    W = 512  # fused rows of q | k | v

    def call(freq=FREQ, g=(A[0], A[1], A[2]), q=A[3], k=A[3] + 512, w=(None, None), pos=None,
             o=(A[4], A[4] + 512, A[4] + 768), dw=(None, None), work=A[6], wb=1 << 30, strides=(W, W, W), **kw):
        c = rotary_desc(strides, **{**dict(norm=True), **kw})
        return L.sc_rotary_backward(ctypes.byref(c), freq.data_ptr(), *g, q, k, *w, pos, *o, *dw, work, wb, None)

    for bad in (dict(q=None), dict(k=None), dict(g=(None, A[1], A[2])), dict(o=(A[4], None, A[4] + 768)),
                dict(o=(None,) * 3, g=(None,) * 3), dict(norm=False, dw=(A[7], None)), dict(norm=False, w=(A[7], None)),
                dict(g=(None, A[1], A[2]), o=(None, A[4] + 512, A[4] + 768), dw=(A[7], None)),
                dict(o=(A[4], A[4] + 510, A[4] + 768)),                 # two bytes of q's row
                dict(o=(A[4], A[4] + 512, A[4] + 770)),                 # two bytes of the next row's q
                dict(o=(A[0], A[4] + 512, A[4] + 768)), dict(o=(A[3], A[4] + 512, A[4] + 768)),
                dict(dw=(A[7], A[7])), dict(dw=(A[4], A[7])), dict(dw=(A[7], A[8]), work=A[7]),
                dict(dw=(A[7], A[8]), work=A[6] + 8), dict(strides=(255, W, W))):
        assert call(**bad) == B.SC_EINVAL, bad
    need = sc.sc_rotary_backward_workspace_size(sc.RotaryDesc(2, 8, 4, 2, norm=True))
    assert need > 0 and sc.sc_rotary_backward_workspace_size(sc.RotaryDesc(2, 8, 4, 2)) == 0
    assert call(dw=(A[7], A[8]), work=None) == B.SC_EWORKSPACE
    assert call(dw=(A[7], A[8]), wb=need - 1) == B.SC_EWORKSPACE


def ffn(**kw):
    return sc.FfnDesc(**{**dict(B=2, n=800, D=64, F=96), **kw})


@pytest.mark.parametrize("i", [0, 1])
def test_ffn_refusals(i):
    L = list(libs())
    if i >= len(L):
        pytest.skip("libsc_debug.so not built")
    L = L[i]

    def call(x=A[0], w=(A[1], A[2], A[3]), y=A[4], saved=None, work=A[5], wb=1 << 32, **kw):
        return L.sc_gated_ffn(ctypes.byref(ffn(**kw).c()), x, *w, y, saved, work, wb, None)

    for bad in (dict(B=0), dict(n=0), dict(D=0), dict(F=0), dict(act=3), dict(act=-1), dict(dtype=2), dict(x=None),
                dict(w=(None, A[2], A[3])), dict(w=(A[1], None, A[3])), dict(w=(A[1], A[2], None)), dict(y=None),
                dict(x=A[0] + 8), dict(w=(A[1], A[2] + 2, A[3])), dict(y=A[4] + 4), dict(saved=A[6] + 8),
                dict(work=A[5] + 8), dict(y=A[0]), dict(y=A[1] + 32), dict(saved=A[0]), dict(saved=A[4]),
                dict(work=A[3]), dict(saved=A[6], D=65, work=A[6])):
        assert call(**bad) == B.SC_EINVAL, bad
    for big in (dict(dtype=sc.SC_F32), dict(B=1 << 16, n=1 << 15), dict(D=(1 << 20) + 1), dict(F=(1 << 20) + 1),
                dict(B=1 << 12, n=1 << 12, F=128), dict(B=1 << 12, n=1 << 12, D=121), dict(D=1 << 16, F=1 << 15),
                dict(B=8193, n=1, valid_len=Addr(A[7]))):
        assert call(**big) == B.SC_EUNSUPPORTED, big
    need = sc.sc_gated_ffn_workspace_size(ffn())
    assert need >= 1600 * 96 * 2 and sc.sc_gated_ffn_workspace_size(ffn(), save=True) == 0
    assert call(work=None) == B.SC_EWORKSPACE and call(wb=need - 1) == B.SC_EWORKSPACE
    assert sc.sc_gated_ffn_saved_size(ffn()) >= 1600 * 96 * 8
    assert sc.sc_gated_ffn_saved_size(ffn(F=0)) == 0 == sc.sc_gated_ffn_workspace_size(ffn(F=0))
    assert L.sc_gated_ffn(None, A[0], A[1], A[2], A[3], A[4], None, A[5], 1 << 32, None) == B.SC_EINVAL


def test_ffn_backward_refusals():
    L = sc.load()

    def call(x=A[0], w=(A[1], A[2], A[3]), saved=A[4], dy=A[5], o=(A[6], A[7], A[8], A[9]), work=A[10], wb=1 << 32, **kw):
        return L.sc_gated_ffn_backward(ctypes.byref(ffn(**kw).c()), x, *w, saved, dy, *o, work, wb, None)

    for bad in (dict(saved=None), dict(dy=None), dict(o=(None,) * 4), dict(dy=A[5] + 2), dict(o=(A[6] + 8, None, None, None)),
                dict(o=(A[0], None, None, None)), dict(o=(A[5], None, None, None)), dict(o=(A[6], A[7], A[7] + 64, None)),
                dict(o=(None, None, None, A[3])), dict(work=A[4]), dict(work=A[6]), dict(work=A[10] + 8),
                dict(o=(A[4] + 16, None, None, None))):
        assert call(**bad) == B.SC_EINVAL, bad
    need = sc.sc_gated_ffn_backward_workspace_size(ffn())
    assert need >= 2 * 1600 * 96 * 2
    assert call(work=None) == B.SC_EWORKSPACE and call(wb=need - 1) == B.SC_EWORKSPACE
    assert call(dtype=sc.SC_F32) == B.SC_EUNSUPPORTED


def test_dropout_refusals():
    for L in libs():
        def call(x=A[0], seed=A[1], res=None, out=A[2], **kw):
            d = sc.DropoutDesc(**{**dict(B=2, n=8, D=64, p=0.1), **kw})
            return L.sc_dropout(ctypes.byref(d.c()), x, seed, res, out, None)
        for bad in (dict(B=0), dict(n=0), dict(D=0), dict(p=-0.1), dict(p=1.0), dict(p=65535.5 / 65536), dict(p=math.nan),
                    dict(dtype=2), dict(res_scale=math.inf), dict(x=None), dict(seed=None), dict(seed=A[1] + 4),
                    dict(out=None), dict(out=A[0] + 16), dict(res=A[2] + 2), dict(out=A[1]),
                    dict(valid_len=Addr(A[2] + 4))):
            if L is not sc.load() and "valid_len" in bad:
                continue  # the debug build reads the lengths first
            assert call(**bad) == B.SC_EINVAL, bad
        assert call(B=1 << 16, n=1 << 15) == B.SC_EUNSUPPORTED


def test_binding_refuses_host_and_wrong_tensors():
    x = torch.zeros((2, 8, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU tensor"):
        sc.sc_gated_ffn(ffn(n=8), x, x, x, x)
    with pytest.raises(ValueError, match="GPU tensor"):
        sc.sc_dropout(sc.DropoutDesc(2, 8, 64, 0.1), x, torch.zeros(1, dtype=torch.int64))
    with pytest.raises(TypeError, match="torch.Tensor"):
        sc.sc_rotary(sc.RotaryDesc(2, 8, 1, 1), FREQ, None)


def test_mask_threshold_counts():
    """16 bits an element: a share of t / 65536 is dropped, t the rounded p."""
    r = np.concatenate([np.asarray(v) for v in philox((np.arange(1 << 14), 0 * np.arange(1 << 14), 0 * np.arange(1 << 14),
                                                      0 * np.arange(1 << 14)), (1, 2))])
    r = np.concatenate([r & np.uint64(0xFFFF), r >> np.uint64(16)])
    for p in (0.1, 0.5):
        assert abs(float((r < round(p * 65536)).mean()) - p) < 5 * math.sqrt(p * (1 - p) / len(r))
