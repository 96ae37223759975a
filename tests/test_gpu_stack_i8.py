"""sc_encoder_stack_i8 against the same layers composed of the public operators (each tested against its own plain
form): every step is deterministic and a row depends on itself alone, so the results are the same bits."""
import math

import pytest
import torch

import paper_2310_07109_amd as sc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(B, n, H, F, layers, seed, extras=True):
    g = torch.Generator()
    g.manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g).to(DEV)  # noqa: E731
    D = H * 64

    def weight(K, N, bias):
        return (*sc.sc_quantize_weight_i8(rnd(K, N) * 0.7 / math.sqrt(K)), 0.1 * rnd(N) if bias else None)
    out = []
    for _ in range(layers):
        v = {}
        if extras:
            v = {k: (0.8 if "gate" in k else 1.0) + 0.1 * rnd(D) if k[-1] != "b" else 0.1 * rnd(D)
                 for k in ("gate1", "ln1_w", "ln1_b", "gate2", "ln2_w", "ln2_b")}
        out.append(sc.LayerI8(weight(D, 3 * D, extras), weight(D, D, extras), weight(D, F, extras),
                              weight(F, D, extras), **v))
    return rnd(B, n, D).to(torch.bfloat16), out


def composed(x, vl, gp, layers, H, F, thetas, windows, res_scale):
    B, n, D = x.shape
    orig = None
    for y, theta, win in zip(layers, thetas, windows):
        d = sc.Desc(B, n, H, win, vl, gp)
        lin = lambda v, w, N, length, act=sc.SC_ACT_NONE: sc.sc_linear_i8(  # noqa: E731
            sc.LinearDesc(B, n, v.shape[-1], N, length, act=act), v, *w)
        qkv = lin(x, y.products["qkv"], 3 * D, vl)
        q, k, v = (t.contiguous().view(B, n, H, 64) for t in qkv.split(D, dim=2))
        o, _, sp, _ = sc.sc_window_attention(d, q, k, v)
        _, nl, ngp, orig, (ok, xk) = sc.sc_ltp_prune_compact(d, sc.sc_ltp_score(d, sp), theta, True,
                                                             [o.view(B, n, D), x], orig_idx_in=orig,
                                                             dsts=[torch.zeros_like(x), torch.zeros_like(x)])

        def norm(res, t, gate, w, b):
            c = sc.NormDesc(B, n, D, nl, gate=sc.SC_GATE_NONE if gate is None else sc.SC_GATE_CHANNEL, res_scale=res_scale)
            return sc.sc_block_norm(c, res, t, gate=gate, pre_w=w, pre_b=b, r=False)[1]
        e = y.vectors
        x1 = norm(xk, lin(ok, y.products["o"], D, nl), e["gate1"], e["ln1_w"], e["ln1_b"])
        h = lin(x1, y.products["w1"], F, nl, sc.SC_ACT_GELU)
        x = norm(x1, lin(h, y.products["w2"], D, nl), e["gate2"], e["ln2_w"], e["ln2_b"])
        vl, gp = nl, ngp
    return x, vl, orig


@pytest.mark.parametrize("B,n,H,F,lens,glob,thetas,windows,extras,scale", [
    (3, 130, 2, 200, (130, 1, 77), 1, (0.0, 0.007, 0.012), (32, 64, 128), True, 1.3),
    (2, 300, 4, 1024, (300, 0), 0, (0.002, 0.003), (64, 64), False, 1.0),
    (5, 1000, 3, 768, (1000, 999, 512, 3, 700), 3, (0.0, 0.0008), (256, 1000), True, 0.9),
])
def test_stack_is_its_operators(B, n, H, F, lens, glob, thetas, windows, extras, scale):
    x, layers = make(B, n, H, F, len(thetas), seed=n, extras=extras)
    vl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    gp = None
    if glob:  # the first tokens; shorter sequences have unused slots
        gp = torch.arange(glob, device=DEV).expand(B, glob)
        gp = torch.where(gp < vl[:, None], gp, -1).to(torch.int32).contiguous()
    d = sc.Desc(B, n, H, windows[0], vl, gp)
    y = torch.full_like(x, 7.0)  # rows beyond the survivors stay as they are
    _, fl, orig, kept = sc.sc_encoder_stack_i8(d, x, layers, F, thetas, windows=windows, res_scale=scale, x_out=y)
    want, wl, worig = composed(x, vl, gp, layers, H, F, thetas, windows, scale)
    assert torch.equal(fl, wl) and torch.equal(kept[-1], wl) and torch.equal(orig, worig)
    assert (fl <= vl).all() and 0 < int(fl.sum()) < int(vl.sum())
    for b in range(B):
        assert torch.equal(y[b, : fl[b]], want[b, : fl[b]]), b
        assert (y[b, fl[b]:] == 7).all()


def test_stack_i8_close_to_bf16_stack():
    """The same random layers in 8 bits and in bf16, nothing pruned: rows keep their direction (cosine above 0.99; two
    8-bit roundings per product leave about 1 % of a row's norm, six products deep)."""
    B, n, H, F, nl = 2, 200, 4, 512, 3
    D = H * 64
    g = torch.Generator()
    g.manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g).to(DEV)  # noqa: E731
    x = rnd(B, n, D).to(torch.bfloat16)
    w = [[(rnd(K, N) * 0.7 / math.sqrt(K)).to(torch.bfloat16) for K, N in ((D, 3 * D), (D, D), (D, F), (F, D))]
         for _ in range(nl)]
    vl = torch.tensor([200, 150], dtype=torch.int32, device=DEV)
    d = sc.Desc(B, n, H, 64, vl)
    y, fl, _, _ = sc.sc_encoder_stack(d, x, *([u[i] for u in w] for i in range(4)), [-1.0] * nl)
    layers = [sc.LayerI8(*(sc.sc_quantize_weight_i8(u) for u in v)) for v in w]
    y8, fl8, _, _ = sc.sc_encoder_stack_i8(d, x, layers, F, [-1.0] * nl)
    assert torch.equal(fl, vl) and torch.equal(fl8, vl)
    for b in range(B):
        cos = torch.nn.functional.cosine_similarity(y[b, : vl[b]].float(), y8[b, : vl[b]].float(), dim=-1)
        assert cos.min() > 0.99, float(cos.min())


def test_stack_i8_captured():
    """Captured once, replayed three times between other work: the eager bits."""
    B, n, H, F = 3, 130, 2, 200
    x, layers = make(B, n, H, F, 2, seed=3)
    vl = torch.tensor([130, 1, 77], dtype=torch.int32, device=DEV)
    d = sc.Desc(B, n, H, 64, vl, torch.zeros((B, 1), dtype=torch.int32, device=DEV))
    ws = torch.empty(sc.sc_encoder_stack_i8_workspace_size(d, 2, F), dtype=torch.uint8, device=DEV)
    step = lambda w: sc.sc_encoder_stack_i8(d, x, layers, F, [0.0, 0.008], workspace=w, x_out=torch.zeros_like(x))  # noqa: E731
    want = [t.clone() for t in step(None)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(ws)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(ws)
    for _ in range(3):
        for o in outs:
            o.fill_(-3)
        ws.fill_(85)
        step(None)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_stack_i8_binding_refusals():
    """Tensors of another type, shape or place never reach the library."""
    B, n, H, F = 2, 64, 2, 200
    x, layers = make(B, n, H, F, 1, seed=5)
    vl = torch.tensor([64, 7], dtype=torch.int32, device=DEV)
    gp = torch.zeros((B, 1), dtype=torch.int32, device=DEV)

    def call(x=x, vl=vl, gp=gp, layers=layers, F=F, th=(0.0,), **kw):
        return sc.sc_encoder_stack_i8(sc.Desc(B, n, H, 32, vl, gp), x, layers, F, th, **kw)
    call()
    q, s, b = layers[0].products["qkv"]
    with_qkv = lambda *w: [sc.LayerI8(w, *(layers[0].products[k] for k in ("o", "w1", "w2")))]  # noqa: E731
    for bad in (dict(vl=vl.long()), dict(vl=vl[:1]), dict(vl=vl.cpu()), dict(gp=gp.long()), dict(gp=gp[:1]),
                dict(x=x.float()), dict(x=x[:, :63]), dict(x=x.cpu()), dict(F=F + 1), dict(th=(0.0, 0.0)),
                dict(layers=with_qkv(q.t(), s, b)), dict(layers=with_qkv(q, s[1:], b)), dict(layers=with_qkv(q, s.half(), b)),
                dict(layers=with_qkv(q, s, b.cpu())), dict(x_out=x[:1]), dict(windows=[32, 32]),
                dict(workspace=torch.empty(16, dtype=torch.uint8, device=DEV))):
        with pytest.raises((TypeError, ValueError)):
            call(**bad)


def test_stack_with_an_odd_feed_forward_width():
    """512 rows of 777 values: beyond the one-launch form of bf16 rows of odd length, within that of 8-bit rows."""
    test_stack_is_its_operators(2, 256, 4, 777, (256, 201), 0, (0.003, 0.004), (64, 64), True, 1.0)
