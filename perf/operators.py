"""Performance cases of the encoder block's operators: 8-bit integer products and block norms.

  linear         out = act((x . W) + bias) with x quantised per token (in the call, or before it where x comes as int8)
                 and W per output channel, sums in whole numbers;
  norm           r = res_scale * x + gate * post(t), y = pre(r): the norms after and before a block with the block's
                 gate and the residual's scale;
  norm_backward  the gradients of x, t, the gate and both norms' weights.

A batch is padded: sequence b holds lens[b] of n rows, the outputs of the others are zero.  Sizes: hidden sizes of
encoders (64 per head, 8 to 16 heads), their fused q|k|v and feed-forward widths, and odd ones; batches from one row to
the largest of the framework's own encoder benchmark (16 files of 2048 tokens).
"""
import math
import statistics

import torch

own = False

EPS = 1e-5
PITCH = 128  # rows of 8-bit values are padded with zeros to a multiple of this


# ------------------------------------------------------------------ cases ----
def _linear(name, B, n, K, N, lens="full", x="bf16", out="bf16", gelu=False, bias=True):
    c = dict(op="linear", B=B, n=n, K=K, N=N, lens=lens, x=x, out=out, gelu=gelu, bias=bias)
    return dict(c, name=name) if name else c


def _norm(name, B, n, D, lens="full", dtype="bf16", kind="layer", gate="none", post=False, pre=True, scale=1.0, r=True,
          backward=False):
    c = dict(op="norm_backward" if backward else "norm", B=B, n=n, D=D, lens=lens, dtype=dtype, kind=kind, gate=gate,
             post=post, pre=pre, scale=scale, r=r)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One token through a fused q|k|v projection: latency.
        _linear("linear-b1-n1-k512-n1536", 1, 1, 512, 1536),
        # What a pruned layer leaves of a batch: a few rows of each of 16 files, widening with GELU.
        _linear("linear-b16-n8-k768-n2304-gelu", 16, 8, 768, 2304, lens="ragged", gelu=True),
        # Odd sizes everywhere, float32 in and out.
        _linear("linear-f32-b3-n501-k500-n1111", 3, 501, 500, 1111, lens="ragged", x="f32", out="f32"),
        # A batch of files of the usual length distribution, much padding; the output projection.
        _linear("linear-b64-n1024-k768-n768-lognormal", 64, 1024, 768, 768, lens="lognormal"),
        # The largest: long files through the widening product with GELU, and the narrowing one, whose input comes
        # quantised from the operator before it.
        _linear("linear-b16-n2048-k1024-n4096-gelu", 16, 2048, 1024, 4096, gelu=True),
        _linear("linear-i8-b16-n2048-k4096-n1024", 16, 2048, 4096, 1024, x="i8"),
        # One token between two blocks (sandwich norm): latency.
        _norm("norm-b1-n1-d512-sandwich", 1, 1, 512, kind="rms", post=True),
        # The residual LayerNorm of a post-norm encoder, files of the usual lengths.
        _norm("norm-b64-n1024-d768-lognormal", 64, 1024, 768, lens="lognormal", scale=1.5, r=False),
        # Long files, norms on both sides, a gate for every channel of each file.
        _norm("norm-b16-n2048-d1024-gated", 16, 2048, 1024, post=True, gate="sequence"),
        # Odd sizes in float32, gated per channel: forward's and backward's ragged ends.
        _norm("norm-backward-f32-b3-n501-d1111", 3, 501, 1111, lens="ragged", dtype="f32", gate="channel", post=True,
              backward=True),
        # Training: a post-norm block of a usual batch, and a gated one with norms on both sides of long files.
        _norm("norm-backward-b16-n512-d768", 16, 512, 768, lens="ragged", scale=1.5, r=False, backward=True),
        _norm("norm-backward-b16-n2048-d1024-gated", 16, 2048, 1024, kind="rms", post=True, gate="sequence",
              backward=True),
    ]


def _size(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _batch(rng, most):
    B = _size(rng, 1, min(64, most))
    return B, _size(rng, 1, min(2048, most // B))


def draw(rng):
    op = rng.choice(("linear", "linear", "norm", "norm_backward"))
    lens = rng.choice(("full", "ragged", "ragged", "lognormal"))
    if op == "linear":
        out = rng.choice(("bf16", "bf16", "f32"))
        B, n = _batch(rng, 16384 if out == "f32" else 32768)
        K = rng.choice((512, 768, 1024, 2048, 4096, _size(rng, 33, 4096)))
        N = rng.choice((512, 768, 1024, 1536, 2304, 4096, _size(rng, 33, 4096)))
        N = min(N, (1 << 22) // K)  # no more work than the widening and narrowing products
        return _linear(None, B, n, K, N, lens=lens, x=rng.choice(("bf16", "bf16", "f32", "i8")), out=out,
                       gelu=rng.random() < 0.4, bias=rng.random() < 0.7)
    dtype = rng.choice(("bf16", "bf16", "f32"))
    gate = rng.choice(("none", "channel", "sequence", "token"))
    B, n = _batch(rng, (32768 if gate != "token" else 24576) // (2 if dtype == "f32" else 1))
    D = rng.choice((512, 768, 1024, _size(rng, 33, 1024)))
    pre = rng.random() < 0.8
    return _norm(None, B, n, D, lens=lens, dtype=dtype, kind=rng.choice(("layer", "rms")), gate=gate,
                 post=rng.random() < 0.5, pre=pre, scale=rng.choice((1.0, 1.5, 0.81)), r=not pre or rng.random() < 0.5,
                 backward=op == "norm_backward")


def _lengths(case):
    """Rows of each sequence, ascending: all of n, evenly spread over the upper half, or the quantiles of the length
    distribution ln L ~ N(5.717, 0.738^2) cut to [1, n]."""
    B, n = case["B"], case["n"]
    if case["lens"] == "full":
        return [n] * B
    if case["lens"] == "lognormal":
        z = statistics.NormalDist(5.717, 0.738)
        return [max(1, min(n, round(math.exp(z.inv_cdf((b + 0.5) / B))))) for b in range(B)]
    return [round((n + 1) // 2 + (n // 2) * (b + 1) / B) for b in range(B)]


def _type(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "i8": torch.int8}[name]


# ----------------------------------------------------------------- inputs ----
def _geometry(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    L = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    L = L[torch.randperm(case["B"], generator=g, device="cuda")].contiguous()
    return g, L


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _pad(q):
    """int8 [..., K] with the row padding that the products expect."""
    return torch.nn.functional.pad(q, (0, -q.shape[-1] % PITCH)).contiguous()


def _hidden(g, B, n, D):
    """Hidden rows as encoders have them: a few channels many times the others, rows of different size."""
    gain = torch.exp(0.3 * _randn(g, D))
    gain[torch.randperm(D, generator=g, device="cuda")[:max(1, D // 128)]] *= 8
    return _randn(g, B, n, D) * gain * torch.exp(0.2 * _randn(g, B, n, 1))


def _prepare_linear(case, seed):
    g, L = _geometry(case, seed)
    B, n, K, N = case["B"], case["n"], case["K"], case["N"]
    x, x_scale = _hidden(g, B, n, K), None
    if case["x"] == "i8":  # what the operator before this one left: rows of int8 and their scales
        x_scale = (x.abs().amax(-1) / 127).contiguous()
        x = _pad(torch.round(x / x_scale[..., None]).to(torch.int8))
    else:
        x = x.to(_type(case["x"])).contiguous()
    w = _randn(g, N, K) * torch.exp(0.3 * _randn(g, N, 1)) / math.sqrt(K)
    w_scale = (w.abs().amax(-1) / 127).contiguous()
    w = _pad(torch.round(w / w_scale[:, None]).to(torch.int8))
    return dict(case=case, lens=L, x=x, x_scale=x_scale, w=w, w_scale=w_scale,
                bias=0.1 * _randn(g, N) if case["bias"] else None)


def _prepare_norm(case, seed):
    g, L = _geometry(case, seed)
    B, n, D, dt = case["B"], case["n"], case["D"], _type(case["dtype"])
    s = dict(case=case, lens=L, x=_hidden(g, B, n, D).to(dt), t=(0.5 * _randn(g, B, n, D)).to(dt), gate=None,
             post_w=None, post_b=None, pre_w=None, pre_b=None, dr=None, dy=None)
    if case["gate"] != "none":
        shape = {"channel": (D,), "sequence": (B, D), "token": (B, n, D)}[case["gate"]]
        s["gate"] = (0.5 + 0.2 * _randn(g, *shape)).to(torch.float32 if case["gate"] == "channel" else dt)
    for name in ("post", "pre"):
        if case[name]:
            s[name + "_w"] = 1 + 0.1 * _randn(g, D)
            s[name + "_b"] = 0.1 * _randn(g, D) if case["kind"] == "layer" else None
    if case["op"] == "norm_backward":
        if case["r"]:
            s["dr"] = _randn(g, B, n, D).to(dt)
        if case["pre"]:
            s["dy"] = _randn(g, B, n, D).to(dt)
    return s


def prepare(case, seed):
    return _prepare_linear(case, seed) if case["op"] == "linear" else _prepare_norm(case, seed)


# ------------------------------------------------------------ plain forms ----
def _valid(s):
    return torch.arange(s["case"]["n"], device="cuda")[None, :, None] < s["lens"][:, None, None]


def _plain_linear(s):
    c = s["case"]
    if c["x"] == "i8":
        q, scale = s["x"][..., :c["K"]].float(), s["x_scale"][..., None]
    else:
        x = s["x"].float()
        amax = x.abs().amax(-1, keepdim=True)
        scale = amax / 127
        # next to a border between two steps 32 bits would take the wrong one
        q = torch.round(127 * x.double() / amax.double()).float()
        q = torch.where(amax > 0, q, 0.0)
    out = torch.matmul(q, s["w"][:, :c["K"]].float().t()) * scale * s["w_scale"]
    if s["bias"] is not None:
        out = out + s["bias"]
    if c["gelu"]:
        out = 0.5 * out * (1 + torch.erf(out * math.sqrt(0.5)))
    return torch.where(_valid(s), out, 0.0).to(_type(c["out"]))


def _normalise(x, kind):
    """(normalised rows, 1 / deviation)"""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    inv = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * inv, inv


def _affine(x, w, b):
    x = x * w
    return x if b is None else x + b


def _plain_gate(s):
    c, gate = s["case"], s["gate"]
    if gate is None:
        return None
    return gate.float()[:, None, :] if c["gate"] == "sequence" else gate.float()


def _plain_norm(s):
    c, valid, dt = s["case"], _valid(s), _type(s["case"]["dtype"])
    u, gate = s["t"].float(), _plain_gate(s)
    if c["post"]:
        u = _affine(_normalise(u, c["kind"])[0], s["post_w"], s["post_b"])
    r = c["scale"] * s["x"].float() + (u if gate is None else gate * u)
    y = _affine(_normalise(r, c["kind"])[0], s["pre_w"], s["pre_b"]) if c["pre"] else None
    return dict(r=torch.where(valid, r, 0.0).to(dt) if c["r"] else None,
                y=torch.where(valid, y, 0.0).to(dt) if c["pre"] else None)


def _norm_input_grad(g, xhat, inv, kind):
    d = g - xhat * (g * xhat).mean(-1, keepdim=True)
    if kind == "layer":
        d = d - g.mean(-1, keepdim=True)
    return inv * d


def _plain_norm_backward(s):
    c, valid, dt = s["case"], _valid(s), _type(s["case"]["dtype"])
    x, u, gate = s["x"].float(), s["t"].float(), _plain_gate(s)
    o = dict(dx=None, dt=None, dgate=None, dpost_w=None, dpost_b=None, dpre_w=None, dpre_b=None)
    if c["post"]:
        that, tinv = _normalise(u, c["kind"])
        u = _affine(that, s["post_w"], s["post_b"])
    grad = torch.where(valid, s["dr"].float(), 0.0) if c["r"] else 0.0
    if c["pre"]:
        r = c["scale"] * x + (u if gate is None else gate * u)
        rhat, rinv = _normalise(r, c["kind"])
        dy = torch.where(valid, s["dy"].float(), 0.0)
        grad = grad + _norm_input_grad(dy * s["pre_w"], rhat, rinv, c["kind"])
        o["dpre_w"] = (dy * rhat).sum((0, 1))
        if s["pre_b"] is not None:
            o["dpre_b"] = dy.sum((0, 1))
    o["dx"] = (c["scale"] * grad).to(dt)
    du = grad
    if gate is not None:
        du = grad * gate
        dg = grad * u
        o["dgate"] = {"channel": lambda: dg.sum((0, 1)), "sequence": lambda: dg.sum(1).to(dt),
                      "token": lambda: dg.to(dt)}[c["gate"]]()
    if c["post"]:
        o["dpost_w"] = (du * that).sum((0, 1))
        if s["post_b"] is not None:
            o["dpost_b"] = du.sum((0, 1))
        du = _norm_input_grad(du * s["post_w"], that, tinv, c["kind"])
    o["dt"] = du.to(dt)
    return o


# -------------------------------------------------- the framework's calls ----
def _own(s):
    import paper_2310_07109_amd as sc
    c = s["case"]
    code = {"f32": sc.SC_F32, "bf16": sc.SC_BF16, "i8": sc.SC_I8}
    if c["op"] == "linear":
        d = sc.LinearDesc(c["B"], c["n"], c["K"], c["N"], valid_len=s["lens"], x_dtype=code[c["x"]],
                          out_dtype=code[c["out"]], act=sc.SC_ACT_GELU if c["gelu"] else sc.SC_ACT_NONE)
        return sc.sc_linear_i8(d, s["x"], s["w"], s["w_scale"], bias=s["bias"], x_scale=s["x_scale"])
    gate = dict(none=sc.SC_GATE_NONE, channel=sc.SC_GATE_CHANNEL, sequence=sc.SC_GATE_SEQUENCE,
                token=sc.SC_GATE_TOKEN)[c["gate"]]
    d = sc.NormDesc(c["B"], c["n"], c["D"], valid_len=s["lens"], post=c["post"], pre=c["pre"], gate=gate, eps=EPS,
                    kind=sc.SC_NORM_LAYER if c["kind"] == "layer" else sc.SC_NORM_RMS, res_scale=c["scale"],
                    dtype=code[c["dtype"]])
    w = dict(gate=s["gate"], post_w=s["post_w"], post_b=s["post_b"], pre_w=s["pre_w"], pre_b=s["pre_b"])
    if c["op"] == "norm":
        r, y, _, _ = sc.sc_block_norm(d, s["x"], s["t"], r=c["r"], y=c["pre"], **w)
        return dict(r=r, y=y)
    g = sc.sc_block_norm_backward(d, s["x"], s["t"], dr=s["dr"], dy=s["dy"], **w)
    return {k: g[k] for k in ("dx", "dt", "dgate", "dpost_w", "dpost_b", "dpre_w", "dpre_b")}


def run(state):
    if own:
        return _own(state)
    return {"linear": _plain_linear, "norm": _plain_norm,
            "norm_backward": _plain_norm_backward}[state["case"]["op"]](state)


# ------------------------------------------------------------------- work ----
def work(case):
    R, T = sum(_lengths(case)), case["B"] * case["n"]
    if case["op"] == "linear":
        K, N = case["K"], case["N"]
        ex, eo = {"f32": 4, "bf16": 2, "i8": 1}[case["x"]], {"f32": 4, "bf16": 2}[case["out"]]
        b = R * K * ex + N * K + T * N * eo + 4 * N * (2 if case["bias"] else 1)
        return dict(bytes=b + (4 * R if case["x"] == "i8" else 0), flops=2 * R * K * N)
    D, e = case["D"], 4 if case["dtype"] == "f32" else 2
    gate = {"none": 0, "channel": 4 * D, "sequence": case["B"] * D * e, "token": R * D * e}[case["gate"]]
    per_norm = 4 * D * (2 if case["kind"] == "layer" else 1)
    weights = per_norm * (case["post"] + case["pre"])
    if case["op"] == "norm":
        outs = T * D * e * (case["r"] + case["pre"])
        return dict(bytes=2 * R * D * e + gate + weights + outs, flops=R * D * (4 + 6 * (case["post"] + case["pre"])))
    ins = R * D * e * (2 + case["r"] + case["pre"])
    out_gate = T * D * e if case["gate"] == "token" else gate
    return dict(bytes=ins + 2 * T * D * e + gate + out_gate + 2 * weights,
                flops=R * D * (6 + 18 * (case["post"] + case["pre"])))


# -------------------------------------------------------------- reference ----
def _exact_linear(case, s):
    rows = [s["x"][b, :L] for b, L in enumerate(s["lens"].tolist())]
    W = s["w"][:, :case["K"]].double() * s["w_scale"].double()[:, None]
    out = torch.zeros((case["B"], case["n"], case["N"]), dtype=torch.float64, device="cuda")
    for b, x in enumerate(rows):
        v = x[:, :case["K"]].double()
        if case["x"] == "i8":
            v = v * s["x_scale"][b, :len(x), None].double()
        else:
            top = v.abs().max(dim=1, keepdim=True).values
            v = torch.where(top > 0, torch.round(v * 127 / top) * (top / 127), 0.0)
        o = v @ W.T
        if s["bias"] is not None:
            o += s["bias"].double()
        out[b, :len(x)] = torch.nn.functional.gelu(o) if case["gelu"] else o
    return out


def _exact_norms(case, s, leaves):
    """(r, y) of the rows of every sequence, in float64, as functions of the leaves."""
    def norm(v, w, b):
        if case["kind"] == "layer":
            return torch.nn.functional.layer_norm(v, (case["D"],), w, b, EPS)
        v = v * (v.pow(2).mean(-1, keepdim=True) + EPS).pow(-0.5) * w
        return v if b is None else v + b
    u = leaves["t"]
    if case["post"]:
        u = norm(u, leaves["post_w"], leaves["post_b"])
    if case["gate"] == "sequence":
        u = leaves["gate"].unsqueeze(1) * u
    elif case["gate"] != "none":
        u = leaves["gate"] * u
    r = case["scale"] * leaves["x"] + u
    return r, norm(r, leaves["pre_w"], leaves["pre_b"]) if case["pre"] else None


def exact(case, seed):
    """The outputs of run() in float64, from the definition."""
    s = prepare(case, seed)
    if case["op"] == "linear":
        return _exact_linear(case, s)
    back = case["op"] == "norm_backward"
    names = ("x", "t", "gate", "post_w", "post_b", "pre_w", "pre_b")
    leaves = {k: None if s[k] is None else s[k].double().requires_grad_(back) for k in names}
    mask = (torch.arange(case["n"], device="cuda") < s["lens"][:, None]).double()[..., None]
    with torch.set_grad_enabled(back):
        r, y = _exact_norms(case, s, leaves)
        if not back:
            return dict(r=r * mask if case["r"] else None, y=y * mask if case["pre"] else None)
        loss = 0.0
        if case["r"]:
            loss = loss + (r * mask * s["dr"].double()).sum()
        if case["pre"]:
            loss = loss + (y * mask * s["dy"].double()).sum()
        have = [k for k in names if leaves[k] is not None]
        grads = dict(zip(have, torch.autograd.grad(loss, [leaves[k] for k in have])))
    return {"d" + k: grads.get(k) for k in ("x", "t", "gate", "post_w", "post_b", "pre_w", "pre_b")}
