"""Cases of layer norm (with the statistics of its gradients) and of the orthogonalised update: what is timed and compared.

Shapes follow the framework's other calls: a leading dimension of M replicas, each with parameters of its own, then b samples
of T rows, then the features; weight matrices are [M, rows, cols].

  layer norm     mu = mean x, r = 1 / sqrt(mean (x - mu)^2 + eps), y = (x - mu) r gamma + beta
  its gradients  xh = (x - mu) r, h = dy gamma:  dx = r (h - mean h - xh mean(h xh)),
                 per sample i  g_i = (sum_t dy xh, sum_t dy),  gbar = mean_i g_i,  n_i = ||g_i||^2,  q_i = <g_i, gbar>
  orthogonalise  X = G / (||G|| + eps), then in each step  A = X X^T,  X <- a X + (b A + c A A) X
  the update     v <- mu v + g,  u = g + mu v,  x <- (1 - lr wd) x - lr scale orth(u)
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LN_EPS, NS_EPS = 1e-5, 1e-7
STEPS, COEF = 5, (3.4445, -4.7750, 2.0315)
MOMENTUM, LR, WD = 0.95, 1e-3, 0.05


def _ln(name, kind, M, b, T, D, dtype, param="f32", stats="none"):
    c = dict(kind=kind, M=M, b=b, T=T, D=D, dtype=dtype, param=param)
    if kind == "ln_bwd":
        c["stats"] = stats
    return dict(c, name=name) if name else c


def _mat(name, kind, M, rows, cols, dtype, grad=None):
    c = dict(kind=kind, M=M, rows=rows, cols=cols, dtype=dtype)
    if kind == "muon":
        c["grad"] = grad or dtype
    return dict(c, name=name) if name else c


def listed():
    return [
        # one replica's norm of a few single tokens, as in serving: all latency
        _ln("ln_tokens", "ln_fwd", 1, 8, 1, 2048, "bf16", "bf16"),
        # a training step's norm: eight replicas, 16 sequences of 512 tokens each
        _ln("ln_train", "ln_fwd", 8, 16, 512, 2048, "bf16"),
        # the fp32 path at sizes that are multiples of nothing
        _ln("ln_odd_f32", "ln_fwd", 3, 37, 27, 777, "f32"),
        # gradients of a small net's norm: single rows per sample, all statistics of the batch tests
        _ln("ln_grad_rows", "ln_bwd", 8, 512, 1, 512, "bf16", stats="inner"),
        # gradients of a language model's norm: samples are sequences, per-sample norms for the norm test
        _ln("ln_grad_train", "ln_bwd", 8, 16, 512, 2048, "bf16", stats="norms"),
        # gradients alone, fp32, odd sizes
        _ln("ln_grad_odd_f32", "ln_bwd", 3, 37, 27, 777, "f32"),
        # the smallest matrices that an update orthogonalises: one head's projection
        _mat("orth_small", "orth", 4, 64, 96, "bf16"),
        # tall and odd, many at once
        _mat("orth_odd", "orth", 12, 1001, 333, "f16"),
        # one large matrix
        _mat("orth_4096", "orth", 1, 4096, 4096, "bf16"),
        # the medium net's hidden layer in fp32: master weights, eight replicas
        _mat("muon_mlp512_f32", "muon", 8, 512, 784, "f32"),
        # a hidden layer of the large net for sixteen replicas, 16-bit weights and gradients, 32-bit momentum
        _mat("muon_mlp2048", "muon", 16, 2048, 2048, "bf16"),
        # a feed-forward matrix, fp32 weights
        _mat("muon_ffn_f32", "muon", 2, 4096, 1024, "f32"),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], its logarithm uniform."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["ln_fwd", "ln_bwd", "ln_bwd", "orth", "orth", "muon"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if kind in ("ln_fwd", "ln_bwd"):
        M, D = _log(rng, 1, 16), _log(rng, 16, 8192)
        T = rng.choice([1, 1, _log(rng, 2, 32), _log(rng, 32, 1024)])
        b = _log(rng, 2, max(2, min(4096, (1 << 26) // (M * D * T))))
        return _ln(None, kind, M, b, T, D, dtype, rng.choice(["f32", dtype]), rng.choice(["none", "norms", "inner"]))
    rows, cols = _log(rng, 16, 3000), _log(rng, 16, 3000)
    most = (1 << 36) // (rows * cols * min(rows, cols))
    return _mat(None, kind, _log(rng, 1, max(1, min(32, most))), rows, cols, dtype, rng.choice([dtype, "f32"]))


# ---- inputs --------------------------------------------------------------------------------------------------------

def _gradients(M, rows, cols, g):
    """Batch gradients as a linear layer has them: signals times inputs over 512 samples, features of falling scale."""
    def side(n):
        t = torch.randn((M, 512, n), device="cuda", generator=g)
        return t * (1.0 + torch.arange(n, device="cuda") % 61).rsqrt()
    return torch.bmm(side(rows).transpose(1, 2).contiguous(), side(cols)) / 512.0


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    M = case["M"]
    if case["kind"] in ("ln_fwd", "ln_bwd"):
        shape, D = (M, case["b"], case["T"], case["D"]), case["D"]
        # activations of a residual stream: an offset, and a few features far larger than the rest
        scale = 1.0 + 7.0 * (torch.rand((M, 1, 1, D), device="cuda", generator=g) < 0.01)
        x = (torch.randn(shape, device="cuda", generator=g) * scale + 0.3).to(dt)
        w = (1.0 + 0.2 * torch.randn((M, D), device="cuda", generator=g)).to(DTYPES[case["param"]])
        s = dict(case=case, x=x, w=w)
        if case["kind"] == "ln_fwd":
            return dict(s, bias=(0.1 * torch.randn((M, D), device="cuda", generator=g)).to(DTYPES[case["param"]]))
        dy = torch.randn(shape, device="cuda", generator=g)
        dy = (dy * (0.5 + torch.rand((M, case["b"], 1, 1), device="cuda", generator=g)) + 0.05).to(dt)
        x32 = x.float()
        mean = x32.mean(-1)
        rstd = ((x32 - mean[..., None]).square().mean(-1) + LN_EPS).rsqrt()
        return dict(s, dy=dy, mean=mean, rstd=rstd)
    grad = _gradients(M, case["rows"], case["cols"], g)
    if case["kind"] == "orth":
        return dict(case=case, g=grad.to(dt))
    x = (torch.rand(grad.shape, device="cuda", generator=g) * 2.0 - 1.0) / math.sqrt(case["cols"])
    v = _gradients(M, case["rows"], case["cols"], g) * 4.0      # what some steps have left
    return dict(case=case, x=x.to(dt), g=grad.to(DTYPES[case["grad"]]), v=v)


# ---- one pass ------------------------------------------------------------------------------------------------------

def _orth32(x):
    """The Newton-Schulz steps on [M, rows, cols] in 32 bits, on the smaller side."""
    x = x / (x.double().square().sum((1, 2), keepdim=True).sqrt().float() + NS_EPS)
    a, b, c = COEF
    wide = x.shape[1] <= x.shape[2]
    for _ in range(STEPS):
        xt = x.transpose(1, 2).contiguous()
        gram = torch.matmul(x, xt) if wide else torch.matmul(xt, x)
        poly = b * gram + c * torch.matmul(gram, gram)
        x = a * x + (torch.matmul(poly, x) if wide else torch.matmul(x, poly))
    return x


def _scale(case):
    return 0.2 * math.sqrt(max(case["rows"], case["cols"]))


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "ln_fwd":
        x = s["x"].float()
        mean = x.mean(-1)
        d = x - mean[..., None]
        rstd = (d.square().mean(-1) + LN_EPS).rsqrt()
        y = d * rstd[..., None] * s["w"].float()[:, None, None] + s["bias"].float()[:, None, None]
        return dict(y=y.to(s["x"].dtype), mean=mean, rstd=rstd)
    if kind == "ln_bwd":
        dy, r = s["dy"].float(), s["rstd"][..., None]
        xh = (s["x"].float() - s["mean"][..., None]) * r
        h = dy * s["w"].float()[:, None, None]
        dx = r * (h - h.mean(-1, keepdim=True) - xh * (h * xh).mean(-1, keepdim=True))
        gw, gb = (dy * xh).sum(2), dy.sum(2)
        out = dict(dx=dx.to(s["x"].dtype), dw=gw.mean(1), db=gb.mean(1))
        if case["stats"] != "none":
            out["n"] = gw.square().sum(-1) + gb.square().sum(-1)
        if case["stats"] == "inner":
            out["q"] = (gw * out["dw"][:, None]).sum(-1) + (gb * out["db"][:, None]).sum(-1)
        return out
    if kind == "orth":
        return dict(o=_orth32(s["g"].float()).to(s["g"].dtype))
    g = s["g"].float()
    s["v"].mul_(MOMENTUM).add_(g)
    o = _orth32(g + MOMENTUM * s["v"])
    s["x"].copy_(((1.0 - LR * WD) * s["x"].float() - (LR * _scale(case)) * o).to(s["x"].dtype))
    return dict(x=s["x"], v=s["v"])


def _own(s):
    import paper_2406_13936_amd as A
    case = s["case"]
    kind = case["kind"]
    if kind == "ln_fwd":
        y, mean, rstd = A.layer_norm(s["x"], s["w"], s["bias"], eps=LN_EPS)
        return dict(y=y, mean=mean, rstd=rstd)
    if kind == "ln_bwd":
        dx, dw, db, n, q = A.layer_norm_backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"],
                                                 want_norms=case["stats"] != "none", want_inner=case["stats"] == "inner")
        out = dict(dx=dx, dw=dw, db=db)
        if n is not None:
            out["n"] = n
        if q is not None:
            out["q"] = q
        return out
    if kind == "orth":
        return dict(o=A.orthogonalize(s["g"], steps=STEPS, eps=NS_EPS))
    A.muon_step(s["x"], s["g"], s["v"], LR, momentum=MOMENTUM, weight_decay=WD, scale=_scale(case), steps=STEPS, eps=NS_EPS)
    return dict(x=s["x"], v=s["v"])


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definition in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "ln_fwd":
        x = s["x"].double()
        var, mean = torch.var_mean(x, dim=-1, correction=0)
        rstd = 1.0 / torch.sqrt(var + LN_EPS)
        y = torch.addcmul(s["bias"].double().view(case["M"], 1, 1, -1), (x - mean.unsqueeze(-1)) / torch.sqrt(var + LN_EPS).unsqueeze(-1),
                          s["w"].double().view(case["M"], 1, 1, -1))
        return dict(y=y, mean=mean, rstd=rstd)
    if kind == "ln_bwd":
        D = case["D"]
        x, dy, w = s["x"].double(), s["dy"].double(), s["w"].double().view(case["M"], 1, 1, -1)
        var, mean = torch.var_mean(x, dim=-1, correction=0, keepdim=True)
        sd = torch.sqrt(var + LN_EPS)
        xh = (x - mean) / sd
        h = dy * w
        dx = (D * h - h.sum(-1, keepdim=True) - xh * (h * xh).sum(-1, keepdim=True)) / (D * sd)
        per = torch.cat([(dy * xh).sum(2), dy.sum(2)], -1)          # [M, b, 2 D]: the gradient of each sample
        bar = per.sum(1) / case["b"]
        out = dict(dx=dx, dw=bar[:, :D], db=bar[:, D:])
        if case["stats"] != "none":
            out["n"] = (per * per).sum(-1)
        if case["stats"] == "inner":
            out["q"] = torch.matmul(per, bar.unsqueeze(-1)).squeeze(-1)
        return out

    def orth(u):
        flip = u.shape[1] > u.shape[2]
        z = u.transpose(1, 2).contiguous() if flip else u
        z = z / (torch.linalg.vector_norm(z, dim=(1, 2), keepdim=True) + NS_EPS)
        a, b, c = COEF
        eye = torch.eye(z.shape[1], dtype=torch.float64, device=z.device)
        for _ in range(STEPS):
            k = torch.matmul(z, z.transpose(1, 2))
            z = torch.matmul(a * eye + torch.matmul(k, b * eye + c * k), z)
        return z.transpose(1, 2).contiguous() if flip else z

    if kind == "orth":
        return dict(o=orth(s["g"].double()))
    g = s["g"].double()
    v = MOMENTUM * s["v"].double() + g
    x = s["x"].double()
    return dict(x=x - LR * (WD * x + _scale(case) * orth(g + MOMENTUM * v)), v=v)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------

def work(case):
    """Bytes: inputs once, outputs once.  Flops: products of the steps, the symmetric ones (A and A A) at half."""
    M, size = case["M"], {"f32": 4, "bf16": 2, "f16": 2}
    e = size[case["dtype"]]
    if case["kind"] in ("ln_fwd", "ln_bwd"):
        rows, D, b = M * case["b"] * case["T"], case["D"], case["b"]
        if case["kind"] == "ln_fwd":
            return {"bytes": rows * (2.0 * D * e + 8) + 2.0 * M * D * size[case["param"]], "flops": 8.0 * rows * D}
        stats = {"none": 0, "norms": 1, "inner": 2}[case["stats"]]
        return {"bytes": rows * (3.0 * D * e + 8) + M * D * (size[case["param"]] + 8.0) + 4.0 * M * b * stats, "flops": 14.0 * rows * D}
    m, n = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    flops = float(M) * STEPS * (3.0 * m * m * n + float(m) ** 3)
    if case["kind"] == "orth":
        return {"bytes": 2.0 * M * m * n * e, "flops": flops}
    return {"bytes": float(M) * m * n * (2 * e + size[case["grad"]] + 8), "flops": flops}
