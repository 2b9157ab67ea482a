"""Cases of the operators of a language model's blocks that stand beside layer norm and the orthogonalised update: token embedding with
the gradient of its table, root-mean-square norm behind a residual's addition, causal attention over packed sequences.

M replicas with parameters of their own, b samples of T tokens each; gradients are of per-sample losses, a parameter's batch gradient
is the mean over the b samples, and n_i, q_i are the statistics that the batch tests take of it.

  embedding      y_t = s table[token_t]  (a token outside the table is padding: zeros, no gradient)
  its gradient   g_i = s sum_t dy_t e(token_t)^T of sample i,  gbar = mean_i g_i,  n_i = ||g_i||^2,  q_i = <g_i, gbar>
  norm           h = x + residual, rounded to its type;  r = 1 / sqrt(mean h^2 + eps),  y = h r w
                 or in 8 bits (e4m3):  c = max(max |y| / 448, 2^-100) of a row,  y / c rounded
  its gradients  hh = h r,  u = dy w:  dx = dh + r (u - hh mean(u hh)),  g_i = sum_t dy hh
  attention      s_ij = a q_i . k_j for j <= i of one sequence,  o_i = sum_j softmax(s_i)_j v_j,  lse_i = log sum_j exp s_ij
  its gradients  p_ij = exp(s_ij - lse_i),  ds_ij = a p_ij (do_i . v_j - do_i . o_i):
                 dv_j = sum p_ij do_i,  dk_j = sum ds_ij q_i,  dq_i = sum ds_ij k_j;  query heads that share a key head add up there
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i32": torch.int32, "i64": torch.int64}
EPS = 1e-6
SMALLEST_SCALE = 2.0 ** -100


def _emb(name, kind, M, b, T, V, D, table, dtype, idx="i64", pad=0.0, stats="none"):
    c = dict(kind=kind, M=M, b=b, T=T, V=V, D=D, dtype=dtype, idx=idx, pad=pad)
    c["table" if kind == "emb_fwd" else "stats"] = table if kind == "emb_fwd" else stats
    return dict(c, name=name) if name else c


def _rms(name, kind, M, b, T, D, dtype, param="f32", add=True, stats="none"):
    c = dict(kind=kind, M=M, b=b, T=T, D=D, dtype=dtype, param=param, add=add)
    if kind == "rms_bwd":
        c["stats"] = stats
    return dict(c, name=name) if name else c


def _attn(name, kind, rows, docs, Hq, Hkv, D, dtype, T=0, tail=0, pack=1, fused=False):
    """docs sequences: of T tokens each (T > 0), or of what `pack` makes of rows - tail tokens; the last `tail` rows are no sequence's."""
    c = dict(kind=kind, rows=rows, docs=docs, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, T=T, tail=tail, pack=pack, fused=fused)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a training step's first layer: fp32 master table, 16-bit activations, four replicas of 8 sequences
        _emb("emb_train", "emb_fwd", 4, 8, 1024, 32000, 1024, "f32", "bf16"),
        # its gradient with all statistics of the batch tests
        _emb("emb_grad_train", "emb_bwd", 4, 8, 1024, 32000, 1024, None, "bf16", stats="inner"),
        # a small net's table in fp32 at sizes that are multiples of nothing, padded samples: latency
        _emb("emb_grad_odd_f32", "emb_bwd", 3, 5, 33, 997, 257, None, "f32", "i32", 0.2, "norms"),
        # the norm of single tokens in front of 8-bit products: all latency
        _rms("rms_tokens_8bit", "rms_8bit", 1, 8, 1, 2048, "bf16", "bf16"),
        # a training step's norm behind the residual's addition: eight replicas, 16 sequences of 512 tokens each
        _rms("rms_train", "rms_fwd", 8, 16, 512, 2048, "bf16"),
        # its gradients, per-sample norms for the norm test
        _rms("rms_grad_train", "rms_bwd", 8, 16, 512, 2048, "bf16", stats="norms"),
        # gradients in fp32, odd sizes, all statistics
        _rms("rms_grad_odd_f32", "rms_bwd", 3, 29, 31, 999, "f32", stats="inner"),
        # a few short sequences of some tokens, among them single ones: latency
        _attn("attn_short", "attn_fwd", 257, 9, 8, 2, 64, "bf16", pack=7),
        # one long sequence
        _attn("attn_prompt", "attn_fwd", 16384, 1, 16, 4, 128, "bf16", T=16384),
        # a step's gradients: four replicas of 8 samples of 1024 tokens, documents packed, q, k and v side by side in one buffer
        _attn("attn_grad_train", "attn_bwd", 32768, 40, 16, 4, 64, "bf16", pack=3, fused=True),
        # odd everything, rows behind the last sequence
        _attn("attn_grad_odd", "attn_bwd", 3001, 7, 6, 3, 80, "f16", tail=37, pack=5),
        # the fp32 path: two replicas of three samples
        _attn("attn_f32", "attn_fwd", 3000, 6, 4, 4, 48, "f32", T=500),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], its logarithm uniform."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["emb_fwd", "emb_bwd", "emb_bwd", "rms_fwd", "rms_8bit", "rms_bwd", "attn_fwd", "attn_fwd", "attn_bwd", "attn_bwd"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if kind.startswith("emb"):
        M, D = _log(rng, 1, 8), _log(rng, 8, 4096)
        V = _log(rng, 50, max(50, min(131072, (1 << 27) // (M * D))))
        T = rng.choice([1, _log(rng, 2, 64), _log(rng, 64, max(64, min(2048, (1 << 24) // (M * D))))])
        b = _log(rng, 2, max(2, min(2048, (1 << 25) // (M * D * T))))
        return _emb(None, kind, M, b, T, V, D, rng.choice(["f32", dtype]), dtype, rng.choice(["i32", "i64"]), rng.choice([0.0, 0.2]),
                    rng.choice(["none", "norms", "inner"]))
    if kind.startswith("rms"):
        M, D = _log(rng, 1, 16), _log(rng, 16, 8192)
        T = rng.choice([1, 1, _log(rng, 2, 32), _log(rng, 32, 1024)])
        b = _log(rng, 2, max(2, min(4096, (1 << 26) // (M * D * T))))
        return _rms(None, kind, M, b, T, D, dtype, rng.choice(["f32", dtype]), rng.random() < 0.7, rng.choice(["none", "norms", "inner"]))
    Hkv, G = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 1, 2, 3, 4])
    D = rng.choice([32, 64, 64, 80, 96, 128, 128, rng.randint(8, 128)])
    # scores: the largest listed has 16 heads of 2^27, of 128 values
    most = (1 << 28) if dtype == "f32" else 800_000_000 if kind == "attn_bwd" else 2_000_000_000
    longest = int(math.sqrt(2.0 * most / (Hkv * G)))
    if rng.random() < 0.4:
        T = _log(rng, 1, min(12000, longest))
        n = _log(rng, 1, max(1, min(48, 2 * most // (Hkv * G * T * T), 40000 // T)))
        return _attn(None, kind, n * T, n, Hkv * G, Hkv, D, dtype, T=T, fused=rng.random() < 0.5)
    rows = _log(rng, 16, min(20000, longest))
    docs = _log(rng, 1, max(1, min(64, rows // 8)))
    return _attn(None, kind, rows, docs, Hkv * G, Hkv, D, dtype, tail=rng.choice([0, 0, rng.randint(0, rows // 8)]),
                 pack=rng.randint(1, 1 << 20), fused=rng.random() < 0.5)


def _lengths(case):
    """Lengths of a case's sequences: all T, or between cuts at random places (some of length zero or one among many)."""
    if case["T"]:
        return [case["T"]] * case["docs"]
    r, n = random.Random(case["pack"]), case["rows"] - case["tail"]
    cuts = sorted(r.randint(0, n) for _ in range(case["docs"] - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [n])]


# ---- inputs --------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    if case["kind"].startswith("emb"):
        M, b, T, V, D = (case[k] for k in ("M", "b", "T", "V", "D"))
        # words by falling frequency: the n-th as often as 1 / n; padded ends of samples
        u = torch.rand((M, b, T), device="cuda", generator=g, dtype=torch.float64)
        tokens = ((V + 1.0) ** u).long().clamp(1, V) - 1
        if case["pad"]:
            keep = 1.0 - case["pad"] * torch.rand((M, b, 1), device="cuda", generator=g)
            tokens = torch.where(torch.arange(T, device="cuda") < keep * T, tokens, -1)
        s = dict(case=case, tokens=tokens.to(DTYPES[case["idx"]]), scale=math.sqrt(D))
        if case["kind"] == "emb_fwd":
            return dict(s, table=(normal(M, V, D) / math.sqrt(D)).to(DTYPES[case["table"]]))
        return dict(s, dy=(normal(M, b, T, D) * (0.5 + torch.rand((M, b, 1, 1), device="cuda", generator=g)) / T).to(dt))
    if case["kind"].startswith("rms"):
        M, b, T, D = (case[k] for k in ("M", "b", "T", "D"))
        # a residual stream: a few features far larger than the rest
        scale = 1.0 + 7.0 * (torch.rand((M, 1, 1, D), device="cuda", generator=g) < 0.01)
        big = (normal(M, b, T, D) * scale).to(dt)
        s = dict(case=case, w=(1.0 + 0.2 * normal(M, D)).to(DTYPES[case["param"]]))
        if case["kind"] != "rms_bwd":
            return dict(s, x=(0.3 * normal(M, b, T, D)).to(dt), residual=big) if case["add"] else dict(s, x=big, residual=None)
        dy = (normal(M, b, T, D) * (0.5 + torch.rand((M, b, 1, 1), device="cuda", generator=g)) + 0.05).to(dt)
        return dict(s, h=big, dy=dy, dh=normal(M, b, T, D).to(dt) if case["add"] else None,
                    rstd=(big.float().square().mean(-1) + EPS).rsqrt())
    R, Hq, Hkv, D = (case[k] for k in ("rows", "Hq", "Hkv", "D"))
    lens = _lengths(case)
    ends = [0]
    for n in lens:
        ends.append(ends[-1] + n)

    def heads(fused, *counts):
        """[R, heads, D] values for each of counts; fused: columns of one buffer"""
        if fused:
            return torch.split(normal(R, sum(counts), D).to(dt), list(counts), dim=1)
        return [normal(R, n, D).to(dt) for n in counts]
    q, k, v = heads(case["fused"], Hq, Hkv, Hkv)
    s = dict(case=case, q=q, k=k, v=v, ends=ends, offsets=None if case["T"] else torch.tensor(ends, dtype=torch.int32, device="cuda"))
    if case["T"]:                                    # sequences of one length: a dimension of their own
        for x in "qkv":
            s[x] = s[x].unflatten(0, (case["docs"], case["T"]))
    if case["kind"] == "attn_bwd":
        s["o"], s["lse"] = _attention(s)
        s["do"] = normal(*s["o"].shape).to(dt)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------

def _rows_of(case, tokens):
    """Each token's row of the tables of all replicas side by side, and which tokens are in one."""
    V = case["V"]
    ok = (tokens >= 0) & (tokens < V)
    first = torch.arange(case["M"], device="cuda").view(-1, 1, 1) * V
    return torch.where(ok, tokens.long(), 0) + first, ok


def _embedding_gradient(s):
    case, D = s["case"], s["case"]["D"]
    rows, ok = _rows_of(case, s["tokens"])
    g = s["dy"].float() * s["scale"] * ok.unsqueeze(-1)
    bar = torch.zeros((case["M"] * case["V"], D), device="cuda").index_add_(0, rows.flatten(), g.view(-1, D)) / case["b"]
    out = dict(dtable=bar.view(case["M"], case["V"], D))
    if case["stats"] == "none":
        return out
    # rows of one sample and token summed first: those that follow each other once sorted
    samples = torch.arange(case["M"] * case["b"], device="cuda").repeat_interleave(case["T"])
    key, order = torch.sort(samples * (case["M"] * case["V"]) + rows.flatten())
    new = torch.cat([torch.ones_like(key[:1]), (key[1:] != key[:-1]).long()])
    each = torch.zeros_like(g.view(-1, D)).index_add_(0, new.cumsum(0) - 1, g.view(-1, D)[order])
    whose = torch.zeros_like(key).scatter_(0, new.cumsum(0) - 1, samples[order])
    out["n"] = torch.zeros(case["M"] * case["b"], device="cuda").index_add_(0, whose, each.square().sum(-1)).view(case["M"], case["b"])
    if case["stats"] == "inner":
        out["q"] = (g * bar[rows]).sum((2, 3))
    return out


def _normed(s):
    x = s["x"].float()
    h = (x if s["residual"] is None else x + s["residual"].float()).to(s["x"].dtype)
    rstd = (h.float().square().mean(-1) + EPS).rsqrt()
    return h, rstd, h.float() * rstd[..., None] * s["w"].float()[:, None, None]


def _pieces(s):
    """(rows of queries, rows of keys, mask) of each sequence, some queries at a time."""
    Hq, dev = s["case"]["Hq"], s["q"].device
    for a, e in zip(s["ends"], s["ends"][1:]):
        step = max(1, (1 << 28) // max(1, Hq * (e - a)))
        for i in range(a, e, step):
            j = min(i + step, e)
            yield slice(i, j), slice(a, j), torch.arange(a, j, device=dev) <= torch.arange(i, j, device=dev)[:, None]


def _by_head(t, groups=1):
    t = t.float().transpose(0, 1)
    return (t.repeat_interleave(groups, 0) if groups > 1 else t).contiguous()


def _attention(s):
    case = s["case"]
    q, k, v = (s[x].reshape(case["rows"], -1, case["D"]) for x in "qkv")
    G, a = case["Hq"] // case["Hkv"], 1.0 / math.sqrt(case["D"])
    o = torch.zeros(q.shape, device="cuda", dtype=q.dtype)
    lse = torch.zeros((case["Hq"], case["rows"]), device="cuda")
    for i, j, mask in _pieces(s):
        t = torch.matmul(_by_head(q[i]), _by_head(k[j], G).transpose(1, 2)) * a
        t = t.masked_fill_(~mask, -math.inf)
        top = t.amax(-1, keepdim=True)
        t = t.sub_(top).exp_()
        total = t.sum(-1, keepdim=True)
        o[i] = (torch.matmul(t, _by_head(v[j], G)) / total).transpose(0, 1).to(o.dtype)
        lse[:, i] = (top + total.log()).squeeze(-1)
    return o.view(s["q"].shape), lse.view((case["Hq"],) + s["q"].shape[:-2])


def _attention_gradients(s):
    case = s["case"]
    Hkv, D, R = case["Hkv"], case["D"], case["rows"]
    q, k, v, o, do = (s[x].reshape(R, -1, D) for x in ("q", "k", "v", "o", "do"))
    lse = s["lse"].view(case["Hq"], R)
    G, a = case["Hq"] // Hkv, 1.0 / math.sqrt(D)
    dq, dk, dv = (torch.zeros(x.shape, device="cuda") for x in (q, k, v))
    for i, j, mask in _pieces(s):
        qi, kj, doi = _by_head(q[i]), _by_head(k[j], G), _by_head(do[i])
        p = torch.matmul(qi, kj.transpose(1, 2)).mul_(a).sub_(lse[:, i, None]).exp_().masked_fill_(~mask, 0.0)
        dv[j] += torch.matmul(p.transpose(1, 2), doi).view(Hkv, G, -1, D).sum(1).transpose(0, 1)
        ds = torch.matmul(doi, _by_head(v[j], G).transpose(1, 2))
        ds = ds.sub_((doi * _by_head(o[i])).sum(-1, keepdim=True)).mul_(p).mul_(a)
        dq[i] = torch.matmul(ds, kj).transpose(0, 1)
        dk[j] += torch.matmul(ds.transpose(1, 2), qi).view(Hkv, G, -1, D).sum(1).transpose(0, 1)
    return {"d" + n: t.to(q.dtype).view(s[n].shape) for n, t in (("q", dq), ("k", dk), ("v", dv))}


def _e4m3(v):
    """The nearest value of four exponent and three mantissa bits, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(v / step) * step


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "emb_fwd":
        rows, ok = _rows_of(case, s["tokens"])
        y = s["table"].view(-1, case["D"])[rows].float() * s["scale"] * ok.unsqueeze(-1)
        return dict(y=y.to(DTYPES[case["dtype"]]))
    if kind == "emb_bwd":
        return _embedding_gradient(s)
    if kind == "rms_fwd":
        h, rstd, y = _normed(s)
        return dict(y=y.to(h.dtype), h=h, rstd=rstd)
    if kind == "rms_8bit":
        h, rstd, _ = _normed(s)
        # (in 64 bits: values next to a border between two of e4m3's)
        y = h.double() * (h.double().square().mean(-1, keepdim=True) + EPS).rsqrt() * s["w"].double()[:, None, None]
        c = (y.abs().amax(-1) / 448.0).clamp(min=SMALLEST_SCALE)
        return dict(y=_e4m3(y / c[..., None]).bfloat16(), scale=c.float(), h=h, rstd=rstd)
    if kind == "rms_bwd":
        dy, r = s["dy"].float(), s["rstd"][..., None]
        hh = s["h"].float() * r
        u = dy * s["w"].float()[:, None, None]
        dx = r * (u - hh * (u * hh).mean(-1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        each = (dy * hh).sum(2)
        out = dict(dx=dx.to(s["h"].dtype), dw=each.mean(1))
        if case["stats"] != "none":
            out["n"] = each.square().sum(-1)
        if case["stats"] == "inner":
            out["q"] = (each * out["dw"][:, None]).sum(-1)
        return out
    if kind == "attn_fwd":
        o, lse = _attention(s)
        return dict(o=o, lse=lse)
    return _attention_gradients(s)


def _own(s):
    import paper_2406_13936_amd as A
    case = s["case"]
    kind = case["kind"]
    if kind == "emb_fwd":
        return dict(y=A.embedding(s["tokens"], s["table"], scale=s["scale"], dtype=DTYPES[case["dtype"]]))
    if kind in ("emb_bwd", "rms_bwd"):
        norms, inner = case["stats"] != "none", case["stats"] == "inner"
        if kind == "emb_bwd":
            dtable, n, q = A.embedding_backward(s["dy"], s["tokens"], case["V"], scale=s["scale"], want_norms=norms, want_inner=inner)
            out = dict(dtable=dtable)
        else:
            dx, dw, n, q = A.rms_norm_backward(s["dy"], s["h"], s["w"], s["rstd"], dh=s["dh"], want_norms=norms, want_inner=inner)
            out = dict(dx=dx, dw=dw)
        if n is not None:
            out["n"] = n
        if q is not None:
            out["q"] = q
        return out
    if kind == "rms_fwd":
        y, h, rstd = A.rms_norm(s["x"], s["w"], residual=s["residual"], eps=EPS)
        return dict(y=y, h=h, rstd=rstd)
    if kind == "rms_8bit":
        y8, c, h, rstd = A.rms_norm_8bit(s["x"], s["w"], residual=s["residual"], eps=EPS)
        return dict(y=y8.bfloat16(), scale=c, h=h, rstd=rstd)      # (bf16 holds every value of e4m3)
    if kind == "attn_fwd":
        o, lse = A.causal_attention(s["q"], s["k"], s["v"], offsets=s["offsets"])
        return dict(o=o, lse=lse)
    dq, dk, dv = A.causal_attention_backward(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], offsets=s["offsets"])
    return dict(dq=dq, dk=dk, dv=dv)


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("emb"):
        M, b, T, V, D = (case[k] for k in ("M", "b", "T", "V", "D"))
        tok = s["tokens"].long()
        inside = ((tok >= 0) & (tok < V)).double()
        tok = tok.clamp(0, V - 1)
        if kind == "emb_fwd":
            return dict(y=torch.stack([s["table"][m][tok[m]].double() * (s["scale"] * inside[m])[..., None] for m in range(M)]))
        dtable = torch.zeros((M, V, D), device="cuda", dtype=torch.float64)
        n = torch.zeros((M, b), device="cuda", dtype=torch.float64)
        signal = s["dy"].double() * (s["scale"] * inside)[..., None]
        for m in range(M):
            dtable[m].index_put_((tok[m].flatten(),), signal[m].reshape(-1, D) / b, accumulate=True)
            for i in range(b if case["stats"] != "none" else 0):
                # ||sum_t x_t e(t)^T||^2 = sum_tu [token_t = token_u] x_t . x_u
                x, t = signal[m, i], tok[m, i]
                n[m, i] = (torch.matmul(x, x.t()) * (t[:, None] == t[None, :])).sum()
        out = dict(dtable=dtable)
        if case["stats"] != "none":
            out["n"] = n
        if case["stats"] == "inner":
            out["q"] = torch.stack([(signal[m] * dtable[m][tok[m]]).sum((1, 2)) for m in range(M)])
        return out
    if kind in ("rms_fwd", "rms_8bit"):
        h = s["x"].double()
        if s["residual"] is not None:
            h = h + s["residual"].double()
        kept = h.to(s["x"].dtype).double()
        rstd = 1.0 / torch.sqrt(torch.linalg.vector_norm(kept, dim=-1) ** 2 / case["D"] + EPS)
        y = torch.einsum("mbtd,mbt,md->mbtd", kept, rstd, s["w"].double())
        if kind == "rms_fwd":
            return dict(y=y, h=h, rstd=rstd)
        c = torch.maximum(torch.amax(torch.abs(y), -1) / 448.0, torch.full_like(rstd, SMALLEST_SCALE))
        v = y / c.unsqueeze(-1)                       # the nearest of e4m3's values: of 2^-6 and more eight to a factor of two
        unit = torch.pow(2.0, torch.clamp(torch.frexp(v).exponent - 4, min=-9).double())
        return dict(y=unit * torch.round(v / unit), scale=c, h=h, rstd=rstd)
    if kind == "rms_bwd":
        h, dy, r = s["h"].double(), s["dy"].double(), s["rstd"].double().unsqueeze(-1)
        u = dy * s["w"].double().view(case["M"], 1, 1, -1)
        dx = r * u - h * r ** 3 * torch.linalg.vecdot(u, h).unsqueeze(-1) / case["D"]
        if s["dh"] is not None:
            dx = dx + s["dh"].double()
        each = (dy * h * r).sum(2)
        bar = each.sum(1) / case["b"]
        out = dict(dx=dx, dw=bar)
        if case["stats"] != "none":
            out["n"] = (each * each).sum(-1)
        if case["stats"] == "inner":
            out["q"] = torch.matmul(each, bar.unsqueeze(-1)).squeeze(-1)
        return out
    # attention, a key head's query heads and some of its queries at a time
    R, Hq, Hkv, D = (case[x] for x in ("rows", "Hq", "Hkv", "D"))
    G, f64 = Hq // Hkv, dict(device="cuda", dtype=torch.float64)
    t = {x: s[x].reshape(R, -1, D) for x in ("q", "k", "v", "o", "do") if x in s}
    lse = s["lse"].view(Hq, R).double() if "lse" in s else None
    out = {"dq": torch.zeros((R, Hq, D), **f64), "dk": torch.zeros((R, Hkv, D), **f64), "dv": torch.zeros((R, Hkv, D), **f64)} if "do" in s \
        else {"o": torch.zeros((R, Hq, D), **f64), "lse": torch.zeros((Hq, R), **f64)}
    start = 0
    for n in _lengths(case):
        for h in range(Hq):
            kk, vv = t["k"][start:start + n, h // G].double(), t["v"][start:start + n, h // G].double()
            for lo in range(0, n, 4096):
                hi = min(n, lo + 4096)
                rows = slice(start + lo, start + hi)
                qq = t["q"][rows, h].double()
                z = torch.matmul(qq, kk[:hi].t()) / math.sqrt(D)
                z = z + torch.full((hi - lo, hi), -math.inf, **f64).triu(lo + 1)
                if "do" not in s:
                    out["lse"][h, rows] = torch.logsumexp(z, 1)
                    out["o"][rows, h] = torch.matmul(torch.softmax(z, 1), vv[:hi])
                    continue
                g = t["do"][rows, h].double()
                p = torch.exp(z - lse[h, rows].unsqueeze(1))
                inner = torch.linalg.vecdot(g, t["o"][rows, h].double()).unsqueeze(1)
                dz = p * (torch.matmul(g, vv[:hi].t()) - inner) / math.sqrt(D)
                out["dq"][rows, h] = torch.matmul(dz, kk[:hi])
                out["dk"][start:start + hi, h // G] += torch.matmul(dz.t(), qq)
                out["dv"][start:start + hi, h // G] += torch.matmul(p.t(), g)
        start += n
    if "do" in s:
        return {x: out[x].view(s[x[1]].shape) for x in out}
    return dict(o=out["o"].view(s["q"].shape), lse=out["lse"].view((Hq,) + s["q"].shape[:-2]))


# ---- what a pass cannot do without ------------------------------------------------------------------------------------

def work(case):
    """Bytes: inputs once (of a table the rows that tokens can name), outputs once.  Flops: of attention the products of the pairs that
    the mask leaves, two forward and five backward."""
    size = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4, "i64": 8}
    e = size[case["dtype"]]
    if case["kind"].startswith("emb"):
        M, V, D, n = case["M"], case["V"], case["D"], case["b"] * case["T"]
        if case["kind"] == "emb_fwd":
            # words of the frequencies above: word i is missing with probability (1 - log(1 + 1/i) / log(V + 1))^n
            named = sum(1.0 - (1.0 - math.log1p(1.0 / i) / math.log(V + 1.0)) ** n for i in range(1, V + 1)) if V <= 200000 else min(n, V)
            return {"bytes": M * (n * (size[case["idx"]] + 1.0 * D * e) + named * D * size[case["table"]]), "flops": 1.0 * M * n * D}
        stats = {"none": 0, "norms": 1, "inner": 2}[case["stats"]]
        return {"bytes": M * (n * (size[case["idx"]] + 1.0 * D * e) + 4.0 * V * D + 4.0 * case["b"] * stats), "flops": M * n * D * (1.0 + 2.0 * stats)}
    if case["kind"].startswith("rms"):
        M, D, rows, p = case["M"], case["D"], case["M"] * case["b"] * case["T"], size[case["param"]]
        if case["kind"] == "rms_bwd":
            stats = {"none": 0, "norms": 1, "inner": 2}[case["stats"]]
            return {"bytes": rows * ((4.0 if case["add"] else 3.0) * D * e + 4) + M * D * (p + 4.0) + 4.0 * M * case["b"] * stats, "flops": 10.0 * rows * D}
        y = 1.0 * D * e if case["kind"] == "rms_fwd" else D + 4.0
        return {"bytes": rows * ((3.0 if case["add"] else 1.0) * D * e + y + 4) + 1.0 * M * D * p, "flops": 5.0 * rows * D}
    pairs = case["Hq"] * sum(n * (n + 1.0) / 2.0 for n in _lengths(case))
    n, heads = sum(_lengths(case)), case["Hq"] + case["Hkv"]
    if case["kind"] == "attn_fwd":
        return {"bytes": n * (2.0 * heads * case["D"] * e + 4.0 * case["Hq"]), "flops": 4.0 * case["D"] * pairs}
    return {"bytes": n * ((4.0 * case["Hq"] + 4.0 * case["Hkv"]) * case["D"] * e + 4.0 * case["Hq"]), "flops": 10.0 * case["D"] * pairs}
