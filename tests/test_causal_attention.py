"""Causal attention over packed sequences with grouped heads and its gradients: refusals on the host, then parity with the definition in 64 bits.

Tolerances count roundings.  U[t] is half a step of a type relative to the value.  A score is a sum of D products in fp32, so a weight p is off by
rel = (D + 4) U32 a sum |q_d k_d| + 8 U32 (1 + |s| + |lse|) of itself, and it and ds are rounded to the type once (in fp16 also by half a step of the smallest
values: 2^-25 of the row's largest weight forward, 2^-37 backward, where weights are held times 2^12).  Results of the exponential below 2^-126, the smallest normal value,
are zeros: TINY of a weight, and of ds that times the difference that it is multiplied with (scores of size 36 give weights of e^-110 = 2^-158)."""
import ctypes as C
import math

import pytest

U32 = 2.0 ** -24
U = {"f32": U32, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = 2.0 ** -126
gpu = pytest.mark.gpu
EINVAL, ENOMEM, EUNSUPPORTED = 1, 2, 5
FAKE, WS = 0x10000000, 0x40000000


def _A():
    import paper_2406_13936_amd as A
    return A


def _dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


# ---- refusals (no GPU call is made) ------------------------------------------------------------------------------------

def _lib():
    from paper_2406_13936_amd import binding as B
    return B.load_library()


def _shape(**k):
    from paper_2406_13936_amd import binding as B
    d = dict(type=0, seqs=3, T=0, Hq=4, Hkv=2, D=16, offsets_type=16, rows=50)
    for n in ("q", "o", "do", "dq"):
        d["ld" + n], d["head_" + n] = 64, 16
    for n in ("k", "v", "dk", "dv"):
        d["ld" + n], d["head_" + n] = 32, 16
    d.update(k)
    return B.AttentionShape(*[d[f] for f, _ in B.AttentionShape._fields_])


@pytest.mark.parametrize("change,status", [
    (dict(type=3), EINVAL), (dict(seqs=0), EINVAL), (dict(rows=0), EINVAL), (dict(Hq=0), EINVAL), (dict(Hkv=0), EINVAL), (dict(D=0), EINVAL),
    (dict(Hkv=3, ldk=48, ldv=48, lddk=48, lddv=48), EINVAL), (dict(offsets_type=3), EINVAL), (dict(offsets_type=0), EINVAL), (dict(offsets_type=0, T=17), EINVAL),
    (dict(ldq=63), EINVAL), (dict(head_k=15), EINVAL), (dict(ldv=-32), EINVAL), (dict(ldo=16), EINVAL),
    (dict(D=129), EUNSUPPORTED), (dict(rows=1 << 31), EUNSUPPORTED), (dict(rows=(1 << 31) - 1, Hq=128, ldq=1 << 11, ldo=1 << 11), EUNSUPPORTED)])
def test_shapes_are_refused(change, status):
    lib, n = _lib(), C.c_size_t(0)
    s = _shape(**change)
    far = [FAKE + i * (1 << 20) for i in range(10)]
    assert lib.abs_causal_attention(C.byref(s), far[0], far[1], far[2], far[3], 0.25, far[4], far[5], 0, WS, 1 << 20, None) == status
    assert lib.abs_causal_attention_backward(C.byref(s), *far[:7], 0.25, *far[7:], 0, WS, 1 << 20, None) == status
    assert lib.abs_causal_attention_workspace_bytes(C.byref(s), 0, C.byref(n)) == status
    assert lib.abs_last_error(None)


@pytest.mark.parametrize("change", [dict(lddo=3), dict(head_dq=8), dict(lddk=31), dict(head_dv=-16)])
def test_strides_of_gradients_are_refused(change):
    lib, n = _lib(), C.c_size_t(0)
    s = _shape(**change)
    assert lib.abs_causal_attention_workspace_bytes(C.byref(s), 0, C.byref(n)) == 0
    assert lib.abs_causal_attention_workspace_bytes(C.byref(s), 1, C.byref(n)) == EINVAL


def test_arguments_are_refused():
    lib, s = _lib(), _shape()
    far = [FAKE + i * (1 << 20) for i in range(12)]

    def fwd(sh=s, scale=0.25, ws=None, nbytes=0, **k):
        d = dict(q=far[0], k=far[1], v=far[2], off=far[3], o=far[4], lse=far[5])
        d.update(k)
        return lib.abs_causal_attention(C.byref(sh), d["q"], d["k"], d["v"], d["off"], scale, d["o"], d["lse"], 0, ws, nbytes, None)
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(off=None), dict(o=None), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(q=far[0] + 2), dict(k=far[1] + 1), dict(off=far[3] + 2), dict(lse=far[5] + 2), dict(o=far[0]), dict(o=far[1] + 64),
                dict(lse=far[4]), dict(o=far[3] - 64), dict(sh=_shape(seqs=65)), dict(sh=_shape(seqs=65), ws=WS + 8, nbytes=1 << 20),
                dict(sh=_shape(seqs=65), ws=far[0] + 256, nbytes=1 << 20), dict(sh=_shape(offsets_type=0, seqs=5, T=10))):
        assert fwd(**bad) == EINVAL, bad
    assert fwd(sh=_shape(seqs=65), ws=WS, nbytes=16) == ENOMEM
    assert lib.abs_causal_attention(None, *far[:4], 0.25, far[4], None, 0, None, 0, None) == EINVAL
    names = ["do", "q", "k", "v", "o", "lse", "off", "dq", "dk", "dv"]

    def bwd(scale=0.25, ws=WS, nbytes=1 << 20, **k):
        d = dict(zip(names, far))
        d.update(k)
        return lib.abs_causal_attention_backward(C.byref(s), *[d[n] for n in names[:7]], scale, *[d[n] for n in names[7:]], 0, ws, nbytes, None)
    for name in names:
        assert bwd(**{name: None}) == EINVAL, name
        assert bwd(**{name: far[11] + 2}) == EINVAL, name
        assert bwd(**{name: WS + 128}) == EINVAL, name
    assert bwd(ws=None) == EINVAL and bwd(ws=WS + 16) == EINVAL and bwd(nbytes=64) == ENOMEM and bwd(scale=0.0) == EINVAL
    for a, b in (("dq", "q"), ("dk", "k"), ("dv", "dk"), ("dq", "do"), ("dk", "o"), ("dv", "lse")):
        assert bwd(**{a: far[names.index(b)]}) == EINVAL, (a, b)
    assert lib.abs_causal_attention_workspace_bytes(C.byref(s), 0, None) == EINVAL


def test_tensors_are_refused():
    import torch
    A = _A()
    q, k = torch.zeros(5, 4, 8), torch.zeros(5, 2, 8)
    with pytest.raises(A.AbsError, match="device memory"):
        A.causal_attention(q, k, k)


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------

def _reference(q, k, v, ends, scale, dtype, do=None, o=None, lse=None):
    """Results and how far they may be off, on [rows, heads, D] tensors: o and lse, or dq, dk and dv."""
    import torch
    q, k, v = (t.double().cpu() for t in (q, k, v))
    R, Hq, D = q.shape
    Hkv = k.shape[1]
    f64 = dict(dtype=torch.float64)
    u = 0.0 if dtype == "f32" else U[dtype]
    if do is None:
        out = {"o": torch.zeros(R, Hq, D, **f64), "lse": torch.zeros(Hq, R, **f64)}
    else:
        do, o, lse = do.double().cpu(), o.double().cpu(), lse.double().cpu()
        out = {"dq": torch.zeros(R, Hq, D, **f64), "dk": torch.zeros(R, Hkv, D, **f64), "dv": torch.zeros(R, Hkv, D, **f64)}
        a1 = do.norm(dim=-1).max() * v.norm(dim=-1).max() if dtype == "f16" else 0.0
    off = {n: torch.zeros_like(t) for n, t in out.items()}
    for a, e in zip(ends, ends[1:]):
        n = e - a
        if n <= 0:
            continue
        mask = torch.ones(n, n).tril().bool()
        for h in range(Hq):
            g = h // (Hq // Hkv)
            qq, kk, vv = q[a:e, h], k[a:e, g], v[a:e, g]
            s = (qq @ kk.T) * scale
            srel = (D + 4) * U32 * scale * (qq.abs() @ kk.abs().T)
            if do is None:
                z = s.masked_fill(~mask, -math.inf)
                top = torch.logsumexp(z, 1)
                p = torch.exp(z - top[:, None])
                rel = torch.where(mask, srel + 8 * U32 * (1 + s.abs() + top.abs()[:, None]), 0.0)
                weight = p * (u + 2 * rel + 2 * rel.amax(1, keepdim=True) + (n + 8) * U32) + mask.double() * TINY
                out["o"][a:e, h], out["lse"][h, a:e] = p @ vv, top
                err = weight @ vv.abs() + (mask.double() * (2.0 ** -25 if dtype == "f16" else 0.0)) @ vv.abs()
                off["o"][a:e, h] = err + U[dtype] * ((p @ vv).abs() + err) + (2.0 ** -25 if dtype == "f16" else 0)
                off["lse"][h, a:e] = 2 * rel.amax(1) + (n + 8) * U32 + 4 * U32 * top.abs()
                continue
            gg, oo, ll = do[a:e, h], o[a:e, h], lse[h, a:e, None]
            p = torch.where(mask, torch.exp(s - ll), 0.0)
            rel = torch.where(mask, srel + 8 * U32 * (1 + s.abs() + ll.abs()), 0.0)
            inner = (gg * oo).sum(1, keepdim=True)
            ds = p * (gg @ vv.T - inner)
            dserr = ds.abs() * (u + 2 * rel + 8 * U32) + p * (D + 4) * U32 * (gg.abs() @ vv.abs().T + (gg * oo).abs().sum(1, keepdim=True))
            perr = p * (u + 2 * rel + 4 * U32) + mask.double() * TINY
            dserr = dserr + mask.double() * TINY * (1 + (gg @ vv.T - inner).abs())
            if dtype == "f16":
                dserr, perr = dserr + mask.double() * 2.0 ** -37 * a1, perr + mask.double() * 2.0 ** -37
            summed = (n * (Hq // Hkv) + 8) * U32
            out["dq"][a:e, h] = scale * ds @ kk
            off["dq"][a:e, h] = scale * (dserr + summed * ds.abs()) @ kk.abs()
            out["dk"][a:e, g] += scale * ds.T @ qq
            off["dk"][a:e, g] += scale * (dserr + summed * ds.abs()).T @ qq.abs()
            out["dv"][a:e, g] += p.T @ gg
            off["dv"][a:e, g] += (perr + summed * p).T @ gg.abs()
    if do is not None:
        for n in out:
            off[n] += U[dtype] * (out[n].abs() + off[n]) + (2.0 ** -25 if dtype == "f16" else 0)
    return out, off


def _check(got, want, off, what):
    import torch
    got = got.double().cpu()
    bad = ~((got - want).abs() <= off + 1e-300)
    assert not bad.any(), (what, int(bad.sum()), torch.nonzero(bad)[:3].tolist(), float(((got - want).abs() / (off + 1e-300)).max()))


def _ends(lens):
    ends = [0]
    for n in lens:
        ends.append(ends[-1] + n)
    return ends


def _tensors(rows, Hq, Hkv, D, dtype, seed=0, size=1.0):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda h: (size * torch.randn((rows, h, D), device="cuda", generator=gen)).to(_dt(dtype))  # noqa: E731
    return r(Hq), r(Hkv), r(Hkv), r(Hq)


LENS = [[1], [2, 1, 3], [31, 32, 33], [0, 63, 0, 64, 65, 0], [127, 128, 129], [300, 5], [1] * 70 + [40] + [0] * 30 + [200], [520]]
HEADS = [(1, 1, 64), (4, 2, 128), (6, 2, 80), (3, 3, 33), (8, 1, 8), (2, 1, 1), (8, 8, 32), (4, 4, 96), (5, 1, 100), (16, 4, 64), (2, 2, 7), (7, 7, 72)]


def _all(q, k, v, do, off, scale, dtype, ends):
    A = _A()
    o, lse = A.causal_attention(q, k, v, offsets=off, scale=scale)
    R, Hq, D = q.shape
    want, err = _reference(q, k, v, ends, scale or 1 / math.sqrt(D), dtype)
    _check(o, want["o"], err["o"], "o")
    _check(lse, want["lse"], err["lse"], "lse")
    grads = A.causal_attention_backward(do, q, k, v, o, lse, offsets=off, scale=scale)
    want, err = _reference(q, k, v, ends, scale or 1 / math.sqrt(D), dtype, do, o, lse)
    for g, n in zip(grads, ("dq", "dk", "dv")):
        _check(g, want[n], err[n], n)
    return (o, lse) + grads


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("which", range(len(LENS)))
def test_packed_sequences(which, dtype):
    import torch
    A = _A()
    lens = LENS[which]
    for Hq, Hkv, D in (HEADS[which % len(HEADS)], HEADS[(which * 5 + 3) % len(HEADS)]):
        ends = _ends(lens)
        q, k, v, do = _tensors(ends[-1], Hq, Hkv, D, dtype, which)
        off = torch.tensor(ends, dtype=torch.int32, device="cuda")
        first = _all(q, k, v, do, off, None, dtype, ends)
        again = A.causal_attention(q, k, v, offsets=off.long())
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
        assert all(torch.equal(a, b) for a, b in zip(A.causal_attention_backward(do, q, k, v, first[0], first[1], offsets=off.long()), first[2:]))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_sequences_of_one_length(heads, dtype):
    import torch
    A = _A()
    Hq, Hkv, D = heads
    for lead, T in (((), 1), ((2,), 45), ((2, 3), 130)):
        n = math.prod(lead)
        q, k, v, do = _tensors(n * T, Hq, Hkv, D, dtype, T)
        ends = _ends([T] * n)
        packed = _all(q, k, v, do, torch.tensor(ends, device="cuda"), 0.3, dtype, ends)
        shaped = [t.view(lead + (T,) + t.shape[1:]) for t in (q, k, v, do)]
        o, lse = A.causal_attention(*shaped[:3], scale=0.3)
        grads = A.causal_attention_backward(shaped[3], *shaped[:3], o, lse, scale=0.3)
        assert lse.shape == (Hq,) + lead + (T,)
        for a, b in zip(packed, (o, lse) + grads):
            assert torch.equal(a.flatten(), b.flatten())


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", [0.01, 6.0])
def test_flat_and_peaked_weights(size, dtype):
    """Scores near zero over long rows (fp16 weights far below 2^-14 of the sum), and scores that one key dominates."""
    import torch
    ends = [0, 1500, 1700]
    q, k, v, do = _tensors(1700, 2, 1, 64, dtype, 4, size)
    v, do = v * (1 / size) if size < 1 else v, do * 2.0 ** -10
    _all(q, k, v, do.to(q.dtype), torch.tensor(ends, device="cuda"), None, dtype, ends)


@gpu
@pytest.mark.parametrize("D", [64, 72, 75])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layouts_and_rows_of_no_sequence(D, dtype):
    import torch
    A = _A()
    ends, R, Hq, Hkv = [3, 70, 70, 201], 230, 6, 2
    q, k, v, do = _tensors(R, Hq, Hkv, D, dtype, D)
    for t in (q, k, v, do):                          # what is in no sequence is not read
        t[:3] = float("nan")
        t[201:] = float("inf")
    off = torch.tensor(ends, dtype=torch.int32, device="cuda")
    o, lse = A.causal_attention(q, k, v, offsets=off)
    grads = A.causal_attention_backward(do, q, k, v, o, lse, offsets=off)
    want, err = _reference(q, k, v, ends, 1 / math.sqrt(D), dtype)
    _check(o, want["o"], err["o"], "o")
    _check(lse, want["lse"], err["lse"], "lse")      # (zeros in rows of no sequence)
    plain = (o, lse) + grads
    for t in plain:
        assert torch.isfinite(t).all()
    for t in (o,) + grads:
        assert (t[:3] == 0).all() and (t[201:] == 0).all() and not (t[3:201] == 0).all()

    def laid(how, *ts):
        if how == "heads":                           # [heads][rows][D]
            return [t.transpose(0, 1).contiguous().transpose(0, 1) for t in ts]
        extra = 8 if how == "columns" else 3
        buf = torch.full((R, sum(t.shape[1] for t in ts), D + extra), 7.0, device="cuda").to(ts[0].dtype)
        views = torch.split(buf, [t.shape[1] for t in ts], dim=1)
        views = [w[..., :D] for w in views]
        for w, t in zip(views, ts):
            w.copy_(t)
        return views
    for how in ("heads", "columns", "odd"):
        q2, k2, v2 = laid(how, q, k, v)
        do2, = laid(how, do)
        out, = laid(how, torch.full_like(o, 5.0))
        o2, lse2 = A.causal_attention(q2, k2, v2, offsets=off, out=out)
        assert o2 is out and (out[:3] == 5).all() and (out[201:] == 5).all()
        assert torch.equal(out[3:201], o[3:201]) and torch.equal(lse2, lse)
        gs = laid(how, *[torch.full_like(t, 5.0) for t in grads])
        got = A.causal_attention_backward(do2, q2, k2, v2, out, lse2, offsets=off, out=tuple(gs))
        for a, b in zip(got, grads):
            assert (a[:3] == 5).all() and (a[201:] == 5).all() and torch.equal(a[3:201], b[3:201])
    with pytest.raises(A.AbsError, match="equally spaced"):
        A.causal_attention(torch.zeros((2, 9, 5, 1, D), device="cuda")[:, :, :4], torch.zeros((2, 9, 4, 1, D), device="cuda"), torch.zeros((2, 9, 4, 1, D), device="cuda"))
    with pytest.raises(A.AbsError, match="offsets"):
        A.causal_attention(q, k, v, offsets=off.float())
    with pytest.raises(A.AbsError, match="rows, heads, D"):
        A.causal_attention(q[None], k[None], v[None], offsets=off)
    with pytest.raises(A.AbsError, match="same type"):
        A.causal_attention(q, k.double().to(torch.float16), v.to(torch.float16))
    with pytest.raises(A.AbsError, match="multiple"):
        A.causal_attention(q[:, :5], k, v)
    with pytest.raises(A.AbsError, match="lse"):
        A.causal_attention_backward(do, q, k, v, o, lse[:, :4])
    with pytest.raises(A.AbsError, match="empty"):
        A.causal_attention(q[:0], k[:0], v[:0])
    with pytest.raises(A.AbsError, match="overlap"):
        A.causal_attention(q, k, v, offsets=off, out=q)


@gpu
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 40), ("f32", 64)])
def test_offsets_that_are_no_list_stay_inside(dtype, D):
    """They are brought into range: whatever comes out, rows outside every sequence stay, and nothing is read or written elsewhere."""
    import torch
    A = _A()
    R = 150
    q, k, v, do = _tensors(R, 2, 2, D, dtype)
    for bad in ([-5, 40, 30, 200], [0, 1 << 30], [100, 20, 20, 10], [0, 150, 0, 150]):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        pad = torch.full((3, R, 2, D), 9.0, device="cuda").to(q.dtype)
        o, lse = A.causal_attention(q, k, v, offsets=off, out=pad[1])
        g = [torch.full((3, R, 2, D), 9.0, device="cuda").to(q.dtype) for _ in range(3)]
        A.causal_attention_backward(do, q, k, v, q, lse, offsets=off, out=tuple(t[1] for t in g))
        for t in [pad] + g:
            assert (t[0] == 9).all() and (t[2] == 9).all()


@gpu
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f16", 80), ("f32", 48)])
@pytest.mark.parametrize("at", [0, 40, 63, 64, 130, 199])
def test_infinities_and_nan_that_a_row_does_not_see(at, dtype, D):
    """A key or value of row `at` is not seen by rows before it; a query's signal reaches keys up to its own only."""
    import torch
    A = _A()
    R = 200
    q, k, v, do = _tensors(R, 2, 1, D, dtype, at)
    o, lse = A.causal_attention(q, k, v)
    for value in (float("inf"), float("nan"), float("-inf")):
        for what in "kv":
            k2, v2 = k.clone(), v.clone()
            (k2 if what == "k" else v2)[at, 0, D // 3] = value
            o2, lse2 = A.causal_attention(q, k2, v2)
            assert torch.equal(o2[:at], o[:at]) and torch.equal(lse2[:, :at], lse[:, :at])
            if what == "v":
                seen = o2[at:, :, D // 3].float()
                # (a weight that is zero in the type makes NaN of an infinity)
                assert (torch.isnan(seen) | (seen == value)).all()
                others = [c for c in range(D) if c != D // 3]
                assert torch.isfinite(o2[:, :, others]).all()
            dq, dk, dv = A.causal_attention_backward(do, q, k2, v2, o, lse)
            dq0 = A.causal_attention_backward(do, q, k, v, o, lse)[0]
            assert torch.equal(dq[:at], dq0[:at])
        base = A.causal_attention_backward(do, q, k, v, o, lse)
        for what in ("q", "do"):
            q2, do2 = q.clone(), do.clone()
            (q2 if what == "q" else do2)[at, 1, D // 3] = value
            dq, dk, dv = A.causal_attention_backward(do2, q2, k, v, o, lse)
            if dtype != "f16" or what == "q":        # (the power of two that holds ds goes by the finite signals)
                assert torch.equal(dk[at + 1:], base[1][at + 1:]) and torch.equal(dv[at + 1:], base[2][at + 1:])
            assert torch.isfinite(dk[at + 1:]).all() and torch.isfinite(dv[at + 1:]).all()
            if what == "do":
                assert not torch.isfinite(dv[:at + 1, 0, D // 3]).any()


@gpu
def test_replayed_graphs_share_nothing_and_streams():
    import torch
    A = _A()
    ends = [[0, 100, 101, 300, 333], [0, 5, 200, 210, 333], [0, 0, 333, 333, 333]]
    sets = [_tensors(333, 4, 2, 64, "f16", s) for s in range(3)]
    q, k, v, do = (t.clone() for t in sets[0])
    many = [torch.tensor(e + [e[-1]] * 80, dtype=torch.int32, device="cuda") for e in ends]
    off = many[0].clone()

    def step(q, k, v, do, off):
        o, lse = A.causal_attention(q, k, v, offsets=off)
        return (o, lse) + A.causal_attention_backward(do, q, k, v, o, lse, offsets=off)
    step(q, k, v, do, off)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step(q, k, v, do, off)
        graphs.append((g, out))
    for i in (1, 2, 0, 2):
        for t, s in zip((q, k, v, do), sets[i]):
            t.copy_(s)
        off.copy_(many[i])
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        want = step(*sets[i], many[i])
        for _, out in graphs:
            assert all(torch.equal(a, c) for a, c in zip(out, want))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = step(*sets[1], many[1])
    s.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, step(*sets[1], many[1])))


@gpu
def test_gradients_against_differences():
    import torch
    A = _A()
    ends = [0, 20, 21, 60]
    q, k, v, c = (t.double() for t in _tensors(60, 4, 2, 16, "f32", 2, 0.7))
    off = torch.tensor(ends, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(6)
    f32 = lambda *t: [x.float() for x in t]  # noqa: E731
    o, lse = A.causal_attention(*f32(q, k, v), offsets=off)
    grads = A.causal_attention_backward(c.float(), *f32(q, k, v), o, lse, offsets=off)
    loss = lambda *t: (A.causal_attention(*f32(*t), offsets=off)[0].double() * c).sum()  # noqa: E731
    e = 2.0 ** -7
    for i, g in enumerate(grads):
        d = torch.randn(g.shape, device="cuda", generator=gen, dtype=torch.float64)
        plus, minus = [q, k, v], [q, k, v]
        plus[i], minus[i] = plus[i] + e * d, minus[i] - e * d
        slope = (loss(*plus) - loss(*minus)) / (2 * e)
        want = (g.double() * d).sum()
        # 3840 results of about 1, off by some 40 U32 each, over e; e^2 / 6 of a third derivative: of 240 rows' weights along scores that d changes by
        # about 3, cubed
        assert abs(slope - want) <= math.sqrt(3840) * 40 * U32 / e * 4 + e * e / 6 * 240 * 27


# ---- many and long sequences --------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("long,D", [(5000, 24), (140000, 8)])
def test_many_sequences_beside_a_long_one(long, D):
    """More than 64 sequences take a list of tiles, in which one of more than 32 tiles is written by a wavefront, and more than 1024 share places.  A sequence's
    results are the same bits alone."""
    import torch
    A = _A()
    lens = [3, 0, 130, 1] * 20 + [long] + [64, 2] * 5
    ends = _ends(lens)
    q, k, v, do = _tensors(ends[-1], 2, 1, D, "bf16", 3)
    off = torch.tensor(ends, device="cuda")
    o, lse = A.causal_attention(q, k, v, offsets=off)
    grads = A.causal_attention_backward(do, q, k, v, o, lse, offsets=off)
    for a, e in zip(ends, ends[1:]):
        if e - a not in (long, 130):
            continue
        one = [t[a:e] for t in (q, k, v, do)]
        o1, lse1 = A.causal_attention(*one[:3])
        assert torch.equal(o[a:e], o1) and torch.equal(lse[:, a:e], lse1)
        for g, g1 in zip(grads, A.causal_attention_backward(one[3], *one[:3], o1, lse1)):
            assert torch.equal(g[a:e], g1)
    a = ends[80]
    for i in (0, 1, long // 2, long - 1):            # some rows of the long one by the definition
        s = (q[a + i].double() @ k[a:a + i + 1, 0].double().T) / math.sqrt(D)
        want = torch.softmax(s, 1) @ v[a:a + i + 1, 0].double()
        # half a step for each weight and the result; scores of these inputs are off by less than 2^-18, sums by i U32
        bound = (torch.softmax(s, 1) @ v[a:a + i + 1, 0].double().abs()) * (2 * U["bf16"] + 2.0 ** -17 + (i + 8) * U32)
        assert ((o[a + i].double() - want).abs() <= bound).all()


@gpu
def test_rows_beyond_32_bits():
    """Heads whose rows end beyond 2^31 values and 2^32 bytes."""
    import torch
    A = _A()
    R, Hq, D, n = 280_000, 64, 128, 100
    q = torch.zeros((R, Hq, D), device="cuda", dtype=torch.bfloat16)
    k, v = torch.zeros((2, R, 1, D), device="cuda", dtype=torch.bfloat16)
    gen = torch.Generator(device="cuda").manual_seed(0)
    for t in (q, k, v):
        t[-n:] = torch.randn(t[-n:].shape, device="cuda", generator=gen).to(torch.bfloat16)
    do = q.flip(1)
    off = torch.arange(0, R + 1, n, dtype=torch.int64, device="cuda")
    o, lse = A.causal_attention(q, k, v, offsets=off)
    grads = A.causal_attention_backward(do, q, k, v, o, lse, offsets=off)
    one = [t[-n:].contiguous() for t in (q, k, v, do)]
    o1, lse1 = A.causal_attention(*one[:3])
    assert torch.equal(o[-n:], o1) and torch.equal(lse[:, -n:], lse1)
    for g, g1 in zip(grads, A.causal_attention_backward(one[3], *one[:3], o1, lse1)):
        assert torch.equal(g[-n:], g1) and (g[:-n] == 0).all()
