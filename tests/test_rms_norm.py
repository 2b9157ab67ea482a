"""Root-mean-square norm behind a residual's addition, its 8-bit results, its gradients and the batch tests' statistics of the gain's: refusals
on the host, then parity with the definition in 64 bits.  Tolerances count roundings as in test_embedding.py."""
import ctypes as C

import pytest

U32 = 2.0 ** -24
U = {"f32": U32, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}
gpu = pytest.mark.gpu
EINVAL, ENOMEM, EUNSUPPORTED = 1, 2, 5
FAKE, WS = 0x10000000, 0x40000000
EPS = 1e-6


def _A():
    import paper_2406_13936_amd as A
    return A


def _dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


# ---- refusals (no GPU call is made) ------------------------------------------------------------------------------------

def _shape(**k):
    from paper_2406_13936_amd import binding as B
    d = dict(M=2, b=3, T=4, D=16, type=0, param_type=0, ldx=16, stride_x=192, ldr=16, stride_r=192, ldh=16, stride_h=192, ldy=16, stride_y=192)
    d.update(k)
    return B.RmsNormShape(*[d[f] for f, _ in B.RmsNormShape._fields_])


def _lib():
    from paper_2406_13936_amd import binding as B
    return B.load_library()


@pytest.mark.parametrize("change,status", [
    (dict(M=0), EINVAL), (dict(b=0), EINVAL), (dict(T=0), EINVAL), (dict(D=0), EINVAL), (dict(type=3), EINVAL), (dict(param_type=1), EINVAL),
    (dict(ldx=15), EINVAL), (dict(stride_x=100), EINVAL), (dict(ldy=-16), EINVAL), (dict(ldr=3), EINVAL), (dict(stride_h=8), EINVAL),
    (dict(M=(1 << 20) + 1), EUNSUPPORTED), (dict(b=1 << 20, T=1 << 12, stride_x=1 << 40, stride_r=1 << 40, stride_h=1 << 40, stride_y=1 << 40), EUNSUPPORTED),
    (dict(D=1 << 27, ldx=1 << 27, ldy=1 << 27), EUNSUPPORTED)])
def test_shapes_are_refused(change, status):
    lib, n = _lib(), C.c_size_t(0)
    s = _shape(**change)
    far = [FAKE + i * (1 << 20) for i in range(8)]
    assert lib.abs_rms_norm(C.byref(s), far[0], far[1], far[2], EPS, far[3], far[4], None, far[5], None) == status
    assert lib.abs_rms_norm_backward(C.byref(s), far[0], far[1], far[2], far[3], far[4], far[5], far[6], None, None, WS, 1 << 20, None) == status
    if not {"ldr", "stride_h"} & set(change):
        assert lib.abs_rms_norm_backward_workspace_bytes(C.byref(s), 1, 1, C.byref(n)) == status
    assert lib.abs_last_error(None)


def test_arguments_are_refused():
    lib, s = _lib(), _shape()
    far = [FAKE + i * (1 << 20) for i in range(12)]

    def fwd(sh=s, eps=EPS, **k):
        d = dict(x=far[0], r=far[1], w=far[2], h=far[3], y=far[4], scale=None, rstd=far[5])
        d.update(k)
        return lib.abs_rms_norm(C.byref(sh), d["x"], d["r"], d["w"], eps, d["h"], d["y"], d["scale"], d["rstd"], None)
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(r=None), dict(h=None), dict(eps=-1.0), dict(eps=float("nan")), dict(x=far[0] + 1),
                dict(r=far[1] + 2), dict(h=far[3] + 2), dict(y=far[4] + 2), dict(w=far[2] + 2), dict(rstd=far[5] + 1), dict(scale=far[6] + 2),
                dict(y=far[3]), dict(h=far[4]), dict(y=far[0] + 64), dict(h=far[1] + 64), dict(y=far[2]), dict(rstd=far[0]), dict(scale=far[5]),
                dict(scale=far[6], y=far[0]), dict(scale=far[6], y=far[0] + 16 * 4 - 1), dict(y=far[0], sh=_shape(ldy=20, stride_y=240)),
                dict(h=far[0], y=far[0])):
        assert fwd(**bad) == EINVAL, bad
    assert lib.abs_rms_norm(None, far[0], None, far[2], EPS, None, far[4], None, None, None) == EINVAL
    names = ["dy", "h", "dh", "w", "rstd", "dx", "dw", "n", "q"]

    def bwd(nbytes=1 << 20, ws=WS, **k):
        d = dict(zip(names, far))
        d.update(k)
        return lib.abs_rms_norm_backward(C.byref(s), *[d[x] for x in names], ws, nbytes, None)
    for name in ("dy", "h", "w", "rstd", "dx", "dw"):
        assert bwd(**{name: None}) == EINVAL, name
    for name in names:
        assert bwd(**{name: far[0] + 2}) == EINVAL, name
        assert bwd(**{name: WS + 128}) == EINVAL, name
    assert bwd(ws=None) == EINVAL and bwd(ws=WS + 16) == EINVAL and bwd(nbytes=16) == ENOMEM
    assert bwd(dx=far[1]) == EINVAL and bwd(dw=far[0] + 64) == EINVAL and bwd(n=far[8]) == EINVAL
    assert lib.abs_rms_norm_backward_workspace_bytes(C.byref(s), 0, 0, None) == EINVAL


def test_tensors_on_the_host_are_refused():
    import torch
    A = _A()
    x, w = torch.zeros(2, 3, 8), torch.zeros(2, 8)
    for call in (A.rms_norm, A.rms_norm_8bit):
        with pytest.raises(A.AbsError, match="device memory"):
            call(x, w)
    with pytest.raises(A.AbsError, match="device memory"):
        A.rms_norm_backward(x, x, w, torch.zeros(2, 3))


# ---- parity ------------------------------------------------------------------------------------------------------------

def _inputs(M, b, T, D, dtype, param, add, seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    x = (0.5 * r(M, b, T, D) + 0.1).to(_dt(dtype))
    res = (r(M, b, T, D) * (1 + 6 * (torch.rand((M, 1, 1, D), device="cuda", generator=gen) < 0.05))).to(_dt(dtype)) if add else None
    w = (1 + 0.3 * r(M, D)).to(_dt(param))
    dy, dh = (r(M, b, T, D) + 0.1).to(_dt(dtype)), r(M, b, T, D).to(_dt(dtype))
    return x, res, w, dy, (dh if add else None)


SIZES = [(1, 1, 1, 1), (2, 3, 4, 7), (3, 5, 1, 128), (2, 7, 3, 129), (2, 2, 19, 520), (1, 3, 5, 1032), (2, 9, 2, 2048), (1, 2, 3, 4100), (1, 3, 1, 8192),
         (2, 2, 2, 8200), (1, 1, 3, 20001)]


@gpu
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("dtype,param", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward(size, dtype, param, add):
    import torch
    A = _A()
    M, b, T, D = size
    x, res, w, _, _ = _inputs(M, b, T, D, dtype, param, add, D)
    y, h, rstd = A.rms_norm(x, w, residual=res, eps=EPS)
    assert torch.equal(h, (x.float() + res.float()).to(x.dtype)) if add else h is x
    h64 = h.double()
    want_r = 1 / torch.sqrt(h64.square().mean(-1) + EPS)
    rel = (D / 2 + 8) * U32                          # a sum of D squares, then a division, a root and an inverse
    assert ((rstd.double() - want_r).abs() <= rel * want_r).all()
    want = h64 * want_r[..., None] * w.double()[:, None, None]
    assert ((y.double() - want).abs() <= want.abs() * (U[dtype] + 2 * rel) + TINY[dtype]).all()
    # 8 bits
    y8, c, h8, r8 = A.rms_norm_8bit(x, w, residual=res, eps=EPS)
    assert torch.equal(h8, h) and torch.equal(r8, rstd) and y8.dtype == torch.float8_e4m3fn
    want_c = (want.abs().amax(-1) / 448).clamp(min=2.0 ** -100)
    assert ((c.double() - want_c).abs() <= 2 * rel * want_c).all()
    got = y8.double() * c.double()[..., None]
    assert ((got - want).abs() <= torch.maximum(want.abs() * 2.0 ** -4, 2.0 ** -10 * c.double()[..., None]) + 4 * rel * want.abs()).all()
    assert torch.isfinite(y8.float()).all() and (y8.float().abs().amax(-1) == 448).all()


@gpu
@pytest.mark.parametrize("dtype,param", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("size", [(2, 7, 3, 129), (1, 40, 64, 2048), (2, 9, 5, 8200), (8, 300, 4, 64)], ids=str)
def test_8_bits_are_the_nearest_values(size, dtype, param):
    """Every value is the nearest of e4m3's to 448 h w / max |h w|, ties to even, next to the borders between two and on them.  h w has at most 48 bits
    and a border 5, so products with 448 = 7 2^6 and of a border with the maximum are exact in 64 bits, and so are comparisons of the two."""
    import torch
    A = _A()
    M, b, T, D = size
    x, _, w, _, _ = _inputs(M, b, T, D, dtype, param, False, D)
    y8 = A.rms_norm_8bit(x, w, eps=EPS)[0].double().cpu()
    p = x.double().cpu() * w.double().cpu()[:, None, None]
    most = p.abs().amax(-1, keepdim=True)
    v = p.abs() * (448 / most)
    units = torch.tensor([2.0 ** e for e in range(-9, 6)], dtype=torch.float64)
    unit = units[torch.clamp(torch.frexp(v).exponent - 4, min=-9).long() + 9]
    low = torch.floor(v / unit)
    side = p.abs() * 448 - (low + 0.5) * unit * most
    n = torch.where(side > 0, low + 1, torch.where(side < 0, low, low + low % 2))
    assert torch.equal(y8, torch.sign(p) * n * unit)


@gpu
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("dtype,param", [("f32", "f32"), ("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("size", SIZES + [(2, 40, 1, 64), (1, 2, 600, 96), (2, 130, 16, 40), (3, 2, 300, 777), (1, 600, 7, 2056)], ids=str)
def test_gradients_and_statistics(size, dtype, param, add):
    import torch
    A = _A()
    M, b, T, D = size
    h, _, w, dy, dh = _inputs(M, b, T, D, dtype, param, True, D + T)
    if not add:
        dh = None
    rstd = (h.float().square().mean(-1) + EPS).rsqrt()
    r, h64, g64, w64 = rstd.double()[..., None], h.double(), dy.double(), w.double()[:, None, None]
    hh, u = h64 * r, g64 * w64
    mean = (u * hh).mean(-1, keepdim=True)
    want = r * (u - hh * mean) + (dh.double() if add else 0)
    # the mean is off by its roundings; every other step by one of its terms
    off = r * hh.abs() * (D + 8) * U32 * (u * hh).abs().mean(-1, keepdim=True) + 8 * U32 * (r * u.abs() + r * (hh * mean).abs() + (dh.double().abs() if add else 0))
    each, mag = (g64 * hh).sum(2), (g64 * hh).abs().sum(2)
    eoff = (T + 4) * U32 * mag
    bar = each.mean(1)
    barerr = (T + b + 8) * U32 * mag.mean(1)
    n, q = each.square().sum(-1), (each * bar[:, None]).sum(-1)
    noff = (2 * each.abs() * eoff + eoff ** 2).sum(-1) + (D + 16) * U32 * n
    qoff = ((mag + eoff) * barerr[:, None] + ((T * D + 16) * U32) * mag * bar.abs()[:, None]).sum(-1)
    first = None
    for norms, inner in ((True, True), (True, False), (False, True), (False, False)):
        dx, dw, n2, q2 = A.rms_norm_backward(dy, h, w, rstd, dh=dh, want_norms=norms, want_inner=inner)
        assert ((dx.double() - want).abs() <= want.abs() * U[dtype] + off * (1 + U[dtype]) + TINY[dtype]).all()
        assert ((dw.double() - bar).abs() <= barerr).all()
        assert (n2 is not None) == norms and (q2 is not None) == inner
        assert n2 is None or ((n2.double() - n).abs() <= noff).all()
        assert q2 is None or ((q2.double() - q).abs() <= qoff).all()
        if first is None:
            first = (dx, dw, n2, q2)
            assert all(torch.equal(a, c) for a, c in zip(first, A.rms_norm_backward(dy, h, w, rstd, dh=dh, want_norms=True, want_inner=True)))


@gpu
@pytest.mark.parametrize("D", [72, 77, 1024, 9000])
def test_layouts_and_results_in_place(D):
    import torch
    A = _A()
    M, b, T = 2, 3, 5
    x, res, w, dy, dh = _inputs(M, b, T, D, "bf16", "f32", True, D)
    y, h, rstd = A.rms_norm(x, w, residual=res)
    y8, c, _, _ = A.rms_norm_8bit(x, w, residual=res)

    def laid(t, how):
        """t's values among others: columns of wider rows, or replicas interleaved by rows"""
        extra = 3 if how == "odd" else 16
        buf = torch.full((b * T, M, D + extra), 99.0, device="cuda").to(t.dtype) if how == "rows" else torch.full((M, b * T, D + extra), 99.0, device="cuda").to(t.dtype)
        v = (buf.transpose(0, 1) if how == "rows" else buf)[..., extra // 2:extra // 2 + D].unflatten(1, (b, T))
        v.copy_(t)
        return v, buf
    for how in ("columns", "rows", "odd"):
        xs, rs, gs, hs = (laid(t, how)[0] for t in (x, res, dy, dh))
        ys, ybuf = laid(torch.zeros_like(x), how)
        got = A.rms_norm(xs, w, residual=rs, out=ys, residual_out=rs)           # h in place of the residual
        assert got[0] is ys and got[1] is rs and torch.equal(rs, h)
        assert torch.equal(ys, y) if how != "odd" and D % 8 == 0 else torch.allclose(ys.float(), y.float(), rtol=2 ** -6)
        assert int((ybuf == 99).sum()) >= ybuf.numel() - y.numel()
        rs.copy_(res)
        o8, obuf = laid(torch.zeros_like(y8), how)
        got8 = A.rms_norm_8bit(xs, w, residual=rs, out=o8)
        assert torch.allclose(got8[1], c, rtol=1e-5) and ((o8.float() - y8.float()).abs() <= y8.float().abs() / 8 + 2 ** -9).all()
        assert torch.equal(A.rms_norm(xs, w, residual=rs, out=xs)[0], ys)       # y in place of x
        want, got = A.rms_norm_backward(dy, h, w, rstd, dh=dh, want_norms=True, want_inner=True), \
            A.rms_norm_backward(gs, laid(h, how)[0], w, rstd, dh=hs, want_norms=True, want_inner=True)
        for a, g in zip(want, got):
            assert torch.allclose(a.float(), g.float(), rtol=2 ** -6, atol=1e-3 * float(a.float().abs().max()))
    with pytest.raises(A.AbsError, match="residual"):
        A.rms_norm(x, w, residual_out=res)
    with pytest.raises(A.AbsError, match="shape and type"):
        A.rms_norm(x, w, residual=res.float())
    with pytest.raises(A.AbsError, match="float8"):
        A.rms_norm_8bit(x, w, out=y)
    with pytest.raises(A.AbsError, match="overlap"):
        A.rms_norm(x, w, residual=res, out=res, residual_out=res)
    with pytest.raises(A.AbsError, match="weight"):
        A.rms_norm(x, w[:1])


@gpu
@pytest.mark.parametrize("D", [40, 2048, 9001])
def test_rows_of_zeros_infinities_and_nan(D):
    import torch
    A = _A()
    x = torch.randn((1, 5, D), device="cuda").to(torch.bfloat16)
    x[0, 0] = 0
    x[0, 1, D // 2] = float("inf")
    x[0, 2, D - 1] = float("nan")
    w = torch.ones((1, D), device="cuda")
    clean = A.rms_norm_8bit(x[:, 3:], w)
    y, _, rstd = A.rms_norm(x, w)
    y8, c, _, _ = A.rms_norm_8bit(x, w)
    assert (y[0, 0] == 0).all() and (y8[0, 0].float() == 0).all() and c[0, 0] == 2.0 ** -100 and abs(float(rstd[0, 0]) - 1000) < 1e-3
    assert torch.isnan(c[0, 1:3]).all() and torch.isnan(y8[0, 1:3].float()).all() and torch.isnan(y[0, 2]).all()
    assert torch.isfinite(y[0, 3:]).all() and torch.equal(y8[:, 3:].float(), clean[0].float()) and torch.equal(c[:, 3:], clean[1])
    # gradients of such rows stay in their sample
    dy = torch.ones_like(x)
    dx, dw, n, q = A.rms_norm_backward(dy, x, w, rstd, want_norms=True, want_inner=True)
    assert torch.isfinite(dx[0, [0, 3, 4]]).all() and torch.isnan(dx[0, 2]).all() and torch.isfinite(n[0, [0, 3, 4]]).all() and torch.isnan(n[0, 2])


@gpu
def test_replayed_graphs_and_another_stream():
    import torch
    A = _A()
    sets = [_inputs(2, 4, 33, 200, "bf16", "f32", True, s) for s in range(3)]
    x, res, w, dy, dh = (t.clone() for t in sets[0])

    def step(x, res, w, dy, dh):
        y, h, rstd = A.rms_norm(x, w, residual=res)
        y8, c, _, _ = A.rms_norm_8bit(x, w, residual=res)
        return (y, h, rstd, y8.float(), c) + A.rms_norm_backward(dy, h, w, rstd, dh=dh, want_norms=True, want_inner=True)
    step(x, res, w, dy, dh)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step(x, res, w, dy, dh)
        graphs.append((g, out))
    for k in (1, 2, 0, 2):
        for t, v in zip((x, res, w, dy, dh), sets[k]):
            t.copy_(v)
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        want = step(*sets[k])
        for _, out in graphs:
            assert all(torch.equal(a, c) for a, c in zip(out, want))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = step(*sets[1])
    s.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, step(*sets[1])))


@gpu
def test_gradients_against_differences():
    import torch
    A = _A()
    x, res, w, c, _ = _inputs(2, 3, 4, 50, "f32", "f32", True, 9)
    gen = torch.Generator(device="cuda").manual_seed(1)
    ch = torch.randn(x.shape, device="cuda", generator=gen)
    d, dw_ = torch.randn(x.shape, device="cuda", generator=gen), torch.randn(w.shape, device="cuda", generator=gen)

    def loss(x, w):
        y, h, rstd = A.rms_norm(x, w, residual=res)
        return (y.double() * c.double()).sum() + (h.double() * ch.double()).sum(), h, rstd
    _, h, rstd = loss(x, w)
    dx, dw, _, _ = A.rms_norm_backward(c, h, w, rstd, dh=ch)
    e = 2.0 ** -8
    for plus, minus, want in (((x + e * d, w), (x - e * d, w), (dx.double() * d.double()).sum()),
                              ((x, w + e * dw_), (x, w - e * dw_), 3 * (dw.double() * dw_.double()).sum())):       # (dw is the mean over b = 3)
        slope = (loss(*plus)[0] - loss(*minus)[0]) / (2 * e)
        # fp32 values of about 1 and 1200 terms: 1200 U32 / e of rounding at most, and e^2 of the third derivative
        assert abs(slope - want) <= 1200 * 8 * U32 / e + 40 * e * e * 24
