"""The operators beside the replicas' step: orthogonalisation, the step with orthogonalised momentum, layer norm with its
gradients and their statistics.  Host-only refusals first, then parity with plain implementations in 64 bits."""
import ctypes as C
import math

import numpy as np
import pytest

U32 = 2.0 ** -24                                     # half a step of fp32, relative
U = {"f32": U32, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}   # half a step of a type relative to the value
COEF = (3.4445, -4.7750, 2.0315)
gpu = pytest.mark.gpu


def _A():
    import paper_2406_13936_amd as A
    return A


def _dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


# ---- refusals (no GPU call is made) ------------------------------------------------------------------------------------

EINVAL, ENOMEM, EUNSUPPORTED = 1, 2, 5
FAKE, WS = 0x10000000, 0x40000000                    # never touched: every call below is refused before a launch


def _lib():
    from paper_2406_13936_amd import binding as B
    return B.load_library()


def _orth(lib, **k):
    d = dict(g=FAKE, gt=0, ldg=16, sg=16 * 16, o=FAKE + (1 << 24), ot=0, ldo=16, so=16 * 16, batch=2, rows=16, cols=16, steps=5,
             coef=None, eps=1e-7, prec=1, ws=WS, nbytes=1 << 24)
    d.update(k)
    return lib.abs_orthogonalize(d["g"], d["gt"], d["ldg"], d["sg"], d["o"], d["ot"], d["ldo"], d["so"], d["batch"], d["rows"],
                                 d["cols"], d["steps"], d["coef"], d["eps"], d["prec"], d["ws"], d["nbytes"], None)


@pytest.mark.parametrize("change,status", [
    (dict(g=None), EINVAL), (dict(o=None), EINVAL), (dict(gt=3), EINVAL), (dict(ot=-1), EINVAL), (dict(batch=0), EINVAL),
    (dict(rows=0), EINVAL), (dict(cols=-1), EINVAL), (dict(steps=0), EINVAL), (dict(steps=33), EINVAL), (dict(eps=0.0), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL), (dict(prec=2), EINVAL), (dict(ws=None), EINVAL),
    (dict(ws=WS + 8), EINVAL), (dict(nbytes=128), ENOMEM), (dict(rows=200, cols=200, ldg=200, ldo=200, sg=40000, so=40000, nbytes=1 << 18), ENOMEM), (dict(ldg=15), EINVAL), (dict(so=100), EINVAL), (dict(sg=-256), EINVAL),
    (dict(g=FAKE + 2), EINVAL), (dict(o=FAKE + 64), EINVAL), (dict(o=FAKE, ot=1), EINVAL), (dict(g=WS), EINVAL),
    (dict(ldg=1 << 40), EINVAL), (dict(rows=1 << 15, cols=1 << 15, ldg=1 << 15, ldo=1 << 15, batch=1), EUNSUPPORTED),
    (dict(coef=(9.0, 9.0, 9.0) * 5), EINVAL),
    # (each step takes what the one before can leave, 1.34, 2.1 and 10, further from 1)
    (dict(steps=4, coef=(4.0, -6.0, 2.6, 3.4, -4.7, 2.0, 2.0, -1.5, 0.5, 1.875, -1.25, 0.375)), EINVAL), (dict(coef=(float("nan"), 0.0, 0.0) * 5), EINVAL), (dict(coef=(0.0, 0.0, 0.0) * 5), EINVAL)])
def test_orthogonalize_refuses(change, status):
    lib = _lib()
    if "coef" in change:
        arr = np.asarray(change["coef"], dtype=np.float32)
        change = dict(change, coef=arr.ctypes.data)
    assert _orth(lib, **change) == status
    assert lib.abs_last_error(None)


def test_orthogonalize_workspace_sizes():
    lib = _lib()
    n = C.c_size_t(0)
    assert lib.abs_orthogonalize_workspace_bytes(3, 150, 200, 1, C.byref(n)) == 0 and n.value > 0
    one = n.value
    assert lib.abs_orthogonalize_workspace_bytes(3, 150, 200, 0, C.byref(n)) == 0 and n.value > one
    assert lib.abs_orthogonalize_workspace_bytes(3, 150, 200, 1, None) == EINVAL
    assert lib.abs_orthogonalize_workspace_bytes(0, 100, 200, 1, C.byref(n)) == EINVAL
    assert lib.abs_orthogonalize_workspace_bytes(1, 1 << 16, 1 << 14, 1, C.byref(n)) == EUNSUPPORTED


@pytest.mark.parametrize("change,status", [
    (dict(x=None), EINVAL), (dict(v=None), EINVAL), (dict(g=FAKE), EINVAL), (dict(v=FAKE + 128), EINVAL), (dict(ws=FAKE), EINVAL),
    (dict(lr=float("nan")), EINVAL), (dict(mu=float("inf")), EINVAL), (dict(wd=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL),
    (dict(xt=7), EINVAL), (dict(gt=7), EINVAL), (dict(nbytes=0), ENOMEM), (dict(v=FAKE + (1 << 24) + 2), EINVAL), (dict(steps=0), EINVAL)])
def test_muon_step_refuses(change, status):
    lib = _lib()
    d = dict(x=FAKE, xt=0, g=FAKE + (1 << 23), gt=0, v=FAKE + (1 << 24), lr=0.1, mu=0.9, wd=0.0, scale=1.0, steps=5, ws=WS, nbytes=1 << 24)
    d.update(change)
    assert lib.abs_muon_step(d["x"], d["xt"], d["g"], d["gt"], d["v"], 2, 16, 16, d["lr"], d["mu"], 1, d["wd"], d["scale"], d["steps"],
                             None, 1e-7, 1, d["ws"], d["nbytes"], None) == status
    assert lib.abs_last_error(None)


def _shape(**k):
    from paper_2406_13936_amd import binding as B
    d = dict(M=2, b=3, T=4, D=16, type=0, param_type=0, ldx=16, stride_x=192, ldy=16, stride_y=192, lddx=16, stride_dx=192)
    d.update(k)
    return B.LayerNormShape(*[d[f] for f, _ in B.LayerNormShape._fields_])


@pytest.mark.parametrize("change,status", [
    (dict(M=0), EINVAL), (dict(b=0), EINVAL), (dict(T=0), EINVAL), (dict(D=0), EINVAL), (dict(type=3), EINVAL),
    (dict(param_type=1), EINVAL), (dict(ldx=15), EINVAL), (dict(stride_x=100), EINVAL), (dict(ldy=-16), EINVAL), (dict(stride_y=0), EINVAL),
    (dict(b=1 << 20, T=1 << 12, stride_x=1 << 40, stride_y=1 << 40), EUNSUPPORTED), (dict(M=(1 << 20) + 1), EUNSUPPORTED),
    (dict(D=1 << 27, ldx=1 << 27, ldy=1 << 27, stride_x=1 << 32, stride_y=1 << 32), EUNSUPPORTED)])
def test_layer_norm_refuses_shapes(change, status):
    lib = _lib()
    s = _shape(**change)
    n = C.c_size_t(0)
    assert lib.abs_layer_norm(C.byref(s), FAKE, FAKE, None, 1e-5, FAKE, None, None, None) == status
    assert lib.abs_layer_norm_backward_workspace_bytes(C.byref(s), 1, 1, C.byref(n)) == status


def test_layer_norm_refuses_arguments():
    lib = _lib()
    s = _shape()
    far = [FAKE + i * (1 << 20) for i in range(10)]
    fwd = lambda x=far[0], g=far[1], be=None, eps=1e-5, y=far[2], m=None, r=None: lib.abs_layer_norm(C.byref(s), x, g, be, eps, y, m, r, None)  # noqa: E731
    for bad in (dict(x=None), dict(g=None), dict(y=None), dict(eps=-1.0), dict(eps=float("nan")), dict(x=far[0] + 1), dict(be=far[3] + 2),
                dict(m=far[3] + 1), dict(y=far[0] + 16)):
        assert fwd(**bad) == EINVAL, bad
    assert lib.abs_layer_norm(None, far[0], far[1], None, 1e-5, far[2], None, None, None) == EINVAL
    names = ["dy", "x", "gamma", "mean", "rstd", "dx", "dgamma", "dbeta", "n", "q"]

    def bwd(nbytes=1 << 20, ws=WS, **k):
        d = dict(zip(names, far))
        d.update(k)
        return lib.abs_layer_norm_backward(C.byref(s), *[d[x] for x in names], ws, nbytes, None)
    for name in ("dy", "x", "gamma", "mean", "rstd", "dx", "dgamma"):
        assert bwd(**{name: None}) == EINVAL, name
    for name in names:
        assert bwd(**{name: far[0] + 2}) == EINVAL, name
    assert bwd(ws=None) == EINVAL and bwd(ws=WS + 16) == EINVAL and bwd(nbytes=16) == ENOMEM
    assert bwd(dx=far[1]) == EINVAL and bwd(dx=far[0] + 64) == EINVAL
    for name in ("dy", "x", "dx"):
        assert bwd(**{name: WS + 128}) == EINVAL, name
    assert lib.abs_layer_norm_backward_workspace_bytes(C.byref(s), 0, 0, None) == EINVAL


def test_tensors_on_the_host_are_refused():
    import torch
    A = _A()
    x = torch.zeros(2, 8, 8)
    with pytest.raises(A.AbsError, match="device memory"):
        A.orthogonalize(x)
    with pytest.raises(A.AbsError, match="device memory"):
        A.muon_step(x, x, x, 0.1)
    with pytest.raises(A.AbsError, match="device memory"):
        A.layer_norm(x, x[:, 0])
    with pytest.raises(A.AbsError, match="float32, bfloat16 or float16"):
        A.orthogonalize(x.double())


def test_sizes_beyond_31_bits_are_refused():
    """(The C entries take 31 bits, and ctypes would drop the rest.)"""
    import torch
    from paper_2406_13936_amd import binding as B
    big = 1 << 32
    with pytest.raises(B.AbsError, match="too large"):
        B._matrices((big + 1, 1, 1), (1, 1, 1), "g")
    with pytest.raises(B.AbsError, match="too large"):
        B._matrices((1 << 16, 1 << 16, 1, 1), (1 << 16, 1, 1, 1), "g")
    with pytest.raises(B.AbsError, match="too large"):
        B._norm_shape(torch.Size((1, big + 2, 4)), (4 * (big + 2), 4, 1), 0, 0, torch.Size((1, big + 2, 4)), (4 * (big + 2), 4, 1), "dy")


# ---- orthogonalisation ----------------------------------------------------------------------------------------------------

def orth64(G, steps=5, coef=None, eps=1e-7):
    """The definition, in 64 bits."""
    X = np.asarray(G, dtype=np.float64)
    X = X / (np.sqrt((X ** 2).sum()) + eps)
    for k in range(steps):
        a, b, c = COEF if coef is None else coef[k]
        A = X @ X.T if X.shape[0] <= X.shape[1] else X.T @ X
        B = b * A + c * (A @ A)
        X = a * X + (B @ X if X.shape[0] <= X.shape[1] else X @ B)
    return X


# Relative errors (2-norm) of the number formats alone, found on the CPU with the roundings put into a 64-bit run: 16-bit operands
# at most 2.4e-3 from 64 rows on (full rank, rank 64, spectra over five decades), hi + lo operands at most 1.3e-5.  Twice that,
# and the rounding of the result.
TOL16, TOL32 = 5e-3, 3e-5


def _orth_tol(prec, m, out):
    return (TOL32 if prec == 0 or m <= 64 else TOL16) + U[out]


def _null_space_tol(G, eps=1e-7):
    """What roundings of X alone can leave in directions in which a low-rank G has nothing: X_k is rounded to fp32 (2^-24 of an
    entry) and held as hi + lo (half a step of hi, 2^-11, and half of lo's, 2^-11 of that), and every later step multiplies what
    lies in those directions by a = 3.4445, 485 over five steps.  (fp32 products leave up to 2.5e-5 in these tests' matrices.)"""
    norms = [np.linalg.norm(orth64(G, steps=k, eps=eps)) for k in range(6)]
    return (2.0 ** -22 + 2.0 ** -24) * sum(COEF[0] ** (5 - k) * norms[k] for k in range(6)) / norms[5]


def _matrix(kind, batch, rows, cols, gen, scale=1.0):
    import torch
    if kind == "full":
        G = torch.randn((batch, rows, cols), generator=gen, dtype=torch.float64)
    else:                                            # rank about an eighth of the smaller side, as a short batch's gradient
        r = max(1, min(rows, cols) // 8)
        G = torch.randn((batch, rows, r), generator=gen, dtype=torch.float64) @ torch.randn((batch, r, cols), generator=gen, dtype=torch.float64)
    return G * scale


def _check_orth(got, G, prec, out, tol=None, **k):
    got = got.double().cpu().numpy()
    for i in range(G.shape[0]):
        want = orth64(G[i].double().cpu().numpy(), **k)
        err, norm = np.linalg.norm(got[i] - want), np.linalg.norm(want)
        assert err <= (tol or _orth_tol(prec, min(want.shape), out)) * norm, (i, err / norm)
        assert np.abs(got[i] - want).max() <= 0.05 * max(np.abs(want).max(), norm / math.sqrt(want.size)), i


@gpu
@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (2, 1, 7), (3, 5, 1), (2, 8, 8), (3, 17, 33), (4, 64, 96), (1, 66, 65), (2, 130, 70),
                                             (3, 72, 129), (2, 333, 129), (1, 127, 128), (2, 256, 512), (1, 520, 264), (2, 300, 1100),
                                             (1, 1030, 515), (1, 640, 640), (17, 40, 24), (4, 1288, 1032), (2, 600, 2056),
                                             (2, 13, 1500), (3, 1300, 30), (2, 50, 1409), (2, 1025, 90), (1, 125, 1100), (1, 2000, 128), (40, 1100, 70), (2, 64, 500), (300, 24, 960)])
@pytest.mark.parametrize("dtype,prec", [("bf16", 1), ("f32", 0), ("f16", None)])
@pytest.mark.parametrize("kind", ["full", "low"])
def test_orthogonalize_against_the_definition(batch, rows, cols, dtype, prec, kind):
    import torch
    A = _A()
    gen = torch.Generator().manual_seed(rows * 1000 + cols)
    G = _matrix(kind, batch, rows, cols, gen).to(_dt(dtype)).cuda()
    keep = G.clone()
    out = A.orthogonalize(G, prec=prec)
    assert out.dtype == G.dtype and torch.equal(G, keep)
    used = 0 if prec is None else prec                # (an fp16 result asks for more than 16-bit products give)
    tol = _orth_tol(used, min(rows, cols), dtype)
    if kind == "low":
        tol += max(_null_space_tol(G[i].double().cpu().numpy()) for i in range(batch))
    _check_orth(out, G, used, dtype, tol=tol)
    assert torch.equal(out, A.orthogonalize(G, prec=prec))              # the same bits every time


@gpu
def test_orthogonalize_types_of_input_and_result():
    import torch
    A = _A()
    gen = torch.Generator().manual_seed(1)
    G = _matrix("full", 2, 96, 136, gen)
    for gt in ("f32", "bf16", "f16"):
        for ot in ("f32", "bf16", "f16"):
            g = G.to(_dt(gt)).cuda()
            out = torch.empty((2, 96, 136), dtype=_dt(ot), device="cuda")
            A.orthogonalize(g, out=out)
            _check_orth(out, g, 1 if ot == "bf16" else 0, ot)


@gpu
@pytest.mark.parametrize("rows,cols", [(24, 40), (40, 24), (100, 72), (65, 203), (200, 136), (136, 200), (150, 161), (300, 264), (9, 1301), (1290, 61)])
def test_orthogonalize_of_strided_and_unaligned_matrices(rows, cols):
    import torch
    A = _A()
    gen = torch.Generator().manual_seed(2)
    for off, ld in ((0, cols + 8), (3, cols + 5), (1, cols), (0, cols)):
        buf = torch.zeros(off + 3 * (rows * ld + 11), dtype=torch.float32, device="cuda")
        g = buf[off:].as_strided((3, rows, cols), (rows * ld + 11, ld, 1))
        g.copy_(_matrix("full", 3, rows, cols, gen))
        for dtype, prec in (("bf16", 1), ("f32", 0)):
            for step in (rows * ld + 11, rows * ld + 16):
                obuf = torch.full((off + 3 * step,), 7.0, device="cuda", dtype=_dt(dtype))
                o = obuf[off:].as_strided((3, rows, cols), (step, ld, 1))
                A.orthogonalize(g, out=o)
                _check_orth(o, g, prec, dtype)
                mask = torch.ones_like(obuf, dtype=torch.bool)
                mask[off:].as_strided((3, rows, cols), (step, ld, 1)).fill_(False)
                assert (obuf[mask] == 7.0).all()                        # nothing outside the matrices is written
        want = A.orthogonalize(g.contiguous())
        A.orthogonalize(g, out=g)                                       # in place
        assert torch.equal(g, want)
    x = torch.zeros((4, 8, 6), device="cuda")
    with pytest.raises(A.AbsError, match="consecutive"):
        A.orthogonalize(x.transpose(1, 2))
    with pytest.raises(A.AbsError, match="equally spaced"):
        A.orthogonalize(torch.zeros((3, 4, 8, 6), device="cuda")[:, ::3])
    with pytest.raises(A.AbsError, match="shape"):
        A.orthogonalize(x, out=torch.zeros((4, 6, 8), device="cuda"))


@gpu
def test_orthogonalize_of_zeros_infinities_and_extreme_sizes():
    import torch
    A = _A()
    gen = torch.Generator().manual_seed(3)
    for rows, cols in ((48, 80), (200, 104), (40, 1200), (1100, 20)):
        G = _matrix("full", 6, rows, cols, gen).float()
        G[1] = 0.0
        G[2, 3, 5] = float("inf")
        G[3, 0, 0] = float("nan")
        G[4] *= 1e34
        G[5] *= 1e-30
        for prec in (0, 1):
            out = A.orthogonalize(G.cuda(), prec=prec, eps=1e-38)
            assert (out[1] == 0).all() and out[2].isnan().all() and out[3].isnan().all()
            for i in (0, 4, 5):
                _check_orth(out[i:i + 1], G[i:i + 1], prec, "f32", eps=1e-38)
        # with the usual eps a tiny matrix stays small: its norm does not reach it
        out = A.orthogonalize(G[5:6].cuda() * 1e24)
        _check_orth(out, G[5:6] * 1e24, 0, "f32", tol=1e-4)


@gpu
def test_orthogonalize_of_very_many_matrices():
    """More than one launch has places for, and more values than 32 bits count."""
    import torch
    A = _A()
    gen = torch.Generator("cuda").manual_seed(5)
    G = torch.randn((4194304 + 3, 1, 1), generator=gen, device="cuda")
    p = G.double() / (G.double().abs() + 1e-7)
    for _ in range(5):
        p = COEF[0] * p + COEF[1] * p ** 3 + COEF[2] * p ** 5
    v, x = torch.zeros_like(G), torch.full_like(G, 2.0)
    assert (A.orthogonalize(G).double() - p).abs().max() <= (TOL32 + U["f32"]) * p.abs().max()
    A.muon_step(x, G, v, 0.5, momentum=0.0, scale=1.0)
    assert torch.equal(v, G) and (x.double() - (2.0 - 0.5 * p)).abs().max() <= 0.5 * TOL32 * p.abs().max() + 2 * 2.5 * U["f32"]
    del G, p, v, x
    G = torch.randn((32771, 264, 256), generator=gen, device="cuda", dtype=torch.bfloat16)
    assert G.numel() > 1 << 31
    out = A.orthogonalize(G)
    some = [0, 1, 32767, 32768, 32770]
    _check_orth(out[some], G[some], 1, "bf16")


@gpu
def test_orthogonalize_with_strides_beyond_32_bits():
    import torch
    A = _A()
    for rows, cols, ld in ((33, 40, 1 << 26), (140, 136, (1 << 24) + 3)):
        step = rows * ld
        buf = torch.empty(step + rows * ld, device="cuda", dtype=torch.bfloat16)
        g = buf.as_strided((2, rows, cols), (step, ld, 1))
        g.copy_(_matrix("full", 2, rows, cols, torch.Generator().manual_seed(6)))
        want = A.orthogonalize(g.contiguous())
        A.orthogonalize(g, out=g)
        assert torch.equal(g, want)


@gpu
@pytest.mark.parametrize("steps,coef", [(1, None), (3, [(1.5, -0.5, 0.0)] * 3), (14, [(1.5, -0.5, 0.0)] * 14), (7, [(1.875, -1.25, 0.375)] * 7),
                                        (4, [COEF, (2.8, -3.0, 1.0), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)]),
                                        (2, [(8.0, 0.0, 0.0), (1.0, 0.0, 0.0)])])
def test_orthogonalize_with_other_coefficients(steps, coef):
    import torch
    A = _A()
    gen = torch.Generator().manual_seed(4)
    for rows, cols in ((40, 56), (136, 80)):
        G = _matrix("full", 2, rows, cols, gen).float().cuda()
        got = A.orthogonalize(G, steps=steps, coefficients=coef)
        _check_orth(got, G, 0, "f32", steps=steps, coef=coef)
        if coef and coef == [coef[0]] * steps:                          # one triple stands for all steps
            assert torch.equal(got, A.orthogonalize(G, steps=steps, coefficients=coef[0]))
    with pytest.raises(A.AbsError, match="triple"):
        A.orthogonalize(G, steps=3, coefficients=[(1.5, -0.5, 0.0)] * 2)
    if steps == 14:                                   # the cubic iteration ends at the orthogonal factor itself
        o = got[0].double().cpu().numpy()
        sv = np.linalg.svd(o, compute_uv=False)
        u, _, vt = np.linalg.svd(G[0].double().cpu().numpy(), full_matrices=False)
        big = sv > 0.999
        assert big.sum() >= 70 and np.abs((u @ vt) - o).max() < 0.5


@gpu
def test_orthogonalize_on_a_stream_and_in_a_graph():
    import torch
    A = _A()
    gen = torch.Generator().manual_seed(5)
    for rows, cols, dtype in ((48, 72, "f32"), (264, 520, "bf16"), (24, 1300, "f32")):
        G = [_matrix("full", 3, rows, cols, gen).to(_dt(dtype)).cuda() for _ in range(3)]
        want = [A.orthogonalize(g) for g in G]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got = [A.orthogonalize(g) for g in G]
            into = G[0].clone()
            out = torch.empty_like(into)
            A.orthogonalize(into, out=out)
        s.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y)
        g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g1):
            A.orthogonalize(into, out=out)
        out2 = torch.empty_like(out)
        with torch.cuda.graph(g2):                    # a second graph of the same shapes has a workspace of its own
            A.orthogonalize(out, out=out2)
        for i in (1, 2, 0, 1):
            into.copy_(G[i])
            g1.replay()
            g2.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want[i])
            assert torch.equal(out2, A.orthogonalize(want[i]))


# ---- the step with orthogonalised momentum ------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 9), (3, 33, 50), (2, 128, 64), (2, 264, 136), (1, 70, 515), (2, 1201, 27)])
@pytest.mark.parametrize("xt,gt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("nesterov", [True, False])
def test_muon_step_against_the_definition(batch, rows, cols, xt, gt, nesterov):
    import torch
    A = _A()
    gen = torch.Generator().manual_seed(rows + cols)
    rnd = lambda s: torch.randn((batch, rows, cols), generator=gen, dtype=torch.float64) * s  # noqa: E731
    x = (rnd(1.0) / math.sqrt(cols)).to(_dt(xt)).cuda()
    v = torch.zeros((batch, rows, cols), device="cuda")
    lr, mu, wd, scale = 0.02, 0.9, 0.1, 0.2 * math.sqrt(max(rows, cols))
    for step in range(3):
        g = rnd(1e-3).to(_dt(gt)).cuda()
        x0, v0 = x.double().cpu().numpy(), v.double().cpu().numpy()
        A.muon_step(x, g, v, lr, momentum=mu, weight_decay=wd, nesterov=nesterov)
        g64 = g.double().cpu().numpy()
        v64 = mu * v0 + g64
        got_v, got_x = v.double().cpu().numpy(), x.double().cpu().numpy()
        mu32 = float(np.float32(mu))                  # the momentum the kernel has: one rounding of the constant, one of the sum
        assert (np.abs(got_v - v64) <= 2 * U32 * (np.abs(v64) + np.abs(mu32 * v0))).all()
        for i in range(batch):
            o = orth64(g64[i] + mu * v64[i] if nesterov else v64[i])
            want = (1.0 - lr * wd) * x0[i] - lr * scale * o
            # the factor's own error, a handful of fp32 roundings of the step, one rounding of x to its type
            tol = lr * scale * np.linalg.norm(o) * _orth_tol(0 if xt == "f32" else 1, min(rows, cols), "f32") + (U[xt] + 6 * U32) * np.linalg.norm(want) \
                + 6 * U32 * np.linalg.norm(x0[i])
            assert np.linalg.norm(got_x[i] - want) <= tol, (step, i)


@gpu
def test_muon_step_alone_on_a_matrix_and_in_a_graph():
    import torch
    A = _A()
    gen = torch.Generator().manual_seed(6)
    x = torch.randn((40, 24), generator=gen).cuda()
    g = [torch.randn((40, 24), generator=gen).cuda() for _ in range(4)]
    v = torch.zeros_like(x)
    ex, ev = x.clone(), v.clone()
    into = g[0].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        A.muon_step(x.clone(), into, v.clone(), 0.1)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.muon_step(x, into, v, 0.1, weight_decay=0.01)
    for i in range(4):
        into.copy_(g[i])
        graph.replay()
        A.muon_step(ex, g[i], ev, 0.1, weight_decay=0.01)
        torch.cuda.synchronize()
        assert torch.equal(x, ex) and torch.equal(v, ev), i
    with pytest.raises(A.AbsError, match="contiguous"):
        A.muon_step(x.t(), g[0].t(), v.t(), 0.1)
    with pytest.raises(A.AbsError, match="float32"):
        A.muon_step(x, g[0], v.to(torch.bfloat16), 0.1)
    with pytest.raises(A.AbsError, match="overlap"):
        A.muon_step(x, x, v, 0.1)


# ---- layer norm ---------------------------------------------------------------------------------------------------------------

DS = [1, 2, 7, 8, 16, 100, 128, 129, 264, 512, 513, 777, 2048, 2050, 2056, 4096, 5000, 8192, 8193, 10008]


def _sums(D):
    """Most roundings on a value's way through a row's sum: a lane adds at most 32 values (or D / 256 of a long row), then lanes
    and wavefronts."""
    return max(32, D // 256 + 1) + 12


def _ln_inputs(M, b, T, D, dtype, ptype, seed=0):
    import torch
    gen = torch.Generator().manual_seed(seed + D)
    x = (torch.randn((M, b, T, D), generator=gen) * 1.5 + 0.7).to(_dt(dtype)).cuda()
    w = (1.0 + 0.3 * torch.randn((M, D), generator=gen)).to(_dt(ptype)).cuda()
    bias = (0.3 * torch.randn((M, D), generator=gen)).to(_dt(ptype)).cuda()
    dy = (torch.randn((M, b, T, D), generator=gen) + 0.2).to(_dt(dtype)).cuda()
    return x, w, bias, dy


def _n(t):
    return t.double().cpu().numpy()


def _check_forward(y, mean, rstd, x, w, bias, eps, dtype):
    x, w = _n(x), _n(w)[:, None, None]
    be = _n(bias)[:, None, None] if bias is not None else np.zeros_like(w)
    D = x.shape[-1]
    k = _sums(D)
    mu = x.mean(-1, keepdims=True)
    d = x - mu
    var = (d ** 2).mean(-1, keepdims=True)
    r = 1.0 / np.sqrt(var + eps)
    e_mu = (k + 2) * U32 * np.abs(x).mean(-1, keepdims=True)
    e_d = e_mu + U32 * np.abs(d)
    e_var = 2 * np.abs(d).mean(-1, keepdims=True) * e_mu + e_mu ** 2 + (k + 4) * U32 * var + 2 * U32 * var
    e_r = r * (e_var / (2 * (var + eps)) + 4 * U32) * 1.01
    want = d * r * w + be
    e_y = np.abs(w) * (e_d * r + np.abs(d) * e_r) * 1.01 + 4 * U32 * (np.abs(d * r * w) + np.abs(be))
    if mean is not None:
        assert (np.abs(_n(mean)[..., None] - mu) <= e_mu).all()
        assert (np.abs(_n(rstd)[..., None] - r) <= e_r).all()
    tiny = 2.0 ** -25 if dtype == "f16" else 0.0      # fp16 results below its normal range
    assert (np.abs(_n(y) - want) <= e_y + U[dtype] * (np.abs(want) + e_y) + tiny).all()


@gpu
@pytest.mark.parametrize("D", DS)
@pytest.mark.parametrize("dtype,ptype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
def test_layer_norm_against_the_definition(D, dtype, ptype):
    import torch
    A = _A()
    for M, b, T in ((1, 1, 1), (3, 5, 7)):
        x, w, bias, _ = _ln_inputs(M, b, T, D, dtype, ptype)
        y, mean, rstd = A.layer_norm(x, w, bias, eps=1e-5)
        _check_forward(y, mean, rstd, x, w, bias, 1e-5, dtype)
        y2, _, _ = A.layer_norm(x, w)
        _check_forward(y2, None, None, x, w, None, 1e-5, dtype)
        z = x.clone()
        A.layer_norm(z, w, bias, out=z)
        assert torch.equal(z, y)


def _check_backward(got, dy, x, w, mean, rstd, has_bias, dtype):
    dx, dw, db, n, q = got
    x, dy, g, mu, r = _n(x), _n(dy), _n(w)[:, None, None], _n(mean)[..., None], _n(rstd)[..., None]
    M, b, T, D = x.shape
    k = _sums(D)
    xh, h = (x - mu) * r, dy * g
    a, c = h.mean(-1, keepdims=True), (h * xh).mean(-1, keepdims=True)
    want = r * (h - a - xh * c)
    e_a = (k + 3) * U32 * np.abs(h).mean(-1, keepdims=True)
    e_c = (k + 6) * U32 * np.abs(h * xh).mean(-1, keepdims=True)
    e = r * (e_a + np.abs(xh) * e_c + 6 * U32 * (np.abs(h) + np.abs(a) + np.abs(xh * c))) * 1.01
    tiny = 2.0 ** -25 if dtype == "f16" else 0.0
    assert (np.abs(_n(dx) - want) <= e + U[dtype] * (np.abs(want) + e) + tiny).all()
    gw, gb = (dy * xh).sum(2), dy.sum(2)
    # sums over rows: no value meets more than one rounding per row of the replica and a few on the way
    N = b * T + 16
    lim = lambda s: (N + 4) * U32 * np.abs(s).sum((1, 2)) / b  # noqa: E731
    bw, bb = gw.mean(1), gb.mean(1)
    assert (np.abs(_n(dw) - bw) <= lim(dy * xh)).all()
    near = lambda p, want, rel: np.linalg.norm(_n(p) - want) <= rel * np.linalg.norm(want) + 1e-30  # noqa: E731
    # (and as a whole far nearer than that bound: roundings do not all point one way)
    assert near(dw, bw, 1e-5)
    if has_bias:
        assert (np.abs(_n(db) - bb) <= lim(dy)).all() and near(db, bb, 1e-5)
    else:
        assert db is None
        gb, bb = np.zeros_like(gb), np.zeros_like(bb)
    e_w = (T + 8) * U32 * np.abs(dy * xh).sum(2)
    e_b = (T + 8) * U32 * np.abs(dy).sum(2) if has_bias else np.zeros_like(gb)
    if n is not None:
        wn = (gw ** 2).sum(-1) + (gb ** 2).sum(-1)
        tol = (2 * np.abs(gw) * e_w + e_w ** 2 + 2 * np.abs(gb) * e_b + e_b ** 2).sum(-1) + (2 * k + 8) * U32 * wn
        assert (np.abs(_n(n) - wn) <= tol).all() and near(n, wn, 1e-5)
    if q is not None:
        wq = (gw * bw[:, None]).sum(-1) + (gb * bb[:, None]).sum(-1)
        e_bw, e_bb = lim(dy * xh)[:, None], (lim(dy) if has_bias else np.zeros_like(bb))[:, None]
        mag = (np.abs(dy * xh).sum(2) * np.abs(bw)[:, None]).sum(-1) + (np.abs(dy).sum(2) * np.abs(bb)[:, None]).sum(-1)
        tol = (e_w * np.abs(bw)[:, None] + np.abs(gw) * e_bw + e_b * np.abs(bb)[:, None] + np.abs(gb) * e_bb).sum(-1) \
            + (T * (D // 16 + 8) + 16) * U32 * mag
        assert (np.abs(_n(q) - wq) <= tol).all()
        assert np.linalg.norm(_n(q) - wq) <= 1e-5 * np.linalg.norm(mag)


@gpu
@pytest.mark.parametrize("D", DS)
@pytest.mark.parametrize("dtype,ptype", [("f32", "f32"), ("bf16", "f32"), ("f16", "f16")])
def test_layer_norm_gradients_and_statistics(D, dtype, ptype):
    A = _A()
    for M, b, T in ((1, 1, 1), (2, 9, 1), (3, 5, 7), (2, 3, 150)):
        x, w, bias, dy = _ln_inputs(M, b, T, D, dtype, ptype)
        _, mean, rstd = A.layer_norm(x, w, bias)
        for has_bias, norms, inner in ((True, True, True), (False, True, True), (True, False, False), (True, True, False), (True, False, True)):
            if (M, b, T) != (3, 5, 7) and not (has_bias and norms and inner):
                continue
            got = A.layer_norm_backward(dy, x, w, mean, rstd, has_bias=has_bias, want_norms=norms, want_inner=inner)
            assert (got[3] is not None) == norms and (got[4] is not None) == inner
            _check_backward(got, dy, x, w, mean, rstd, has_bias, dtype)


@gpu
@pytest.mark.parametrize("M,b,T,D", [(1, 4000, 1, 96), (2, 1500, 3, 200), (8, 2, 700, 520), (1, 3, 2000, 40), (300, 4, 2, 24), (1, 2, 5000, 16),
                                     (2, 1, 300, 2304)])
def test_layer_norm_gradients_of_many_rows(M, b, T, D):
    import torch
    A = _A()
    x, w, bias, dy = _ln_inputs(M, b, T, D, "f32", "f32")
    y, mean, rstd = A.layer_norm(x, w, bias)
    _check_forward(y, mean, rstd, x, w, bias, 1e-5, "f32")
    for norms, inner in ((True, True), (False, False)):
        got = A.layer_norm_backward(dy, x, w, mean, rstd, want_norms=norms, want_inner=inner)
        _check_backward(got, dy, x, w, mean, rstd, True, "f32")
        again = A.layer_norm_backward(dy, x, w, mean, rstd, want_norms=norms, want_inner=inner)
        for p, r in zip(got, again):
            assert p is None or torch.equal(p, r)


@gpu
def test_layer_norm_gradient_against_differences():
    """(f(x + h) - f(x - h)) / 2h of f = sum_i <dy_i, y_i> along random directions of x, gamma and beta, in 64 bits."""
    A = _A()
    M, b, T, D = 1, 3, 4, 24
    x, w, bias, dy = _ln_inputs(M, b, T, D, "f32", "f32")
    _, mean, rstd = A.layer_norm(x, w, bias, eps=1e-5)
    dx, dw, db, _, _ = A.layer_norm_backward(dy, x, w, mean, rstd)
    x, w, bias, dy = _n(x), _n(w), _n(bias), _n(dy)

    def f(x, w, be):
        d = x - x.mean(-1, keepdims=True)
        return (dy * (d / np.sqrt((d ** 2).mean(-1, keepdims=True) + 1e-5) * w[:, None, None] + be[:, None, None])).sum()
    rng = np.random.default_rng(0)
    for name, at, grad, scale in (("x", 0, _n(dx), 1.0), ("w", 1, _n(dw), b), ("b", 2, _n(db), b)):
        args = [x, w, bias]
        v = rng.standard_normal(args[at].shape)
        eps = 1e-5
        lo, hi = list(args), list(args)
        lo[at], hi[at] = args[at] - eps * v, args[at] + eps * v
        num = (f(*hi) - f(*lo)) / (2 * eps)
        assert abs(num - scale * (grad * v).sum()) <= 1e-4 * np.abs(scale * grad * v).sum(), name


@gpu
def test_layer_norm_of_strided_rows():
    import torch
    A = _A()
    for D, ld, off in ((24, 24, 1), (40, 48, 0), (33, 37, 2), (264, 272, 8), (600, 601, 0),
                       (3, 5, 1), (7, 7, 3), (9, 11, 1), (1501, 1503, 1), (5001, 5001, 2), (8190, 8191, 1)):
        M, b, T = 2, 3, 4
        big = torch.randn(off + M * (b * T * ld + 5), device="cuda", generator=torch.Generator("cuda").manual_seed(D)).to(torch.bfloat16)
        x = big[off:].as_strided((M, b, T, D), (b * T * ld + 5, T * ld, ld, 1))
        w, bias = torch.randn((M, D), device="cuda"), torch.randn((M, D), device="cuda")
        y, mean, rstd = A.layer_norm(x, w, bias)
        ref = A.layer_norm(x.contiguous(), w, bias)
        _check_forward(y, mean, rstd, x, w, bias, 1e-5, "bf16")
        dy = big.flip(0)[:off + M * (b * T * ld + 5)][off:].as_strided((M, b, T, D), (b * T * ld + 5, T * ld, ld, 1))
        got = A.layer_norm_backward(dy, x, w, ref[1], ref[2], want_norms=True, want_inner=True)
        _check_backward(got, dy, x, w, ref[1], ref[2], True, "bf16")
        obig = torch.full_like(big, 3.0)
        o = obig[off:].as_strided((M, b, T, D), (b * T * ld + 5, T * ld, ld, 1))
        A.layer_norm(x, w, bias, out=o)
        assert torch.equal(o, y)
        mask = torch.ones_like(obig, dtype=torch.bool)
        mask[off:].as_strided((M, b, T, D), (b * T * ld + 5, T * ld, ld, 1)).fill_(False)
        assert (obig[mask] == 3.0).all()
    with pytest.raises(A.AbsError, match="equally spaced"):
        A.layer_norm(torch.zeros((2, 4, 6, 8), device="cuda")[:, :, ::2][:, :, :2], torch.zeros((2, 8), device="cuda"))
    with pytest.raises(A.AbsError, match="consecutive"):
        A.layer_norm(torch.zeros((2, 4, 8, 6), device="cuda").transpose(2, 3), torch.zeros((2, 8), device="cuda"))
    with pytest.raises(A.AbsError, match=r"\[M, D\]"):
        A.layer_norm(torch.zeros((2, 4, 8), device="cuda"), torch.zeros((2, 9), device="cuda"))


@gpu
def test_layer_norm_beyond_32_bits():
    """Strides, and numbers of values, that 32 bits do not hold."""
    import torch
    A = _A()
    gen = torch.Generator("cuda").manual_seed(7)
    for D in (40, 1000, 9000):
        M, b, ld, step = 2, 3, 1 << 29, 1 << 31
        bufs = [torch.empty(step + 2 * ld + D, device="cuda", dtype=torch.bfloat16) for _ in range(3)]
        x, dy, y = (t.as_strided((M, b, 1, D), (step, ld, ld, 1)) for t in bufs)
        for t in (x, dy):
            t.copy_(torch.randn((M, b, 1, D), generator=gen, device="cuda"))
        w, bias = torch.randn((M, D), generator=gen, device="cuda"), torch.randn((M, D), generator=gen, device="cuda")
        want = A.layer_norm(x.contiguous(), w, bias)
        got = A.layer_norm(x, w, bias, out=y)
        assert all(torch.equal(p, r) for p, r in zip(got, want))
        ref = A.layer_norm_backward(dy.contiguous(), x.contiguous(), w, *want[1:], want_norms=True, want_inner=True)
        got = A.layer_norm_backward(dy, x, w, *want[1:], want_norms=True, want_inner=True)
        assert all(torch.equal(p, r) for p, r in zip(got, ref))
        del bufs, x, dy, y
    n, D = (1 << 20) + 5, 2056
    x = torch.randn((1, n, D), generator=gen, device="cuda", dtype=torch.bfloat16)
    dy = torch.randn((1, n, D), generator=gen, device="cuda", dtype=torch.bfloat16)
    w, bias = torch.randn((1, D), generator=gen, device="cuda"), torch.randn((1, D), generator=gen, device="cuda")
    y, mean, rstd = A.layer_norm(x, w, bias)
    dx, _, _, ni, _ = A.layer_norm_backward(dy, x, w, mean, rstd, want_norms=True)
    tail = slice(n - 7, n)
    assert y.numel() > 1 << 31
    for p, r in zip((y, mean, rstd), A.layer_norm(x[:, tail], w, bias)):
        assert torch.equal(p[:, tail], r)
    part = A.layer_norm_backward(dy[:, tail], x[:, tail], w, mean[:, tail].contiguous(), rstd[:, tail].contiguous(), want_norms=True)
    assert torch.equal(dx[:, tail], part[0]) and torch.equal(ni[:, tail], part[3])


@gpu
@pytest.mark.parametrize("D", [24, 300, 1024, 9000])
def test_layer_norm_keeps_rows_apart(D):
    """A row with an infinity or NaN, constant rows and rows of huge values do not reach the others."""
    import torch
    A = _A()
    x, w, bias, dy = _ln_inputs(1, 6, 2, D, "f32", "f32")
    good = A.layer_norm(x, w, bias)[0]
    y0 = x.clone()
    y0[0, 1, 0, D // 2] = float("nan")
    y0[0, 2, 1, 0] = float("inf")
    y0[0, 3, 0] = 5.0
    y0[0, 4, 1] = 0.0
    y, mean, rstd = A.layer_norm(y0, w, bias)
    assert y[0, 1, 0].isnan().all() and not y[0, 2, 1].isfinite().any()
    assert torch.equal(y[0, 3, 0], bias[0]) and torch.equal(y[0, 4, 1], bias[0])
    for i, t in ((0, 0), (0, 1), (1, 1), (2, 0), (3, 1), (4, 0), (5, 0), (5, 1)):
        assert torch.equal(y[0, i, t], good[0, i, t]), (i, t)
    dx, dw, db, n, q = A.layer_norm_backward(dy, y0, w, mean, rstd, want_norms=True)
    base = A.layer_norm_backward(dy, x, w, *A.layer_norm(x, w, bias)[1:], want_norms=True)
    assert torch.equal(dx[0, 0], base[0][0, 0]) and torch.equal(dx[0, 5], base[0][0, 5])
    assert n[0, 1].isnan() and not n[0, 2].isfinite() and torch.equal(n[0, [0, 5]], base[3][0, [0, 5]]) and n[0, 3].isfinite()
    assert torch.equal(db, base[2])


@gpu
def test_layer_norm_on_a_stream_and_in_a_graph():
    import torch
    A = _A()
    for M, b, T, D in ((2, 5, 1, 96), (2, 3, 140, 320), (1, 2, 3, 9000)):
        ins = [_ln_inputs(M, b, T, D, "bf16", "f32", seed=s) for s in range(3)]

        def both(x, w, bias, dy):
            y, mean, rstd = A.layer_norm(x, w, bias)
            return (y,) + A.layer_norm_backward(dy, x, w, mean, rstd, want_norms=True, want_inner=True)
        want = [both(*i) for i in ins]
        buf = [t.clone() for t in ins[0]]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got = both(*buf)
        s.synchronize()
        for p, r in zip(got, want[0]):
            assert torch.equal(p, r)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = both(*buf)
        for i in (1, 2, 0, 1):
            for t, src in zip(buf, ins[i]):
                t.copy_(src)
            graph.replay()
            torch.cuda.synchronize()
            for p, r in zip(out, want[i]):
                assert torch.equal(p, r), i


# ---- together -----------------------------------------------------------------------------------------------------------------

@gpu
def test_a_block_trained_with_norms_statistics_steps_and_averages():
    """Two replicas of y = W ln(x) by the framework's calls: forward, gradients of the norm and of the weights, the statistics of
    both together against explicit per-sample gradients, an orthogonalised step and the replica average."""
    import torch
    A = _A()
    M, b, fin, fout = 2, 12, 40, 24
    gen = torch.Generator().manual_seed(9)
    x = torch.randn((M, b, fin), generator=gen).to(torch.bfloat16).cuda()
    w = (1.0 + 0.1 * torch.randn((M, fin), generator=gen)).cuda()
    bias = (0.1 * torch.randn((M, fin), generator=gen)).cuda()
    W = (torch.randn((M, fout, fin), generator=gen) / math.sqrt(fin)).to(torch.bfloat16).cuda()
    delta = torch.randn((M, b, fout), generator=gen).to(torch.bfloat16).cuda()      # signals at y
    a, mean, rstd = A.layer_norm(x, w, bias)
    res, n1, q1, G = A.layer_stats([a], [delta], want_per_sample=True, want_gbar=True)
    da = torch.bmm(delta.float(), W.float()).to(torch.bfloat16)
    dx, dw, db, n2, q2 = A.layer_norm_backward(da, x, w, mean, rstd, want_norms=True, want_inner=True)
    a64, d64, da64 = _n(a), _n(delta), _n(da)
    xh = (_n(x) - _n(mean)[..., None]) * _n(rstd)[..., None]
    for m in range(M):
        per = np.concatenate([(d64[m][:, :, None] * a64[m][:, None, :]).reshape(b, -1), da64[m] * xh[m], da64[m]], 1)
        bar = per.mean(0)
        S1, S2 = (per ** 2).sum(), (bar ** 2).sum()
        assert abs(float(n1[m].sum() + n2[m].sum()) - S1) <= 1e-4 * S1
        got2 = res[m].gbar_sq + float((dw[m].double() ** 2).sum() + (db[m].double() ** 2).sum())
        assert abs(got2 - S2) <= 1e-4 * S2
        q = (q1[m] + q2[m]).double().cpu().numpy()
        # (the linear layer's products take gbar rounded to bf16)
        assert np.linalg.norm(q - per @ bar) <= 4e-3 * np.linalg.norm(np.abs(per) @ np.abs(bar))
    g = G.view(M, fout, fin)
    v = torch.zeros((M, fout, fin), device="cuda")
    W0 = _n(W)
    A.muon_step(W, g, v, 0.05, momentum=0.9)
    for m in range(M):
        want = W0[m] - 0.05 * 0.2 * math.sqrt(fin) * orth64(1.9 * _n(g)[m])
        assert np.linalg.norm(_n(W)[m] - want) <= (2 * U["bf16"]) * np.linalg.norm(want)
    P = W.reshape(M, -1)
    mean_w = P.float().mean(0)
    A.average_bf16(P)
    assert torch.equal(P[0], P[1]) and (P[0].float() - mean_w).abs().max() <= 2 * U["bf16"] * mean_w.abs().max()


# ---- as the replicas' inner optimizer -------------------------------------------------------------------------------------------

def test_muon_configurations_without_a_gpu():
    from paper_2406_13936_amd import binding as B
    lib = B.load_library()

    def size(dims, opt, prec=B.PREC_F32):
        d = (C.c_int * len(dims))(*dims)
        cfg = B._Config(len(dims) - 1, d, 1, 1, prec, 2, 64, opt, 0.9, 0.9, 0.999, 1e-8, 0, 1, None, None, 0)
        n = C.c_size_t(0)
        return lib.abs_workspace_bytes(C.byref(cfg), 100, C.byref(n)), n.value
    st, muon = size((24, 16, 4), 4)
    st2, adam = size((24, 16, 4), 2)
    assert st == 0 and st2 == 0 and muon > adam
    assert size((24, 4), 4)[0] == EINVAL and b"hidden layer" in lib.abs_last_error(None)
    assert size((24, 16, 4), 5)[0] == EINVAL
    assert size((1 << 16, 1 << 14, 4), 4)[0] == EUNSUPPORTED


def _muon_case(dims, prec, b, M, hb=True, mu=0.9, wd=0.05):
    from oracle import abs_oracle as O
    from paper_2406_13936_amd import workloads as W
    w = W.Workload("muon", dims, W.ACT_GELU, hb, prec, N=1024, M=M, H=1, rounds=1, b0=b, b_cap=b + 5, opt=W.OPT_MUON, lr=0.02,
                   momentum=mu, weight_decay=wd, test=W.TEST_IP, theta=0.9, data="teacher_mlp", seed=21)
    X, y = W.make_dataset(w)
    x0 = W.make_x0(w)
    return w, X, y, x0, _A().Replicas.from_workload(w, X, y, x0), O.Net(w.dims, w.act, hb)


def _check_muon_step(w, net, before, after, g, state0, state1, t, prec):
    """One worker's step from its own batch gradient g (fp32 values, taken as they are): parameters and optimizer state."""
    L = len(w.dims) - 1
    parts = lambda z: net.unpack(np.asarray(z, dtype=np.float64))  # noqa: E731  (one (W, beta) per layer)
    x, y, g, (v0, m0), (v1, m1) = parts(before), parts(after), parts(g), [parts(s) for s in state0], [parts(s) for s in state1]
    lr, wd, mu = w.lr, w.weight_decay, w.momentum

    def adam(x, y, g, v0, m0, v1, m1):
        m, v = w.beta1 * m0 + (1 - w.beta1) * g, w.beta2 * v0 + (1 - w.beta2) * g * g
        # beta1 in fp32 is off by up to 2^-24 of itself, and 1 - beta1 (exact from there) by as much absolutely; two products and their
        # sum are rounded: 2^-24 (beta1 |g| + 2 beta1 |m0| + (1 - beta1) |g| + |m|), where the two may cancel
        p, q = w.beta1 * np.abs(m0), (1 - w.beta1) * np.abs(g)
        assert (np.abs(m1 - m) <= 1.01 * U32 * (w.beta1 * np.abs(g) + 2 * p + q + np.abs(m)) + 1e-30).all()
        np.testing.assert_allclose(v1, v, rtol=1e-4, atol=1e-7 * np.abs(v).max() + 1e-30)
        want = x * (1 - lr * wd) - lr * (m / (1 - w.beta1 ** t)) / (np.sqrt(v / (1 - w.beta2 ** t)) + w.eps)
        big = np.abs(g) > 1e-4 * np.abs(g).max()      # (a first step is lr times the gradient's sign, noise or not)
        assert np.abs(y - want)[big].max(initial=0.0) <= 1e-3 * lr + 1e-6 * np.abs(x).max()
    for l in range(L):
        if net.has_bias:
            adam(*[p[l][1] for p in (x, y, g, v0, m0, v1, m1)])
        if l == L - 1:
            adam(*[p[l][0] for p in (x, y, g, v0, m0, v1, m1)])
            continue
        G = g[l][0]
        v = mu * v0[l][0] + G
        assert (np.abs(v1[l][0] - v) <= 3 * U32 * (np.abs(G) + np.abs(v0[l][0]))).all() and not m1[l][0].any()
        u = G + mu * v
        o = orth64(u)
        scale = 0.2 * math.sqrt(max(u.shape))
        want = (1 - lr * wd) * x[l][0] - lr * scale * o
        rel = _orth_tol(prec, min(u.shape), "f32") + _null_space_tol(u)
        tol = lr * scale * np.linalg.norm(o) * rel + 8 * U32 * np.linalg.norm(x[l][0])
        assert np.linalg.norm(y[l][0] - want) <= tol, (l, np.linalg.norm(y[l][0] - want) / (lr * scale * np.linalg.norm(o)))


MUON_NETS = [((40, 24, 16, 7), 0, 37, 3, True), ((72, 130, 5), 0, 150, 2, False), ((136, 264, 72, 100), 1, 300, 2, True),
             ((384, 256, 256, 12), 1, 64, 3, True), ((64, 32, 10), 1, 24, 2, False),
             ((1203, 24, 1030, 5), 0, 40, 2, True), ((1208, 24, 1032, 10), 1, 48, 3, True)]


@gpu
@pytest.mark.parametrize("dims,prec,b,M,hb", MUON_NETS)
@pytest.mark.parametrize("mode", ["plain", "ragged", "micro", "graphed"])
def test_muon_as_inner_optimizer(dims, prec, b, M, hb, mode):
    import torch
    from oracle import abs_oracle as O
    from paper_2406_13936_amd import workloads as W
    A = _A()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):                     # (steps are captured on a created stream only)
        w, X, y, x0, rep, net = _muon_case(dims, prec, b, M, hb)
        orc = O.Replicas(net, x0, X, y, M, opt=O.OPT_SGD, mixed=prec == 1, want_ip=True, gram_max_b=256 if mode != "micro" else 0)
        try:
            for t in range(1, 5):
                idx = W.step_indices(w, 0, t, b)
                before = [rep.get_params(m) for m in range(M)]
                state0 = [[rep.get_opt_state(m, i) for i in range(2)] for m in range(M)]
                orc.x = np.stack(before).astype(np.float64)
                if mode == "ragged":
                    rows = [r[:max(2, b - 3 * m)] for m, r in enumerate(idx)]
                    rep.local_step_ragged(rows, w.lr)
                    orc.local_step(rows, 0.0)
                else:
                    if mode == "micro":
                        rep.local_step_accumulated(idx, b // 2 + (b % (b // 2) == 1), w.lr)
                    elif mode == "graphed":
                        d, _ = rep.upload_indices(idx)
                        rep.local_step_graphed_dev(d, b, w.lr)
                    else:
                        rep.local_step(idx, w.lr)
                    orc.local_step(idx, 0.0)
                res = rep.inner_product_test(w.theta)
                for m in range(M):
                    g = rep.get_grad(m)
                    assert np.linalg.norm(g - orc.grads[m]) <= (2e-3 if prec else 1e-5) * np.linalg.norm(orc.grads[m]), (t, m)
                    for got, want in ((res[m].sum_sq, orc.stats[m]["S1"]), (res[m].gbar_sq, orc.stats[m]["S2"])):
                        assert abs(got - want) <= (2e-3 if prec else 1e-4) * abs(want), (t, m)
                    _check_muon_step(w, net, before[m], rep.get_params(m), g, state0[m],
                                     [rep.get_opt_state(m, i) for i in range(2)], t, prec)
            if mode == "graphed":
                assert rep.graph_count() == 1
            rep.average_replicas()
            p = np.stack([rep.get_params(m) for m in range(M)])
            assert (p == p[0]).all() and rep.guard_intact()
            with pytest.raises(A.AbsError, match="fused"):
                rep.set_fused_update(True)
            rep.set_fused_update(False)
        finally:
            rep.close()


@gpu
def test_muon_replayed_steps_are_the_direct_ones_and_its_workers_stand_alone():
    import torch
    from paper_2406_13936_amd import workloads as W
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        w, X, y, x0, rep, _ = _muon_case((136, 264, 72, 100), 1, 96, 3)
        _, _, _, _, ref, _ = _muon_case((136, 264, 72, 100), 1, 96, 3)
        try:
            for t in range(6):
                idx = W.step_indices(w, 0, t, 96)
                d, _ = rep.upload_indices(idx)
                lr = 0.02 / (t + 1)                   # (a captured step reads the rate from memory)
                rep.local_step_graphed_dev(d, 96, lr)
                ref.local_step(idx, lr)
                rep.norm_test(0.5)
                ref.norm_test(0.5)
                for m in range(3):
                    assert np.array_equal(rep.get_params(m), ref.get_params(m)), (t, m)
        finally:
            rep.close()
            ref.close()
