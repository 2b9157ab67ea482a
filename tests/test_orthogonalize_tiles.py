"""Orthogonalisation launch by launch: every kind of product kernel (tile, ring, operand layout, pairs or not, with and without the
update) at sizes that are multiples of nothing, against the definition in 64 bits."""
import ctypes as C
import math

import pytest

from paper_2406_13936_amd import binding as B
from test_operators import COEF, TOL32, U, U32, _dt, _matrix

gpu = pytest.mark.gpu

CASES = [(1, 131, 129), (1, 129, 133), (48, 130, 129), (29, 137, 129), (29, 132, 143), (44, 257, 136), (39, 221, 194), (35, 513, 558),
         (52, 635, 386), (57, 280, 262), (8, 520, 700), (11, 520, 1032), (2, 2100, 2300), (1, 3901, 4037), (1, 4037, 3001)]


def _routes(batch, rows, cols, prec):
    """The product kernels that a call takes: (product, layout, pairs, tile and ring), or who takes the matrix instead."""
    lib = B.load_library()
    small, slices, shape = (lib["_ZN4absk" + n] for n in ("15orth_small_fitsEiii", "15orth_slices_fitEiii", "18orth_product_shapeEiiiii"))
    small.restype = slices.restype = C.c_bool
    if small(batch, rows, cols):
        return {"one launch"}
    if slices(batch, rows, cols):
        return {"slices"}
    pairs, wide = prec == B.PREC_F32 or min(rows, cols) <= 128, rows <= cols
    unit, f, layout = 32 if pairs else 8, 2 if pairs else 1, "wide" if wide else "tall"
    rp, cp = (-(-n // unit) * unit for n in (rows, cols))
    mp = min(rp, cp)
    return {("A", layout, pairs, shape(mp, mp, max(rp, cp) * f, batch, 1)), ("B", "", pairs, shape(mp, mp, mp * f, batch, 1)),
            ("X", layout, pairs, shape(rp, cp, mp * f, batch, 0))}


def test_the_cases_reach_every_kind_of_product():
    tiles = (6424, 6422, 12822, 12812, 25612)
    every = {(product, layout, pairs, t) for product, layouts in (("A", ("wide", "tall")), ("B", ("",)), ("X", ("wide", "tall")))
             for layout in layouts for pairs in (False, True) for t in tiles}
    reached = set().union(*(_routes(*c, prec) for c in CASES for prec in (B.PREC_F32, B.PREC_BF16)))
    assert reached == every


def test_the_rule_for_tiles():
    """Both sides of each line."""
    shape = B.load_library()["_ZN4absk18orth_product_shapeEiiiii"]
    assert shape(1024, 1024, 1024, 1, 0) == 6424 and shape(1024, 1088, 1024, 1, 0) == 6422         # 256 tiles of 64 x 64, 272
    assert shape(1024, 1536, 1024, 1, 0) == 6422 and shape(1024, 1600, 1024, 1, 0) == 12822        # 384, 400
    assert shape(2048, 2048, 480, 1, 0) == 12822 and shape(2048, 2176, 480, 1, 0) == 12812         # 256 of 128 x 128, 272
    assert shape(4096, 4096, 504, 1, 0) == 12812 and shape(4096, 4096, 512, 1, 0) == 25612         # a reduction of 512
    assert shape(4096, 4096, 4096, 1, 1) == 25612 and shape(3968, 3968, 4096, 1, 1) == 12812       # 136 of 256 x 256 and 528 or 496 of 128 x 128


def _orth(G, norms=None):
    """The definition in 64 bits, on the device; the norm of X before each step and at the end goes to `norms`."""
    import torch
    X = G / (torch.linalg.vector_norm(G) + 1e-7)
    a, b, c = COEF
    for _ in range(5):
        if norms is not None:
            norms.append(float(X.norm()))
        if X.shape[0] <= X.shape[1]:
            A = X @ X.T.contiguous()
            X = a * X + (b * A + c * (A @ A)) @ X
        else:
            A = X.T.contiguous() @ X
            X = a * X + X @ (b * A + c * (A @ A))
    if norms is not None:
        norms.append(float(X.norm()))
    return X


# Relative error (2-norm) of 16-bit products: abs.h says at most 1.6e-3 (their number formats alone, with the roundings put into a 64-bit run
# on the CPU: 1.52e-3 for full rank at 129 x 129, less for larger sides, lower ranks and falling spectra).
TOL16 = 1.6e-3


def _tol(prec, rows, cols):
    return TOL32 if prec == B.PREC_F32 or min(rows, cols) <= 128 else TOL16


@pytest.fixture
def guarded(monkeypatch):
    """Workspaces with guard bytes behind them; the check that they are as they were."""
    import torch
    kept = []

    def workspace(nbytes, device):
        t = torch.full((nbytes + 256 + 4096,), 0xA5, dtype=torch.uint8, device=device)
        base = (t.data_ptr() + 255) // 256 * 256
        kept.append(t[base - t.data_ptr() + nbytes:])
        return t, base
    monkeypatch.setattr(B, "_workspace", workspace)

    def intact():
        assert kept and all(bool((t == 0xA5).all()) for t in kept)
        kept.clear()
    return intact


@gpu
@pytest.mark.parametrize("batch,rows,cols", CASES)
@pytest.mark.parametrize("prec", [B.PREC_BF16, B.PREC_F32])
@pytest.mark.parametrize("kind", ["full", "low"])
def test_products_of_ragged_matrices(batch, rows, cols, prec, kind, guarded):
    import torch
    gen = torch.Generator().manual_seed(rows * 10000 + cols)
    G = _matrix(kind, batch, rows, cols, gen).float().cuda()
    out = B.orthogonalize(G, prec=prec)
    for i in range(batch):
        norms = []
        want = _orth(G[i].double(), norms)
        tol = _tol(prec, rows, cols) + U32
        if kind == "low":
            # what roundings of X leave where a low-rank G has nothing: X_k to fp32 and to hi + lo (2^-24 and 2^-22 of an entry), which every
            # later step multiplies by a
            tol += (2.0 ** -22 + 2.0 ** -24) * sum(COEF[0] ** (5 - k) * norms[k] for k in range(6)) / norms[5]
        err = (out[i].double() - want).norm() / want.norm()
        assert err <= tol, (i, float(err), tol)
        assert (out[i].double() - want).abs().max() <= 0.05 * want.abs().max(), i
    for _ in range(2):
        assert torch.equal(out, B.orthogonalize(G, prec=prec))          # the same bits every time
    # rows of other lengths and places, each matrix followed by values that are none of its own
    ld, step = cols + 3, rows * (cols + 3) + 5
    buf = torch.full((1 + batch * step,), 7.0, device="cuda")
    view = buf[1:].as_strided((batch, rows, cols), (step, ld, 1))
    B.orthogonalize(G, prec=prec, out=view)
    assert torch.equal(view, out)
    view.fill_(7.0)
    assert (buf == 7.0).all()
    guarded()


@gpu
@pytest.mark.parametrize("batch,rows,cols", CASES)
@pytest.mark.parametrize("xt,gt", [("f32", "f32"), ("bf16", "f16")])
def test_the_update_by_products_of_ragged_matrices(batch, rows, cols, xt, gt, guarded):
    import torch
    gen = torch.Generator().manual_seed(rows * 10000 + cols + 1)
    G = _matrix("full", batch, rows, cols, gen, 0.01).to(_dt(gt)).cuda()
    x = (torch.rand((batch, rows, cols), generator=gen) / math.sqrt(cols)).to(_dt(xt)).cuda()
    v = torch.randn((batch, rows, cols), generator=gen).cuda() * 0.02
    x0, v0 = x.clone(), v.clone()
    lr, mu, wd, scale = 0.02, 0.9, 0.1, 0.2 * math.sqrt(max(rows, cols))
    B.muon_step(x, G, v, lr, momentum=mu, weight_decay=wd)
    prec = B.PREC_F32 if xt == "f32" else B.PREC_BF16
    for i in range(batch):
        g, old = G[i].double(), x0[i].double()
        v64 = mu * v0[i].double() + g
        # (one rounding of the constant, one of the sum)
        assert ((v[i].double() - v64).abs() <= 2 * U32 * (v64.abs() + (mu * v0[i].double()).abs())).all(), i
        o = _orth(g + mu * v64)
        want = (1.0 - lr * wd) * old - lr * scale * o
        # the factor's own error, a handful of fp32 roundings of the step, one rounding of x to its type
        tol = lr * scale * o.norm() * (_tol(prec, rows, cols) + U32) + (U[xt] + 6 * U32) * want.norm() + 6 * U32 * old.norm()
        assert (x[i].double() - want).norm() <= tol, (i, float((x[i].double() - want).norm()), float(tol))
    guarded()


@gpu
def test_many_large_ragged_matrices_in_a_graph():
    """The pipelined tiles of both layouts, replayed with other inputs."""
    import torch
    gen = torch.Generator("cuda").manual_seed(3)
    for batch, rows, cols in ((35, 513, 558), (52, 635, 386)):
        for dtype, prec in ((torch.bfloat16, B.PREC_BF16), (torch.float32, B.PREC_F32)):
            G = [torch.randn((batch, rows, cols), generator=gen, device="cuda").to(dtype) for _ in range(3)]
            want = [B.orthogonalize(g, prec=prec) for g in G]
            into, out = G[0].clone(), torch.empty_like(G[0])
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                B.orthogonalize(into, prec=prec, out=out)
            for i in (1, 2, 0, 1):
                into.copy_(G[i])
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(out, want[i]), i


@gpu
@pytest.mark.parametrize("rows,cols", [(65, 65), (96, 640), (1500, 97), (128, 513), (530, 128), (128, 128)])
def test_short_sides_take_products_of_both_parts(rows, cols):
    """Up to 128 rows or columns 16-bit products are those of fp32 class all the same, whichever kernel has the matrix."""
    import torch
    gen = torch.Generator().manual_seed(rows + cols)
    for batch in (1, 40):
        G = _matrix("full", batch, rows, cols, gen).float().cuda()
        out = B.orthogonalize(G, prec=B.PREC_BF16)
        for i in range(batch):
            want = _orth(G[i].double())
            assert (out[i].double() - want).norm() <= (TOL32 + U32) * want.norm(), i
        assert torch.equal(out, B.orthogonalize(G, prec=B.PREC_F32))


@gpu
@pytest.mark.parametrize("batch,rows,cols", [(3, 48, 80), (2, 128, 100), (3, 40, 1200), (2, 1100, 20), (3, 200, 144), (1, 264, 600), (1, 1000, 1000)])
@pytest.mark.parametrize("prec", [B.PREC_BF16, B.PREC_F32])
def test_matrices_whose_norm_is_about_eps_or_below(batch, rows, cols, prec):
    """X_k is held to 2^-40 (later, where its bound is above 1, 2^-39) of 1, an entry; N entries are off by sqrt(N) times that, which each later
    step multiplies by 3.4445 like X itself: 2^-40 sqrt(N) / |X_0| (1 + 2 / 3.4 + 2 / 3.4^2 + ..) of the result, at most 2 of the first term."""
    import torch
    gen = torch.Generator().manual_seed(rows)
    G = _matrix("full", batch, rows, cols, gen).cuda()
    G /= torch.linalg.vector_norm(G, dim=(1, 2), keepdim=True)
    for eps in (1e-7, 1e-3):
        for ratio in (1.0, 1e-3, 1e-6):
            g = (G * (eps * ratio)).float()
            out = B.orthogonalize(g, prec=prec, eps=eps)
            for i in range(batch):
                x = g[i].double() / (torch.linalg.vector_norm(g[i].double()) + eps)
                held = 2.0 * 2.0 ** -40 * math.sqrt(rows * cols) / float(x.norm())
                for _ in range(5):
                    k = x @ x.T.contiguous()
                    x = COEF[0] * x + (COEF[1] * k + COEF[2] * (k @ k)) @ x
                err = float((out[i].double() - x).norm() / x.norm())
                assert err <= _tol(prec, rows, cols) + U32 + held, (eps, ratio, i, err, held)


@gpu
@pytest.mark.parametrize("rows,cols,blocks", [(23000, 23000, 92), (13000, 41000, 50), (41000, 13000, 50)])
@pytest.mark.parametrize("prec", [B.PREC_BF16, B.PREC_F32])
def test_matrices_of_almost_as_many_values_as_are_taken(rows, cols, blocks, prec):
    """Blocks that meet in no row or column, scattered over the matrix: each is taken for itself, with the norm of all of them, and what
    lies in none stays zero."""
    import torch
    gen = torch.Generator("cuda").manual_seed(rows)
    r, c = rows // blocks, cols // blocks
    P = torch.randn((blocks, r, c), generator=gen, device="cuda")
    ri = torch.randperm(rows, generator=gen, device="cuda").view(blocks, r)
    ci = torch.randperm(cols, generator=gen, device="cuda").view(blocks, c)
    G = torch.zeros((rows, cols), device="cuda")
    for k in range(blocks):
        G[ri[k][:, None], ci[k]] = P[k]
    x = P.double() / (torch.linalg.vector_norm(P.double()) + 1e-7)
    for _ in range(5):
        k = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = COEF[0] * x + torch.matmul(COEF[1] * k + COEF[2] * torch.matmul(k, k), x)
    out = B.orthogonalize(G[None], prec=prec)[0]
    del G
    got = torch.stack([out[ri[k][:, None], ci[k]] for k in range(blocks)])
    assert (got.double() - x).norm() <= (_tol(prec, rows, cols) + U32) * x.norm()
    for k in range(blocks):
        out[ri[k][:, None], ci[k]] = 0.0
    assert int(torch.count_nonzero(out)) == 0
    with pytest.raises(B.AbsError, match="2\\^29"):
        B.orthogonalize(torch.empty((1, 1 << 15, 1 << 14), device="cuda"))
