"""Token embedding, the gradient of its tables and the batch tests' statistics of it: refusals on the host, then parity with the
definition in 64 bits.  Tolerances count roundings: U[t] is half a step of a type relative to the value; a sum of k values in fp32 is off by
at most k U32 of the sum of their magnitudes."""
import ctypes as C
import itertools

import pytest

U32 = 2.0 ** -24
U = {"f32": U32, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}          # half a step of the smallest values
gpu = pytest.mark.gpu
EINVAL, ENOMEM, EUNSUPPORTED = 1, 2, 5
FAKE, WS = 0x10000000, 0x40000000                            # never touched: every call with them is refused before a launch


def _A():
    import paper_2406_13936_amd as A
    return A


def _dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i32": torch.int32, "i64": torch.int64}[name]


# ---- refusals (no GPU call is made) ------------------------------------------------------------------------------------

def _shape(**k):
    from paper_2406_13936_amd import binding as B
    d = dict(M=2, b=3, T=4, V=10, D=16, token_type=16, type=0, table_type=0, ldy=16, stride_y=192)
    d.update(k)
    return B.EmbeddingShape(*[d[f] for f, _ in B.EmbeddingShape._fields_])


def _lib():
    from paper_2406_13936_amd import binding as B
    return B.load_library()


@pytest.mark.parametrize("change,status", [
    (dict(M=0), EINVAL), (dict(b=0), EINVAL), (dict(T=0), EINVAL), (dict(V=0), EINVAL), (dict(D=0), EINVAL), (dict(token_type=0), EINVAL),
    (dict(type=3), EINVAL), (dict(ldy=15), EINVAL), (dict(stride_y=100), EINVAL), (dict(ldy=-16), EINVAL),
    (dict(M=(1 << 20) + 1), EUNSUPPORTED), (dict(V=(1 << 30) + 1), EUNSUPPORTED), (dict(b=1 << 25), EUNSUPPORTED),
    (dict(b=1 << 20, T=1 << 12, stride_y=1 << 40), EUNSUPPORTED)])
def test_shapes_are_refused(change, status):
    lib, n = _lib(), C.c_size_t(0)
    s = _shape(**change)
    assert lib.abs_embedding(C.byref(s), FAKE, FAKE + (1 << 20), 1.0, FAKE + (1 << 21), None) == status
    assert lib.abs_embedding_backward_workspace_bytes(C.byref(s), 1, 1, C.byref(n)) == status
    assert lib.abs_last_error(None)


def test_arguments_are_refused():
    lib, s = _lib(), _shape()
    far = [FAKE + i * (1 << 20) for i in range(8)]
    fwd = lambda tok=far[0], tab=far[1], scale=1.0, y=far[2], sh=s: lib.abs_embedding(C.byref(sh), tok, tab, scale, y, None)  # noqa: E731
    for bad in (dict(tok=None), dict(tab=None), dict(y=None), dict(scale=float("nan")), dict(scale=float("inf")), dict(tok=far[0] + 2), dict(tab=far[1] + 2),
                dict(y=far[2] + 2), dict(y=far[0]), dict(y=far[1] + 64), dict(sh=_shape(table_type=5)), dict(sh=_shape(token_type=17), tok=far[0] + 4)):
        assert fwd(**bad) == EINVAL, bad
    assert lib.abs_embedding(None, far[0], far[1], 1.0, far[2], None) == EINVAL

    def bwd(nbytes=1 << 20, ws=WS, scale=1.0, **k):
        d = dict(dy=far[0], tokens=far[1], dtable=far[2], n=far[3], q=far[4])
        d.update(k)
        return lib.abs_embedding_backward(C.byref(s), d["dy"], d["tokens"], scale, d["dtable"], d["n"], d["q"], ws, nbytes, None)
    for name in ("dy", "tokens", "dtable"):
        assert bwd(**{name: None}) == EINVAL, name
    for name in ("dy", "tokens", "dtable", "n", "q"):
        assert bwd(**{name: far[0] + 2}) == EINVAL, name
        assert bwd(**{name: WS + 128}) == EINVAL, name
    assert bwd(ws=None) == EINVAL and bwd(ws=WS + 8) == EINVAL and bwd(nbytes=16) == ENOMEM and bwd(scale=float("nan")) == EINVAL
    assert bwd(dtable=far[0]) == EINVAL and bwd(n=far[4]) == EINVAL
    assert lib.abs_embedding_backward_workspace_bytes(C.byref(s), 0, 0, None) == EINVAL


def test_tensors_are_refused():
    import torch
    A = _A()
    tok, table, dy = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 5, 8), torch.zeros(2, 3, 8)
    with pytest.raises(A.AbsError, match="device memory"):
        A.embedding(tok, table)
    with pytest.raises(A.AbsError, match="int32 or int64"):
        A.embedding(tok.float(), table)
    with pytest.raises(A.AbsError, match="device memory"):
        A.embedding_backward(dy, tok, 5)


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------

def _reference(dy, tokens, V, scale):
    """(gbar, n, q), and the largest errors of sums in fp32 of each."""
    import torch
    M, b = tokens.shape[:2]
    D = dy.shape[-1]
    tok, y = tokens.reshape(M, b, -1).long().cpu(), dy.reshape(M, b, -1, D).double().cpu()
    g, gabs = torch.zeros(M, V, D, dtype=torch.float64), torch.zeros(M, V, D, dtype=torch.float64)
    n, nerr = torch.zeros(M, b, dtype=torch.float64), torch.zeros(M, b, dtype=torch.float64)
    inside = (tok >= 0) & (tok < V)
    count = torch.zeros(M, V, dtype=torch.float64)
    for m, i in itertools.product(range(M), range(b)):
        t, v = tok[m, i][inside[m, i]], y[m, i][inside[m, i]] * scale
        words, where = torch.unique(t, return_inverse=True)
        each = torch.zeros(len(words), D, dtype=torch.float64).index_add_(0, where, v)
        mag = torch.zeros(len(words), D, dtype=torch.float64).index_add_(0, where, v.abs())
        k = torch.bincount(where, minlength=len(words)).double()[:, None]
        off = (k + 2) * U32 * mag
        n[m, i] = (each ** 2).sum()
        # sums of D squares in fp32 and in fp64 over column tiles, rounded once
        nerr[m, i] = (2 * each.abs() * off + off ** 2).sum() + (D + 16) * U32 * n[m, i]
        g[m].index_add_(0, words, each / b)
        gabs[m].index_add_(0, words, mag / b)
        count[m].index_add_(0, words, k[:, 0])
    gerr = (count[..., None] + 4) * U32 * gabs
    q, qerr = torch.zeros(M, b, dtype=torch.float64), torch.zeros(M, b, dtype=torch.float64)
    for m, i in itertools.product(range(M), range(b)):
        t, v = tok[m, i][inside[m, i]], y[m, i][inside[m, i]] * scale
        q[m, i] = (v * g[m][t]).sum()
        qerr[m, i] = (v.abs() * (gerr[m][t] + (len(t) * D + 8) * U32 * (g[m][t].abs() + gerr[m][t]))).sum()
    return (g, n, q), (gerr, nerr + 1e-300, qerr + 1e-300)


def _tokens(shape, V, idx, gen, pad=0.0, words=None):
    import torch
    u = torch.rand(shape, device="cuda", generator=gen, dtype=torch.float64)
    t = (((words or V) + 1.0) ** u).long().clamp(1, words or V) - 1
    if pad:
        t = torch.where(torch.rand(shape, device="cuda", generator=gen) < pad, torch.where(t % 2 == 0, -1 - t, V + t), t)
    return t.to(_dt(idx))


# M, b, T, V, D, type, tokens, padding, words in use
CASES = [
    (1, 2, 1, 1, 1, "f32", "i32", 0.0, None), (1, 1, 1, 50, 8, "bf16", "i64", 0.0, None), (2, 3, 5, 7, 9, "f16", "i32", 0.3, None),
    (3, 5, 33, 997, 257, "f32", "i32", 0.2, None), (2, 4, 64, 50, 128, "bf16", "i64", 0.1, None), (1, 40, 1, 3, 33, "f32", "i32", 0.0, None),
    (2, 3, 700, 5000, 64, "f16", "i64", 0.0, None), (2, 3, 701, 40000, 129, "bf16", "i32", 0.5, None), (1, 4, 999, 2048, 520, "f16", "i32", 0.1, None),
    (1, 5, 901, 2047, 1024, "bf16", "i64", 0.0, None), (1, 3, 1500, 3, 1032, "bf16", "i32", 0.0, None), (1, 3, 1500, 4194305, 16, "f32", "i64", 0.01, None),
    (1, 2, 2500, 9, 24, "f16", "i32", 0.0, 1), (3, 1, 129, 300, 2050, "bf16", "i64", 1.0, None), (5, 2, 17, 100, 4096, "f32", "i32", 0.0, None),
    (2, 130, 20, 60, 40, "bf16", "i32", 0.05, 5)]


@gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c))
def test_gradient_and_statistics(case):
    import torch
    A = _A()
    M, b, T, V, D, dtype, idx, pad, words = case
    gen = torch.Generator(device="cuda").manual_seed(M + 10 * b + T)
    tok = _tokens((M, b, T), V, idx, gen, pad, words)
    dy = (torch.randn((M, b, T, D), device="cuda", generator=gen) + 0.2).to(_dt(dtype))
    scale = 1.7
    (g, n, q), (gerr, nerr, qerr) = _reference(dy, tok, V, scale)
    got = A.embedding_backward(dy, tok, V, scale=scale, want_norms=True, want_inner=True)
    assert ((got[0].double().cpu() - g).abs() <= gerr).all()
    assert ((got[1].double().cpu() - n).abs() <= nerr).all(), (got[1], n)
    assert ((got[2].double().cpu() - q).abs() <= qerr).all(), (got[2], q)
    # the same bits again, and whatever else is asked for
    for norms, inner in ((True, True), (True, False), (False, True), (False, False)):
        g2, n2, q2 = A.embedding_backward(dy, tok, V, scale=scale, want_norms=norms, want_inner=inner)
        if norms:
            assert torch.equal(g2, got[0]) and torch.equal(n2, got[1])
        assert ((g2.double().cpu() - g).abs() <= gerr).all()
        assert (n2 is not None) == norms and (q2 is not None) == inner
        assert q2 is None or ((q2.double().cpu() - q).abs() <= qerr).all()


@gpu
@pytest.mark.parametrize("D", [1, 7, 64, 65, 1000, 2048, 2056])
@pytest.mark.parametrize("table", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_lookup(D, table, dtype):
    import torch
    A = _A()
    M, b, T, V = 3, 5, 13, 41
    gen = torch.Generator(device="cuda").manual_seed(D)
    tok = _tokens((M, b, T), V, "i64", gen, 0.2)
    w = torch.randn((M, V, D), device="cuda", generator=gen).to(_dt(table))
    y = A.embedding(tok, w, scale=3.3, dtype=_dt(dtype))
    inside = ((tok >= 0) & (tok < V))[..., None]
    want = torch.stack([w[m].double()[tok[m].clamp(0, V - 1)] for m in range(M)]) * 3.3 * inside
    # (the scale is an fp32 value, one product, one rounding to the type)
    assert ((y.double() - want).abs() <= want.abs() * (U[dtype] + 3 * U32) + TINY[dtype]).all()
    assert (y[~inside.expand_as(y)] == 0).all() and y.dtype == _dt(dtype)
    assert torch.equal(A.embedding(tok.int(), w, scale=3.3, dtype=_dt(dtype)), y)


@gpu
def test_rows_with_gaps_and_samples_of_several_dimensions():
    import torch
    A = _A()
    M, b, T, V, D = 2, 6, 10, 30, 48
    gen = torch.Generator(device="cuda").manual_seed(3)
    tok = _tokens((M, b, 2, 5), V, "i32", gen)
    w = torch.randn((M, V, D), device="cuda", generator=gen)
    plain = A.embedding(tok, w)
    for lay in ("columns", "interleaved", "odd"):
        buf = torch.full((b * T, M, D + 24), -7.0, device="cuda") if lay == "interleaved" else torch.full((M, b * T, D + 24 + (lay == "odd")), -7.0, device="cuda")
        y = (buf.transpose(0, 1) if lay == "interleaved" else buf)[..., 1 if lay == "odd" else 8:][..., :D].unflatten(1, (b, 2, 5))
        y_rows = A.embedding(tok, w, out=y)
        assert y_rows is y and torch.equal(y, plain)
        assert int((buf == -7.0).sum()) == buf.numel() - plain.numel()
        want = A.embedding_backward(plain, tok, V, want_norms=True, want_inner=True)
        got = A.embedding_backward(y, tok, V, want_norms=True, want_inner=True)
        assert all(torch.equal(a, c) for a, c in zip(want, got)) or lay == "odd"
        assert all(torch.allclose(a, c, rtol=1e-5, atol=1e-6) for a, c in zip(want, got))
    with pytest.raises(A.AbsError, match="equally spaced"):
        A.embedding(tok, w, out=torch.zeros((M, b, 2, 7, D), device="cuda")[:, :, :, :5])
    with pytest.raises(A.AbsError, match="contiguous"):
        A.embedding(tok, w.transpose(0, 1).contiguous().transpose(0, 1))
    with pytest.raises(A.AbsError, match="must be"):
        A.embedding_backward(plain[:, :, :1], tok, V)
    with pytest.raises(A.AbsError, match="out must be"):
        A.embedding(tok, w, dtype=torch.bfloat16, out=plain)
    with pytest.raises(A.AbsError):
        A.embedding(tok[:, :0], w)


@gpu
def test_unusual_values_stay_where_they_are():
    import torch
    A = _A()
    tok = torch.tensor([[[0, 1, 2, 1], [3, 3, 9, -1]]], device="cuda")
    dy = torch.ones((1, 2, 4, 72), device="cuda", dtype=torch.bfloat16)
    dy[0, 0, 2] = float("nan")
    dy[0, 1, 2:] = float("inf")                      # words outside the table: no part in anything
    g, n, q = A.embedding_backward(dy, tok, 6, want_norms=True, want_inner=True)
    assert torch.isnan(g[0, 2]).all() and torch.isfinite(g[0, [0, 1, 3, 4, 5]]).all()
    assert torch.equal(g[0, :, 0].cpu()[[0, 1, 3, 4, 5]], torch.tensor([0.5, 1.0, 1.0, 0.0, 0.0]))
    assert torch.isnan(n[0, 0]) and torch.isnan(q[0, 0]) and n[0, 1] == 4 * 72 and q[0, 1] == 2 * 72
    # guards behind the operands
    table = torch.full((1, 6, 72), float("inf"), device="cuda")
    table[0, :4] = 1.0
    assert torch.isfinite(A.embedding(tok, table)).all()


@gpu
def test_replayed_graphs_of_two_calls_share_nothing():
    import torch
    A = _A()
    M, b, T, V, D = 2, 8, 400, 500, 96
    gen = torch.Generator(device="cuda").manual_seed(5)
    toks = [_tokens((M, b, T), V, "i32", gen) for _ in range(3)]
    dys = [torch.randn((M, b, T, D), device="cuda", generator=gen) for _ in range(3)]
    tok, dy = toks[0].clone(), dys[0].clone()
    w = torch.randn((M, V, D), device="cuda", generator=gen)
    A.embedding_backward(dy, tok, V, want_norms=True, want_inner=True)
    graphs = []
    for scale in (1.0, 2.0):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = A.embedding_backward(dy, tok, V, scale=scale, want_norms=True, want_inner=True) + (A.embedding(tok, w, scale=scale),)
        graphs.append((scale, g, out))
    for k in (1, 2, 0, 1):
        tok.copy_(toks[k])
        dy.copy_(dys[k])
        for scale, g, out in graphs:
            g.replay()
        torch.cuda.synchronize()
        for scale, g, out in graphs:
            want = A.embedding_backward(dys[k], toks[k], V, scale=scale, want_norms=True, want_inner=True) + (A.embedding(toks[k], w, scale=scale),)
            assert all(torch.equal(a, c) for a, c in zip(out, want))


@gpu
def test_gradient_against_differences():
    """Sample i's loss sum_t c_t . y_t: its directional derivative along a table is <g_i, direction>."""
    import torch
    A = _A()
    M, b, T, V, D = 2, 4, 9, 12, 20
    gen = torch.Generator(device="cuda").manual_seed(8)
    tok = _tokens((M, b, T), V, "i64", gen)
    w, c, d = (torch.randn(s, device="cuda", generator=gen) for s in ((M, V, D), (M, b, T, D), (M, V, D)))
    g, _, _ = A.embedding_backward(c, tok, V, scale=0.5)
    loss = lambda t: (A.embedding(tok, t, scale=0.5).double() * c.double()).sum((1, 2, 3)) / b  # noqa: E731
    eps = 0.5                                        # (linear: any step will do)
    slope = (loss(w + eps * d) - loss(w - eps * d)) / (2 * eps)
    want = (g.double() * d.double()).sum((1, 2))
    # 2 T b rows of D products of fp32 values, each a few roundings of values up to |w| + eps |d|
    bound = 8 * U32 / eps * ((w.abs() + d.abs()).amax() * c.abs().double().sum((1, 2, 3)) / b) + (T * b + 8) * U32 * (g.abs() * d.abs()).double().sum((1, 2))
    assert ((slope - want).abs() <= bound).all()
