"""Layer norm where its numbers or its rows are at the edge of what the entry points take."""
import pytest

from test_operators import DS, _A, _check_backward, _check_forward, _dt, _ln_inputs

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("D", DS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_constant_rows_of_huge_values(D, dtype):
    """x - mean is zero in them, and 1 / sqrt(eps) times the mean is beyond fp32: lanes without a column of the row multiply it with dy = 0.
    (Powers of two: sums of up to 2^24 of them are exact, and so are the means.)"""
    import torch
    A = _A()
    for M, b, T in ((1, 1, 1), (2, 9, 1), (2, 3, 7), (2, 2, 150)):
        x, w, bias, dy = _ln_inputs(M, b, T, D, dtype, "f32")
        x = torch.full_like(x, 2.0 ** 113)
        y, mean, rstd = A.layer_norm(x, w, bias, eps=1e-12)
        assert torch.equal(y, bias[:, None, None].to(y.dtype).expand_as(y)) and (mean == 2.0 ** 113).all() and (rstd > 9e5).all()
        got = A.layer_norm_backward(dy, x, w, mean, rstd, want_norms=True, want_inner=True)
        _check_backward(got, dy, x, w, mean, rstd, True, dtype)


@gpu
def test_more_long_rows_than_a_launch_takes():
    """(A block to a row would be more threads than a grid counts from 2^24 rows on, which fit the card in place.)"""
    import torch
    A = _A()
    M, b, D = 2, (1 << 17) + 5, 8193
    gen = torch.Generator("cuda").manual_seed(1)
    x = torch.randn((M, b, D), generator=gen, device="cuda", dtype=torch.bfloat16)
    w, bias = (torch.randn((M, D), generator=gen, device="cuda") for _ in range(2))
    keep = x.clone()
    y, mean, rstd = A.layer_norm(x, w, bias, out=x)
    for i in (slice(0, 3), slice(b - 12, b)):
        for p, r in zip((y, mean, rstd), A.layer_norm(keep[:, i], w, bias)):
            assert torch.equal(p[:, i], r)
    _check_forward(y[:, -9:, None], mean[:, -9:, None], rstd[:, -9:, None], keep[:, -9:, None], w, bias, 1e-5, "bf16")


@gpu
@pytest.mark.parametrize("D", [8, 40, 256, 1024, 2048, 4096, 8192, 8200])
@pytest.mark.parametrize("dtype,ptype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
def test_gains_and_sums_that_no_vector_begins_on(D, dtype, ptype):
    """Rows of whole vectors beside gains, biases, batch gradients and statistics one value off any; and without the outputs that may be absent."""
    import ctypes as C
    import torch
    from paper_2406_13936_amd import binding as B
    A = _A()
    M, b, T = 2, 5, 3
    x, w, bias, dy = _ln_inputs(M, b, T, D, dtype, ptype)

    def off(t):
        buf = torch.zeros(t.numel() + 1, device="cuda", dtype=t.dtype)
        v = buf[1:].view(t.shape)
        return v.copy_(t)
    y, mean, rstd = A.layer_norm(x, w, bias)
    for p, r in zip(A.layer_norm(x, off(w), off(bias)), (y, mean, rstd)):
        assert torch.equal(p, r)
    want = A.layer_norm_backward(dy, x, w, mean, rstd, want_norms=True, want_inner=True)
    got = [off(torch.zeros_like(t)) for t in want]
    got[0] = torch.empty_like(want[0])
    lib = B.load_library()
    kind = lambda s: {"f32": 0, "bf16": 1, "f16": 2}[s]  # noqa: E731
    s = B.LayerNormShape(M, b, T, D, kind(dtype), kind(ptype), D, b * T * D, D, b * T * D, D, b * T * D)
    n = C.c_size_t(0)
    assert lib.abs_layer_norm_backward_workspace_bytes(C.byref(s), 1, 1, C.byref(n)) == 0
    keep, ws = B._workspace(n.value, x.device)
    stream = torch.cuda.current_stream().cuda_stream
    ins = [dy, x, off(w), off(mean), off(rstd)]
    assert lib.abs_layer_norm_backward(C.byref(s), *[t.data_ptr() for t in ins + got], ws, n.value, stream) == 0
    for p, r in zip(got, want):
        assert torch.equal(p, r)
    z = torch.empty_like(y)
    assert lib.abs_layer_norm(C.byref(s), x.data_ptr(), w.data_ptr(), bias.data_ptr(), 1e-5, z.data_ptr(), None, None, stream) == 0
    assert torch.equal(z, y)
