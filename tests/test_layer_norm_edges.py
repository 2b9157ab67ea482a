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
