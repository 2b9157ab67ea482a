"""The 8-bit result of the root-mean-square norm at gains that are infinite or NaN, or whose products with the rows pass fp32's range."""
import pytest

from test_rms_norm import EPS, U32, _A, _inputs

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dtype,param", [("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "f32")])
@pytest.mark.parametrize("D", [1, 100, 129, 1000, 2048, 4100, 8192, 8200])
def test_gains_that_are_infinite_or_nan(D, dtype, param):
    """Such a gain leaves every row of its replica an infinity or NaN: the scale is NaN, and what is held in 8 bits with it."""
    import torch
    A = _A()
    x, res, w, _, _ = _inputs(3, 4, 5, D, dtype, param, True, D)
    x[1, 2, 3] = 0
    res[1, 2, 3] = 0                                  # (a row of zeros: 0 times infinity)
    want8, want_c, h, rstd = A.rms_norm_8bit(x, w, residual=res, eps=EPS)
    assert torch.isfinite(want_c).all()
    for at in {0, D // 2, D - 1}:
        for value in (float("nan"), float("inf"), float("-inf")):
            w2 = w.clone()
            w2[1, at] = value
            y8, c, h2, r2 = A.rms_norm_8bit(x, w2, residual=res, eps=EPS)
            assert torch.equal(h2, h) and torch.equal(r2, rstd)
            assert torch.isnan(c[1]).all() and torch.isnan(y8[1].float()).all()
            for m in (0, 2):
                assert torch.equal(c[m], want_c[m]) and torch.equal(y8[m].float(), want8[m].float())


@gpu
@pytest.mark.parametrize("D", [16, 100, 129, 1000, 2048, 4100, 8192, 8200])
def test_infinities_in_a_row_where_its_gain_is_zero(D):
    """Infinity times 0 is NaN in that place, and so is the scale; other rows, and those whose squares pass fp32's range, keep theirs."""
    import torch
    A = _A()
    x, _, w, _, _ = _inputs(2, 5, 7, D, "bf16", "f32", False, D)
    w[:, D // 2] = 0
    x[0, 0, 0] = 2.0 ** 100                           # (1 / sqrt(infinity) = 0: zeros)
    want8, want_c, _, _ = A.rms_norm_8bit(x, w, eps=EPS)
    assert want_c[0, 0, 0] == 2.0 ** -100 and (want8[0, 0, 0].float() == 0).all()
    rows = torch.zeros(x.shape[:-1], dtype=torch.bool, device="cuda")
    for m, i, t, value in ((0, 0, 1, float("inf")), (0, 3, 6, float("-inf")), (1, 4, 0, float("inf")), (1, 4, 1, float("nan"))):
        x[m, i, t, D // 2] = value
        rows[m, i, t] = True
    y8, c, _, _ = A.rms_norm_8bit(x, w, eps=EPS)
    assert torch.isnan(c[rows]).all() and torch.isnan(y8.float()[rows]).all()
    assert torch.equal(c[~rows], want_c[~rows]) and torch.equal(y8.float()[~rows], want8.float()[~rows])


@gpu
@pytest.mark.parametrize("D", [16, 200, 2048, 8200])
@pytest.mark.parametrize("row,gain,eps", [(1e10, 1e30, 1e-6), (3e-5, 1e-41, 0.0), (1e-18, 1e-27, 0.0), (1e-17, 3e-28, 0.0), (1e15, 1e25, 0.0)])
def test_products_of_rows_and_gains_beyond_fp32(row, gain, eps, D):
    """max |h w| may be above fp32's range, or among its last bits, where max |h r w| / 448 is not: the scale is right in both, and so are the values."""
    import torch
    A = _A()
    gen = torch.Generator(device="cuda").manual_seed(D)
    x = row * (0.5 + torch.rand((2, 3, 4, D), device="cuda", generator=gen)) * (2.0 * (torch.rand((2, 3, 4, D), device="cuda", generator=gen) < 0.5) - 1.0)
    w = gain * (0.5 + torch.rand((2, D), device="cuda", generator=gen))
    y8, c, _, rstd = A.rms_norm_8bit(x, w, eps=eps)
    p = x.double() * w.double()[:, None, None]
    r = 1 / torch.sqrt(x.double().square().mean(-1) + eps)
    # squares of 1e-18 are held to half of 2^-149 of 1e-36 and more: 2^-30; the root halves it
    rel = (D / 2 + 8) * U32 + 2.0 ** -30
    assert ((rstd.double() - r).abs() <= rel * r).all()
    want_c = (p.abs().amax(-1) * r / 448).clamp(min=2.0 ** -100)
    assert ((c.double() - want_c).abs() <= 2 * rel * want_c).all()
    v = p * r[..., None] / want_c[..., None]
    got = y8.double()
    assert torch.isfinite(got).all() and ((got - v).abs() <= torch.maximum(v.abs() * (2.0 ** -4 + 4 * rel), torch.full_like(v, 2.0 ** -10 * (1 + rel)))).all()


@gpu
@pytest.mark.parametrize("D", [16, 129, 1000, 2048, 8192, 8200])
def test_rows_whose_squares_are_below_fp32(D):
    """Without eps r is infinite and y infinite or NaN: the scale is NaN, also where all gains are zero; with eps such rows are as small as they are."""
    import torch
    A = _A()
    x = torch.full((3, 2, 3, D), 1e-30, device="cuda")
    w = torch.ones((3, D), device="cuda")
    w[1] = 0
    w[2, ::2] = 0
    y8, c, _, rstd = A.rms_norm_8bit(x, w, eps=0.0)
    assert torch.isinf(rstd).all() and torch.isnan(c).all() and torch.isnan(y8.float()).all()
    y8, c, _, rstd = A.rms_norm_8bit(x, w, eps=EPS)
    # y = 1e-27, c = 1e-27 / 448 = 2.2e-30 above 2^-100, and the quotients 448 and 0
    r = 1e-30 / EPS ** 0.5 / 448
    assert ((c[[0, 2]].double() - r).abs() <= 16 * U32 * r).all() and (c[1] == 2.0 ** -100).all()
    assert (y8[0].float() == 448).all() and (y8[1].float() == 0).all() and torch.equal(y8[2].float(), 448 * w[2].expand(2, 3, D))
