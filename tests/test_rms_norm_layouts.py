"""Root-mean-square norm: results in the place of operands, and the same bits whatever the rows lie among."""
import pytest

from test_rms_norm import _A, _inputs

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("D", [40, 2048, 9000])
def test_h_that_the_result_took_the_place_of_is_not_returned(D):
    """Without a residual h is x: where y is written over it there is none to return, and a backward pass that takes it is refused."""
    import torch
    A = _A()
    x, res, w, dy, _ = _inputs(2, 3, 4, D, "bf16", "f32", True, D)
    y, h, rstd = A.rms_norm(x, w)
    assert h is x
    for view in (False, True):
        x2 = x.clone()
        y2, h2, r2 = A.rms_norm(x2, w, out=x2.view(x2.shape) if view else x2)
        assert h2 is None and torch.equal(y2, y) and torch.equal(x2, y) and torch.equal(r2, rstd)
        with pytest.raises(A.AbsError):
            A.rms_norm_backward(dy, h2, w, r2)
    other = torch.empty_like(x)
    assert A.rms_norm(x, w, out=other)[1] is x
    y, h, rstd = A.rms_norm(x, w, residual=res)       # h has a place of its own
    x2 = x.clone()
    y2, h2, _ = A.rms_norm(x2, w, residual=res, out=x2)
    assert torch.equal(h2, h) and torch.equal(y2, y)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [(2, 3, 5, 72), (3, 4, 33, 77), (2, 5, 6, 1024), (2, 40, 1, 264), (1, 2, 3, 9000)], ids=str)
def test_gradients_and_statistics_are_the_same_bits_in_other_layouts(size, dtype):
    """Rows among wider ones, and replicas interleaved by rows: the same reads and sums where rows begin on the same kind of places."""
    import torch
    A = _A()
    M, b, T, D = size
    h, _, w, dy, dh = _inputs(M, b, T, D, dtype, "f32", True, D)
    rstd = (h.float().square().mean(-1) + 1e-6).rsqrt()

    def laid(t, interleaved):
        buf = torch.full((b * T, M, D + 16) if interleaved else (M, b * T, D + 16), 99.0, device="cuda").to(t.dtype)
        v = (buf.transpose(0, 1) if interleaved else buf)[..., 8:8 + D].unflatten(1, (b, T))
        v.copy_(t)
        return v
    for norms, inner in ((True, True), (True, False), (False, True), (False, False)):
        want = A.rms_norm_backward(dy, h, w, rstd, dh=dh, want_norms=norms, want_inner=inner)
        for how in ((False, False, False), (True, True, True), (True, False, True), (False, True, False)):
            got = A.rms_norm_backward(laid(dy, how[0]), laid(h, how[1]), w, rstd, dh=laid(dh, how[2]), want_norms=norms, want_inner=inner)
            for a, g in zip(want, got):
                assert (a is None and g is None) or torch.equal(a, g)
