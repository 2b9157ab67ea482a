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
