"""The operators beside torch's autograd: outside its graph, but what they change in place counts as changed."""
import pytest

from test_operators import _A

pytestmark = pytest.mark.gpu


def test_what_is_changed_in_place_cannot_be_used_by_a_backward_pass():
    import torch
    A = _A()
    new = lambda *s: torch.randn(s, device="cuda")  # noqa: E731
    x = torch.nn.Parameter(new(40, 24))
    v, g = torch.zeros_like(x, requires_grad=False), new(40, 24)
    loss = (x * x).sum()
    A.muon_step(x, g, v, 0.1)
    assert x._version == 1 and v._version == 1 and g._version == 0
    with pytest.raises(RuntimeError, match="inplace operation"):
        loss.backward()
    (x * x).sum().backward()
    assert torch.equal(x.grad, 2 * x.detach())
    out = torch.empty_like(g)
    A.orthogonalize(g, out=out)
    assert out._version == 1 and g._version == 0
    A.orthogonalize(g, out=g)
    assert g._version == 1
    t, w = new(2, 3, 24), new(2, 24)
    z = torch.empty_like(t)
    A.layer_norm(t, w, out=z)
    assert z._version == 1 and t._version == 0
    A.layer_norm(t, w, out=t)
    assert t._version == 1
    with torch.inference_mode():                      # (tensors that have no counter)
        y = new(40, 24)
        A.orthogonalize(y, out=y)
        A.muon_step(y, new(40, 24), torch.zeros_like(y), 0.1)


def test_results_require_no_gradient():
    import torch
    A = _A()
    x, w = (torch.randn(s, device="cuda", requires_grad=True) for s in ((2, 3, 24), (2, 24)))
    y, mean, rstd = A.layer_norm(x, w)
    dx, dw, db, n, q = A.layer_norm_backward(torch.ones_like(x), x, w, mean, rstd, want_norms=True, want_inner=True)
    for t in (y, mean, rstd, dx, dw, db, n, q, A.orthogonalize(x)):
        assert not t.requires_grad
