"""Bytes and calls that a profiled step counts where the hidden weights take steps with orthogonalised momentum."""
import pytest

from test_operators import _muon_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dims,prec,hb", [((72, 136, 40, 5), 0, True), ((72, 136, 40, 5), 1, True), ((64, 32, 10), 1, False)])
def test_a_profiled_step_counts_what_the_update_moves(dims, prec, hb):
    import torch
    from paper_2406_13936_amd import workloads as W
    M, b, steps = 2, 48, 3
    with torch.cuda.stream(torch.cuda.Stream()):
        w, _, _, _, rep, _ = _muon_case(dims, prec, b, M, hb)
        try:
            rep.profile_enable(True)
            for t in range(steps):
                rep.local_step(W.step_indices(w, 0, t, b), w.lr)
            got = rep.profile_read()
        finally:
            rep.close()
    hidden = sum(i * o for i, o in zip(dims[:-2], dims[1:-1]))
    rest = dims[-2] * dims[-1] + (sum(dims[1:]) if hb else 0)
    # AdamW's step: x, v, m read and written, g read (and the bf16 copy written); of hidden weights the gradient is read for its norm
    want = steps * M * (rest * (28 + 2 * prec) + 4 * hidden)
    assert got["update"]["bytes"] == want and got["update"]["calls"] == steps
    # momentum and weights read and written, g read (and the bf16 copy written), a call to each hidden layer
    assert got["muon"]["bytes"] == steps * M * hidden * (20 + 2 * prec) and got["muon"]["calls"] == steps * (len(dims) - 2)
