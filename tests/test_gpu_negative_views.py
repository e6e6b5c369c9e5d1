"""A tensor whose memory holds its numbers with the other sign (the imaginary part of a conjugate) is refused: the kernels read
the memory."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_refused_and_taken_once_resolved():
    import paper_2208_09151_amd as g
    c = torch.randn((40, 1), dtype=torch.complex64, device="cuda")
    x = c.conj().imag
    assert x.is_neg() and x.shape == (40, 1)        # (one column: any stride will do)
    w, ids = torch.ones((1, 3), device="cuda"), torch.arange(40, device="cuda")
    r = g.route(torch.zeros((40, 1), dtype=torch.int64, device="cuda"), 2)
    for call in (lambda t: g.linear(t, w), lambda t: g.linear_backward(t, torch.ones((3, 1), device="cuda")), lambda t: g.bias_gradient(t),
                 lambda t: g.layer_norm(t), lambda t: g.layer_norm_backward(t, t, torch.ones((40, 2), device="cuda"))[0],
                 lambda t: g.lookup(t, ids), lambda t: g.lookup_backward(t, ids, 40), lambda t: g.expert_layer(t, w.mT, w[None].expand(3, 1, 3), 1),
                 lambda t: g.dispatch(t, r), lambda t: g.restore(g.compress(t)), lambda t: g.activate(t, "relu")[0]):
        with pytest.raises(ValueError, match="other sign"):
            call(x)
        call(x.resolve_neg())
    assert torch.equal(g.lookup(x.resolve_neg(), ids), -c.imag)
