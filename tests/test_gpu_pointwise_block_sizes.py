"""The pointwise block with layer norm at sizes that no group norm takes, gradients against 64-bit autograd; orthogonal updates first called in a
capture."""
import pytest
import torch

from tests import layer_norm_ref
from tests import pointwise_ref as ref
from tests.test_gpu_pointwise_block_forms import prepared

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,HW,C,H", [(3, 5, 4096, 24), (65537, 1, 16, 24)])
def test_gradients_against_autograd(B, HW, C, H):
    M = B * HW
    blk, x, dy = prepared("f32", B, HW, C, H, act=ref.ACTS.index("gelu"))
    y = blk.forward(x.cuda())
    dx = blk.backward(x.cuda(), dy.cuda())
    P = {k: v.double().cpu().requires_grad_() for k, v in blk.p32.items()}
    X = x.double().reshape(M, C).requires_grad_()
    h = layer_norm_ref.forward(X, P["gamma"], P["beta"], blk.ln.eps)[0]
    Y = X + ref.act("gelu", h @ P["W1"].t() + P["b1"]) @ P["W2"].t() + P["b2"]
    (Y * dy.double().reshape(M, C)).sum().backward()
    # five fp32 calls in a row, each within some tens of roundings of its largest terms: 1e-5 of the results' norm
    near = lambda got, want: (got.double().cpu() - want).norm() <= 1e-5 * want.norm()  # noqa: E731
    assert near(y.reshape(M, C), Y.detach())
    assert near((dx + dy.cuda()).reshape(M, C), X.grad)
    for k, w in P.items():
        assert near(blk.grad[k], w.grad), k


@pytest.mark.parametrize("prepared_before", [False, True])
def test_a_first_orthogonal_update_within_a_capture(prepared_before):
    """The momentum begins at zero with the first update that runs, captured or not, and no replay clears it again."""
    pair = [prepared("bf16", 2, 20, 72, 136, mx=True)[0] for _ in range(2)]
    g = torch.Generator().manual_seed(3)
    for k, w in pair[0].grad.items():
        w.copy_(torch.randn(w.shape, generator=g))
        pair[1].grad[k].copy_(w)
    if prepared_before:
        pair[0].prepare_muon()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pair[0].muon(0.02, 0.01)
    for turn in range(6):
        graph.replay() if turn % 3 else pair[0].muon(0.02, 0.01)   # the first to run is not the captured one
        pair[1].muon(0.02, 0.01)
        torch.cuda.synchronize()
        for k, w in pair[1].p32.items():
            assert torch.equal(pair[0].p32[k], w) and torch.isfinite(w).all(), (k, turn)
        assert all(torch.equal(a, b) for a, b in zip(pair[0].v, pair[1].v)), turn
        pair[0].grad["W1"].mul_(0.9), pair[1].grad["W1"].mul_(0.9)
