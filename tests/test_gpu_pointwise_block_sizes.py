"""The pointwise block with layer norm at sizes that no group norm takes: gradients against 64-bit autograd."""
import pytest

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
