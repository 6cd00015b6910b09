"""The pointwise block: its gradients against 64-bit autograd through the same steps, and training from quantised caches."""
import pytest
import torch

from paper_2402_14139_amd import binding as nf
from tests import pointwise_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
def test_gradients_against_autograd(act):
    from paper_2402_14139_amd.pointwise import PointwiseBlock
    B, HW, C, H, G, p, step = 3, 10, 24, 40, 4, 0.25, 7
    blk = PointwiseBlock(nf.NF_F32, B, HW, C, H, G, act=ref.ACTS.index(act), p=p, seed=5)
    g = torch.Generator().manual_seed(1)
    for k in ("gamma", "beta", "b1", "b2"):
        blk.p32[k] += 0.3 * torch.randn(blk.p32[k].shape, generator=g).cuda()
    x, dy = torch.randn(B, HW, C, generator=g), torch.randn(B, HW, C, generator=g)
    y = blk.forward(x.cuda(), step)
    dx = blk.backward(x.cuda(), dy.cuda(), step)
    P = {k: v.double().cpu().requires_grad_() for k, v in blk.p32.items()}
    X = x.double().requires_grad_()
    v = X.reshape(B, HW, G, C // G)
    v = v - v.mean((1, 3), keepdim=True)
    v = (v * (v.square().mean((1, 3), keepdim=True) + blk.norm.eps).rsqrt()).reshape(B, HW, C)
    h = ref.act(act, v * P["gamma"] + P["beta"]).reshape(B * HW, C)
    a = ref.act(act, h @ P["W1"].t() + P["b1"]) * ref.keep_scale(B * HW, H, p, 10, step)
    Y = X.reshape(B * HW, C) + (a @ P["W2"].t() + P["b2"]) * ref.keep_scale(B * HW, C, p, 11, step)
    (Y * dy.double().reshape(B * HW, C)).sum().backward()
    # five fp32 calls in a row, each within some tens of roundings of its largest terms: 1e-5 of the results' norm
    close = lambda got, want: (got.double().cpu() - want).norm() <= 1e-5 * want.norm()  # noqa: E731
    assert close(y.reshape(B * HW, C), Y.detach())
    assert close(dx.reshape(B, HW, C) + dy.cuda(), X.grad)
    for k, w in P.items():
        assert close(blk.grad[k], w.grad), k


@pytest.mark.parametrize("fmt,p", [(nf.NF_Q_INT8, 0.0), (nf.NF_Q_E4M3, 0.05), (nf.NF_Q_E2M1, 0.0)])
def test_training_from_a_quantised_cache(fmt, p):
    from paper_2402_14139_amd.pointwise import fit
    losses = fit(fmt=fmt, p=p)
    assert all(0 < v < 10 for v in losses) and losses[-1] < 0.7 * losses[0], losses


@pytest.mark.parametrize("B", [1, 31, 41, 47])
def test_a_smaller_batch_than_the_blocks(B):
    """A block of 48 maps on fewer: all calls run in its workspace, to the bits that a block of that batch gives."""
    from paper_2402_14139_amd.pointwise import PointwiseBlock
    args = dict(HW=49, C=72, H=100, groups=12, p=0.1, seed=2)
    large, own = PointwiseBlock(nf.NF_BF16, 48, **args), PointwiseBlock(nf.NF_BF16, B, **args)
    g = torch.Generator().manual_seed(B)
    x, dy = (torch.randn(B, 49, 72, generator=g).bfloat16().cuda() for _ in range(2))
    for b in (large, own):
        b.out = b.forward(x, 3).clone(), b.backward(x, dy, 3).clone()
    assert all(torch.equal(u, v) for u, v in zip(large.out, own.out))
    assert all(torch.equal(large.grad[k], own.grad[k]) for k in own.grad)
