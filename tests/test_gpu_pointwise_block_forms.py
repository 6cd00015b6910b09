"""The pointwise block with layer norm, products on 4-bit operands and orthogonal updates, in training, in graphs and in serving.  Every stage is
held against 64 bits from the operands that the stage before left: one step of fp32 for each term of a sum, half a step of the results' type."""
import pytest
import torch

from paper_2402_14139_amd import binding as nf
from paper_2402_14139_amd.pointwise import MUON_STEPS, PointwiseBlock, fit
from tests import layer_norm_ref, mx_ref, orth_ref
from tests import pointwise_ref as ref
from tests.pointwise_ref import DT, FUNC, HALF, SUM, TINY, TYPES
from tests.test_gpu_pointwise import close

pytestmark = pytest.mark.gpu


def prepared(t, B, HW, C, H, p=0.0, seed=5, **more):
    blk = PointwiseBlock(DT[t], B, HW, C, H, 1, p=p, seed=seed, norm="layer", **more)
    g = torch.Generator().manual_seed(1)
    for k in ("gamma", "beta", "b1", "b2"):
        blk.p32[k] += 0.3 * torch.randn(blk.p32[k].shape, generator=g).cuda()
    x, dy = (torch.randn(B, HW, C, generator=g).to(TYPES[t]) for _ in range(2))
    return blk, x, dy


@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
def test_gradients_against_autograd(act):
    B, HW, C, H, p, step = 3, 10, 24, 40, 0.25, 7
    blk, x, dy = prepared("f32", B, HW, C, H, p, act=ref.ACTS.index(act))
    y = blk.forward(x.cuda(), step)
    dx = blk.backward(x.cuda(), dy.cuda(), step)
    P = {k: v.double().cpu().requires_grad_() for k, v in blk.p32.items()}
    X = x.double().reshape(B * HW, C).requires_grad_()
    h = layer_norm_ref.forward(X, P["gamma"], P["beta"], blk.ln.eps)[0]
    a = ref.act(act, h @ P["W1"].t() + P["b1"]) * ref.keep_scale(B * HW, H, p, 10, step)
    Y = X + (a @ P["W2"].t() + P["b2"]) * ref.keep_scale(B * HW, C, p, 11, step)
    (Y * dy.double().reshape(B * HW, C)).sum().backward()
    # five fp32 calls in a row, each within some tens of roundings of its largest terms: 1e-5 of the results' norm
    near = lambda got, want: (got.double().cpu() - want).norm() <= 1e-5 * want.norm()  # noqa: E731
    assert near(y.reshape(B * HW, C), Y.detach())
    assert near((dx + dy.cuda()).reshape(B * HW, C), X.grad)
    for k, w in P.items():
        assert near(blk.grad[k], w.grad), k


def four(x):
    """x's rows as their 4 bits stand for them."""
    return torch.from_numpy(mx_ref.quantise(x.double().cpu().numpy())[2])


def check_product(name, t, got, a, b, bias=0.0, more=0.0):
    """a b^T + bias, and a residual; the sum's order is the kernel's own."""
    want, size = a @ b.t() + bias, a.abs() @ b.abs().t() + torch.as_tensor(bias).abs()
    err = (a.shape[1] + 2) * SUM * size
    total = want + more
    close(name, got.double().cpu(), total, err + (HALF[t] + 2 * SUM) * (total.abs() + err) + TINY[t])


SIZES = [(3, 10, 24, 40), (1, 33, 100, 70), (5, 49, 72, 260), (2, 500, 512, 136)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("B,HW,C,H", SIZES)
def test_four_bit_training(t, B, HW, C, H):
    M = B * HW
    blk, x, dy = prepared(t, B, HW, C, H, mx=True)
    x, dy = x.cuda(), dy.cuda()
    y = blk.forward(x)
    x64, P = x.double().cpu().reshape(M, C), {k: v.double().cpu() for k, v in blk.p32.items()}
    h, a = blk.h.clone(), blk.a.clone()
    want = layer_norm_ref.forward(x64, P["gamma"], P["beta"], blk.ln.eps)[0]
    # C terms in either sum, a product and a sum behind them; the row's values are below 8 times its spread
    close("h", h.double().cpu(), want, (C + 16) * SUM * (8 * P["gamma"].abs() + P["beta"].abs()) + HALF[t] * want.abs() + TINY[t])
    W1, W2 = four(blk.p32["W1"]), four(blk.p32["W2"])
    check_product("z1", t, blk.z1, four(h), W1, P["b1"])
    check_product("y", t, y.reshape(M, C), four(a), W2, P["b2"], x64)
    dx = blk.backward(x, dy)
    assert torch.equal(blk.dz2, dy.reshape(M, C))   # neither activation nor dropout
    dz1 = blk.a                                     # its room is used again
    check_product("da", t, blk.da, four(blk.dz2), four(blk.p32["W2"].t()))
    check_product("dh", t, blk.dh, four(dz1), four(blk.p32["W1"].t()))
    check_product("dW2", "f32", blk.grad["W2"], four(blk.dz2.t()), four(a.t()))
    check_product("dW1", "f32", blk.grad["W1"], four(dz1.t()), four(h.t()))
    d64 = blk.dh.double().cpu()
    mean, rstd = blk.mean.double().cpu(), blk.rstd.double().cpu()
    want, dgamma, dbeta = layer_norm_ref.gradients(d64, x64, P["gamma"], mean, rstd)
    g = (d64 * P["gamma"]).abs()
    size = rstd[:, None] * (g + g.mean(1, keepdim=True) + 8 * (8 * g).mean(1, keepdim=True))   # |xhat| below 8
    close("dx", dx.double().cpu().reshape(M, C), want, (C + 16) * SUM * size + HALF[t] * want.abs() + TINY[t])
    close("dgamma", blk.grad["gamma"].double().cpu(), dgamma, (M + 4) * SUM * (8 * d64.abs()).sum(0) + TINY["f32"])
    close("dbeta", blk.grad["beta"].double().cpu(), dbeta, (M + 4) * SUM * d64.abs().sum(0) + TINY["f32"])


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("C,H", [(24, 40), (72, 260)])
def test_orthogonal_updates(mx, C, H):
    blk, x, dy = prepared("bf16", 4, 30, C, H, mx=mx)
    v = {k: torch.zeros_like(w).double().cpu() for k, w in blk.p32.items()}
    lr, mu, wd, sgd = 0.05, 0.9, 0.1, 0.01
    for step in range(3):
        blk.forward(x.cuda())
        blk.backward(x.cuda(), dy.cuda())
        was, grad = ({k: w.double().cpu() for k, w in ws.items()} for ws in (blk.p32, blk.grad))
        blk.muon(lr, sgd, mu, wd)
        for k, w in blk.p32.items():
            if k in ("W1", "W2"):
                v[k] = mu * v[k] + grad[k]
                m = grad[k] + mu * v[k]
                scale = lr * max(1.0, m.shape[0] / m.shape[1]) ** 0.5
                new = lambda u: was[k] * (1 - lr * wd) - scale * u.double()  # noqa: E731
                want = new(orth_ref.steps(m, MUON_STEPS, blk.orth.eps))
                # the steps' own amplification of roundings as fp32 shows it, operands at 2^-22, both doubled; some roundings of the momentum and of the result
                off = (new(orth_ref.steps(m.float(), MUON_STEPS, blk.orth.eps)) - want).norm()
                assert (w.double().cpu() - want).norm() <= 8 * off + 8 * SUM * (want.norm() + was[k].norm()) + scale * 2.0 ** -20 * m.shape[0] ** 0.5, (k, step)
            else:
                want = was[k] - sgd * grad[k]
                close(k, w.double().cpu(), want, 4 * SUM * (want.abs() + (sgd * grad[k]).abs()))
        for k in ("W1", "W2"):
            assert torch.equal(blk.w[k], blk.p32[k].bfloat16())
            if mx:
                n, room = blk.p32[k].shape[1], nf.nf_qcache_row_bytes(nf.NF_Q_E2M1, blk.p32[k].shape[1])
                codes = blk.q[k][0].pair[0].view(-1, room[0]).cpu()
                assert (mx_ref.unpack(codes, n) == mx_ref.quantise(blk.p32[k].double().cpu().numpy())[0]).all()


def test_training_in_a_graph():
    """Forward, backward and update captured once and replayed, with other work in between, to the bits of the same steps run one by one."""
    pair = [prepared("bf16", 4, 100, 72, 136, p=0.1, mx=True)[0] for _ in range(2)]
    x, dy = (t.cuda() for t in prepared("bf16", 4, 100, 72, 136)[1:])

    def step(b):
        b.dxs = b.backward(x, (b.forward(x, 3).float() + dy).to(x.dtype), 3)
        b.muon(0.01, 0.01)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(pair[0])
    for k in range(4):
        graph.replay()
        step(pair[1])
        torch.cuda.synchronize()
        assert torch.equal(pair[0].dxs, pair[1].dxs), k
        for n, w in pair[1].p32.items():
            assert torch.equal(pair[0].p32[n], w) and torch.isfinite(w).all(), (n, k)
        assert all(torch.equal(a, b) for a, b in zip(pair[0].v, pair[1].v))
        x.mul_(0.9)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows", [1, 2, 9, 17, 32, 33, 70])
def test_serving(t, rows):
    blk, _, _ = prepared(t, 5, 14, 130, 264, mx=True)
    x = torch.randn(rows, 130, generator=torch.Generator().manual_seed(rows)).to(TYPES[t]).cuda()
    y = blk.predict(x)
    P = {k: v.double().cpu() for k, v in blk.p32.items()}
    z = four(blk.h[:rows]) @ four(blk.p32["W1"]).t()
    want = ref.act("gelu", z + P["b1"])
    size = four(blk.h[:rows]).abs() @ four(blk.p32["W1"]).abs().t() + P["b1"].abs()
    err = 1.13 * 132 * SUM * size + FUNC * (z + P["b1"]).abs()
    close("a", blk.a[:rows].double().cpu(), want, err + (HALF[t] + 2 * SUM) * (want.abs() + err) + TINY[t])
    check_product("y", t, y, four(blk.a[:rows]), four(blk.p32["W2"]), P["b2"], x.double().cpu())


def test_serving_its_own_results():
    blk, x, _ = prepared("bf16", 1, 40, 64, 96, mx=True)
    y = blk.predict(x.cuda().view(40, 64))
    with pytest.raises(ValueError):
        blk.predict(y[:3])
    assert torch.isfinite(blk.predict(y[:3].clone())).all()


def test_a_row_served_is_a_row_trained():
    """What is kept for the gradients changes no bit."""
    blk, x, _ = prepared("f16", 2, 40, 64, 96, mx=True)
    want = blk.forward(x.cuda(), train=False).clone()
    assert torch.equal(blk.predict(x.cuda().view(80, 64)), want.view(80, 64))
    with pytest.raises(RuntimeError):
        blk.backward(x.cuda(), x.cuda())
    blk.forward(x.cuda())
    blk.backward(x.cuda(), x.cuda())


@pytest.mark.parametrize("more", [dict(norm="layer"), dict(norm="layer", muon_lr=0.02), dict(norm="layer", muon_lr=0.02, mx=True, fmt=nf.NF_Q_E2M1),
                                  dict(muon_lr=0.02, mx=True)])
def test_the_example_runs(more):
    losses = fit(items=128, epochs=2, **more)
    assert len(losses) == 2 and all(0 < v < 100 for v in losses), losses
