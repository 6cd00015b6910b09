"""In which order a pointwise block's calls may come, and on what, without a GPU: its bookkeeping on host memory, with kernels that do nothing."""
import pytest
import torch

from paper_2402_14139_amd import binding as nf
from paper_2402_14139_amd import pointwise as pw

FORMS = [dict(), dict(norm="layer"), dict(norm="layer", mx=True), dict(mx=True)]
B, HW, C, H = 3, 4, 16, 24


@pytest.fixture
def idle(monkeypatch):
    for name in nf.EXPORTS:
        if not name.endswith("_bytes"):
            monkeypatch.setattr(nf, name, lambda *a, **k: None, raising=False)
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    return lambda **k: pw.PointwiseBlock(nf.NF_BF16, B, HW, C, H, 2, device="cpu", **k)


def maps():
    return torch.zeros(B, HW, C, dtype=torch.bfloat16)


@pytest.mark.parametrize("more", FORMS)
def test_one_backward_pass_for_a_forward_pass(idle, more):
    block = idle(**more)
    with pytest.raises(RuntimeError):   # uninitialised buffers
        block.backward(maps(), maps())
    for _ in range(2):
        block.forward(maps())
        block.backward(maps(), maps())
        with pytest.raises(RuntimeError):   # the second layer's input is gone: dW2 would be wrong
            block.backward(maps(), maps())


@pytest.mark.parametrize("more", FORMS)
def test_forward_refuses_its_own_results(idle, more):
    """They would be written over while the residual is read, and backward() would normalise the new ones."""
    block = idle(**more)
    y = block.forward(maps())
    for train in (True, False):
        for own in (y, y[1:], block.y.view(B, HW, C)[:2]):
            with pytest.raises(ValueError):
                block.forward(own, train=train)
    block.forward(y.clone())


@pytest.mark.parametrize("more", FORMS)
def test_no_backward_pass_behind_a_forward_pass_without_its_dropout(idle, more):
    """Masks would be applied to the gradients that no result had."""
    block = idle(p=0.2, **more)
    block.forward(maps(), train=False)
    with pytest.raises(RuntimeError):
        block.backward(maps(), maps())
    block.forward(maps())
    block.backward(maps(), maps())
    block = idle(**more)   # no dropout: the same function either way
    block.forward(maps(), train=False)
    block.backward(maps(), maps())


@pytest.mark.parametrize("more", FORMS)
def test_backward_is_of_the_same_batch_and_masks(idle, more):
    block = idle(p=0.2, **more)
    block.forward(maps(), 5)
    for x, step in ((maps()[:2], 5), (maps(), 4)):
        with pytest.raises(RuntimeError):
            block.backward(x, x, step)
    block.backward(maps(), maps(), 5)
    block = idle(**more)
    block.forward(maps()[:2], 5)
    with pytest.raises(RuntimeError):
        block.backward(maps(), maps(), 5)
    block.backward(maps()[:2], maps()[:2], 4)   # no masks to choose
