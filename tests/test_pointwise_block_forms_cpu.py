"""The pointwise block's layer norm, 4-bit products and orthogonal updates without a GPU: refusals, and the workspace for every batch."""
import pytest
import torch

from paper_2402_14139_amd import binding as nf
from paper_2402_14139_amd import pointwise as pw
from tests.test_pointwise_block_cpu import BF16, block, no_kernels  # noqa: F401


def serving(**more):
    b = block()
    b.kind, b.mx = "layer", True
    for k, v in more.items():
        setattr(b, k, v)
    return b


BAD = {"more rows than the buffers": torch.zeros(25, 8, dtype=BF16), "no rows": torch.zeros(0, 8, dtype=BF16), "other type": torch.zeros(3, 8),
       "strided": torch.zeros(8, 3, dtype=BF16).t(), "short rows": torch.zeros(3, 7, dtype=BF16), "other device": torch.zeros(3, 8, dtype=BF16, device="meta")}


@pytest.mark.parametrize("why", BAD)
def test_predict_refuses(no_kernels, why):  # noqa: F811
    with pytest.raises(ValueError):
        serving().predict(BAD[why])


def test_predict_refuses_other_blocks(no_kernels):  # noqa: F811
    for more in (dict(kind="group"), dict(mx=False)):
        with pytest.raises(ValueError):
            serving(**more).predict(torch.zeros(3, 8, dtype=BF16))


@pytest.mark.parametrize("why", ["more maps than the buffers", "other type"])
def test_training_refuses(no_kernels, why):  # noqa: F811
    from tests.test_pointwise_block_cpu import BAD as MAPS
    with pytest.raises(ValueError):
        serving().forward(MAPS[why])
    with pytest.raises(ValueError):
        serving().backward(torch.zeros(4, 6, 8, dtype=BF16), MAPS[why])


def test_no_backward_pass_behind_predict(no_kernels):  # noqa: F811
    x, b = torch.zeros(4, 6, 8, dtype=BF16), serving(kept=False)
    with pytest.raises(RuntimeError):
        b.backward(x, x)
    b.kept = True
    with pytest.raises(AttributeError):   # on its way to the kernels, which this block has no buffers for
        b.backward(x, x)


def test_unknown_norm():
    with pytest.raises(ValueError):
        pw.PointwiseBlock(nf.NF_BF16, 1, 1, 8, 8, 1, norm="batch")


@pytest.mark.parametrize("dtype", [nf.NF_F32, nf.NF_BF16])
@pytest.mark.parametrize("B,HW,C,H", [(48, 49, 72, 100), (3, 1, 2048, 512), (33, 67, 1030, 520), (1, 4096, 32, 64), (9, 1000, 512, 2048)])
def test_workspace_holds_every_batch(dtype, B, HW, C, H):
    up, down = (nf.LinearDesc(dtype=dtype, K=k, N=n, act=0) for k, n in ((C, H), (H, C)))
    room = pw.mx_workspace_bytes(up, down, B, HW)
    for M in range(1, B * HW + 1):
        for d in (up, down):
            assert nf.nf_mx_linear_workspace_bytes(d, M) <= room, M
    for M in range(HW, B * HW + 1, HW):
        for k, n in ((C, H), (H, C)):
            assert nf.nf_mx_product_workspace_bytes(nf.LinearDesc(dtype=dtype, K=n, N=k, act=0), M) <= room
            assert nf.nf_mx_product_workspace_bytes(nf.LinearDesc(dtype=nf.NF_F32, K=M, N=k, act=0), n) <= room
