"""What a pointwise block asks room for, and which sizes it takes, without a GPU: its constructor on host memory, where no kernel runs."""
import pytest
import torch

from paper_2402_14139_amd import binding as nf
from paper_2402_14139_amd import pointwise as pw
from tests.test_pointwise_block_cpu import no_kernels  # noqa: F401


@pytest.fixture
def on_host(no_kernels, monkeypatch):  # noqa: F811
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    return lambda *a, **k: pw.PointwiseBlock(*a, device="cpu", **k)


# rows wider than a group, more maps than a group norm takes
@pytest.mark.parametrize("B,HW,C,H", [(2, 3, 4096, 16), (1, 1, 1 << 16, 8), (65536, 1, 8, 8)])
def test_layer_norms_own_limits(on_host, B, HW, C, H):
    block = on_host(nf.NF_BF16, B, HW, C, H, 1, norm="layer")
    need = max(max(nf.nf_layernorm_workspace_bytes(block.ln, b * HW), *(nf.nf_linear_workspace_bytes(d, b * HW) for d in (block.up, block.down)))
               for b in {1, 2, B // 3 + 1, B})
    assert block.ws.numel() >= need
    with pytest.raises(nf.NfError):
        on_host(nf.NF_BF16, B, HW, C, H, 1)
