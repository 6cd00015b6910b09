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


@pytest.mark.parametrize("more", [dict(), dict(norm="layer")])
def test_a_block_without_orthogonal_updates_has_no_room_for_them(on_host, monkeypatch, more):
    """Neither their workspace nor the momentum, nor their limits: only muon() asks."""
    C, H, B, HW = 256, 1024, 2, 8
    orth = nf.nf_orthogonalise_workspace_bytes(nf.orth_desc(pw.MUON_STEPS), [(H, C), (C, H)])

    def refuses(*a):
        raise nf.NfError(nf.NF_ERR_UNSUPPORTED, "nf_orthogonalise_workspace_bytes")

    monkeypatch.setattr(nf, "nf_orthogonalise_workspace_bytes", refuses)
    block = on_host(nf.NF_BF16, B, HW, C, H, 8, **more)
    need = pw.workspace_bytes(block.ln if more else block.norm, block.up, block.down, B, HW)
    assert block.ws.numel() == max(need, 1) < orth and block.v is None
    with pytest.raises(nf.NfError):
        block.muon(0.1, 0.1)
    assert block.v is None   # a second call asks again


def test_momentum_is_made_once(on_host):
    block = on_host(nf.NF_BF16, 2, 8, 64, 128, 8)
    block.prepare_muon()
    v, ws = block.v, block.muon_ws
    assert [t.shape for t in v] == [(128, 64), (64, 128)] and not any(t.any() for t in v)
    assert ws.numel() == nf.nf_orthogonalise_workspace_bytes(block.orth, [(128, 64), (64, 128)])
    with pytest.raises(AssertionError):   # on its way to the kernels
        block.muon(0.1, 0.1)
    assert block.v is v and block.muon_ws is ws
