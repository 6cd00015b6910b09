"""Steps of orthogonal updates whose results leave the range that products of fp16 pieces keep their digits in are refused, and so are sizes
beyond 32 bits."""
import pytest
import torch

from paper_2402_14139_amd import binding as nf

ONE = (1.0, 0.0, 0.0)
# far below 1 between steps or at the end, far above, and both; the last ones' polynomials matter among such singular values, too
GOOD = {"small": [(2e-6, 0.0, 0.0), (5e5, 0.0, 0.0)], "small at the end": [ONE, (3e-6, -1e-6, 0.0)], "large": [(100.0, 0.0, 0.0)] * 4 + [ONE], "large, then not":
        [(100.0, 0.0, 0.0)] * 4 + [(1e-8, 0.0, 0.0)], "large, then small": [(100.0, 0.0, 0.0)] * 4 + [(1.1e-14, 0.0, 0.0)], "large, then bent":
        [(100.0, 0.0, 0.0)] * 4 + [(2e-8, -1e-24, 0.0)], "small, then bent": [(1e-3, 0.0, 0.0), (1.01e-3, 0.0, 0.0), (2.0, -1e12, 0.0)], "nothing": [(0.0, 0.0, 0.0), ONE]}
BAD = {"too small": [(1e-15, 0.0, 0.0), (1e15, 0.0, 0.0)], "too small at the end": [(5e-7, 0.0, 0.0)], "vanishing": [ONE, (1e-25, -1e-25, 0.0)],
       "too large": [(100.0, 0.0, 0.0)] * 4 + [(20.0, 0.0, 0.0)], "large, then too small": [(100.0, 0.0, 0.0)] * 4 + [(1e-15, 0.0, 0.0)]}


@pytest.mark.parametrize("which", GOOD)
def test_accepted(which):
    assert nf.nf_orthogonalise_workspace_bytes(nf.orth_desc(GOOD[which]), [(8, 8)]) > 0


@pytest.mark.parametrize("which", BAD)
def test_refused(which):
    with pytest.raises(nf.NfError) as e:
        nf.nf_orthogonalise_workspace_bytes(nf.orth_desc(BAD[which]), [(8, 8)])
    assert e.value.status == nf.NF_ERR_UNSUPPORTED


@pytest.mark.parametrize("rows,cols", [(1, 2 ** 32 + 64), (2 ** 32 + 64, 1), (2 ** 33 + 8, 2 ** 33 + 8), (8, 2 ** 31)])
def test_sizes_beyond_32_bits(rows, cols):
    with pytest.raises(nf.NfError) as e:
        nf.nf_orthogonalise_workspace_bytes(nf.orth_desc([ONE]), [(rows, cols)])
    assert e.value.status == nf.NF_ERR_UNSUPPORTED


def test_a_tensor_beyond_32_bits():
    """The sizes that the calls take from their tensors."""
    t = torch.empty(1, 2 ** 32 + 64, dtype=torch.bfloat16, device="meta")
    rows, cols = nf._as_matrices([t, torch.empty(64, 3, 3, 3, device="meta")])
    assert list(rows) == [1, 64] and list(cols) == [2 ** 31 - 1, 27]
