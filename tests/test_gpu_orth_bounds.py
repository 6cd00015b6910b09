"""Orthogonal updates whose singular values are far from 1 between the steps keep their digits, in one launch and in many."""
import pytest
import torch

from paper_2402_14139_amd import binding as nf
from tests import orth_ref
from tests.test_orth_bounds_cpu import GOOD

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(16, 40), (64, 200), (300, 500)])
@pytest.mark.parametrize("which", GOOD)
def test_digits(which, rows, cols):
    steps = GOOD[which]
    g = orth_ref.gradient(torch.Generator().manual_seed(1), rows, cols)
    d, y = nf.orth_desc(steps), torch.empty(rows, cols, device="cuda")
    ws = torch.full((nf.nf_orthogonalise_workspace_bytes(d, [(rows, cols)]),), 255, dtype=torch.uint8, device="cuda")
    nf.nf_orthogonalise(d, nf.NF_F32, [g.cuda()], [y], ws)
    want = orth_ref.steps(g.double(), steps, d.eps)
    off = (orth_ref.steps(g, steps, d.eps).double() - want).norm()   # the steps' own amplification of roundings; ours are at 2^-22 for 2^-24, both doubled
    assert (y.double().cpu() - want).norm() <= 8 * off + 2.0 ** -20 * want.norm()
