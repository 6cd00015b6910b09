"""Steps of orthogonal updates whose results are far from 1."""
import pytest

from paper_2402_14139_amd import binding as nf

ONE = (1.0, 0.0, 0.0)
# far below 1 between steps or at the end, far above, and both; the last ones' polynomials matter among such singular values, too
GOOD = {"small": [(2e-6, 0.0, 0.0), (5e5, 0.0, 0.0)], "small at the end": [ONE, (3e-6, -1e-6, 0.0)], "large": [(100.0, 0.0, 0.0)] * 4 + [ONE], "large, then not":
        [(100.0, 0.0, 0.0)] * 4 + [(1e-8, 0.0, 0.0)], "large, then small": [(100.0, 0.0, 0.0)] * 4 + [(1.1e-14, 0.0, 0.0)], "large, then bent":
        [(100.0, 0.0, 0.0)] * 4 + [(2e-8, -1e-24, 0.0)], "small, then bent": [(1e-3, 0.0, 0.0), (1.01e-3, 0.0, 0.0), (2.0, -1e12, 0.0)], "nothing": [(0.0, 0.0, 0.0), ONE]}


@pytest.mark.parametrize("which", GOOD)
def test_accepted(which):
    assert nf.nf_orthogonalise_workspace_bytes(nf.orth_desc(GOOD[which]), [(8, 8)]) > 0
