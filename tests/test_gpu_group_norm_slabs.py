"""Every kernel of group norm, named by the measurement's records, against 64 bits: small groups, slabs of one to many groups whose
vectors lie in one group, in several or start anywhere, last slabs of fewer channels, and slabs in chunks."""
import pytest

from paper_2402_14139_amd import binding as nf
from tests import test_gpu_pointwise as tp

pytestmark = pytest.mark.gpu

# (B, HW, C, G): kernels forward and backward of fp32, then of 16 bits
CASES = {
    (1, 1, 68, 1): ("few_256", "few_256", "few_256", "few_256"),
    (1, 1, 261, 1): ("few_1024", "few_1024", "few_1024", "few_1024"),
    (1, 5, 606, 1): ("few_1024_deep", "few_1024_deep", "few_1024_deep", "few_1024_deep"),
    (3, 25, 12, 4): ("few_64", "few_64", "few_64", "few_64"),
    (1, 1, 1045, 1): ("tiny_odd", "tiny_odd", "tiny_odd", "tiny_odd"),
    (1, 1, 1176, 1): ("tiny", "tiny", "tiny", "tiny"),
    (1, 3, 1423, 1): ("slab_odd", "slab_odd", "small_odd", "small_odd"),
    (1, 3, 1608, 1): ("slab", "slab", "small", "small"),
    (1, 34, 692, 2): ("slab_mixed", "split_mixed", "slab_odd", "slab_odd"),
    (1, 5594, 9, 3): ("slab_odd", "split_odd", "slab_odd", "split_odd"),
    (1, 33, 1704, 1): ("split", "split", "slab", "split"),
    (1, 4279, 8, 2): ("slab", "slab", "slab_mixed", "split_mixed"),
    (1, 3042, 24, 3): ("slab", "slab", "slab", "slab"),
    (1, 2060, 57, 1): ("split_odd", "split_odd", "split_odd", "split_odd"),
    (1, 69, 1880, 4): ("split_mixed", "split_mixed", "split_mixed", "split_mixed"),
    (3, 5000, 40, 5): ("slab", "split", "slab", "slab"),
    (1, 99, 1280, 1): ("split", "split", "split", "split"),
    (1, 1637, 30, 3): ("slab_odd", "split_odd", "slab_odd", "slab_odd"),
    (1, 4602, 12, 3): ("slab", "slab", "slab_odd", "split_odd"),
    (2, 86, 360, 2): ("slab", "slab", "slab_mixed", "slab_mixed"),
    (33, 675, 72, 12): ("slab_mixed", "slab_mixed", "slab_mixed", "slab_mixed"),
    (23, 75, 912, 304): ("tiny_mixed", "tiny_mixed", "tiny_mixed", "tiny_mixed"),
    (298, 44, 120, 2): ("small", "small", "small_mixed", "small_mixed"),
    (282, 60, 93, 93): ("tiny_odd", "tiny_odd", "tiny_odd", "tiny_odd"),
    (356, 158, 28, 14): ("small_mixed", "small_mixed", "small_odd", "small_odd"),
    (12, 67, 1960, 245): ("small", "small", "tiny", "tiny"),
    (4, 213, 1850, 370): ("small_odd", "small_odd", "small_odd", "small_odd"),
    (155, 48, 212, 212): ("tiny_mixed", "tiny_mixed", "tiny_odd", "tiny_odd"),
    (19, 391, 216, 54): ("small", "small", "small_mixed", "small_mixed"),
    (1, 5745, 24, 6): ("slab", "slab", "slab_mixed", "split_mixed"),
    (210, 625, 12, 12): ("slab_mixed", "slab_mixed", "slab_odd", "slab_odd"),
    (39, 791, 51, 17): ("slab_odd", "slab_odd", "slab_odd", "slab_odd"),
    (149, 8, 1320, 220): ("tiny_mixed", "tiny_mixed", "tiny_mixed", "tiny_mixed"),
    (68, 58, 399, 133): ("tiny_odd", "tiny_odd", "tiny_odd", "tiny_odd"),
    (28, 251, 224, 28): ("tiny", "tiny", "tiny", "tiny"),
    (4, 349, 1128, 141): ("small", "small", "small", "small"),
    (276, 2, 2856, 357): ("tiny", "tiny", "tiny", "tiny"),
    (416, 223, 17, 17): ("small_odd", "small_odd", "small_odd", "small_odd"),
    (25, 881, 72, 18): ("slab", "slab", "slab_mixed", "slab_mixed"),
    (4, 1024, 512, 32): ("slab", "slab", "slab", "slab"),
    (64, 1001, 512, 32): ("slab", "slab", "slab", "slab"),
    (110, 1212, 12, 3): ("slab", "slab", "slab_odd", "slab_odd"),
}


def expected(direction, kernel):
    """A slab in chunks takes two kernels."""
    if not kernel.startswith("split"):
        return {f"groupnorm_{direction}_{kernel}"}
    return {f"groupnorm_{direction}_{k}{kernel[5:]}" for k in ("stats", "apply")}


@pytest.mark.parametrize("t", tp.TYPES)
@pytest.mark.parametrize("shape", CASES)
def test_kernels(t, shape):
    fwd, bwd = CASES[shape][:2] if t == "f32" else CASES[shape][2:]
    nf.nf_prof_begin()
    try:
        tp.test_group_norm(t, *shape)
    finally:
        got = {r["kernel"] for r in nf.nf_prof_end()}
    want = expected("fwd", fwd) | expected("bwd", bwd)
    assert want <= got and not got - want - {"groupnorm_bwd_sums", "groupnorm_bwd_chunk_sums"}, got


def test_every_kernel_is_among_these_cases():
    kinds = {k + r for k in ("tiny", "small", "slab", "split") for r in ("", "_mixed", "_odd")} | {"few_64", "few_256", "few_1024", "few_1024_deep"}
    for i in range(4):
        assert {c[i] for c in CASES.values()} == kinds, i


@pytest.mark.parametrize("t,shape,fwd,bwd", [
    ("f32", (192, 16, 512, 32), True, True), ("f32", (384, 16, 256, 16), True, True), ("f32", (385, 16, 256, 16), False, False),
    ("f32", (48, 256, 128, 32), False, False), ("bf16", (218, 100, 48, 4), False, False), ("bf16", (7, 905, 64, 8), True, True),
    ("bf16", (39, 105, 264, 8), True, True), ("f16", (28, 144, 96, 8), True, False), ("f32", (16, 64, 64, 8), True, True)])
def test_both_sides_of_the_rule_for_small_groups(t, shape, fwd, bwd):
    nf.nf_prof_begin()
    try:
        tp.test_group_norm(t, *shape)
    finally:
        got = {r["kernel"] for r in nf.nf_prof_end() if not r["kernel"].endswith("sums")}
    assert {k.split("_")[1]: "_few_" in k for k in got} == {"fwd": fwd, "bwd": bwd}, got
