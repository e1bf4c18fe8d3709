"""The kernels of the norm that the library holds are those that some width chooses."""
import re

import pytest

import paper_2510_21956_amd as la

ALIKE = {(8, 1), (16, 1), (32, 1), (64, 1)}  # lanes to a row (0: a workgroup), steps


@pytest.mark.parametrize("kernel,shapes", [("k_norm", ALIKE | {(64, 2), (0, 2)}),
                                           ("k_norm_back", ALIKE | {(128, 1), (0, 1), (0, 2)})])
def test_no_kernel_that_no_width_chooses(kernel, shapes):
    with open(la.library_path(), "rb") as f:
        names = re.findall(rb"_ZN2la12_GLOBAL__N_1%d%sI(ff|tf|tt)Li(\d+)ELi(\d+)EEE" % (len(kernel), kernel.encode()), f.read())
    assert {(t, int(lanes), int(steps)) for t, lanes, steps in names} == {(t, *s) for t in (b"ff", b"tf", b"tt") for s in shapes}
