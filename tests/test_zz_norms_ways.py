"""Every kernel of the norms is chosen by a size of the tests: the host code that chooses is asked for a wide range of sizes and for the tests' own; the sizes below are those that the other file's list
leaves out."""
import pytest

import test_zz_norms as N
from test_zz_experts import gpu
from test_zz_norms_launches import Launches


# rows, width, dtype, extra between rows, shift: kernels that no size of the other file takes
SIZES = [(5, 5001, "f32", 0, 0), (3, 8191, "f32", 1, 1), (4, 9001, "bf16", 0, 0), (3, 9999, "f16", 0, 1), (700, 1501, "f32", 0, 0), (600, 3001, "f16", 3, 1), (601, 2049, "bf16", 0, 0),
         (33, 2000, "f32", 0, 0), (11, 2075, "f32", 0, 3), (4, 8217, "f32", 0, 0), (6, 17001, "f32", 1, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_kernel_of_the_norms_is_chosen(dtype, tmp_path):
    launches = Launches(tmp_path)
    there, gone = {}, set()
    for what in range(3):
        for rows in (1, 2, 600):
            for width in list(range(1, 40)) + list(range(40, 40000, 37)) + [64 * i for i in range(1, 600)] + [1 << 24]:
                for launch in launches.of(what, dtype, rows, width):
                    there.setdefault((launch[0], launch[4]), (rows, width))
        for rows, width, kind, *_ in N.SIZES + SIZES:
            if (kind == "f32") == (dtype == "f32"):
                gone |= {(launch[0], launch[4]) for launch in launches.of(what, dtype, rows, width)}
    assert len(there) > 20
    assert {kernel: size for kernel, size in there.items() if kernel not in gone} == {}


@gpu
@pytest.mark.parametrize("residual,weighted", [(True, True), (False, False)])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_norms(size, residual, weighted):
    N.test_norms(*size, residual, weighted)
    N.test_norms_in_8_bits(*size, residual, weighted)
    N.test_gradients(*size, residual, weighted)


@gpu
@pytest.mark.parametrize("width", [2049, 5001, 9001])
def test_in_place(width):
    N.test_sum_in_place_of_an_input_and_norm_in_place_of_the_other(width)
