"""Wide rows of the norm and its gradient between others, on the GPU: in a
matrix of three rows or more the middle ones are read in pieces where they are
off 16-byte boundaries, the first and the last are not.  The checks and the
tolerances are those of tests/test_gpu_rmsnorm.py."""

import pytest

pytest.importorskip("torch")

from tests import test_gpu_rmsnorm as narrow

pytestmark = pytest.mark.gpu

SIZES = [(5, 4097), (6, 6000), (5, 8193), (160, 8191), (7, 9999), (4, 12001), (3, 16387), (4, 33000)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_wide_rows(rows, cols, dtype):
    narrow.test_forward(rows, cols, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_gradient_of_wide_rows(rows, cols, dtype):
    narrow.test_gradient(rows, cols, dtype)
