"""Extents at the edges of what the training-step operators take: on the CPU what
is refused or only described, on the GPU what runs."""

import pytest

torch = pytest.importorskip("torch")

from tests.test_training_refusals import BASE, UNSUPPORTED, L, mat, ref  # noqa: F401


def test_more_channels_than_the_norm_counts(L):  # noqa: F811
    """(No memory is behind these matrices: what passes the checks of extents is
    refused for its addresses, or for want of a device.)"""
    lib = L.load_library()

    def both(cols):
        x, w = mat(L, rows=1, cols=cols), L.LmTensor(BASE, 1, cols, 0)
        return (lib.lm_rmsnorm(ref(x), None, None, 1e-6, None, ref(x), None, None, None),
                lib.lm_rmsnorm_grad(ref(x), ref(x), None, BASE, None, None, ref(x), ref(w), BASE, 1 << 40, None))

    for cols in (0x7FFFFF00, 0x7FFFFC01, (1 << 31) - 65535):
        assert both(cols) == (UNSUPPORTED, UNSUPPORTED)
    assert UNSUPPORTED not in both((1 << 31) - 65536)
