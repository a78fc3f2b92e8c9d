"""Sizes at which the adapters' calls end, by their workspace queries: nothing is launched."""
import ctypes

import pytest

from test_adapt_args import ct  # noqa: F401


@pytest.mark.parametrize("name", ["ct_adapters_workspace", "ct_adapters_grad_workspace"])
def test_rows_whose_counts_would_pass_32_bits(ct, name):  # noqa: F811
    """Slots and the ends of tiles are counted in 32 bits, up to a step past the last row."""
    f, n = getattr(ct.lib(), name), ctypes.c_size_t()
    for t in (2 ** 31 - 1, 2 ** 31 - 64, 2 ** 31 - 2 ** 16 + 1):
        assert f(t, 3, 16, 64, 64, ctypes.byref(n)) == 5, t
    assert f(2 ** 31 - 2 ** 16, 3, 16, 64, 64, ctypes.byref(n)) == 0
