"""How many values the norms' 32-bit sums may have: a block's values, by the size of the workspace that holds a part for each block."""
import ctypes

import pytest

from test_adapt_args import ct  # noqa: F401


@pytest.mark.parametrize("values", [10 ** 6, 3 * 10 ** 8, 318767105, 10 ** 9, 10 ** 12])
def test_a_thread_adds_at_most_1024_values(ct, values):  # noqa: F811
    w = ctypes.c_size_t()
    assert ct.lib().ct_clip_grads_workspace(1, values, ctypes.byref(w)) == 0
    blocks = w.value // 16 - 2                       # 16 bytes for each whole block, two more
    # a thread of 256 has its share of a block's 16-byte units, a value before them and one behind
    most = values // blocks // 1024 * 1024           # blocks are multiples of 1024 values
    for unit in (4, 8):
        assert -(-most // (unit * 256)) * unit + 2 <= 1024, (values, most)
