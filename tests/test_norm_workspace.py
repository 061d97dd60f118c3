"""The size of the norm's workspace over the numbers of rows (no GPU)."""
import ctypes

import pytest

from paper_2405_14852_b200 import binding as B


@pytest.mark.parametrize("cols", [1, 64, 100, 128, 256, 257, 1000, 2048, 4096, 8192, 8193, 20000, 32768])
def test_the_workspace_of_any_number_of_rows_is_the_largest(cols):
    def need(rows):
        return B.lib().pvt_norm_workspace_bytes(ctypes.byref(B.pvt_norm(rows=rows, cols=cols)))

    sizes = [need(rows) for rows in [*range(1, 700), *(2 ** i + 1 for i in range(10, 31))]]
    assert sizes == sorted(sizes) and need(2 ** 31 - 1) == sizes[-1] <= 64 << 20
