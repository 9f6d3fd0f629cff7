"""The streamed dense products over the longest reductions: their slices of k (no GPU needed)."""
import os

import pytest

from paper_2512_14080_amd import binding as B
from test_dense_launches import launches

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libsonicmoe.so not built")


@pytest.mark.parametrize("T", [1, 4, 8, 9, 16])
def test_slices_of_long_reductions(T, tmp_path):
    """64 columns of k rows, up to the most that is not refused: 16 slices and their join on either side of where k times a
    row's 256 bytes passes 2^31 (k = 2^23)."""
    ks = [1 << 16, (1 << 23) - 128, 1 << 23, (1 << 23) + 8, (1 << 24) - 8]
    for k, got in zip(ks, launches([["fwd", T, k, 64, "none"] for k in ks], tmp_path)):
        assert "linear_few" in got[0][0] and got[0][2] == 16, (k, got)
        assert len(got) == 2 and "join" in got[1][0], (k, got)
