"""What a refused size of a checkpoint is said to be wrong with."""
import pytest

from paper_2512_14080_amd import binding as B
from test_block8_cpu import built

GOOD = (16, 128, 64, 8, 2)


@built
@pytest.mark.parametrize("dims,capacity,flags,word", [(GOOD, 0, 0, "capacity"), (GOOD, -1, 0, "capacity"),
                                                      (GOOD, 32, 2, "flags"), ((16, 100, 64, 8, 2), 32, 0, "d must")])
def test_refused_sizes_of_a_checkpoint(dims, capacity, flags, word):
    assert B.lib().moe_qexperts_bytes(B.dims(16, 128, 63, 8, 2)) == 0  # (an error of another call before)
    assert B.lib().moe_ckpt_bytes(B.dims(*dims), capacity, flags) == 0
    assert word in B.moe_last_error()


@built
def test_a_refused_checkpoint_names_its_capacity():
    with pytest.raises(B.MoEError, match="capacity must be >= 1"):
        B.Checkpoint(B.dims(*GOOD), 0, device="cpu")
