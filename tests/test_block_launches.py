"""CPU-only: what the gated projections' gradients launch, and on which addresses (the launches are recorded, none is
made)."""

import os
import shutil

import pytest

from block_launches import gradients

pytestmark = [
    pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++ for the host link"),
    pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="for machines without a GPU: the recorder calls entry "
                       "points with fake device pointers"),
]


@pytest.mark.parametrize("n", [1, 2, 3, 4, 7, 33, 65, 130, 2309, 6529])
@pytest.mark.parametrize("packed", [False, True])
def test_columns_maxima_are_aligned(n, packed):
    """A lane reads those of four columns at once: 16 bytes, at a multiple of them."""
    found = [at for _, _, _, at in gradients(n, 72, 2056, dtype=1, packed=packed) if at is not None]
    assert len(found) == 1 and found[0] % 16 == 0


def _products(n, k, f, **how):
    """Workgroups of dx's product in tiles of 256 and of 128, 0 for none."""
    found = {256: 0, 128: 0}
    for name, groups, _, _ in gradients(n, k, f, dw=False, **how):
        if "rows_kernel" in name:
            found[256 if "Li256ELi256E" in name else 128] += groups
    return found


# columns' tiles that divide a round of 256 workgroups, and 17, 43 and 160 of them
@pytest.mark.parametrize("n,k,both", [(4096 + 256, 4096, True), (4096 + 1792, 4096, True), (4096 + 2048, 4096, False),
                                      (4096, 4352, True), (2048, 11000, False), (3584, 11000, False), (512, 40960, False),
                                      (1536, 11000, True)])
def test_last_round_in_smaller_tiles(n, k, both):
    """A last round of the larger tiles is left to the smaller ones where it is at most 448 of them: 448 take two
    rounds, of less than half of one of the larger each."""
    found = _products(n, k, 1024)
    assert found[256] > 0
    assert (found[128] > 0) == both and found[128] <= 448
    if not both:  # whole: one launch over every row
        assert found[256] == -(-n // 256) * -(-k // 256)
