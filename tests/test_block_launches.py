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
