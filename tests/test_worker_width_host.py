"""An embedding block of rows that cannot be pulled is refused when it is made, before any memory is asked for."""
import pytest

import paper_2205_11048_amd as gba
from paper_2205_11048_amd.worker import EmbeddingBlock


@pytest.mark.parametrize("D", [-4, 0, 1, 33, 258, 260, 1024])
def test_width(D):
    with pytest.raises(gba.GBAError, match="multiple of 4"):
        EmbeddingBlock(16, D, 100)
