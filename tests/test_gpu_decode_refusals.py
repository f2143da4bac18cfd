"""What the attention block and the serving loop refuse because its results would be wrong."""
import pytest
import torch

from test_gpu_decode import blocks

pytestmark = pytest.mark.gpu


def test_requests_longer_than_the_angles():
    """A position behind the last angle's is neither rotated nor cached: the tokens behind it would attend to what lay in its place before."""
    from paper_2007_12216_amd.decode import DecodingBatch
    stack = blocks(1, 8, 100) + blocks(1, 8, 70, seed=1)
    DecodingBatch(stack, 1, 70)
    with pytest.raises(ValueError, match="angles"):
        DecodingBatch(stack, 1, 71)
