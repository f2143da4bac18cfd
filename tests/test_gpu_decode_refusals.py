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


def test_parts_that_do_not_belong_together():
    """An attention over another cache than the one that the block writes, and a rotation of other heads than the projection's."""
    from paper_2007_12216_amd.decode import AttentionBlock, rotation_angles
    from paper_2007_12216_amd.decoder import CacheAttention, QKNormRope
    a, b = blocks(1, 4, 70)[0], blocks(1, 4, 70, seed=1)[0]
    AttentionBlock(a.qkv, a.rope, a.cache, CacheAttention(a.cache, 6), a.out)
    with pytest.raises(ValueError, match="cache"):
        AttentionBlock(a.qkv, a.rope, a.cache, b.attention, a.out)
    for q, kv, dim in ((2, 4, 64), (14, 2, 32), (1, 2, 128)):
        with pytest.raises(ValueError, match="heads"):
            AttentionBlock(a.qkv, QKNormRope(q, kv, dim, rotation_angles(70, dim)), a.cache, a.attention, a.out)
