"""Results that the card has no room for are torch's own error, as from any other allocation."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_no_room_for_the_results():
    from paper_2007_12216_amd.decoder import Cache4
    cache = Cache4(1, 16, 64, 256)
    slots = torch.full((1 << 25,), -1, dtype=torch.int64, device="cuda")  # 1 TiB of keys
    with pytest.raises(torch.cuda.OutOfMemoryError):
        cache.read(slots)
    assert (cache.read(slots[:4])[0] == 0).all()
