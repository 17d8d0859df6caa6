"""Arguments of PackedAttention that are refused."""
import pytest

pytestmark = pytest.mark.gpu


def test_devices_other_than_cuda_are_refused():
    import paper_2503_21817_b200 as sk
    for device in ("cpu", "meta"):
        with pytest.raises(ValueError):
            sk.PackedAttention([0, 5], 4, 2, 64, device=device)
    assert sk.PackedAttention([0, 5], 4, 2, 64, device="cuda:0").device == sk.PackedAttention([0, 5], 4, 2, 64).device
