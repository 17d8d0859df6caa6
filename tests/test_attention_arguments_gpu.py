"""Arguments of PackedAttention that are refused."""
import pytest

pytestmark = pytest.mark.gpu


def test_devices_other_than_cuda_are_refused():
    import paper_2503_21817_b200 as sk
    for device in ("cpu", "meta"):
        with pytest.raises(ValueError):
            sk.PackedAttention([0, 5], 4, 2, 64, device=device)
    assert sk.PackedAttention([0, 5], 4, 2, 64, device="cuda:0").device == sk.PackedAttention([0, 5], 4, 2, 64).device


def test_offsets_that_are_no_integers_are_refused():
    import numpy as np
    import torch
    import paper_2503_21817_b200 as sk
    for cu in ([0, 4.5], [0.0, 4.0], torch.tensor([0.0, 4.0]), np.array([0.0, 4.5]), ["0", "4"]):
        with pytest.raises(TypeError):
            sk.PackedAttention(cu, 4, 2, 64)
    for cu in ([0, 4], (0, 4), torch.tensor([0, 4]), torch.tensor([0, 4], dtype=torch.int32), np.array([0, 4])):
        assert sk.PackedAttention(cu, 4, 2, 64).tokens == 4
