"""Arguments of the decoder's generate (host only)."""
import pytest
import torch


def test_generate_arguments():
    from paper_2607_24953_amd.decoder import Decoder
    model = Decoder(layers=1, hidden=64, heads=1, kv_heads=1, device="cpu")
    some = torch.tensor([1, 2])
    for prompts, count in (([some, some[:0]], 3), ([], 3), ([some], -1)):
        with pytest.raises(ValueError):
            model.generate(prompts, count)
    assert model.generate([some, some], 0).shape == (2, 0)
