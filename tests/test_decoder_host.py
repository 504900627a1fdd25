"""The 8-bit decoder's checks of its prompts, which come before anything reaches the GPU (an index outside the embedding is an
error there that ends the process's use of it)."""
import pytest
import torch

from paper_2203_12091_gb300.decoder import Decoder


@pytest.fixture
def model():
    m = Decoder.__new__(Decoder)  # (its checks alone: no layers, no GPU)
    m.embed, m.pages, m.max_tokens = torch.zeros(10, 4), torch.zeros(2, 3, dtype=torch.int32), 20
    return m


@pytest.mark.parametrize("prompts,count", [([[10]], 1), ([[0, 9], [3, 11, 2]], 1), ([[-1]], 1), ([], 1), ([[]], 1), ([[1], []], 2), ([[1]], 0),
                                           ([[1] * 20], 1), ([[1]], 20), ([[1], [2], [3]], 1)])
def test_prompts_are_refused(model, prompts, count):
    with pytest.raises(ValueError):
        model.generate(prompts, count)
