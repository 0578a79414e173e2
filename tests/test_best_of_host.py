"""What best_of refuses before anything is on a GPU."""
import pytest
import torch

from paper_2605_20600_amd.best_of import generate


@pytest.mark.parametrize("prompt,images,steps", (
    (torch.zeros(0, dtype=torch.int64), 2, 3), (torch.zeros((1, 4), dtype=torch.int64), 2, 3),
    (torch.zeros(4, dtype=torch.int64), 0, 3), (torch.zeros(4, dtype=torch.int64), 2, 0),
    (torch.zeros(4, dtype=torch.int64), -1, 3)))
def test_nothing_to_generate(prompt, images, steps):
    with pytest.raises(ValueError, match="at least 1"):
        generate(None, prompt, images, steps)
