"""Verification at temperatures next to the least and the largest that are taken: all the
probability lies on the largest logits, equal ones in equal parts, or is spread evenly."""
import pytest
import torch

from test_gpu_verify import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("model", (True, False))
@pytest.mark.parametrize("t", (8.1e-309, 1e-308, 1e-307, 2.5e-307, 2.7e-307, 1e-300, 1e-40, 1e300,
                               1.7e308))
def test_temperatures_of_any_size(dtype, model, t):
    x, tokens, u, y = _inputs(12, 4, 5000, dtype, 8, model, masked=100)
    for r in range(12):  # equal largest ones, in one block's logits and in several; good drafts
        top = x[r].max(1).values
        for n, at in enumerate((130 + r, 2500, 4999 - r)[:1 + r % 3]):
            x[r, :, at] = top + 1
            if model:
                y[r, 1:, at] = x[r, 1:4, at] if n < 2 else y[r, 1:, at]
        if r % 2:
            tokens[r] = 130 + r
    _, count = _check(x.cuda(), tokens, u, None if y is None else y.cuda(), t=t)
    assert bool((count >= 1).all())
    if t < 1:
        assert int(count.max()) > 1
