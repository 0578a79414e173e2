"""Norms of small rows: without an eps down to means of squares of 2^-120, below which fp32 does
not hold them (headkv.h), with one down to bf16's subnormal numbers.

The bounds of test_gpu_rotary.py (its head derives them); rows differ in size, the small ones
beside others, and a row's result does not depend on its neighbours.
"""
import pytest
import torch

from paper_2605_20600_amd.rotary import Rotary
from test_gpu_rotary import _check, _want

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm", ("rms", "layer"))
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("eps,least", ((0.0, -58), (1e-12, -124)))
def test_small_rows(norm, d, eps, least):
    g = torch.Generator().manual_seed(d)
    power = torch.tensor([p for p in (0, -40, -49, -50, -51, -52, -58, -62, -63, -64, -66, -70, -74,
                                      -75, -80, -100, -120, -124, 10, 40) if p >= least])
    x = torch.randn((3, 2, len(power), d), generator=g) * 2.0 ** power[:, None]
    x = x.to(torch.bfloat16)
    pos = torch.randint(0, 100, (3, 2, 1), generator=g, dtype=torch.int32)
    rot = Rotary(d, d // 2, norm=norm, eps=eps)
    got, _ = rot(x.cuda(), None, pos.cuda())
    eps = float(torch.tensor(eps, dtype=torch.float32))
    _check(got, _want(x, pos, d // 2, "half", 1, norm, None, None, eps=eps))
    for h in range(len(power)):
        alone, _ = rot(x[:, :, h:h + 1].contiguous().cuda(), None, pos.cuda())
        assert torch.equal(alone[:, :, 0], got[:, :, h])
    # nothing to divide
    none, _ = rot(torch.zeros((1, 1, 1, d), dtype=torch.bfloat16, device="cuda"), None,
                  pos[:1, :1].cuda().contiguous())
    assert bool(none.isnan().all() if eps == 0 else (none == 0).all())
