"""The sines and cosines of the rotary calls, seen through results of bf16.

A pair (1, 0) becomes (cos t, sin t), which bf16 rounds once.  Beside a whole quarter of a turn one
of the two is small, and bf16's steps there are far finer than fp32's beside 1: whoever works
the sine out from a rest that is not small, or to some 2^-23 whatever its size, rounds many of
them to the wrong side.  With the nearest quarter taken off in 64 bits the rest x, |x| <= 0.4,
has the relative errors of its rounding to fp32 (u = 2^-24), of 2 pi in fp32 (u / 2) and of
their product (u); the sine's series adds at most x^2 / 6 < 0.03 of it with four roundings
and a last rounding (u): below 4 u of the sine.  A cosine, 0.92 and more, has x^2 of the rest's
errors, x^2 / 2 with two roundings and half a unit of 2^-24: below 2 u.  The angle itself is a
product of 64 bits, off by 2^-53 of its turns.  So a result may lie on the wrong side of a border
between two bf16 where it is nearer to it than 2^-22 of itself and 2 pi 2^-52 of its turns,
and nowhere else.
"""
import math

import pytest
import torch

from paper_2605_20600_amd.rotary import Rotary

pytestmark = pytest.mark.gpu


def _unit(turns):
    """(cos, sin) of angles in turns, 64 bits, and the rest of the nearest quarter."""
    quarter = torch.round(4 * turns)
    rest = turns - quarter / 4  # exact
    c, s = torch.cos(2 * math.pi * rest), torch.sin(2 * math.pi * rest)
    q = torch.remainder(quarter, 4)
    cos = torch.where(q == 0, c, torch.where(q == 1, -s, torch.where(q == 2, -c, s)))
    sin = torch.where(q == 0, s, torch.where(q == 1, c, torch.where(q == 2, -s, -c)))
    return cos, sin, rest


@pytest.mark.parametrize("d,layout,far", ((128, "half", 0), (64, "pairs", 0), (128, "pairs", 1 << 17),
                                          (64, "half", -(1 << 17))))
def test_angles_beside_whole_quarters(d, layout, far):
    n = d // 2
    g = torch.Generator().manual_seed(d)
    rot = Rotary(d, layout=layout)
    # pair j: some quarters a position, and 2^-18 to 2^-13 of a turn or that less (far
    # positions: so little that their rests are as small)
    j = torch.arange(n, dtype=torch.float64)
    small = 2.0 ** (-18 + 4 * j / n) * (1 + torch.rand(n, generator=g, dtype=torch.float64))
    if far:
        small = small * 2.0 ** -10
    table = (j % 8) / 4 + torch.where(j % 3 == 0, -small, small)
    rot.turns.copy_(table)
    p = far + torch.cat((torch.arange(1, 1000), torch.arange(-1000, 0)))
    x = torch.zeros((1, len(p), 1, d), dtype=torch.bfloat16)
    x[..., :n if layout == "half" else d:1 if layout == "half" else 2] = 1
    got, _ = rot(x.cuda(), None, p.to(torch.int32).cuda()[None])
    got = got[0, :, 0].cpu().double()
    got = (got[:, :n], got[:, n:]) if layout == "half" else (got[:, 0::2], got[:, 1::2])
    t = p.double()[:, None] * table
    cos, sin, rest = _unit(t)
    there = rest.abs() <= 0.4 / (2 * math.pi)
    told = 0
    for y, z in zip((cos, sin), got):
        size = y.abs().clamp(min=1e-30)
        half = 2.0 ** (torch.floor(torch.log2(size)) - 8)
        slack = 2.0 ** -22 * size + 2 * math.pi * 2.0 ** -52 * t.abs()
        off = (z - y).abs() - half
        assert bool((off <= slack)[there].all()), float((off / slack)[there].max())
        # those that an error of 2^-23 could take across
        border = (torch.remainder(size / (2 * half), 1) - 0.5).abs() * 2 * half
        told += int(((border < 2.0 ** -23) & (border > slack) & there).sum())
    assert int(there.sum()) > 50000 and told > 150, (int(there.sum()), told)


def test_angles_of_a_whole_turn():
    # |x| up to pi / 4: the rest's errors are 2.5 u |x| in the angle, at most 0.56 of which reach
    # either result, the series' terms with their roundings below 0.7 u and the last rounding
    # half a unit of 2^-24: below 3 u of 1
    d, n = 128, 64
    rot = Rotary(d)
    table = torch.rand(n, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    rot.turns.copy_(table)
    p = torch.arange(-1000, 1000)
    x = torch.zeros((1, len(p), 1, d), dtype=torch.bfloat16)
    x[..., :n] = 1
    got, _ = rot(x.cuda(), None, p.to(torch.int32).cuda()[None])
    t = p.double()[:, None] * table
    for y, z in zip(_unit(t), got[0, :, 0].cpu().double().split(n, 1)):
        half = 2.0 ** (torch.floor(torch.log2(y.abs().clamp(min=1e-30))) - 8)
        off = (z - y).abs() - half
        assert bool((off <= 3 * 2.0 ** -24 + 2 * math.pi * 2.0 ** -52 * t.abs()).all())
