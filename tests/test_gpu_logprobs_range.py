"""headkv_token_logprobs with logits and temperatures that are large or small but
finite: masks of any large negative number, largest logits of any size, quotients
x / temperature far past what fp32 holds to one unit.  Bounds as in
test_gpu_logprobs.py."""
import math

import pytest
import torch

from test_gpu_logprobs import _check, _logits

pytestmark = pytest.mark.gpu
DTYPES = (torch.bfloat16, torch.float32)
TINY = float(torch.tensor(3e-39))  # as fp32 holds it
LARGE = (3e5, 1e9, 9e9, 1e10, 1e20, 1e30)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", (1000, 6000, 40000))
def test_masks_of_large_numbers(dtype, vocab):
    # rows that hold nothing else, half rows, whole segments of 16384 logits, all but
    # one token
    x, t = _logits(4 * len(LARGE), vocab, dtype, 11)
    for i, big in enumerate(LARGE):
        x[4 * i] = -big
        x[4 * i + 1, :vocab // 2] = -big
        x[4 * i + 2, :16384 * (vocab // 16384)] = -big
        x[4 * i + 3] = -big
        x[4 * i + 3, vocab // 3] = 2.5
        t[4 * i + 2] = 5
        t[4 * i + 3] = vocab // 3
    _check(x, t, 32)
    _check(x, t, 0, 0.7)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", (1000, 40000, 65536))
def test_largest_logits_of_any_size(dtype, vocab):
    # of both signs, all equal or only one, in one segment of the row or in all
    x, t = _logits(4 * len(LARGE), vocab, dtype, 12)
    for i, big in enumerate(LARGE):
        x[4 * i, vocab - 7] = big
        x[4 * i + 1] = big
        x[4 * i + 2] = x[4 * i + 2].double().sub(8).mul(big).to(dtype)
        x[4 * i + 3, :vocab // 2] = -big
        x[4 * i + 3, vocab // 2:] = big
        t[4 * i] = vocab - 7
    _check(x, t, 7)
    _check(x, t, 7, 3.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("temperature", (1e-5, 1e-6, 1e-8, 1e-9, 1e-10, 1e-20, 1e-30))
def test_small_temperatures(dtype, temperature):
    temperature = float(torch.tensor(temperature))  # as fp32 holds it
    for vocab in (700, 20000):
        x, t = _logits(6, vocab, dtype, 13)
        x[0] += 20.3
        x[1] -= 30
        x[2] = x[2].double().mul(temperature).to(dtype)  # quotients of order one
        x[3] = 20.3
        x[4, :vocab // 2] = -math.inf
        t[0] = int(x[0].argmax())
        _check(x, t, 4, temperature)


@pytest.mark.parametrize("sign", (-1, 1))
def test_quotients_that_differ_by_little_though_large(sign):
    # steps of a unit in the last place of 3e10, which the temperature makes 2
    vocab = 40000
    g = torch.Generator().manual_seed(14)
    x = sign * (3e10 + 2048.0 * torch.randint(0, 12, (5, vocab), generator=g)).float()
    x[1, :16384] = -2e10 if sign < 0 else 4e10  # one segment away from the others
    x[2, 16384:32768] = -4e10 if sign < 0 else 2e10
    x[3, 20000:] = -math.inf
    x[4, :16384] = 3.0                          # and one of ordinary numbers
    t = torch.randint(0, vocab, (5,), generator=g).to(torch.int32)
    _check(x, t, 20, 1024.0)


@pytest.mark.parametrize("sign", (-1, 1))
@pytest.mark.parametrize("span", (3, 25))
def test_segments_about_the_bound(sign, span):
    # 2^24 in log2 units is where sums leave the product rounded once for all:
    # segments on this side of it and on that, quotients of one to span apart
    vocab = 5 * 16384
    g = torch.Generator().manual_seed(span)
    middle = float(int(2 ** 24 * math.log(2)))
    x = torch.empty((4, vocab))
    for r in range(4):
        for s in range(5):
            at = sign * middle + (s - 2) * (1, -1, 4, -4)[r]
            x[r, s * 16384:(s + 1) * 16384] = at + torch.randint(-span, span + 1, (16384,),
                                                                 generator=g)
    t = torch.randint(0, vocab, (4,), generator=g).to(torch.int32)
    _check(x, t, 9)


@pytest.mark.parametrize("dtype", DTYPES)
def test_temperatures_whose_inverse_is_nearly_too_large(dtype):
    # 1 / 3e-39 is finite, 1 / 3e-39 in log2 units is not; differences of under one, so
    # that log p is a number of fp32
    x = torch.rand((3, 20000), generator=torch.Generator().manual_seed(15)).to(dtype)
    x[1] = 0
    x[2] = -0.25
    x[2, 17777] = 0
    _check(x, torch.tensor([4, 5, 17777], dtype=torch.int32), 3, TINY)


@pytest.mark.parametrize("vocab", (600, 20000))
def test_differences_past_the_largest_number(vocab):
    # x - max is -6e38, and so no number, but log p is: -12 and the like
    x = 3e38 * (2 * torch.rand((4, vocab), generator=torch.Generator().manual_seed(16)) - 1)
    x[1, :vocab // 2], x[1, vocab // 2:] = 3e38, -3e38
    x[2] = torch.finfo(torch.float32).min
    x[2, 3] = torch.finfo(torch.float32).max
    t = torch.tensor([7, vocab - 1, 9, 11], dtype=torch.int32)
    _check(x, t, 5, float(torch.tensor(5e37)))
