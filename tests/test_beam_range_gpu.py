"""Beam search's selection for logits of every size: words that a constraint has set to a large
negative number, products of logit and scale up to the type's largest."""
import math

import pytest
import torch

from beamexact import check
from test_beam_gpu import TYPES, _select

pytestmark = pytest.mark.gpu
LOG2E = 1 / math.log(2)


def _check(x, s, m, **kw):
    out = _select(x, s, m, **kw)
    check(out, x, s, m, **kw)
    return out


def _normal(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * 3


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("fill", [-1e5, -1e6, -1e9, -1e10, -1e11, -1e12, -1e13, -1e16, -1e20, -1e30,
                                  -1e36, -1e37, -3e38])
def test_forbidden_words_of_a_large_number(fill, dtype):
    """One run, all runs but one, all words but a few, all words."""
    x = _normal(2, 4, 6000, seed=1)
    x[0, 1, 2048:4096] = fill
    x[0, 2, 2048:] = fill
    few = x[0, 3, 4999:5003].clone()
    x[0, 3] = fill
    x[0, 3, 4999:5003] = few
    x[1] = fill                                    # the beams' words are all alike ...
    x[1, 2, 17] = fill * 0.5                       # ... but for one of this beam
    x = x.to(TYPES[dtype]).cuda()
    s = torch.tensor([[-11.0, -11.5, -12.0, -12.5], [-3.0, -2.0, -40.0, -5.0]], device="cuda")
    for m in (4, 20):
        out = _check(x, s, m)
        # words 0, 1, ... of beam 1, whose last word was the likeliest
        assert out[1][1].tolist() == [5] * m and out[2][1].tolist() == list(range(m))
    # the only beam that is left
    one = torch.full_like(s, -math.inf)
    one[:, 3] = s[:, 3]
    out = _check(x, one, 6)
    assert sorted(out[2][0].tolist()[:4]) == [4999, 5000, 5001, 5002]
    assert out[2][0].tolist()[4:] == [0, 1]


@pytest.mark.parametrize("dtype,scale,low,high", [
    ("f16", 1e6, 4e3, 6e4), ("f16", 1e5, 2e4, 6.5e4), ("f16", 3e4, -6.5e4, 6.5e4),
    ("f16", 1e6, -6.5e4, -6e4), ("f32", 1e6, 7000.0, 7001.0), ("f32", 1e6, 12345.0, 12346.0),
    ("f32", 1e6, -3e4, -2e4), ("f32", 1.0, 1e10, 1.0001e10), ("f32", 1e-6, 1e16, 1.0001e16),
    ("f32", 1e-6, -2e38, 3e38), ("f32", 1e6, 1e30, 3e38), ("f32", 1e6, -3e38, -1e30),
    ("bf16", 1e6, 100.0, 30000.0), ("bf16", 1.0, 1e9, 1e11), ("bf16", 1.0, -1e20, -1e19),
    ("bf16", 0.37, 1e36, 3e38)])
def test_large_products(dtype, scale, low, high):
    """Logits between two bounds, in several beams of several runs; the largest ones more than once."""
    g = torch.Generator().manual_seed(7)
    x = low + (high - low) * torch.rand(3, 5, 5000, generator=g)
    x[0, 2, 4001], x[0, 2, 30] = x[0, 2].max(), x[0, 2].max()
    s = -1.0 - torch.rand(3, 5, generator=g)
    _check(x.to(TYPES[dtype]).cuda(), s.cuda(), 5, scale=scale)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("power", [20, 22, 23, 24, 26, 28, 29, 30, 31, 32, 40, 64, 100, 120, 122, 123])
def test_exponents_around_a_power_of_two(power, sign):
    """Neighbouring fp32 logits whose exponents in base 2 lie around a power of 2: runs on both sides of
    any border, with words one step and a few steps below the largest."""
    at = torch.tensor(sign * 2.0 ** power / LOG2E)
    steps = torch.tensor([0, -1, 1, 2, -2, 5])
    ulp = 2.0 ** (math.floor(math.log2(abs(float(at)))) - 23)
    g = torch.Generator().manual_seed(power)
    x = float(at) + ulp * (steps.view(1, 6, 1) - torch.randint(0, 40, (1, 6, 4200), generator=g)).double()
    x = x.float().cuda()
    s = -1.0 - torch.arange(6).view(1, 6) * 0.01
    for m in (1, 6, 30):
        _check(x, s.cuda(), m)


def test_differences_past_the_types_range():
    """A word far above all others of its beam, and far below: results by name."""
    x = _normal(1, 2, 3000, seed=3)
    x[0, 0, :] = -3e38
    x[0, 0, 77] = 3e38
    best = int(x[0, 1].argmax())
    x, s = x.cuda(), torch.tensor([[-11.5, -11.9]], device="cuda")
    for scale in (1e-6, 1e-3, 1.0, 1e3, 1e6):
        out = _check(x, s, 2, scale=scale)
        assert out[1][0].tolist() == [0, 1] and out[2][0].tolist() == [77, best]
        assert float(out[0][0, 0]) == -11.5


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("weight", [1.5e-45, 1e-40, 1.2e-38, 1e-36, 1e-30, 1e-20, 1e20, 1e30, 8e37, 9e37,
                                    1.6e38, 1.8e38, 3.4e38])
def test_weights_of_every_size(weight, dtype):
    """The threshold that a run's words have to reach is found in fp32, by a division by the weight."""
    g = torch.Generator().manual_seed(11)
    x = (torch.randn(3, 4, 9000, generator=g) * 3).to(TYPES[dtype]).cuda()
    s = (-10 - 2 * torch.rand(3, 4, generator=g)).cuda()
    s[2] = 0.0
    w = (weight * (1 - 0.01 * torch.rand(3, 4, generator=g))).clamp(min=1.5e-45).cuda()
    w[1] = torch.tensor([1.0, weight, 1e-3, weight])
    for m in (2, 4, 16, 40):
        _check(x, s, m, weight=w)
        _check(x, s, m, weight=w, scale=1e-6)


def test_weights_with_scores_next_to_0():
    """A beam's likeliest word has nearly all of its mass: l is 0 or a few units of 2^-149 after
    weighting, and so small that fp32 has no bits for its product with the weight."""
    x = torch.full((1, 4, 9000), -1e4)
    x[0, :, ::2500] = torch.tensor([0.0, -16.0, -17.0, -18.0])
    s = -torch.tensor([[1.0, 1.3, 1.7, 2.1]])
    for size in (1e-7, 1e-15, 1e-25, 1e-38, 1e-43):
        for weight in (1e-38, 1e-30, 1e-20, 1e-10, 1.0, 1e38):
            w = torch.full((1, 4), weight).cuda()
            for m in (1, 2, 4, 9):
                out = _check(x.cuda(), (s * size).cuda(), m, weight=w)
                assert out[1][0, 0] == 0 and out[2][0, 0] == 0
