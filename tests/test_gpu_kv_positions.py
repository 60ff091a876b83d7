"""Rotary angles at any position, against exact arithmetic."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
PI = Fraction(314159265358979323846264338327950288419716939937510582097494459, 10 ** 62)


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    return R


@pytest.mark.parametrize("hd", [64, 66])     # in whole eights of elements, and not
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_positions(R, hd, layout):
    """Pairs (1, 0), which become the angle's cosine and sine: half a step of float32 of the half turns (an angle of
    pi 2^-25), two steps of the sine and cosine, and no more however far the position is."""
    rot = 64
    freqs, _ = R.riftkv_rope_freqs(rot)
    freqs[1:4] = 5.578125, 3.0, 0.9      # the first: its turns as one float64, times 2^31, are 1.2e-6 radians off
    rng = np.random.default_rng(5)
    # (the first five: among those where a rounded product of position and turns is furthest off, 4e-7 at 3 radians a position)
    pos = [2137390034, 2141675906, 2143803342, 2130796829, -2131155304, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 0, -1] + [int(x) for x in rng.integers(-2 ** 31, 2 ** 31, 40)] + \
          [int(x) for x in rng.integers(2 ** 26, 2 ** 28, 20)]
    x = torch.zeros(len(pos), 1, hd, device="cuda")
    first = torch.arange(rot // 2) if layout == "half" else 2 * torch.arange(rot // 2)
    second = first + rot // 2 if layout == "half" else first + 1
    x[..., first.cuda()] = 1.0
    y = torch.empty_like(x)
    R.riftkv_rope(x, None, torch.tensor(pos, dtype=torch.int32, device="cuda"), freqs, y, layout=layout)
    torch.cuda.synchronize()
    turns = [[Fraction(p) * Fraction(float(f)) / (2 * PI) for f in freqs] for p in pos]
    turns = torch.tensor([[float(t - round(t)) for t in row] for row in turns], dtype=torch.float64)
    angle = 2 * math.pi * turns
    y = y[:, 0].double().cpu()
    bound = math.pi * 2.0 ** -25 + 2 * 2.0 ** -24 + 2.0 ** -40
    off = torch.maximum((y[:, first] - torch.cos(angle)).abs(), (y[:, second] - torch.sin(angle)).abs())
    assert float(off.max()) <= bound, float(off.max())


@pytest.mark.parametrize("low", [0.0, 1e-9, 2.0 ** -1060, 1e9])
def test_frequencies_of_any_size(R, low):
    """Frequencies of nothing, subnormal ones and ones of many turns a position."""
    freqs = np.array([low, -low, 3.0, 0.25])
    pos = [0, 1, -7, 2 ** 20 + 3]
    x = torch.zeros(len(pos), 1, 8, device="cuda")
    x[..., :4] = 1.0
    y = torch.empty_like(x)
    R.riftkv_rope(x, None, torch.tensor(pos, dtype=torch.int32, device="cuda"), freqs, y)
    torch.cuda.synchronize()
    turns = [[Fraction(p) * Fraction(float(f)) / (2 * PI) for f in freqs] for p in pos]
    turns = torch.tensor([[float(t - round(t)) for t in row] for row in turns], dtype=torch.float64)
    y = y[:, 0].double().cpu()
    bound = math.pi * 2.0 ** -25 + 2 * 2.0 ** -24 + 2.0 ** -40
    off = torch.maximum((y[:, :4] - torch.cos(2 * math.pi * turns)).abs(), (y[:, 4:] - torch.sin(2 * math.pi * turns)).abs())
    assert float(off.max()) <= bound, float(off.max())
