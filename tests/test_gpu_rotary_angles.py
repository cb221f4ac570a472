"""The rotation's angle alone, against the product of position and frequency reduced with whole numbers.

A head of (1, 0, ..) turns into (cos t, sin t), without another rounding.  Tolerance, in units of 2^-24: the angle's one
rounding to fp32 is half a step of at most half a turn, 2^-26 turns, 2 pi 2^-26 = 1.58 units of a cosine; the sine and cosine
are off by a unit in the last place, 1 below 1: under 2.6.  What the reduction in 64 bits loses is below 2^-40 turns."""
import math

import numpy as np
import pytest
import torch

import paper_2501_16007_b200 as tl

pytestmark = pytest.mark.gpu
DEV = "cuda"
ALLOWED = 2.6 * 2.0 ** -24
BITS = 400


def arctan_inverse(n, one):
    total, term, k = 0, one // n, 1
    while term:
        total += term // k if k % 4 == 1 else -(term // k)
        term //= n * n
        k += 2
    return total


ONE = 1 << BITS
PI = 4 * (4 * arctan_inverse(5, ONE) - arctan_inverse(239, ONE))
PER_TURN = ONE * ONE // (2 * PI)                       # 1 / (2 pi), times 2^BITS


def turns(position, freq):
    """The fraction of a turn that position * freq comes to, exact to far below 2^-100."""
    m, e = math.frexp(float(freq))
    m = int(m * 2 ** 24)                               # freq = m 2^(e - 24)
    v, shift = position * m * PER_TURN, BITS - (e - 24)
    return (v & ((1 << shift) - 1)) * 2 ** 80 // (1 << shift) / 2.0 ** 80


def check(positions, freq, dim, pairing):
    """Every channel pair's cosine and sine at every position."""
    half = len(freq)
    first, second = (np.arange(half), np.arange(half) + half) if pairing == "halves" else (2 * np.arange(half),
                                                                                          2 * np.arange(half) + 1)
    q = torch.zeros((len(positions), 1, dim), device=DEV)
    q[:, :, torch.from_numpy(first).to(DEV)] = 1
    out, _ = tl.toploc_norm_rotary_prompt(q, q.clone(), torch.tensor(positions, dtype=torch.int32, device=DEV),
                                          torch.tensor(freq, dtype=torch.float32, device=DEV), pairing=pairing)
    out = out[:, 0].double().cpu().numpy()
    t = np.array([[turns(p, f) for f in freq] for p in positions]) * 2 * math.pi
    off = max(np.abs(out[:, first] - np.cos(t)).max(), np.abs(out[:, second] - np.sin(t)).max())
    assert off <= ALLOWED, off / 2.0 ** -24


def some_positions(seed, low, high, count):
    r = np.random.default_rng(seed)
    return [low, high] + [int(v) for v in r.integers(low, high, count)]


@pytest.mark.parametrize("dim,pairing", [(128, "halves"), (128, "neighbours"), (2, "halves"), (34, "neighbours")])
@pytest.mark.parametrize("low,high", [(0, 1000), (10 ** 5, 10 ** 6), (2 ** 30, 2 ** 31 - 1), (-2 ** 31, -2 ** 30)])
def test_positions(dim, pairing, low, high):
    freq = [float(np.float32(10000.0 ** (-i / (dim // 2)))) for i in range(dim // 2)]
    check(some_positions(dim, low, high, 400), freq, dim, pairing)


@pytest.mark.parametrize("dim", [16, 2])
def test_frequency_one_at_the_farthest(dim):
    check(some_positions(3, 2 ** 30, 2 ** 31 - 1, 4000), [1.0] * (dim // 2), dim, "halves")


@pytest.mark.parametrize("scale", [3.0, 1e3, 1e6, 2.0 ** 33])
def test_frequencies_above_one(scale):
    r = np.random.default_rng(4)
    freq = [float(np.float32(scale * f)) for f in r.uniform(0.5, 1, 32)]
    check(some_positions(5, 0, 2 ** 31 - 1, 300), freq, 64, "halves")
    check(some_positions(6, 0, 10000, 300), freq, 64, "neighbours")


def test_frequencies_below_one():
    freq = [float(np.float32(2.0 ** -i)) for i in (1, 10, 24, 31, 40, 100, 126, 140)]   # to a subnormal one
    check(some_positions(7, -2 ** 31, 2 ** 31 - 1, 300), freq, 16, "halves")
