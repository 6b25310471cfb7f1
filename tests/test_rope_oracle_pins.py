"""Pins of the rotary oracle and of the tables of frequencies (CPU)."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import rope_oracle as ro
from paper_2404_11068_amd import rope


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_gradients_are_those_of_differences(interleaved, norm):
    rng = np.random.default_rng(0)
    x, dy = rng.standard_normal((2, 3, 2, 8)), rng.standard_normal((2, 3, 2, 8))
    w = 1 + 0.3 * rng.standard_normal(8)
    pos, freq = rng.integers(-50, 50, (2, 3)), [1.0, 0.3, 0.01]
    kw = dict(interleaved=interleaved, amplitude=1.3, norm=norm, eps=1e-3)
    f = lambda x, w: float(np.sum(dy * ro.forward(x, pos, freq, w=w if norm else None, **kw)))
    dx, dw = ro.backward(dy, x, pos, freq, w=w if norm else None, **kw)
    step = 1e-6

    def slope(at, which):
        hi, lo = [x.copy(), w.copy()], [x.copy(), w.copy()]
        hi[which][at] += step
        lo[which][at] -= step
        return (f(*hi) - f(*lo)) / (2 * step)

    for at in [(0, 0, 0, 0), (1, 2, 1, 5), (0, 1, 1, 3), (1, 0, 0, 7)]:
        assert abs(slope(at, 0) - dx[at]) < 1e-7
    if norm:
        for at in range(8):
            assert abs(slope((at,), 1) - dw[at]) < 1e-7
    else:
        assert dw is None


def test_rotation_keeps_lengths_and_depends_on_differences():
    rng = np.random.default_rng(1)
    freq = rope.rope_frequencies(16)
    q, k = rng.standard_normal((1, 1, 1, 16)), rng.standard_normal((1, 1, 1, 16))
    dots = []
    for shift in (0, 17, 100000):
        a = ro.rotate(q, np.array([[5 + shift]]), freq, False)
        b = ro.rotate(k, np.array([[2 + shift]]), freq, False)
        assert abs(np.linalg.norm(a) - np.linalg.norm(q)) < 1e-12
        dots.append(float(np.sum(a * b)))
    assert max(dots) - min(dots) < 1e-9
    assert np.array_equal(ro.rotate(q, np.array([[0]]), freq, True), q)


def _pi():
    """pi to 80 digits by Machin's formula."""
    def arctan(n):
        power, total, k = 10 ** 90 // n, 0, 0
        while power:
            total += (-1) ** k * (power // (2 * k + 1))
            power //= n * n
            k += 1
        return total
    return Fraction(4 * (4 * arctan(5) - arctan(239)), 10 ** 90)


def test_steps_are_the_frequencies_turns():
    pi = _pi()
    freq = rope.rope_frequencies(64) + [0.0, -1.0, 7.5, 2 * math.pi]
    steps = rope.rope_steps(freq, device="cpu")
    assert steps.dtype == torch.int64 and steps.shape == (36,)
    for f, s in zip(freq, steps.tolist()):
        turns = Fraction(f) / (2 * pi) * 2 ** 64
        off = (turns - s) % 2 ** 64
        assert min(off, 2 ** 64 - off) <= Fraction(1, 2) + Fraction(1, 2 ** 40), f
    # a tensor gives the same
    assert torch.equal(rope.rope_steps(torch.tensor(freq, dtype=torch.float64)), steps)
    assert rope.rope_steps([], device="cpu").shape == (0,)


def test_frequencies():
    f = rope.rope_frequencies(8, 10000.0)
    assert np.allclose(f, [1.0, 0.1, 0.01, 0.001], rtol=1e-15)
    assert np.allclose(rope.rope_frequencies(8, factor=4.0), np.array(f) / 4)
    b = rope.rope_frequencies(8, factor=4.0, scaling="base")
    assert b[0] == 1.0 and abs(b[-1] * 4 / f[-1] - 1) < 1e-12
    t = rope.rope_frequencies(8, factor=4.0, scaling="turns", trained_length=4096)
    # 652, 65, 6.5 and 0.65 turns: the first two are kept, the last is divided
    assert t[:2] == f[:2] and t[3] == f[3] / 4 and f[2] / 4 < t[2] < f[2]
    share = math.log(4096 * f[2] / (2 * math.pi)) / math.log(32)
    assert abs(t[2] - f[2] * (share + (1 - share) / 4)) < 1e-15
    assert rope.rope_amplitude(1.0) == 1.0 and abs(rope.rope_amplitude(4.0) - 1.138629436) < 1e-9
    assert rope.rope_frequencies(0) == [] and rope.rope_frequencies(2, factor=2.0, scaling="base") == [1.0]
    for bad in (dict(rot_dim=3), dict(rot_dim=-2), dict(rot_dim=8, base=0.0), dict(rot_dim=8, factor=0.0),
                dict(rot_dim=8, scaling="other"), dict(rot_dim=8, scaling="turns", fast=1.0)):
        with pytest.raises(ValueError):
            rope.rope_frequencies(**bad)
    for bad in ([math.nan], [math.inf]):
        with pytest.raises(ValueError):
            rope.rope_steps(bad, device="cpu")
