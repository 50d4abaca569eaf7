"""How exact the angles of the rotation are, by the kernels' expression in IEEE doubles against rationals (CPU)."""
import random
import re
from fractions import Fraction
from pathlib import Path

import numpy as np
import pytest

from paper_2512_10411_b200.build import CSRC

TURNS = 1 / (2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459"))  # 1 / 2 pi to 60 digits


def source():
    """(the constant of the kernels' expression, what the comment beside it promises up to 2^30 and beyond)."""
    text = (Path(CSRC) / "swaa_rope.cuh").read_text()
    constant, = re.findall(r"const double t = \(double\)position \* \(double\)f\[i\] \* (0\.\d+);", text)
    near, far = re.search(r"keeps its fraction to 2\^-(\d+) for positions up to 2\^30 and to 2\^-(\d+) for every other", text).groups()
    return float(constant), Fraction(1, 2 ** int(near)), Fraction(1, 2 ** int(far))


def off(position, f, constant):
    """Error of the fraction that sincospif gets, in turns: position * f and * constant rounded to double, the rest exact, rounded to fp32."""
    t = float(position) * float(f) * constant
    got = Fraction(float(np.float32(t - np.rint(t))))
    d = (got - position * Fraction(float(f)) * TURNS) % 1
    return min(d, 1 - d)


@pytest.mark.parametrize("top", [2 ** 17, 2 ** 24, 2 ** 30, 2 ** 31])
def test_fraction_of_a_turn(top):
    rng = random.Random(top)
    constant, near, far = source()
    bound = near if top <= 2 ** 30 else far
    worst = Fraction(0)
    for i in range(20000):
        position = rng.choice((-1, 1)) * (top - 1 - rng.randrange(top // (2 if i % 2 else 64)))
        f = np.float32(1.0 if i % 10 == 0 else rng.uniform(0.5, 1) if i % 3 else 10 ** rng.uniform(-7, 0))
        worst = max(worst, off(position, f, constant))
    assert worst <= bound, float(worst / bound)


def test_a_position_beyond_2_to_the_30():
    """2^-24 of a turn does not hold for every 32-bit position."""
    constant, near, far = source()
    assert Fraction(1, 2 ** 24) < off(2108850679, np.float32(0.9973107576370239), constant) <= far
