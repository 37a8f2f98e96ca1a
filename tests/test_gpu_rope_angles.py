"""The bound that include/iso.h states for a rotary angle, near half a turn, where sines are
small and so show the angle's own error: a sine of 2^-11 or less is rounded by 2^-34."""
import math
import os
import re
from fractions import Fraction

import pytest
import torch

import paper_2607_19331_gb300 as iso

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# 1 / (2 pi) to 60 digits
INV = Fraction(159154943091895335768883763372514362034459645740456448747667, 10 ** 60)


def _stated(p):
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "iso.h")) as f:
        text = re.sub(r"\s*\n \*\s*", " ", f.read())
    first, second, far = re.search(r"\|error\| <= 2\^-(\d+) \+ 2\^-(\d+) \+ \|p\| 2\^-(\d+) turns", text).groups()
    return 2.0 ** -int(first) + 2.0 ** -int(second) + abs(p) * 2.0 ** -int(far)


@pytest.mark.parametrize("inverse", [False, True])
def test_angles_are_as_near_as_stated(inverse):
    n, rows = 64, 120
    g = torch.Generator().manual_seed(11)
    # fractions of a turn 0.4999 .. 0.5001 at position 1; further odd positions stay near half a turn for those next to it
    freq = [2 * math.pi * (0.5 + (float(x) - 0.5) * 10 ** -(4 + i % 6)) for i, x in enumerate(torch.rand(n, generator=g))]
    plan = iso.RopePlan(2 * n, freq, [0] * n, 1)
    pos = [1, -1] + [2 * (int(p) >> r % 40) + 1 for r, p in enumerate(torch.randint(-2 ** 40, 2 ** 40, (rows - 2,), generator=g))]
    x = torch.zeros(rows, 2 * n, device=DEV)
    x[:, :n] = 1
    y = (iso.rope_grad if inverse else iso.rope)(x, torch.tensor(pos, device=DEV), plan).double().cpu()
    turns = [Fraction(f) * INV for f in freq]
    checked = 0
    for r, p in enumerate(pos):
        for i, t in enumerate(turns):
            a = (t * p * (-1 if inverse else 1)) % 1
            if abs(a - Fraction(1, 2)) > Fraction(1, 15000):
                continue
            checked += 1
            # y = (cos, sin) of the angle taken: its distance from a, in turns
            d = float(a - Fraction(1, 2)) * 2 * math.pi
            got = math.atan2(-float(y[r, n + i]), -float(y[r, i]))
            assert abs(got - d) / (2 * math.pi) <= _stated(p) + 2.0 ** -34
    assert checked >= 100
