"""How far a number in a scaled cache may be off after its block's scale has grown: the rule in 64 bits, without a GPU."""
import pytest
import torch

from scaled_testlib import codes_of, numbers, step_of


def held(y, kind, scales):
    """What is left of the numbers y that were written under scales[0] while the block's scale grew to scales[-1]."""
    c = codes_of(y / scales[0], kind)
    for old, new in zip(scales, scales[1:]):
        c = codes_of(numbers(c, kind) * (old / new), kind)
    return numbers(c, kind) * scales[-1]


GROWTHS = [[1, 2], [1, 4], [1, 2, 4], [1, 2, 4, 8, 16, 32, 64], [1, 8, 16, 512], [1, 2.0 ** 20], [2.0 ** k for k in range(24)]]


@pytest.mark.parametrize("scales", GROWTHS, ids=lambda s: "-".join("%g" % x for x in s[:4]))
def test_e4m3(scales):
    """2^-4 of itself, or 2^-9 of the scale in all.  A number that is rounded again is below the smallest normal one, 2^-6, of
    the first such scale s1, so its first rounding was off by at most 2^-11 s1; each further one adds at most 2^-10 of its scale,
    and the scales at least double: 2^-10 (2 - 2^-n) of the last one, n roundings later."""
    y = torch.cat([torch.linspace(0, 448, 300001, dtype=torch.float64), torch.logspace(-16, 9, 300001, base=2, dtype=torch.float64)])
    y = y[y <= 448]
    err = (held(y, "e4m3", scales) - y).abs()
    assert (err <= torch.maximum(2.0 ** -4 * y, torch.tensor(2.0 ** -9 * scales[-1], dtype=torch.float64))).all()


def test_e4m3_needs_that_allowance():
    """14.51 * 2^-9 becomes 15 * 2^-9 under a scale of 1 and 16 * 2^-9 under 2: 2^-10 of the scale would not cover it."""
    y = torch.tensor([14.51 * 2.0 ** -9], dtype=torch.float64)
    assert numbers(codes_of(y, "e4m3"), "e4m3") == 15 * 2.0 ** -9 and held(y, "e4m3", [1, 2]) == 16 * 2.0 ** -9
    assert float((held(y, "e4m3", [1, 2]) - y).abs()) > max(2.0 ** -4 * float(y), 2.0 ** -10 * 2)


@pytest.mark.parametrize("scales", GROWTHS, ids=lambda s: "-".join("%g" % x for x in s[:4]))
def test_int8(scales):
    """Half of every scale: less than the last one in all."""
    y = torch.linspace(-127, 127, 300001, dtype=torch.float64)
    assert ((held(y, "int8", scales) - y).abs() <= scales[-1]).all()


@pytest.mark.parametrize("first", [0.75, 0.999, 1.3])
def test_a_scale_that_was_no_power_of_two(first):
    """Every number is rounded twice then: e4m3 is off by 2^-4 twice (and their product), integers as above."""
    new = 2.0 if first > 1 else 1.0
    y = torch.linspace(-1, 1, 300001, dtype=torch.float64)
    x = y * 448 * first
    bound = torch.maximum((2.0 ** -3 + 2.0 ** -8) * x.abs(), torch.tensor(2.0 ** -9 * new, dtype=torch.float64))
    assert ((held(x, "e4m3", [first, new]) - x).abs() <= bound).all()
    x = y * 127 * first
    assert ((held(x, "int8", [first, new]) - x).abs() <= new).all()
    assert step_of(torch.tensor([1.0], dtype=torch.float64), "e4m3") == 2.0 ** -3
