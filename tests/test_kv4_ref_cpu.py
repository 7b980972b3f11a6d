"""The 64-bit reference of rows in 4 bits against exact fractions, group by group."""
from fractions import Fraction

import pytest
import torch

from tests import kv4_ref


def _exact(xs):
    """codes, s, z of 32 bf16 numbers by fractions alone (the range is exact: these rows need no rounding to 32 bits)."""
    x = [Fraction(float(v)) for v in xs]
    low, high = min(x + [Fraction(0)]), max(x + [Fraction(0)])
    e = -100
    while 15 * Fraction(15, 8) * Fraction(2) ** e < high - low:
        e += 1
    s = next(c for c in (Fraction(n, 8) * Fraction(2) ** e for n in range(8, 16)) if 15 * c >= high - low)
    z = round(-low / s)  # (of a Fraction: ties to even)
    return [min(max(round(v / s) + z, 0), 15) for v in x], s, z


@pytest.mark.parametrize("kind", ["normal", "outlier", "positive", "negative", "zero", "ties", "tiny", "edges"])
def test_against_fractions(kind):
    g = torch.Generator().manual_seed(3)
    x = torch.randn(30, 128, generator=g)
    if kind == "outlier":
        x[:, ::17] *= 40
    elif kind == "positive":
        x = x.abs() + 3
    elif kind == "negative":
        x = -x.abs() - 0.01
    elif kind == "zero":
        x[:, 32:64] = 0
    elif kind == "ties":  # multiples of half a step
        x = torch.randint(-15, 16, (30, 128), generator=g) * 0.5 * 1.375
    elif kind == "tiny":
        x = x * 2.0 ** torch.randint(-108, -95, (30, 1), generator=g)
    elif kind == "edges":  # ranges that are 15 scales, or just above
        x = torch.randint(0, 16, (30, 128), generator=g) * torch.tensor([1.0, 1.125, 1.875, 0.0625 * 1.25])[torch.arange(30) % 4, None]
        x[::3, ::32] = 15.0625
    x = x.to(torch.bfloat16)
    codes, s, z = kv4_ref.quantise(x)
    for i in range(len(x)):
        for j in range(4):
            want, ws, wz = _exact(x[i, 32 * j:32 * j + 32])
            assert codes[i, j].tolist() == want and Fraction(float(s[i, j])) == ws and int(z[i, j]) == wz
    held = kv4_ref.values(codes, s, z)
    assert bool(((held - x.double()).abs() <= s.repeat_interleave(32, -1) / 2).all())
    assert torch.equal(held.to(torch.bfloat16).double(), held)  # a bf16 number


def far_apart():
    """Groups whose largest and smallest values are so far apart that fp32 rounds their difference: to 15 scales, where the exact one is
    above (or below) them, and to others."""
    x = torch.zeros(64, 128)
    for i in range(64):
        top = 15.0 * (1 + i % 8 / 8) * 2.0 ** (i % 5 - 2)
        for j in range(4):
            sign = 1 if (i + j) % 2 else -1
            x[i, 32 * j + i % 32] = sign * top
            x[i, 32 * j + (i + 7) % 32] = -sign * top * 2.0 ** -(17 + 3 * j + i // 16)
            x[i, 32 * j + (i + 9) % 32] = sign * top * 0.5
    return x.to(torch.bfloat16)


def test_the_range_is_rounded():
    x = far_apart()
    codes, s, z = kv4_ref.quantise(x)
    rounded = 0
    scales = [Fraction(n, 8) * Fraction(2) ** e for e in range(-8, 8) for n in range(8, 16)]
    for i in range(len(x)):
        for j in range(4):
            g = x[i, 32 * j:32 * j + 32]
            wide = Fraction(float(g.max().float() - g.min().float()))
            rounded += wide != Fraction(float(g.max())) - Fraction(float(g.min()))
            want = next(c for c in scales if 15 * c >= wide)
            zero = round(-Fraction(float(g.min())) / want)
            assert Fraction(float(s[i, j])) == want and int(z[i, j]) == zero
            assert codes[i, j].tolist() == [min(max(round(Fraction(float(v)) / want) + zero, 0), 15) for v in g]
    assert rounded > 100
    held = kv4_ref.values(codes, s, z)
    assert bool(((held - x.double()).abs() <= s.repeat_interleave(32, -1) / 2).all())
    assert float(kv4_ref.quantise(torch.tensor([15.0, -2.0 ** -30] + [0.0] * 126).to(torch.bfloat16))[1][0]) == 1


def test_values_that_are_not_finite():
    x = torch.ones(3, 128, dtype=torch.bfloat16)
    x[0, 5], x[1, 40], x[2, 100] = float("nan"), float("inf"), float("-inf")
    held = kv4_ref.held(x)
    for i, g in enumerate((0, 1, 3)):
        nan = held[i].isnan().unflatten(0, (4, 32)).all(1)
        assert nan.tolist() == [k == g for k in range(4)]


def test_bytes():
    x = torch.arange(128).to(torch.bfloat16)[None, None] % 16
    codes, scales = kv4_ref.row_bytes(*kv4_ref.quantise(x))
    # range 15, so s = 1, z = 0: the codes are the numbers themselves, 0 2 4 6 1 3 5 7 from the low nibble on
    assert codes[0, 0, :8].tolist() == [0x20, 0x64, 0x31, 0x75, 0xA8, 0xEC, 0xB9, 0xFD]
    assert scales[0, 0].tolist() == [0x80, 0x3F] * 4
