"""The scales of 4-bit quantisation next to the borders between two of them, against exact fractions: each is the value of its type nearest to the
exact quotient, ties to even, so scales and zero points are compared for equality and codes with the quotients by them."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2406_03853_b200 as eesd

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def nearest(x, bits):
    """the value with `bits` significant bits (fp32's exponents) nearest to the fraction x > 0, ties to even"""
    e = max(x.numerator.bit_length() - x.denominator.bit_length() - 1, -126)
    while x >= Fraction(2) ** (e + 1):
        e += 1
    step = Fraction(2) ** (e - bits + 1)
    n, rest = divmod(x, step)
    if rest * 2 > step or (rest * 2 == step and n % 2):
        n += 1
    return n * step


def rows(scale, seed):
    """extremes (hi, lo) of groups: quotients on a border of the scale's type, and beside it by less than double precision tells"""
    g = np.random.default_rng(seed)
    bits = 8 if scale == "bf16" else 24
    out = []
    for _ in range(40):
        m = (int(g.integers(2 ** (bits - 1), 2 ** bits)) * 2 + 1) * 2.0 ** int(g.integers(-60, 40))   # halfway between two scales
        top = 15 * Fraction(m)
        hi = float(np.float32(float(top)))
        if Fraction(hi) > top:
            hi = float(np.nextafter(np.float32(hi), np.float32(0)))
        rest = float(top - Fraction(hi))                                                          # (0 for bf16: 13 bits)
        for lo in (rest, float(np.nextafter(np.float32(rest), np.float32(np.inf))), rest + hi * 2.0 ** -60 if rest == 0 else rest, float(np.nextafter(np.float32(rest), np.float32(-1)))):
            lo = max(float(np.float32(lo)), 0.0)
            out += [(hi, -lo), (lo, -hi)]
    out += [(15.05859375, -1e-20), (1e-20, -15.05859375), (15.05859375, 0.0), (15.17578125, -1e-20), (15.17578125, 0.0), (2.0 ** -140, -2.0 ** -149), (22 * 2.0 ** -149, 0.0),
            (3.4e38, -3.4e38), (3.4028234663852886e38, -1e-45)]
    for _ in range(100):
        out.append((float(np.float32(abs(g.standard_normal()) * 2.0 ** int(g.integers(-30, 30)))), -float(np.float32(abs(g.standard_normal()) * 2.0 ** int(g.integers(-30, 30))))))
    return out


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("scale", ["f32", "bf16"])
def test_scales_at_the_borders(scale, group):
    pairs = rows(scale, 5)
    w = np.zeros((len(pairs), group), np.float32)
    rest = np.random.default_rng(1).random((len(pairs), group))
    for i, (hi, lo) in enumerate(pairs):
        w[i] = (lo * rest[i] if hi < -lo else hi * rest[i]) * 0.9
        w[i, i % group], w[i, (i + 7) % group] = hi, lo
    bits = 8 if scale == "bf16" else 24
    m = eesd.W4Matrix.quantize(torch.from_numpy(w).cuda(), group=group, scale_dtype=DT[scale], zero_point=True)
    got, z, codes = m.scales().double().cpu().numpy()[:, 0], m.zeros().cpu().numpy()[:, 0], m.codes().cpu().numpy()
    for i in range(len(pairs)):
        hi, lo = Fraction(float(max(w[i].max(), 0))), Fraction(float(min(w[i].min(), 0)))
        s = nearest((hi - lo) / 15, bits) if hi > lo else Fraction(0)
        assert Fraction(float(got[i])) == s, (pairs[i], got[i], float(s))
        want = min(max(round(-lo / s), 0), 15) if s else 0          # (round of a fraction: ties to even)
        assert z[i] == want, pairs[i]
        assert codes[i].tolist() == [min(max(round(Fraction(float(x)) / s) + want, 0), 15) if s else 0 for x in w[i]], pairs[i]
    # symmetric: the larger magnitude over 7
    for i, (hi, lo) in enumerate(pairs):
        w[i] = np.clip(w[i], -max(hi, -lo), max(hi, -lo))
    m = eesd.W4Matrix.quantize(torch.from_numpy(w).cuda(), group=group, scale_dtype=DT[scale])
    got = m.scales().double().cpu().numpy()[:, 0]
    for i in range(len(pairs)):
        top = Fraction(float(np.abs(w[i]).max()))
        assert Fraction(float(got[i])) == (nearest(top / 7, bits) if top else 0), pairs[i]
