"""Angles of far positions: rows whose pairs are (1, 0) become (cos, sin), which are compared with exact arithmetic.

How far a channel may be, in radians unless it is said:
  angle    turns of a position are a product of whole numbers of 2^-64 turns, of which the lower 32 bits are cut off (2^-32 of a turn at most);
           a frequency is half a unit off, and half a unit more where it comes from a base of 1 or more (test_rope_launch_host.py): 2^31 times
           2^-64 is 2^-33 of a turn at most; a frequency of a smaller base is rounded to 64 bits, its exponent too: (|ln f| + 2) f 2^-64
  sine     the angle is rounded to 32 bits, 2^-24 of it; the hardware's sine and cosine are 1.3e-7 off at most
  rows     products with 1 and 0 and their sum are exact; half a step of the output
"""
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2512_24086_amd import rf2
from tests import rope_ref as ref
from tests.test_rope_launch_host import ONE, TWO_PI, exact_frequency

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


def positions(f, rng):
    """Places where a frequency's turns are next to whole ones, as far away as there are, and others."""
    x, before, q, found = Fraction(f.numerator * ONE, f.denominator * TWO_PI), 0, 1, []
    while q <= MOST and len(found) < 60:        # denominators of the continued fraction
        found.append(q)
        x -= x.numerator // x.denominator
        if x == 0:
            break
        x = 1 / x
        before, q = q, (x.numerator // x.denominator) * q + before
    far = found[-4:] + [found[-1] * (MOST // found[-1]), MOST, -MOST - 1] + rng.integers(-MOST - 1, MOST + 1, 3).tolist()
    return far + [-p for p in found[-2:]] + [0, 1]


def expected(pos, f):
    """Cosine and sine, and the fraction of a turn with a sign."""
    unit, part = (f.numerator * ONE << 192) // (f.denominator * TWO_PI), np.empty(len(pos))              # turns per position, in units of 2^-192
    for i, p in enumerate(pos):
        t = p * unit % (1 << 192)
        part[i] = (t - (1 << 192) if t >> 191 else t) / 2.0 ** 192
    return np.cos(2 * np.pi * part), np.sin(2 * np.pi * part), part


@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("name", ["base 10,000", "base 1,000,000", "base 100", "base 0.01", "table to 1", "table to 16", "table to 65,536"])
def test_angles_of_far_positions(name, halves):
    rng = np.random.default_rng(len(name))
    d, kind, size = 128, name.split()[0], float(name.split()[-1].replace(",", ""))
    if kind == "base":
        table, freq = None, [exact_frequency(size, j, d) for j in range(d // 2)]
    else:
        table = np.exp2(rng.uniform(np.log2(size) - 6, np.log2(size), d // 2))
        table[:3] = size, np.nextafter(size, 0), -0.7 * size
        freq = [Fraction(float(f)) for f in table]
    pos = sorted({p for f in freq for p in positions(abs(f), rng)})
    plan = rf2.RopePlan(heads=1, kv_heads=1, head_dim=d, axis_dims=(d,), theta=size if kind == "base" else 10000.0, inv_freq=table, norm=rf2.RF2_NORM_NONE,
                        pairing=rf2.RF2_ROPE_HALVES if halves else rf2.RF2_ROPE_PAIRS)
    first = slice(0, d // 2) if halves else slice(0, d, 2)
    second = slice(d // 2, d) if halves else slice(1, d, 2)
    x = torch.zeros(len(pos), 1, d, dtype=torch.bfloat16, device="cuda")
    x[..., first] = 1
    at = torch.tensor(pos, dtype=torch.int64).to(torch.int32)[:, None].cuda()
    out, back = torch.empty_like(x), torch.empty_like(x)
    plan.rf2_rope_apply(x, None, at, out, None)
    plan.rf2_rope_backward(None, None, at, x, None, back, None)
    got, back = out[:, 0].cpu().double().numpy(), back[:, 0].cpu().double().numpy()
    far = np.abs(np.array(pos, dtype=np.float64))
    for i, f in enumerate(freq):
        cos, sin, part = expected(pos, f)
        f = abs(float(f))
        rounding = (abs(np.log(f)) + 2) * f * 2.0 ** -64 if kind == "base" and size < 1 else 2 * np.pi * 2.0 ** -65 * (1 if table is None else 0)
        angle = 2 * np.pi * (2.0 ** -32 + np.abs(part) * 2.0 ** -24 + far * 2.0 ** -65) + far * rounding
        error = angle + 1.3e-7
        for value, want in ((got[:, first][:, i], cos), (got[:, second][:, i], sin), (back[:, first][:, i], cos), (back[:, second][:, i], -sin)):
            off = np.abs(value - want) / ref.rounded(want, error, torch.bfloat16)
            assert off.max() <= 1.0, (f, pos[int(off.argmax())], float(off.max()))
