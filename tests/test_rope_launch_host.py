"""The rotations' tables of frequencies against exact arithmetic, and how many workgroups a call asks for, on the host."""
import ctypes as C
import decimal
import os
import subprocess
from fractions import Fraction

import numpy as np
import pytest

from paper_2512_24086_amd import build as b
from paper_2512_24086_amd import rf2

HERE = os.path.dirname(os.path.abspath(__file__))
ONE = 1 << 256                                  # of numbers with 256 bits behind the point


def arctan_of_one_over(n):
    total, term, k = 0, ONE // n, 1
    while term:
        total += term // k if k % 4 == 1 else -(term // k)
        term, k = term // (n * n), k + 2
    return total


TWO_PI = 8 * (4 * arctan_of_one_over(5) - arctan_of_one_over(239))                    # Machin: pi / 4 = 4 arctan 1/5 - arctan 1/239


def exact_turns(f):
    """A frequency's turns per position, in units of 2^-192, whole turns left out."""
    f = Fraction(f)
    return (f.numerator * ONE << 192) // (f.denominator * TWO_PI) % (1 << 192)


def exact_frequency(theta, j, dim):
    with decimal.localcontext() as context:
        context.prec = 70
        return Fraction(decimal.Decimal(theta) ** (decimal.Decimal(-2 * j) / decimal.Decimal(dim)))


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    objs = [os.path.join(b.PKG, "_build", os.path.splitext(s)[0] + ".o") for s in b.SOURCES]
    if not all(os.path.exists(o) for o in objs):
        b.build(verbose=False)
    folder = tmp_path_factory.mktemp("rope_launch")
    lib = str(folder / "rope_launch.so")
    subprocess.run([b.hipcc(), *b.FLAGS, "-c", os.path.join(HERE, "rope_launch_host.cpp"), "-o", str(folder / "driver.o")], check=True, capture_output=True)
    subprocess.run([b.hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-Wl,-Bsymbolic", str(folder / "driver.o"), *objs, "-o", lib], check=True, capture_output=True)
    return C.CDLL(lib)


def config(**over):
    a = dict(dict(heads=4, kv_heads=2, head_dim=128, norm=rf2.RF2_NORM_RMS, dims=(128,), theta=10000.0), **over)
    return rf2.rf2_rope_config(a["heads"], a["kv_heads"], a["head_dim"], 0, 0, a["norm"], 1e-6, 0, len(a["dims"]), (C.c_int32 * 4)(*a["dims"]), a["theta"])


def tables(library, freq=None, **over):
    """Turns of a plan's pairs per position, in units of 2^-64 modulo 2^64, both ways."""
    pairs = np.dtype([("turns", "<i4", 64), ("rest", "<i4", 64), ("axis", "u1", 64)])
    out = np.zeros(2, dtype=pairs)
    cfg = config(**over)
    assert library.rope_tables(C.byref(cfg), None if freq is None else (C.c_double * 64)(*freq), out.ctypes.data_as(C.c_void_p), out.nbytes) == 0
    return [[((int(t) << 32) + int(r)) % (1 << 64) for t, r in zip(way["turns"], way["rest"])] for way in out]


def off(units, exact):
    """How far a table's entry is from exact turns, in units of 2^-64."""
    x = ((units << 128) - exact) % (1 << 192)
    return min(x, (1 << 192) - x) / (1 << 128)


@pytest.mark.parametrize("low, high", [(-40, 0), (0, 4), (4, 10), (10, 16)], ids=str)
def test_turns_of_a_table_of_frequencies_are_the_nearest(library, low, high):
    # (half a unit, and what 126 bits of 1 / 2 pi leave out: 2^16 2^64 2^-128 of one)
    freq = np.exp2(np.random.default_rng(abs(low)).uniform(low, high, 64))
    freq[:8] = [min(x, 65536.0) for x in (2.0 ** low, 2.0 ** high, 100.0, 1000.3, 65535.9, 65536.0, 2 * np.pi, 355.0)]
    freq[::3] *= -1
    for way, sign in zip(tables(library, freq), (1, -1)):
        for f, units in zip(freq, way):
            assert off(units, exact_turns(sign * Fraction(float(f)))) <= 0.5 + 2.0 ** -40, f


@pytest.mark.parametrize("theta", [1.0, 100.0, 10000.0, 500000.0, 1e6, 1e30])
def test_turns_of_a_base(library, theta):
    # f, rounded to 64 bits from an exponent rounded to 64 bits: off by |ln f| f 2^-64 and 2 f 2^-64 at most, so 2.4 2^-64, less than half a
    # unit of turns, beside half a unit
    for way, sign in zip(tables(library, theta=theta, dims=(60, 68)), (1, -1)):
        pairs = [(j, 60) for j in range(30)] + [(j, 68) for j in range(34)]
        for (j, dim), units in zip(pairs, way):
            assert off(units, exact_turns(sign * exact_frequency(theta, j, dim))) <= 1.0, (theta, j, dim)


def grids(library, backward, batch, tokens, layout, **over):
    """Workgroups of each launch of a call on dense rows; `layout` is the order of tokens and heads, or the strides of both."""
    cfg = config(**over)
    rows = []
    for _ in range(3 if backward else 2):
        for heads in (cfg.heads, cfg.kv_heads):
            token, head = {"bnhd": (heads * cfg.head_dim, cfg.head_dim), "bhnd": (cfg.head_dim, tokens * cfg.head_dim)}.get(layout, layout)
            rows += [1 << 20, tokens * heads * cfg.head_dim, token, head]
    out = (C.c_uint32 * 16)()
    n = library.rope_grids(C.byref(cfg), int(backward), batch, tokens, (C.c_int64 * len(rows))(*rows), out)
    assert n >= 0, n
    return list(out[:n])


@pytest.mark.parametrize("layout", ["bnhd", "bhnd", (0, 128), (8, 4096), (1 << 40, 128)], ids=str)
@pytest.mark.parametrize("heads, kv, d, workgroups", [(8, 2, 64, 2), (40, 40, 128, 20), (7, 1, 128, 8), (32, 8, 128, 10), (16, 16, 64, 4)])
def test_one_token_is_rows_of_heads_side_by_side(library, heads, kv, d, workgroups, layout):
    # a wavefront's 64 / (d / 8) rows are heads, as many as divide all, whatever the stride of the only token is
    sizes = dict(heads=heads, kv_heads=kv, head_dim=d, dims=(d,))
    assert grids(library, False, 1, 1, layout, **sizes) == [workgroups]
    # the gradients' sums of one workgroup need no launch of their own
    alone = heads <= 512 // d and kv <= 512 // d
    assert grids(library, True, 1, 1, layout, **sizes) == ([workgroups] if alone else [workgroups, d // 4])


def test_few_tokens_keep_their_layout(library):
    assert grids(library, False, 1, 4, "bhnd", heads=8, kv_heads=8) == [16] and grids(library, False, 1, 4, "bnhd", heads=8, kv_heads=8) == [4]
    assert grids(library, False, 4, 1, "bnhd", heads=8, kv_heads=8) == [4]
