"""Packed prompts at the ends of their range: groups whose range 32 bits cannot hold exactly, values and queries of very
different or extreme sizes, logits far below zero.  The definitions are those of include/shotkv.h, in exact fractions or 64 bits."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import kv4_reference as R
import paper_2502_01941_b200 as skv
from test_kv4_gpu import f64, packed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2502_01941_b200.build import build_library
    build_library()
    c = skv.Context(0)
    yield c
    c.close()


# ------------------------------------------------------------------------------------------------ the scale
def bf16_at_least(x):
    """The least positive bf16 number that is no less than the fraction x (a normal one)."""
    e = 0
    while Fraction(2) ** (e + 1) <= x:
        e += 1
    while Fraction(2) ** e > x:
        e -= 1
    step = Fraction(2) ** (e - 7)
    return -(-x // step) * step


def exact_grid(group):
    """A group of float64 (bf16 values) -> its scale and every c + z, in exact fractions."""
    x = [Fraction(float(v)) for v in group]
    s = bf16_at_least(max((max(x) - min(x)) / 15, max(map(abs, x)) / 240, Fraction(1, 1 << 100)))
    return s, [(v / s + Fraction(1, 2)).__floor__() for v in x]


def groups_next_to_a_scale():
    """(max, min) with 15 s = max for a bf16 number s, and the other end too small for 32 bits to tell from zero; and such whose
    ends are alike in size, or on the same side of zero."""
    rng = np.random.default_rng(11)
    out = [(15.0, -2.0 ** -30), (0.9375, -2.0 ** -30), (2.0 ** -30, -15.0), (15.0, -2.0 ** -120), (15.0, 2.0 ** -30), (-2.0 ** -30, -15.0),
           (15.0, -2.0 ** -9), (15.0, -2.0 ** -8), (240.0, 225.0), (7.5, -7.5), (15.0, 0.0), (15.0, -2.0 ** -133)]
    for _ in range(180):
        at = 2.0 ** int(rng.integers(-40, 60))
        top, low = 15.0 * rng.integers(1, 18) * at, rng.integers(128, 256) * 2.0 ** -float(rng.integers(10, 70)) * at
        out.append([(top, -low), (low, -top), (top, low), (-low, -top)][rng.integers(4)])
    return out


@pytest.mark.parametrize("d", [64, 128])
def test_the_scale_goes_by_the_range_of_the_numbers_themselves(ctx, d):
    ends = groups_next_to_a_scale()
    rng = np.random.default_rng(d)
    rows = np.empty((len(ends), d))
    for r, (top, low) in enumerate(ends):
        rows[r] = torch.from_numpy(low + (top - low) * rng.random(d)).to(torch.bfloat16).double().clamp(low, top).numpy()
        rows[r, 5::32], rows[r, 20::32] = top, low
    K = torch.from_numpy(rows).to(torch.bfloat16).cuda().reshape(1, 1, 1, len(ends), d)
    assert np.array_equal(f64(K)[0, 0, 0], rows)
    n = len(ends)
    K4, V4 = packed(ctx, skv.make_dims(1, 1, 1, 1, d, n, 1, 0), K, K, None, np.full((1, 1), n, np.int32), n)
    for tiles, keys in ((K4, True), (V4, False)):
        c, s, z = R.read_tiles(tiles.cpu().numpy()[0, 0, 0], d, keys)
        for r in range(n):
            for at in range(0, d, 32 if keys else d):
                g = slice(at, at + (32 if keys else d))
                scale, whole = exact_grid(rows[r, g])
                assert Fraction(s[r, at]) == scale, ends[r]
                assert (c[r, g] + z[r, g]).tolist() == whole and z[r, at] == min(whole) + 8, ends[r]
