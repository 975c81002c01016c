"""Packed prompts at the ends of their range: groups whose range 32 bits cannot hold exactly, values and queries of very
different or extreme sizes, logits far below zero.  The definitions are those of include/shotkv.h, in exact fractions or 64 bits."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import kv4_reference as R
import paper_2502_01941_b200 as skv
from test_kv4_gpu import Step, f64, normal, packed

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


# ------------------------------------------------------------------------------------------------ the steps
def check_outputs(s, scores=True):
    """A step's outputs and scores against 64 bits.  The allowance is kv4_reference.step's for sums in 32 bits, and for a weight's
    place in the product: it enters with its value's scale as two f16 numbers, the second of them off by 2^-25 in units of a power
    of two that is no more than the largest scale and no more than 2^8 times the row's own, while the row's largest weight is
    2^10 or more: 2^-35 of that weight and the largest scale, or 2^-27 of it and the own scale, times a code of up to 8."""
    m, n = s.M, s.n_old + 1
    acc, out = s.acc.cpu().numpy(), s.out.cpu().numpy()
    for b in range(s.B):
        for l in range(s.L):
            kk, kv = f64(s.K[b, l]), f64(s.V[b, l])
            kd, vd = f64(s.Kd[b, l, :, :n]), f64(s.Vd[b, l, :, :n])
            scale = R.quantise(kv)[1]                                   # [Hkv, M]
            keys = np.concatenate([R.values_of(kk, True), kd], 1)
            w, w_off, o, o_off = R.step(f64(s.q[b, l]), keys, np.concatenate([R.values_of(kv, False), vd], 1), m,
                                        np.concatenate([R.sizes_of(kk, True), np.abs(kd)], 1),
                                        np.concatenate([R.sizes_of(kv, False), np.abs(vd)], 1))
            x = np.einsum("hgd,htd->hgt", f64(s.q[b, l]).reshape(s.Hkv, s.G, s.d), keys) / np.sqrt(s.d)
            p = np.exp(x - x.max(-1, keepdims=True))
            largest = 1 / p.sum(-1)                                     # [Hkv, G]
            product = 8 * np.minimum(2.0 ** -35 * scale.max(-1, keepdims=True), 2.0 ** -27 * scale).sum(-1)
            o_off = o_off + (largest * product[:, None]).reshape(-1, 1)
            assert np.isfinite(out[b, l]).all()
            err = np.abs(out[b, l] - o)
            assert np.all(err <= o_off), f"outputs of {b}, {l}: off by {(err / o_off).max()} of what they may be"
            if scores:
                old = np.append(s.before[b, l, :n - 1], 0.0)
                assert np.all(np.abs(acc[b, l, :n] - (old + w)) <= w_off + 2.0 ** -22 * (old + w)), "scores"


def bf(t):
    return t.to(torch.bfloat16).contiguous()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 7])
@pytest.mark.parametrize("exponent", [6, 10, 20, 28, 32, 60, -10, -28, -60, -90])
@pytest.mark.parametrize("every", [1, 3, 40])
def test_values_far_from_the_others_that_have_no_weight(ctx, every, exponent, G, d):
    """Rows (all of a block of 40, or every third or fortieth) whose values are larger or smaller by a power of two and whose keys point
    away from every query: the others' outputs are as they would be alone."""
    M = 333
    K, V, q = (normal(i, 1, 2, 2, r, d).float() for i, r in ((1, M), (2, M), (3, G)))
    far = torch.zeros(M, dtype=torch.bool, device="cuda")
    far[slice(60, 100) if every == 1 else slice(2, None, every)] = True
    V[:, :, :, far] *= 2.0 ** exponent
    q[..., 0], K[..., 0] = 20.0, 0.0
    K[:, :, :, far], K[:, :, :, far, 0] = 0.0, -60.0
    s = Step(ctx, 1, 2, 2, G, d, M, 30, counts=np.full((1, 2), M, np.int32), keys=bf(K), values=bf(V), q=bf(q.reshape(1, 2, 2 * G, d)))
    s.run(True)
    check_outputs(s)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 8])
@pytest.mark.parametrize("M", [31, 700])
def test_values_of_every_size_at_once(ctx, M, G, d):
    """Scales from 2^-70 to 2^40 from row to row, weights and scales independent."""
    g = torch.Generator(device="cuda").manual_seed(5)
    V = normal(2, 1, 1, 2, M, d).float() * torch.exp2(110 * torch.rand(1, 1, 2, M, 1, generator=g, device="cuda") - 70)
    s = Step(ctx, 1, 1, 2, G, d, M, 20, counts=np.full((1, 1), M, np.int32), values=bf(V))
    s.run(True)
    check_outputs(s)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 8])
@pytest.mark.parametrize("exponent", [-40, -62, -80, -95, 40, 90])
def test_values_of_any_one_size(ctx, exponent, G, d):
    """All values, the entries' too, are the same power of two smaller or larger than one: so are the outputs."""
    M = 200
    s = Step(ctx, 1, 1, 2, G, d, M, 20, counts=np.full((1, 1), M, np.int32), values=bf(normal(2, 1, 1, 2, M, d).float() * 2.0 ** exponent))
    for t in (s.Vd, s.v):
        t *= 2.0 ** exponent
    s.run(True)
    check_outputs(s)


def test_rows_of_zeros_among_values(ctx):
    """A row of zeros has the least scale there is; it adds nothing, and does not disturb the others."""
    V = normal(2, 1, 1, 2, 300, 128)
    V[:, :, :, ::7] = 0
    V[:, :, :, 64:96] = 0
    s = Step(ctx, 1, 1, 2, 4, 128, 300, 20, counts=np.full((1, 1), 300, np.int32), values=V)
    s.run(True)
    check_outputs(s)


def one_sided(ctx, sign, key_exponent, query_exponent, G, d, M=150, n_old=20):
    """A step whose logits are +-15 n 2^(key_exponent + query_exponent) / sqrt(d), n of 1 to 17 from row to row, of kept rows and entries
    alike: every one exact in bf16 and in 4 bits.  Returns it and the rows and entries with the greatest."""
    K = torch.zeros(1, 1, 2, M, d)
    n = torch.randint(1, 18, (2, M + n_old + 1), generator=torch.Generator().manual_seed(G))
    n[:, ::5] = 1 if sign < 0 else 17
    k = sign * 15.0 * n * 2.0 ** key_exponent
    K[0, 0, :, :, 3] = k[:, :M]
    q = torch.zeros(1, 1, 2 * G, d)
    q[..., 3] = 2.0 ** query_exponent
    s = Step(ctx, 1, 1, 2, G, d, M, n_old, counts=np.full((1, 1), M, np.int32), keys=bf(K).cuda(), q=bf(q).cuda())
    s.Kd.zero_(), s.k.zero_()
    s.Kd[0, 0, :, :n_old, 3] = k[:, M:M + n_old].to(torch.bfloat16).cuda()
    s.k[0, 0, :, 3] = k[:, -1].to(torch.bfloat16).cuda()
    return s, (n == (1 if sign < 0 else 17)).numpy()


def check_one_sided(s, wins, attend, off):
    """Of a row's weights those of the greatest logits are alike, the others are 0; `off` is how far a weight may be from its own,
    relative to it (2^-20 for the exponential and the division, and 32 bits' sums)."""
    off += (wins.shape[1] + 8) * 2.0 ** -23 + 2.0 ** -19
    n = s.n_old + 1
    weight = wins / wins.sum(1, keepdims=True)                          # [Hkv, M + n]
    old = np.append(s.before[0, 0, :n - 1], 0.0)
    want = old + s.G * weight[:, s.M:].sum(0)
    assert np.all(np.abs(s.acc.cpu().numpy()[0, 0, :n] - want) <= off * want)
    if attend:
        v = np.concatenate([R.values_of(f64(s.V[0, 0]), False), f64(s.Vd[0, 0, :, :n])], 1)
        size = np.concatenate([R.sizes_of(f64(s.V[0, 0]), False), np.abs(f64(s.Vd[0, 0, :, :n]))], 1)
        o, o_off = (np.einsum("ht,htd->hd", weight, t).repeat(s.G, 0) for t in (v, size))
        assert np.all(np.abs(s.out.cpu().numpy()[0, 0] - o) <= off * o_off)


@pytest.mark.parametrize("attend", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 7])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("exponents", [(0, 12), (11, 11), (14, 14), (17, 19), (20, 20), (30, 30), (50, 50), (60, 46), (-20, 119), (10, 100)])
def test_logits_of_any_size(ctx, exponents, sign, G, d, attend):
    """Those of 2^24 and more are apart by more than 32 bits' steps of one there, those of some -10^30 lie below what a row begins with."""
    s, wins = one_sided(ctx, sign, *exponents, G, d)
    s.run(attend)
    # a logit, in units of powers of two, is rounded once on the way to an entry's weight, by 2^-24 of itself; from 2^23 on all are
    # rounded alike
    largest = 15 * (1 if sign < 0 else 17) * 2.0 ** sum(exponents) / np.sqrt(d) * 1.4427
    check_one_sided(s, wins, attend, 2.0 ** -23 * largest if largest < 2.0 ** 23 else 0.0)


@pytest.mark.parametrize("attend", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [4, 7])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("exponents", [(-92, 114), (-92, 115), (-97, 120), (-100, 122), (-100, 127), (-60, 125), (-7, 121)])
def test_queries_of_any_size(ctx, exponents, sign, G, d, attend):
    """Queries up to bf16's largest, some heads' a little smaller.  (Keys in 4 bits are multiples of 2^-100, so all logits are beyond 2^23.)"""
    s, wins = one_sided(ctx, sign, *exponents, G, d)
    s.q[0, 0, 1::2] *= 2.0 ** -4
    s.run(attend)
    check_one_sided(s, wins, attend, 0.0)


@pytest.mark.parametrize("attend", [False, True])
@pytest.mark.parametrize("G", [4, 7])
@pytest.mark.parametrize("words", ["bytes", "zeros", "least", "below", "greatest", "negative", "nan", "mixed"])
def test_a_cache_that_was_never_packed_ends_the_step(ctx, words, G, attend):
    """What such a step gives is of no meaning, but it ends, and it leaves the entries' rows, other units and the next step as they are."""
    M, n_old = 300, 20
    s = Step(ctx, 1, 1, 2, G, 64, M, n_old, counts=np.full((1, 1), M, np.int32))
    good = s.K4.clone(), s.V4.clone()
    g = torch.Generator(device="cuda").manual_seed(3)
    tile = s.V4[0, 0, 0].view(torch.int32)[:, 4 * 64:]                    # one unit's words of the values' scales
    fill = {"zeros": 0, "least": 1, "below": (20 << 23) | 5, "greatest": 0x7F7FFFFF, "negative": -(1 << 31) + (100 << 23), "nan": 0x7FC00001}
    if words == "bytes":
        for t in (s.K4, s.V4):
            t[0, 0, 0] = torch.randint(0, 256, t[0, 0, 0].shape, generator=g, device="cuda", dtype=torch.uint8)
    elif words == "mixed":
        tile.copy_(torch.tensor(list(fill.values()), device="cuda", dtype=torch.int32).repeat(tile.numel() // 6 + 1)[:tile.numel()].view_as(tile))
    else:
        tile.fill_(fill[words])
    s.run(attend)
    torch.cuda.synchronize()
    assert torch.equal(s.Kd[:, :, :, n_old], s.k) and torch.equal(s.Vd[:, :, :, n_old], s.v)
    bad = s.out.clone()
    s.K4.copy_(good[0]), s.V4.copy_(good[1])
    s.st.T = s.st.n_dec = n_old
    s.acc.copy_(torch.from_numpy(s.before))
    s.run(attend)
    s.check(attend)
    if attend:
        assert torch.equal(bad[0, 0, G:], s.out[0, 0, G:])                # the other unit's
