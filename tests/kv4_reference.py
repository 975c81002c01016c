"""The 4-bit form of a compressed prompt, and a decode step over it, in 64-bit floating point on the CPU, from their
definitions in include/shotkv.h: nothing here is shared with the library."""
import numpy as np


def bf16_up(x):
    """The least bf16 number >= x (x >= 0, float64), as float64."""
    f = x.astype(np.float32)
    bits = f.view(np.uint32)
    out = (bits & np.uint32(0xFFFF0000)).view(np.float32).astype(np.float64)
    short = out < x
    nxt = ((bits & np.uint32(0xFFFF0000)) + np.uint32(0x10000)).view(np.float32).astype(np.float64)
    return np.where(short, nxt, out)


def quantise(x):
    """x [..., group] float64 (bf16 values) -> codes -8..7, s, z (float64); NaN scales where the group has no grid."""
    with np.errstate(invalid="ignore", over="ignore"):
        wide = (x.max(-1) - x.min(-1)).astype(np.float32).astype(np.float64)
        fine = np.isfinite(x).all(-1) & np.isfinite(wide)
        y = np.where(fine[..., None], x, 0.0)
        s = bf16_up(np.maximum(np.maximum((y.max(-1) - y.min(-1)) / 15, np.abs(y).max(-1) / 240), 2.0 ** -100))
        c = np.floor(y / s[..., None] + 0.5)
    z = c.min(-1) + 8
    assert (c - z[..., None] <= 7).all() and (np.abs(z) <= 256).all()
    return c - z[..., None], np.where(fine, s, np.nan), z


def values_of(rows, keys):
    """What rows [..., d] (float64, bf16 values) read as once they are held in 4 bits, float64."""
    d = rows.shape[-1]
    c, s, z = quantise(rows.reshape(*rows.shape[:-1], d // 32 if keys else 1, 32 if keys else d))
    return (s[..., None] * (c + z[..., None])).reshape(rows.shape)


def tile_bytes(d, keys):
    return 32 * (d // 2 + (d // 8 if keys else 4))


def places(d, keys):
    """Word and nibble of every row and dimension of a tile, and the word of its group."""
    r, i = np.meshgrid(np.arange(32), np.arange(d), indexing="ij")
    if keys:
        lane, j = 4 * (r % 8) + i // 8 % 4, 2 * (i // 32) + i // 4 % 2
        n = r // 8 % 2 + 2 * (i // 2 % 2) + 4 * (i % 2)
        group = 4 * d + r * (d // 32) + i // 32
    else:
        lane, j = 4 * (i // 8 % 8) + r // 2 % 4, 4 * (i // 64) + i // 2 % 4
        n = i % 2 + 2 * (r // 8 % 2) + 4 * (r % 2)
        group = 4 * d + r
    return ((r // 16 * (d // 64) + j // 4) * 32 + lane) * 4 + j % 4, n, group


def read_tiles(tiles, d, keys):
    """uint8 [..., T, bytes] -> codes, s, z of rows [..., T * 32, d], float64."""
    words = np.ascontiguousarray(tiles).view("<u4")
    word, nibble, group = places(d, keys)
    codes = (words[..., word] >> (4 * nibble).astype(np.uint32) & 15).astype(np.float64) - 8
    meta = words[..., group]
    s = (meta & np.uint32(0xFFFF0000)).view(np.float32).astype(np.float64)
    z = (meta << np.uint32(16)).view(np.float32).astype(np.float64)
    lead = tiles.shape[:-2]
    return tuple(a.reshape(*lead, -1, d) for a in (codes, s, z))


def write_tiles(rows, keys):
    """Rows [..., R, d] (float64, bf16 values; R a multiple of 32) -> uint8 [..., R / 32, bytes]."""
    d, lead = rows.shape[-1], rows.shape[:-2]
    groups, wide = (d // 32, 32) if keys else (1, d)
    c, s, z = quantise(rows.reshape(*lead, -1, 32, groups, wide))
    c = (c + 8).astype(np.uint32).reshape(*c.shape[:-2], d)
    s32 = s.astype(np.float32).view(np.uint32) & np.uint32(0xFFFF0000)
    meta = s32 | (z.astype(np.float32).view(np.uint32) >> np.uint32(16))
    words = np.zeros((*c.shape[:-2], tile_bytes(d, keys) // 4), np.uint32)
    word, nibble, group = places(d, keys)
    for n in range(8):                                       # each word has one element in every nibble
        at = nibble == n
        words[..., word[at]] |= c[..., at] << np.uint32(4 * n)
    words[..., 4 * d:] = meta.reshape(*meta.shape[:-2], -1)
    return words.view(np.uint8)


def step(q, keys, values, M, size_of_keys=None, size_of_values=None, steepest=0.0):
    """One (sequence, layer): q [H, d], keys and values [Hkv, t, d] (the M kept rows, then the decode entries), float64.
    Returns the entries' weights summed over all heads, the outputs [H, d], and how far sums in 32 bits may be off both:
    each of a logit's d products is added with an error of 2^-23 at most of the sum of all magnitudes (24 bits, of which a matrix
    unit cuts off what does not fit), which makes d 2^-23 of that sum for the logit, and as much relative to itself for the
    weight; a row's sum of t weights adds t 2^-24 at most, the exponential and the weights' 22 bits 2^-20.  A weight below
    2^-126, float32's least normal number, may be 0: with up to 64 heads that makes 2^-120 of an entry's sum.
    `size_of_*`: the magnitudes that are added for an element of a row in 4 bits.  s (c + z) is added in two parts, the sum over
    p s c and the sum over p s z, each in 32 bits and the first with the weights' 22: s (|c| + |z|), which is what both
    are rounded by, and more than |s (c + z)| where c and z are of opposite sign (all of it where the element is 0).
    `steepest`: the largest s of a value.  A weight times its s enters the product with the codes as two f16 numbers; the second
    of them is off by half of f16's least step, 2^-25, in units in which the row's largest weight is 2^10 or more and the
    largest s is 1 or more: 2^-35 of that weight times that s, for each of t rows, times a code of up to 8."""
    H, d = q.shape
    Hkv, t, _ = keys.shape
    G = H // Hkv
    with np.errstate(invalid="ignore"):
        x = np.einsum("hgd,htd->hgt", q.reshape(Hkv, G, d), keys) / np.sqrt(d)
        size = np.einsum("hgd,htd->hgt", np.abs(q.reshape(Hkv, G, d)), np.abs(keys) if size_of_keys is None else size_of_keys) / np.sqrt(d)
        p = np.exp(x - x.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        # the weighted mean of logit errors moves the row's sum as far
        off = d * 2.0 ** -23 * size
        off = off + (p * off).sum(-1, keepdims=True) + t * 2.0 ** -24 + 2.0 ** -20
        weights, weights_off = p[..., M:].sum((0, 1)), (p * off)[..., M:].sum((0, 1)) + 2.0 ** -120
        if values is None:
            return weights, weights_off, None, None
        out = np.einsum("hgt,htd->hgd", p, values).reshape(H, d)
        # the output's own sum: t products, each added as above
        out_off = np.einsum("hgt,htd->hgd", p * off, np.abs(values))
        rounded = np.einsum("hgt,htd->hgd", p * (t * 2.0 ** -23 + 2.0 ** -21), np.abs(values) if size_of_values is None else size_of_values)
        out_off = (out_off + rounded + t * 2.0 ** -35 * p.max(-1)[..., None] * steepest * 8).reshape(H, d)
    return weights, weights_off, out, out_off


def sizes_of(rows, keys):
    """s (|c| + |z|) of every element of rows [..., d]."""
    d = rows.shape[-1]
    c, s, z = quantise(rows.reshape(*rows.shape[:-1], d // 32 if keys else 1, 32 if keys else d))
    return (s[..., None] * (np.abs(c) + np.abs(z[..., None]))).reshape(rows.shape)
