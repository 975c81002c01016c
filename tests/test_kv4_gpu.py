"""The compressed prompt in 4 bits: packing, unpacking and the decode steps over it, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import kv4_reference as R
import paper_2502_01941_b200 as skv
from paper_2502_01941_b200 import workloads as wl
import parity as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2502_01941_b200.build import build_library
    build_library()
    c = skv.Context(0)
    yield c
    c.close()


def normal(seed, *shape, gain=1.0, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * gain + mean).to(torch.bfloat16)


def f64(t):
    return wl.bf16_to_f64(t) if t.dtype != torch.float32 else t.cpu().numpy().astype(np.float64)


def counts_of(B, L, M, seed):
    """Kept counts between none and all of M rows, both of them among the counts where there are two or more."""
    n = np.random.default_rng(seed).integers(0, M + 1, (B, L)).astype(np.int32)
    n[0, 0] = M
    if B * L > 1:
        n[-1, -1] = 0
    return n


def packed(ctx, dims, K, V, idx, counts, M, fill=0xA5):
    K4, V4 = skv.alloc_kv4(dims, M)
    K4.fill_(fill)
    V4.fill_(fill)
    skv.shotkv_compact_kv4(ctx, dims, K, V, idx, torch.from_numpy(counts).cuda(), M, K4, V4)
    return K4, V4


def check_tiles(tiles, rows, count, keys, fill=0xA5):
    """tiles [T, bytes] hold `rows` [count, d]: the definition's very numbers; zeros to the end of the last tile; the rest untouched."""
    d = rows.shape[-1]
    c, s, z = R.read_tiles(tiles, d, keys)
    ref = R.values_of(rows, keys) if count else rows
    got = s * (c + z)
    assert np.array_equal(got[:count], ref, equal_nan=True)
    last = -(-count // 32)
    assert (got[count:last * 32] == 0).all()
    assert (tiles[last:] == fill).all()


# ------------------------------------------------------------------------------------------------ packing
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,L,Hkv,N,M", [(1, 1, 1, 1, 1), (1, 1, 2, 40, 31), (2, 1, 1, 64, 32), (1, 2, 3, 100, 33), (2, 3, 2, 777, 301),
                                         (1, 2, 8, 900, 900)])
@pytest.mark.parametrize("gathered", [True, False])
def test_packed_rows_are_the_definition_s(ctx, d, B, L, Hkv, N, M, gathered):
    K, V = normal(1, B, L, Hkv, N, d, gain=2.0, mean=0.3), normal(2, B, L, Hkv, N, d)
    counts = counts_of(B, L, M, N)
    rng = np.random.default_rng(M)
    idx = np.full((B, L, M), -1, np.int32)
    for b in range(B):
        for l in range(L):
            idx[b, l, :counts[b, l]] = np.sort(rng.permutation(N)[:counts[b, l]]) if gathered else np.arange(counts[b, l])
    dims = skv.make_dims(B, L, Hkv, Hkv, d, N, 1, 0)
    K4, V4 = packed(ctx, dims, K, V, torch.from_numpy(idx).cuda() if gathered else None, counts, M)
    Kc, Vc = (torch.full((B, L, Hkv, M, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    skv.shotkv_unpack_kv4(ctx, dims, K4, V4, torch.from_numpy(counts).cuda(), M, Kc, Vc)
    for tiles, rows, back, keys in ((K4, K, Kc, True), (V4, V, Vc, False)):
        t, x, y = tiles.cpu().numpy(), f64(rows), f64(back)
        for b in range(B):
            for l in range(L):
                n = counts[b, l]
                for h in range(Hkv):
                    kept = x[b, l, h][idx[b, l, :n]]
                    check_tiles(t[b, l, h], kept, n, keys)
                    want = torch.from_numpy(R.values_of(kept, keys)).to(torch.bfloat16) if n else torch.zeros(0, d, dtype=torch.bfloat16)
                    assert np.array_equal(y[b, l, h, :n], f64(want)) and (y[b, l, h, n:] == 7).all()


def special_rows(d):
    """Rows where a grid can go wrong."""
    rng = np.random.default_rng(d)
    rows = [np.zeros(d), np.full(d, 3.25), np.full(d, -1e-30), -np.zeros(d), np.full(d, 2.0 ** -130),
            np.where(np.arange(d) % 2, 2.0 ** -133, 0), np.linspace(-7.5, 7.5, d), np.arange(d) % 16 * 1.0, np.arange(d) % 16 * 0.5 - 100,
            np.where(np.arange(d) % 2, 1.0, 1.0078125), np.where(np.arange(d) % 2, 1.9921875, 2.0), rng.standard_normal(d) * 1e37,
            np.where(np.arange(d) % 2, 3e38, -3e38), np.where(np.arange(d) % 2, 1.6e38, -1.6e38), rng.standard_normal(d) * 1e-38,
            np.exp(rng.standard_normal(d) * 8) * rng.choice([-1, 1], d)]
    # ties: with a range of 15 and both ends on the grid the scale is 1 and the halves are half-way
    half = np.arange(d) % 31 * 0.5
    rows += [half, -half, half - 7.5, half - 7.0]
    for bad in (np.inf, -np.inf, np.nan):
        for at in (0, 31, d - 1):
            r = rng.standard_normal(d)
            r[at] = bad
            rows.append(r)
    r = np.where(np.arange(d) < 32, np.inf, 1.0)
    rows.append(r)
    return torch.from_numpy(np.array(rows, np.float64).astype(np.float32)).to(torch.bfloat16)


@pytest.mark.parametrize("d", [64, 128])
def test_rows_where_a_grid_can_go_wrong(ctx, d):
    rows = special_rows(d)
    n = rows.shape[0]
    K = torch.cat([rows, rows.flip(0)]).cuda().reshape(1, 1, 2, n, d).contiguous()
    dims = skv.make_dims(1, 1, 2, 2, d, n, 1, 0)
    K4, V4 = packed(ctx, dims, K, K, None, np.full((1, 1), n, np.int32), n)
    for h in range(2):
        for tiles, keys in ((K4, True), (V4, False)):
            check_tiles(tiles.cpu().numpy()[0, 0, h], f64(K[0, 0, h]), n, keys)


@pytest.mark.parametrize("d", [64, 128])
def test_every_bf16_quotient_is_rounded_as_defined(ctx, d):
    """Groups that hold a maximum and its negative and every number of three binades below, at many scales: all ties and all
    numbers next to one."""
    rng = np.random.default_rng(3)
    rows = []
    for top in (128, 135, 151, 192, 200, 225, 240, 255):
        for low in (-top, 0, -top / 2, top * 0.75):
            mant = (rng.integers(128, 256, (24, d)) * 2.0 ** -rng.integers(0, 4, (24, d))) * rng.choice([-1, 1], (24, d))
            r = np.clip(mant, min(low, top), top)
            r[:, ::32], r[:, 1::32] = top, low
            rows.append(r * 2.0 ** int(rng.integers(-40, 40)))
    x = torch.from_numpy(np.concatenate(rows).astype(np.float32)).to(torch.bfloat16)
    n = x.shape[0]
    K = x.cuda().reshape(1, 1, 1, n, d)
    K4, V4 = packed(ctx, skv.make_dims(1, 1, 1, 1, d, n, 1, 0), K, K, None, np.full((1, 1), n, np.int32), n)
    check_tiles(K4.cpu().numpy()[0, 0, 0], f64(x), n, True)
    check_tiles(V4.cpu().numpy()[0, 0, 0], f64(x), n, False)


def test_rows_outside_the_prompt_become_zeros(ctx):
    d, N, M = 64, 50, 40
    K, V = normal(5, 1, 1, 2, N, d), normal(6, 1, 1, 2, N, d)
    idx = np.arange(M, dtype=np.int32)[None, None].copy()
    idx[0, 0, [0, 7, 20, 35]] = [-1, N, 2 ** 31 - 1, -(2 ** 31)]
    dims = skv.make_dims(1, 1, 2, 2, d, N, 1, 0)
    K4, _ = packed(ctx, dims, K, V, torch.from_numpy(idx).cuda(), np.full((1, 1), M, np.int32), M)
    rows = f64(K)[0, 0, 1][np.clip(idx[0, 0], 0, N - 1)]
    rows[[0, 7, 20, 35]] = 0
    check_tiles(K4.cpu().numpy()[0, 0, 1], rows, M, True)


# ------------------------------------------------------------------------------------------------ steps
class Step:
    """A decode state over a packed prompt, and the definition's answer to its next step."""

    def __init__(self, ctx, B, L, Hkv, G, d, M, n_old, counts=None, seed=0, Dcap=None, Mcap=None, keys=None, values=None, q=None,
                 every=1 << 20, r_d=1.0):
        self.ctx, self.B, self.L, self.Hkv, self.G, self.d, self.n_old = ctx, B, L, Hkv, G, d, n_old
        H, self.M = Hkv * G, M
        self.Mcap = Mcap or M
        self.counts = counts_of(B, L, M, seed) if counts is None else counts
        rows = max(self.Mcap, 1)
        self.K = normal(seed + 1, B, L, Hkv, rows, d, gain=1.3, mean=0.2) if keys is None else keys
        self.V = normal(seed + 2, B, L, Hkv, rows, d) if values is None else values
        self.q = normal(seed + 3, B, L, H, d) if q is None else q
        self.k, self.v = normal(seed + 4, B, L, Hkv, d), normal(seed + 5, B, L, Hkv, d)
        Dcap = Dcap or n_old + 3
        self.Kd, self.Vd = normal(seed + 6, B, L, Hkv, Dcap, d), normal(seed + 7, B, L, Hkv, Dcap, d)
        self.acc = torch.rand(B, L, Dcap, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed + 8))
        self.born = torch.arange(Dcap, device="cuda", dtype=torch.int32).expand(B, L, Dcap).contiguous()
        self.count = torch.from_numpy(self.counts).cuda()
        self.dims = skv.make_dims(B, L, H, Hkv, d, rows, 1, 0)
        self.K4, self.V4 = packed(ctx, self.dims, self.K, self.V, None, self.counts, rows) if self.Mcap else (None, None)
        self.ws = torch.empty(skv.shotkv_decode_workspace_bytes(self.dims, Dcap), dtype=torch.uint8, device="cuda")
        self.out = torch.full((B, L, H, d), float("nan"), device="cuda")
        self.st = skv.shotkv_decode_init(ctx, self.dims, skv.make_policy(r_d=r_d, recompress_every=every), Dcap, self.Mcap, self.Kd,
                                         self.Vd, self.acc, self.born, self.ws)
        self.st.T = self.st.n_dec = n_old
        self.before = self.acc.cpu().numpy().astype(np.float64)

    def run(self, attend, stream=None):
        a = (self.ctx, self.st, self.q, self.k, self.v, self.K4)
        if attend:
            return skv.shotkv_decode_step_attend_kv4(*a, self.V4, self.count, self.out, stream)
        return skv.shotkv_decode_step_kv4(*a, self.count, stream)

    def check(self, attend, units=None):
        n = self.n_old + 1
        assert (self.st.T, self.st.n_dec) == (n, n)
        acc, out = self.acc.cpu().numpy(), self.out.cpu().numpy()
        assert torch.equal(self.Kd[:, :, :, n - 1], self.k) and torch.equal(self.Vd[:, :, :, n - 1], self.v)
        assert (self.born[:, :, n - 1] == n - 1).all()
        for b, l in units or [(b, l) for b in range(self.B) for l in range(self.L)]:
            m = int(self.counts[b, l])
            kept_k, kept_v = f64(self.K[b, l, :, :m]), f64(self.V[b, l, :, :m])
            sk = sv = kept_k
            steepest = R.quantise(kept_v)[1].max(initial=0.0)
            if m:
                sk, sv = R.sizes_of(kept_k, True), R.sizes_of(kept_v, False)
                kept_k, kept_v = R.values_of(kept_k, True), R.values_of(kept_v, False)
            kd, vd = f64(self.Kd[b, l, :, :n]), f64(self.Vd[b, l, :, :n])
            w, w_off, o, o_off = R.step(f64(self.q[b, l]), np.concatenate([kept_k, kd], 1), np.concatenate([kept_v, vd], 1) if attend else None, m,
                                        np.concatenate([sk, np.abs(kd)], 1), np.concatenate([sv, np.abs(vd)], 1), steepest)
            old = np.append(self.before[b, l, :n - 1], 0.0)
            assert np.all(np.abs(acc[b, l, :n] - (old + w)) <= w_off + 2.0 ** -22 * (old + w)), "scores"
            if attend:
                err = np.abs(out[b, l] - o)
                assert np.all(err <= o_off), f"outputs of {b}, {l}: off by {(err / o_off).max()} of what they may be"


SHAPES = [  # B, L, Hkv, G, M, n_old
    (1, 1, 1, 1, 1, 0), (1, 1, 1, 8, 15, 1), (1, 1, 2, 2, 16, 15), (2, 1, 2, 3, 17, 16), (1, 2, 4, 4, 31, 33), (2, 2, 1, 7, 33, 64),
    (1, 1, 8, 4, 64, 3), (3, 1, 2, 4, 204, 128), (1, 1, 1, 5, 2049, 100), (2, 3, 8, 4, 500, 200), (1, 1, 2, 4, 100, 900), (4, 8, 8, 4, 333, 40),
    (9, 16, 2, 2, 130, 20)]


@pytest.mark.parametrize("attend", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,L,Hkv,G,M,n_old", SHAPES)
def test_step_is_the_definition_s(ctx, B, L, Hkv, G, d, M, n_old, attend):
    s = Step(ctx, B, L, Hkv, G, d, M, n_old, seed=M + G)
    s.run(attend)
    units = [(0, 0), (B - 1, L - 1), (B // 2, L // 2), (B - 1, 0), (0, L - 1)]
    s.check(attend, units)


@pytest.mark.parametrize("attend", [False, True])
def test_step_without_a_prompt(ctx, attend):
    s = Step(ctx, 2, 1, 2, 4, 64, 0, 37, counts=np.zeros((2, 1), np.int32), Mcap=0)
    s.run(attend)
    s.check(attend)


@pytest.mark.parametrize("d", [64, 128])
def test_counts_beyond_the_cap_are_cut(ctx, d):
    s = Step(ctx, 1, 2, 2, 4, d, 70, 10, counts=np.full((1, 2), 70, np.int32))
    s.count.fill_(1000)
    s.run(True)
    s.check(True)
    s = Step(ctx, 1, 2, 2, 4, d, 70, 10, counts=np.zeros((1, 2), np.int32))
    s.count.fill_(-3)
    s.run(True)
    s.check(True)


@pytest.mark.parametrize("attend", [False, True])
@pytest.mark.parametrize("fill", [0x00, 0x7F, 0xFF])
def test_what_lies_behind_the_kept_rows_is_not_looked_at(ctx, fill, attend):
    """Tiles that were packed with more rows than are kept now, and tiles never written: their scales may be anything."""
    M, kept = 160, 37
    s = Step(ctx, 1, 1, 2, 4, 128, M, 20, counts=np.full((1, 1), M, np.int32))
    word = torch.full((1,), fill, dtype=torch.uint8, device="cuda")
    s.K4[:, :, :, 2:] = word
    s.V4[:, :, :, 2:] = word
    for t, keys, groups in ((s.K4, True, 4), (s.V4, False, 1)):          # the rest of the last tile: codes stay, scales go
        at = 2048 + (kept - 32) * groups * 4
        t[:, :, :, 1, at:] = word
    s.count.fill_(kept)
    s.counts[:] = kept
    s.run(attend)
    s.check(attend)


@pytest.mark.parametrize("attend", [False, True])
def test_what_was_not_kept_may_be_anything(ctx, attend):
    B, L, Hkv, G, d, N, M = 1, 2, 2, 4, 64, 90, 40
    K, V = normal(1, B, L, Hkv, N, d), normal(2, B, L, Hkv, N, d)
    idx = torch.arange(0, 2 * M, 2, device="cuda", dtype=torch.int32).expand(B, L, M).contiguous()
    s = Step(ctx, B, L, Hkv, G, d, M, 12, counts=np.full((B, L), M, np.int32), keys=K[:, :, :, 0:2 * M:2].contiguous(),
             values=V[:, :, :, 0:2 * M:2].contiguous())
    for t in (K, V):
        t[:, :, :, 1::6] = float("nan")
        t[:, :, :, 3::6] = float("inf")
        t[:, :, :, 5::6] = torch.finfo(torch.bfloat16).min
    skv.shotkv_compact_kv4(ctx, skv.make_dims(B, L, Hkv * G, Hkv, d, N, 1, 0), K, V, idx, s.count, M, s.K4, s.V4)
    s.run(attend)
    s.check(attend)


@pytest.mark.parametrize("attend", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", ["sink", "rising", "falling", "small_q", "large_q", "values", "tiny_values", "far_keys"])
def test_ranges(ctx, case, d, attend):
    """Logits and values of very different sizes: what the steps keep in range goes out of it and comes back."""
    B, L, Hkv, G, M, n_old = 1, 1, 2, 4, 700, 50
    K, V = normal(1, B, L, Hkv, M, d).float(), normal(2, B, L, Hkv, M, d).float()
    q = normal(3, B, L, Hkv * G, d).float()
    ramp = torch.linspace(0, 1, M, device="cuda")[:, None]
    towards = q.reshape(B, L, Hkv, G, d).mean(3, keepdim=True)
    if case == "sink":                                       # the first key takes nearly all weight and its value is small
        K[:, :, :, 0] = 6 * towards[:, :, :, 0]
        V[:, :, :, 0] *= 0.01
    elif case == "rising":
        K += 6 * ramp * towards
    elif case == "falling":
        K += 6 * (1 - ramp) * towards
    elif case == "small_q":
        q *= 1e-20
    elif case == "large_q":
        q *= 100
        q[..., ::7] *= 1e-6
    elif case == "values":
        V *= torch.exp2(24 * torch.rand(M, 1, device="cuda", generator=torch.Generator(device="cuda").manual_seed(9)) - 12)
    elif case == "tiny_values":
        V *= 1e-15 * torch.exp2(40 * ramp)
    elif case == "far_keys":                                 # channels far from zero, groups that hardly vary
        K[..., ::5] += 40
        K[..., :32] = K[..., :32] * 0.01 - 25
        q *= 0.05
    bf = lambda t: t.to(torch.bfloat16).contiguous()         # noqa: E731
    s = Step(ctx, B, L, Hkv, G, d, M, n_old, counts=np.full((B, L), M, np.int32), keys=bf(K), values=bf(V), q=bf(q))
    s.run(attend)
    s.check(attend)


@pytest.mark.parametrize("attend", [False, True])
def test_numbers_that_are_not_finite_are_not_hidden(ctx, attend):
    """A kept key, value or query that is not finite leaves no finite output behind; in the scores it leaves what it leaves in
    the bf16 steps (a row without a sum has no weights)."""
    for what in ("key", "value", "query"):
        if what == "value" and not attend:
            continue
        K, V, q = normal(1, 1, 1, 1, 90, 64), normal(2, 1, 1, 1, 90, 64), normal(3, 1, 1, 2, 64)
        {"key": K, "value": V, "query": q}[what][..., -1, 5] = float("nan")
        s = Step(ctx, 1, 1, 1, 2, 64, 90, 4, counts=np.full((1, 1), 90, np.int32), keys=K, values=V, q=q)
        s.run(attend)
        t = Step(ctx, 1, 1, 1, 2, 64, 90, 4, counts=np.full((1, 1), 90, np.int32), keys=K, values=V, q=q)
        if attend:
            skv.shotkv_decode_step_attend(ctx, t.st, q, t.k, t.v, K, V, t.count, t.out)
            assert torch.isnan(s.out[:, :, 1] if what != "key" else s.out).any(-1).all(), what
            assert not torch.isfinite(s.out)[torch.isnan(t.out)].any(), what
        else:
            skv.shotkv_decode_step(ctx, t.st, q, t.k, t.v, K, t.count)
        assert torch.equal(torch.isnan(s.acc), torch.isnan(t.acc)), what


@pytest.mark.parametrize("attend", [False, True])
def test_caches_beyond_four_gigabytes(ctx, attend):
    """Every unit but the last has no rows; the last one's tiles lie beyond 2^32 bytes."""
    B, L, Hkv, G, d, M = 8, 32, 8, 1, 64, 65536
    counts = np.zeros((B, L), np.int32)
    counts[-1, -1] = 1000
    dims = skv.make_dims(B, L, Hkv * G, Hkv, d, M, 1, 0)
    assert skv.shotkv_kv4_value_bytes(dims, M) > 1 << 32
    K4, V4 = (torch.empty(B, L, Hkv, M // 32, R.tile_bytes(d, k), dtype=torch.uint8, device="cuda") for k in (True, False))
    s = Step(ctx, B, L, Hkv, G, d, 1, 5, counts=np.zeros((B, L), np.int32))
    K, V = normal(1, Hkv, 1000, d), normal(2, Hkv, 1000, d)
    for t, x, keys in ((K4, K, True), (V4, V, False)):
        rows = np.zeros((Hkv, 1024, d))
        rows[:, :1000] = f64(x)
        t[-1, -1, :, :32] = torch.from_numpy(R.write_tiles(rows, keys)).cuda()
    s.K4, s.V4, s.counts = K4, V4, counts
    s.count.copy_(torch.from_numpy(counts))
    s.st.Mcap = M
    s.run(attend)
    full = torch.zeros(B, L, Hkv, 1, d, dtype=torch.bfloat16)
    s.K = s.V = full

    class At:                                                # the last unit's rows where check() looks for them
        def __init__(self, x):
            self.x = x

        def __getitem__(self, i):
            b, l, _, m = i
            return self.x[:, :m.stop] if (b, l) == (B - 1, L - 1) else full[i]
    s.K, s.V = At(K), At(V)
    s.check(attend, [(0, 0), (B - 1, L - 1), (B - 1, L - 2)])


@pytest.mark.parametrize("B,L,Hkv,G,d,M,steps", [(2, 2, 2, 4, 128, 150, 70), (12, 3, 8, 5, 64, 90, 22), (1, 1, 8, 8, 128, 700, 15)])
def test_many_steps_with_evictions_are_the_bf16_steps(ctx, B, L, Hkv, G, d, M, steps):
    """Rows that 4 bits and bf16 both hold as they are: the two forms of the prompt take a generation through the same states.
    The prompt's form changes in mid-generation for a third state."""
    g = torch.Generator(device="cuda").manual_seed(4)
    K, V = (torch.randint(-8, 8, (B, L, Hkv, M, d), generator=g, device="cuda").float() for _ in range(2))
    for t in (K, V):                                         # every group reaches over the whole grid, of a scale of 1/8
        t[..., ::32], t[..., 1::32] = -8, 7
    K, V = (K / 8).to(torch.bfloat16), (V / 8).to(torch.bfloat16)
    counts = counts_of(B, L, M, 3)
    cfg = wl.DecodeConfig("kv4", B=B, L=L, H=Hkv * G, Hkv=Hkv, d=d, steps=steps, r_d=0.4, recompress_every=7, cfg_id=31)
    runs = [Step(ctx, B, L, Hkv, G, d, M, 0, counts=counts, keys=K, values=V, Dcap=80, every=7, r_d=0.4) for _ in range(3)]
    for i in range(steps):
        for k, s in enumerate(runs):
            s.q, s.k, s.v = wl.decode_step_inputs(cfg, i, "cuda")
            if k == 0 or (k == 2 and i % 20 < 10):
                skv.shotkv_decode_step_attend(ctx, s.st, s.q, s.k, s.v, s.K, s.V, s.count, s.out)
            else:
                s.run(k == 1 or i % 2 == 0)
        n = runs[0].st.n_dec
        for s in runs[1:]:
            assert s.st.n_dec == n
            assert torch.equal(s.born[:, :, :n], runs[0].born[:, :, :n]), f"step {i}"
            assert torch.equal(s.Kd[:, :, :, :n], runs[0].Kd[:, :, :, :n]) and torch.equal(s.Vd[:, :, :, :n], runs[0].Vd[:, :, :, :n])
            torch.testing.assert_close(s.acc[:, :, :n], runs[0].acc[:, :, :n], rtol=2e-5, atol=1e-6)
        # weights to 2^-17 there, and to 32-bit sums on both sides
        torch.testing.assert_close(runs[1].out, runs[0].out, rtol=1e-4, atol=2e-5)


# ------------------------------------------------------------------------------------------------ as programs call them
@pytest.mark.parametrize("groups", [0, 3])
@pytest.mark.parametrize("tokens", [False, True])
@pytest.mark.parametrize("units", ["shots", "sentences"])
def test_compressing_into_4_bits_is_compressing_and_packing(ctx, groups, tokens, units):
    S, lo, hi = (6, 60, 250) if units == "shots" else (60, 5, 30)
    cfg = wl.PrefillConfig("kv4", B=3, L=2, H=8, Hkv=2, d=64, N=1100, W=16, S=S, shot_dist="uniform", shot_lo=lo, shot_hi=hi,
                           question_len=80, r_p=0.4, cfg_id=27)
    Q, K, V, off = wl.prefill_batch(cfg, "cuda")
    dims, pol = P.dims_of(cfg), skv.make_policy(r_p=cfg.r_p)
    M = skv.shotkv_kept_capacity(dims, pol, off)
    a, b = (skv.alloc_prefill_outputs(dims, M, token_importance=tokens) for _ in range(2))
    (K4, V4), (K4b, V4b) = skv.alloc_kv4(dims, M), skv.alloc_kv4(dims, M)
    flags = skv.FLAG_TOKEN_IMPORTANCE if tokens else 0
    skv.shotkv_set_pipeline_groups(ctx, groups)
    try:
        skv.shotkv_prefill_compress(ctx, dims, pol, Q, K, V, off, a["shot_scores"], a["keep"], a["kept_idx"], a["kept_count"], M, a["Kc"],
                                    a["Vc"], a["token_importance"], flags, a["ws"])
        skv.shotkv_prefill_compress_kv4(ctx, dims, pol, Q, K, V, off, b["shot_scores"], b["keep"], b["kept_idx"], b["kept_count"], M, K4,
                                        V4, b["token_importance"], flags, b["ws"])
    finally:
        skv.shotkv_set_pipeline_groups(ctx, 0)
    compact = skv.make_dims(cfg.B, cfg.L, cfg.H, cfg.Hkv, cfg.d, M, 1, 0)
    skv.shotkv_compact_kv4(ctx, compact, a["Kc"], a["Vc"], None, a["kept_count"], M, K4b, V4b)
    for k in ("keep", "kept_idx", "kept_count"):
        assert torch.equal(a[k], b[k])
    assert torch.equal(K4, K4b) and torch.equal(V4, V4b)
    assert int(a["kept_count"].min()) > 0


@pytest.mark.parametrize("attend", [False, True])
@pytest.mark.parametrize("B,Hkv,M,n_old", [(1, 2, 300, 20), (40, 8, 100, 3)])
def test_a_captured_step_replays(ctx, B, Hkv, M, n_old, attend):
    """Packing and a step in one graph, replayed on other contents of the same tensors."""
    s = Step(ctx, B, 1, Hkv, 4, 128, M, n_old)
    s.run(attend)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    s.st.T = s.st.n_dec = n_old
    with torch.cuda.graph(graph):
        skv.shotkv_compact_kv4(ctx, s.dims, s.K, s.V, None, s.count, M, s.K4, s.V4)
        s.run(attend)
    for seed in (50, 60):
        s.K.copy_(normal(seed, *s.K.shape)), s.V.copy_(normal(seed + 1, *s.V.shape)), s.q.copy_(normal(seed + 2, *s.q.shape))
        s.counts[:] = counts_of(B, 1, M, seed)
        s.count.copy_(torch.from_numpy(s.counts))
        s.acc.uniform_()
        s.before = s.acc.cpu().numpy().astype(np.float64)
        s.out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        s.check(attend, [(0, 0), (B - 1, 0), (B // 2, 0)])


def test_first_calls_may_be_captured():
    """A process whose first calls of all are captured ones."""
    import subprocess
    import sys
    code = (
        "import sys; sys.path[:0] = ['tests', '.']\n"
        "import numpy as np, torch, paper_2502_01941_b200 as skv, test_kv4_gpu as T, test_norm_rope_gpu as N\n"
        "ctx = skv.Context(0)\n"
        "pack, T.packed = T.packed, lambda ctx, dims, K, V, idx, counts, M: skv.alloc_kv4(dims, M)\n"
        "s, r = T.Step(ctx, 2, 1, 2, 4, 64, 90, 10), N.Layer(2, 1, 4, 2, 64, 30, 5, 0, 30, 64)\n"
        "Kc, Vc = torch.zeros_like(s.K), torch.zeros_like(s.V)\n"
        "torch.cuda.synchronize()\n"
        "g = torch.cuda.CUDAGraph()\n"
        "with torch.cuda.graph(g):\n"
        "    r.run(ctx)\n"
        "    skv.shotkv_compact_kv4(ctx, s.dims, s.K, s.V, None, s.count, 90, s.K4, s.V4)\n"
        "    skv.shotkv_unpack_kv4(ctx, s.dims, s.K4, s.V4, s.count, 90, Kc, Vc)\n"
        "    s.run(True)\n"
        "g.replay(); torch.cuda.synchronize()\n"
        "s.check(True); r.check(); assert Kc.abs().sum() > 0\n"
        "del g\n")
    done = subprocess.run([sys.executable, "-c", code], cwd=__file__.rsplit("/tests/", 1)[0], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


def test_steps_on_streams_of_their_own(ctx):
    """Two states on two streams at once, each packed and stepped without a wait in between."""
    streams = [torch.cuda.Stream() for _ in range(2)]
    steps = [Step(ctx, 3, 2, 4, 4, 64, 400, 30, seed=k) for k in range(2)]
    torch.cuda.synchronize()
    for s in steps:
        s.K4.zero_(), s.V4.zero_()
    torch.cuda.synchronize()
    for s, stream in zip(steps, streams):
        skv.shotkv_compact_kv4(ctx, s.dims, s.K, s.V, None, s.count, 400, s.K4, s.V4, stream)
        s.run(True, stream)
    torch.cuda.synchronize()
    for s in steps:
        s.check(True, [(0, 0), (1, 1), (2, 1)])


@pytest.mark.parametrize("shape", [(1, 1, 1, 4, 128, 4000, 20), (30, 8, 8, 4, 128, 2000, 20)])
def test_a_wait_that_gives_up_leaves_the_context_usable(ctx, shape):
    """With a limit of one cycle the waits for tiles (and for a cluster's messages) may give up: the step ends, the next call says so
    once, and a new state steps as ever."""
    s = Step(ctx, *shape)
    torch.cuda.synchronize()
    skv.shotkv_set_wait_limit(ctx, 1)
    try:
        s.run(True)
        torch.cuda.synchronize()
    finally:
        skv.shotkv_set_wait_limit(ctx, 0)
    try:
        t = Step(ctx, *shape)                                # its packing is a call, too
    except skv.ShotKVError as e:
        assert e.code == skv.ERR_TIMEOUT
        t = Step(ctx, *shape)
    t.run(True)
    t.check(True, [(0, 0), (shape[0] - 1, shape[1] - 1)])


def test_both_ways_of_marshalling(ctx, monkeypatch):
    """Through the module and through ctypes: the same results, and the same exceptions."""
    from paper_2502_01941_b200 import binding
    import test_norm_rope_gpu as N
    assert binding._native is not None
    results = []
    for native in (binding._native, None):
        monkeypatch.setattr(binding, "_native", native)
        s, r = Step(ctx, 2, 1, 2, 4, 64, 90, 10), N.Layer(2, 1, 4, 2, 64, 30, 5, 0, 30, 64, all_q=True)
        Kc, Vc = torch.zeros_like(s.K), torch.zeros_like(s.V)
        r.run(ctx)
        skv.shotkv_unpack_kv4(ctx, s.dims, s.K4, s.V4, s.count, 90, Kc, Vc)
        s.run(True)
        first = (s.out.clone(), s.acc.clone())
        s.st.T = s.st.n_dec = 10
        s.run(False)
        results.append([s.K4, s.V4, Kc, Vc, *first, s.acc, r.K, r.V, r.Qwin, r.q_out])
        for call in (lambda: skv.shotkv_compact_kv4(ctx, s.dims, s.K, s.V, None, s.count, 90, s.K4.cpu(), s.V4),
                     lambda: skv.shotkv_unpack_kv4(ctx, s.dims, s.K4.cpu(), s.V4, s.count, 90, Kc, Vc),
                     lambda: skv.shotkv_decode_step_kv4(ctx, s.st, s.q, s.k, s.v, s.K4.cpu(), s.count)):
            with pytest.raises(ValueError, match="K4"):
                call()
        with pytest.raises(TypeError, match="positions"):
            skv.shotkv_norm_rope(ctx, r.dims, r.rope, r.q, r.k, r.v, r.wq, r.wk, r.table, torch.zeros(2, 30, device="cuda"), r.Qwin, r.K, r.V)
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_results_do_not_change_from_call_to_call(ctx):
    for shape in ((1, 1, 8, 4, 128, 1500, 100), (8, 8, 8, 4, 64, 200, 30)):
        outs = []
        for _ in range(3):
            s = Step(ctx, *shape)
            s.run(True)
            outs.append((s.out.clone(), s.acc.clone()))
        assert all(torch.equal(a, outs[0][0]) and torch.equal(b, outs[0][1]) for a, b in outs)


def test_refusals(ctx):
    s = Step(ctx, 1, 1, 2, 4, 64, 40, 3)
    L = skv.lib()
    # pointers, alignment
    for arg, t in (("K4", s.K4), ("V4", s.V4)):
        off = torch.zeros(t.numel() + 16, dtype=torch.uint8, device="cuda")[8:8 + t.numel()].view(t.shape)
        a = dict(K4=s.K4, V4=s.V4, **{}) | {arg: off}
        with pytest.raises(skv.ShotKVError, match="aligned"):
            skv.shotkv_decode_step_attend_kv4(ctx, s.st, s.q, s.k, s.v, a["K4"], a["V4"], s.count, s.out)
        with pytest.raises(skv.ShotKVError, match="aligned"):
            skv.shotkv_compact_kv4(ctx, s.dims, s.K, s.V, None, s.count, 40, a["K4"], a["V4"])
        a[arg] = None
        with pytest.raises(skv.ShotKVError, match="NULL"):
            skv.shotkv_decode_step_attend_kv4(ctx, s.st, s.q, s.k, s.v, a["K4"], a["V4"], s.count, s.out)
        with pytest.raises(skv.ShotKVError, match="NULL"):
            skv.shotkv_compact_kv4(ctx, s.dims, s.K, s.V, None, s.count, 40, a["K4"], a["V4"])
        with pytest.raises(skv.ShotKVError, match="NULL"):
            skv.shotkv_unpack_kv4(ctx, s.dims, a["K4"], a["V4"], s.count, 40, s.K, s.V)
    with pytest.raises(skv.ShotKVError, match="attn_out"):
        skv.shotkv_decode_step_attend_kv4(ctx, s.st, s.q, s.k, s.v, s.K4, s.V4, s.count, None)
    with pytest.raises(skv.ShotKVError, match="NULL"):
        skv.shotkv_decode_step_kv4(ctx, s.st, s.q, s.k, s.v, s.K4, None)
    # types
    with pytest.raises(TypeError, match="K4"):
        skv.shotkv_decode_step_kv4(ctx, s.st, s.q, s.k, s.v, s.K4.view(torch.int8), s.count)
    with pytest.raises(ValueError, match="K4"):
        skv.shotkv_compact_kv4(ctx, s.dims, s.K, s.V, None, s.count, 40, s.K4[..., ::2], s.V4)
    with pytest.raises(TypeError, match="V4"):
        skv.shotkv_compact_kv4(ctx, s.dims, s.K, s.V, None, s.count, 40, s.K4, s.V4.float())
    # shapes
    for bad, code in ((skv.make_dims(1, 1, 8, 2, 96, 40, 1, 0), skv.ERR_UNSUPPORTED_SHAPE), (skv.make_dims(1, 1, 8, 0, 64, 40, 1, 0), skv.ERR_INVALID_ARG),
                      (skv.make_dims(1, 1, 8, 2, 64, 0, 1, 0), skv.ERR_INVALID_ARG), (skv.make_dims(300, 300, 8, 2, 64, 40, 1, 0), skv.ERR_UNSUPPORTED_SHAPE)):
        with pytest.raises(skv.ShotKVError) as e:
            skv.shotkv_compact_kv4(ctx, bad, s.K, s.V, None, s.count, 40, s.K4, s.V4)
        assert e.value.code == code
    for cap in (0, -1):
        with pytest.raises(skv.ShotKVError, match="Mcap"):
            skv.shotkv_compact_kv4(ctx, s.dims, s.K, s.V, None, s.count, cap, s.K4, s.V4)
        with pytest.raises(skv.ShotKVError, match="Mcap"):
            skv.shotkv_unpack_kv4(ctx, s.dims, s.K4, s.V4, s.count, cap, s.K, s.V)
    s.st.n_dec = s.st.Dcap
    with pytest.raises(skv.ShotKVError, match="full"):
        s.run(True)
    s.st.n_dec = 3
    assert s.st.T == 3
    s.run(True)
    s.check(True)
    assert L.shotkv_compact_kv4(None, None, None, None, None, None, 1, None, None, None) == skv.ERR_INVALID_ARG
