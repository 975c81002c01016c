"""Norm, rotation and layout of projected heads against the definition in 64 bits, and the whole run of calls they begin."""
import numpy as np
import pytest
import torch

import kv4_reference as R
import paper_2502_01941_b200 as skv
from oracle import shotkv_oracle as O
from paper_2502_01941_b200 import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2502_01941_b200.build import build_library
    build_library()
    c = skv.Context(0)
    yield c
    c.close()


def table_of(rows, rot, theta=10000.0):
    angle = np.arange(rows)[:, None] * theta ** (-np.arange(0, rot, 2) / max(rot, 1))
    return torch.from_numpy(np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float32)).cuda()


def turned(x, weight, cs, rot, interleaved, eps):
    """x [B, rows, heads, d] float64, cs [B, rows, rot / 2, 2] -> rows and how far 32 bits and one rounding to bf16 may be off."""
    d = x.shape[-1]
    with np.errstate(invalid="ignore"):
        if weight is not None:
            x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
        y, size = x.copy(), np.abs(x)
        i = np.arange(rot // 2)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        cos, sin = cs[:, :, None, :, 0], cs[:, :, None, :, 1]
        y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
        size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    # half a step of bf16, and in 32 bits: the mean of d squares (half of its error in the root), root, weight and two products
    return y, np.abs(y) * 2.0 ** -8 + size * (d / 2 + 8) * 2.0 ** -24


class Layer:
    """Projected rows of one layer and the tensors they go to, filled with a mark."""

    def __init__(self, B, L, H, Hkv, d, N, W, first, rows, rot, layer=0, interleaved=False, norm=True, all_q=False, given=False,
                 fused=True, seed=0, eps=1e-5):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.__dict__.update(B=B, L=L, H=H, Hkv=Hkv, d=d, N=N, W=W, first=first, rows=rows, rot=rot, layer=layer, interleaved=interleaved, eps=eps)

        def draw(*shape):
            return (torch.randn(*shape, generator=g, device="cuda") * 2).to(torch.bfloat16)

        if fused:                                            # views of one projection, rows a little wider than their heads
            x = draw(B, rows + 1, H + 2 * Hkv + 1, d)
            self.q, self.k, self.v = x[:, :rows, :H], x[:, :rows, H:H + Hkv], x[:, :rows, H + Hkv:H + 2 * Hkv]
        else:
            self.q, self.k, self.v = draw(B, rows, H, d), draw(B, rows, Hkv, d), draw(B, rows, Hkv, d)
        self.wq, self.wk = (draw(d), draw(d)) if norm else (None, None)
        self.positions = torch.randint(0, 5000, (B, rows), generator=g, device="cuda", dtype=torch.int32) if given else None
        self.table = table_of(5000 if given else N, rot) if rot else None
        mark = lambda *s: torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda")     # noqa: E731
        self.Qwin, self.K, self.V = mark(B, L, H, W, d), mark(B, L, Hkv, N, d), mark(B, L, Hkv, N, d)
        self.q_out = mark(B, rows, H, d) if all_q else None
        self.dims = skv.make_dims(B, L, H, Hkv, d, N, W, 0)
        self.rope = skv.make_rope(rows=rows, rot=rot, first=first, layer=layer, interleaved=interleaved, eps=eps)

    def run(self, ctx, stream=None):
        return skv.shotkv_norm_rope(ctx, self.dims, self.rope, self.q, self.k, self.v, self.wq, self.wk, self.table, self.positions,
                                    self.Qwin, self.K, self.V, self.q_out, stream)

    def check(self):
        B, rows, first = self.B, self.rows, self.first
        pos = self.positions.cpu().numpy() if self.positions is not None else np.broadcast_to(first + np.arange(rows), (B, rows))
        cs = self.table.cpu().numpy().astype(np.float64) if self.rot else np.zeros((1, 0, 2))
        inside = (pos >= 0) & (pos < cs.shape[0])
        cs = cs[np.where(inside, pos, 0)] if self.rot else np.zeros((B, rows, 0, 2))
        if self.rot:
            cs[~inside] = np.nan
        w = [None if t is None else wl.bf16_to_f64(t) for t in (self.wq, self.wk)]
        q, q_off = turned(wl.bf16_to_f64(self.q), w[0], cs, self.rot, self.interleaved, self.eps)
        k, k_off = turned(wl.bf16_to_f64(self.k), w[1], cs, self.rot, self.interleaved, self.eps)

        def near(got, want, off):
            got = wl.bf16_to_f64(got)
            assert np.array_equal(np.isnan(got), np.isnan(want))
            with np.errstate(invalid="ignore"):
                assert not (np.abs(got - want) > off).any(), (np.abs(got - want) / off).max()

        def untouched(t):
            assert (t == 7).all()

        at = slice(first, first + rows)
        near(self.K[:, self.layer, :, at].transpose(1, 2), k, k_off)
        assert torch.equal(self.V[:, self.layer, :, at].transpose(1, 2), self.v)
        for t in (self.K, self.V):
            untouched(t[:, self.layer, :, :first]), untouched(t[:, self.layer, :, first + rows:])
        start = self.N - self.W
        lo, hi = min(max(first - start, 0), self.W), max(first + rows - start, 0)
        untouched(self.Qwin[:, self.layer, :, :lo]), untouched(self.Qwin[:, self.layer, :, hi:])
        if hi > lo:
            t0 = lo + start - first
            near(self.Qwin[:, self.layer, :, lo:hi].transpose(1, 2), q[:, t0:t0 + hi - lo], q_off[:, t0:t0 + hi - lo])
        for t in (self.Qwin, self.K, self.V):
            for l in range(self.L):
                if l != self.layer:
                    untouched(t[:, l])
        if self.q_out is not None:
            near(self.q_out, q, q_off)


CASES = [  # B, L, H, Hkv, d, N, W, first, rows, rot, more
    (1, 1, 1, 1, 64, 1, 1, 0, 1, 64, {}),
    (8, 1, 32, 8, 128, 1, 1, 0, 1, 128, dict(given=True)),
    (3, 2, 8, 2, 64, 1, 1, 0, 1, 32, dict(given=True, layer=1, interleaved=True)),
    (1, 1, 32, 8, 128, 300, 32, 0, 300, 128, {}),
    (2, 3, 6, 2, 64, 101, 7, 0, 101, 48, dict(layer=1, all_q=True)),
    (2, 1, 7, 7, 128, 100, 33, 11, 57, 16, dict(interleaved=True)),            # no row of the window
    (2, 1, 24, 8, 128, 100, 33, 11, 60, 96, dict(given=True)),                  # its first rows
    (1, 2, 17, 1, 64, 50, 50, 3, 40, 64, dict(norm=False, all_q=True)),         # the window is the prompt
    (2, 1, 8, 4, 128, 64, 5, 60, 4, 0, {}),                                     # no rotation
    (1, 1, 4, 2, 64, 40, 3, 37, 3, 0, dict(norm=False)),                        # neither
    (2, 1, 40, 5, 64, 70, 9, 0, 70, 64, dict(fused=False, interleaved=True, all_q=True)),
]


@pytest.mark.parametrize("B,L,H,Hkv,d,N,W,first,rows,rot,more", CASES)
def test_rows_are_the_definition_s(ctx, B, L, H, Hkv, d, N, W, first, rows, rot, more):
    s = Layer(B, L, H, Hkv, d, N, W, first, rows, rot, seed=H + N, **more)
    s.run(ctx)
    s.check()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 16), (64, 48), (128, 80), (128, 112), (128, 128)])
def test_every_rotated_part(ctx, d, rot, interleaved):
    s = Layer(1, 1, 3, 3, d, 20, 4, 0, 20, rot, interleaved=interleaved, all_q=True)
    s.run(ctx)
    s.check()


def test_one_weight_alone(ctx):
    for which in ("wq", "wk"):
        s = Layer(1, 1, 4, 2, 64, 30, 5, 0, 30, 64, all_q=True)
        setattr(s, which, None)
        s.run(ctx)
        s.check()


@pytest.mark.parametrize("interleaved", [False, True])
def test_positions_outside_the_table_are_nan(ctx, interleaved):
    s = Layer(2, 1, 4, 2, 128, 30, 30, 0, 30, 64, interleaved=interleaved, given=True)
    s.positions[0, 3], s.positions[0, 4], s.positions[1, 7], s.positions[1, 8] = -1, 5000, 2 ** 31 - 1, -(2 ** 31)
    s.run(ctx)
    s.check()
    assert torch.isnan(s.K[0, 0, :, 3, :64]).all() and not torch.isnan(s.K[0, 0, :, 3, 64:]).any()


def test_zeros_and_numbers_that_are_not_finite(ctx):
    """A head of zeros stays zeros; what is not finite stays in its head, and past the rotated part in its place."""
    s = Layer(1, 1, 2, 2, 128, 6, 6, 0, 6, 64, norm=False, fused=False)
    s.k[0, 0] = 0
    s.k[0, 1, 0, 100] = float("inf")
    s.k[0, 2, 1, 3] = float("nan")
    s.run(ctx)
    K = s.K[0, 0]
    assert (K[:, 0] == 0).all() and torch.isinf(K[0, 1, 100]) and int((~torch.isfinite(K[:, 1])).sum()) == 1
    assert torch.isnan(K[1, 2, 3]) and torch.isnan(K[1, 2, 35]) and int((~torch.isfinite(K[:, 2])).sum()) == 2
    s = Layer(1, 1, 2, 2, 64, 6, 6, 0, 6, 64)
    s.k[0, 0] = 0
    s.run(ctx)
    assert (s.K[0, 0, :, 0] == 0).all()


def test_prompts_beyond_two_to_the_31_elements(ctx):
    """Strides and places past 32 bits: the last rows of the last prompt of a large projection."""
    B, H, Hkv, d, N = 2, 8, 8, 128, 600000
    s = Layer(B, 1, H, Hkv, d, N, 4, N - 6, 6, 128, given=True)
    big = torch.zeros(B, N, H + 2 * Hkv, d, dtype=torch.bfloat16, device="cuda")      # 7.4 GB
    big[:, N - 6:, :] = torch.cat([s.q, s.k, s.v], 2)
    s.q, s.k, s.v = big[:, N - 6:, :H], big[:, N - 6:, H:H + Hkv], big[:, N - 6:, H + Hkv:]
    assert (B * Hkv * N * d) > 1 << 30 and big.numel() > 1 << 31
    s.run(ctx)
    s.check()


def test_parts_of_a_prompt_make_the_prompt(ctx):
    whole = Layer(2, 1, 8, 2, 64, 90, 40, 0, 90, 64, fused=False)
    whole.run(ctx)
    parts = Layer(2, 1, 8, 2, 64, 90, 40, 0, 90, 64, fused=False)
    q, k, v = parts.q, parts.k, parts.v
    for a, b in ((0, 13), (13, 14), (14, 71), (71, 90)):
        parts.q, parts.k, parts.v = q[:, a:b], k[:, a:b], v[:, a:b]
        parts.rope.first, parts.rope.rows = a, b - a
        parts.run(ctx)
    for n in ("Qwin", "K", "V"):
        assert torch.equal(getattr(whole, n), getattr(parts, n))


def test_captured_and_on_another_stream(ctx):
    s = Layer(2, 1, 8, 2, 128, 50, 9, 0, 50, 128, fused=False, given=True)
    s.run(ctx)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run(ctx)
    s.q.normal_(), s.k.normal_(), s.v.normal_(), s.positions.random_(0, 5000)
    graph.replay()
    torch.cuda.synchronize()
    s.check()
    side = torch.cuda.Stream()
    s.k.normal_()
    torch.cuda.synchronize()
    s.run(ctx, side)
    torch.cuda.synchronize()
    s.check()


def test_refusals(ctx):
    def make(**more):
        return Layer(2, 2, 8, 2, 64, 30, 5, 3, 20, 32, fused=False, **more)

    def bad(match, code=skv.ERR_INVALID_ARG, **fields):
        s = make()
        for k, x in fields.items():
            setattr(s.rope if hasattr(s.rope, k) else s, k, x)
        with pytest.raises(skv.ShotKVError, match=match) as e:
            s.run(ctx)
        assert e.value.code == code

    bad("layer", layer=2)
    bad("layer", layer=-1)
    bad("first", first=11)
    bad("first", first=-1)
    bad("eps", eps=float("nan"))
    bad("eps", eps=-1.0)
    bad("interleaved", interleaved=2)
    bad("NULL", table=None)
    bad("NULL", K=None)
    bad("NULL", Qwin=None)
    bad("aligned", K=torch.zeros(10000, dtype=torch.bfloat16, device="cuda")[1:])
    bad("head dimension", code=skv.ERR_UNSUPPORTED_SHAPE, dims=skv.make_dims(2, 2, 8, 2, 32, 30, 5, 0),
        **{n: torch.zeros(2, 20, h, 32, dtype=torch.bfloat16, device="cuda") for n, h in (("q", 8), ("k", 2), ("v", 2))})
    bad("W exceeds", dims=skv.make_dims(2, 2, 8, 2, 64, 30, 31, 0))
    for rot in (8, 24, 80, -16):
        s = make()
        s.rope.rot = rot
        s.table = torch.zeros(30, max(rot // 2, 0), 2, device="cuda")
        with pytest.raises((skv.ShotKVError, ValueError)):
            s.run(ctx)
    s = make()
    s.table = s.table[:, :8].contiguous()
    with pytest.raises(ValueError, match="cos_sin"):
        s.run(ctx)
    s = make()
    s.q = s.q[:, :, :7]
    with pytest.raises(ValueError, match="q"):
        s.run(ctx)
    s = make()
    s.k = s.k.transpose(2, 3).contiguous().transpose(2, 3)
    with pytest.raises(ValueError, match="k"):
        s.run(ctx)
    s = make()
    s.v = s.v.float()
    with pytest.raises(TypeError, match="v"):
        s.run(ctx)
    s = make()
    s.q = torch.zeros(2, 20, 8 * 64 + 4, dtype=torch.bfloat16, device="cuda")[:, :, :512].unflatten(2, (8, 64))
    with pytest.raises(skv.ShotKVError, match="strides"):
        s.run(ctx)


# ------------------------------------------------------------------------------------------------ the whole run
@pytest.mark.parametrize("d,Hkv,G", [(64, 2, 3), (128, 2, 4)])
def test_a_generation_from_its_projections(ctx, d, Hkv, G):
    """Two layers' prompts: normed and rotated in two parts, scored and packed in 4 bits; then a dozen tokens whose projections are
    normed, rotated and stepped over the packed prompt, one layer after the other, with evictions.  Every layer's outputs are
    those of 64-bit attention over the definition's rows."""
    B, L, N, W, steps, every, r_d, r_p = 2, 2, 400, 16, 12, 4, 0.5, 0.4
    H = Hkv * G
    g = torch.Generator(device="cuda").manual_seed(d)
    off = np.stack([np.array([0, 60, 130, 220, 300], np.int32), np.array([10, 90, 140, 200, 310], np.int32)])
    dims, pol = skv.make_dims(B, L, H, Hkv, d, N, W, 4), skv.make_policy(r_p=r_p, r_d=r_d, recompress_every=every)
    table = table_of(N + steps, d)
    wq, wk = ((1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(torch.bfloat16) for _ in range(2))
    Qwin = torch.empty(B, L, H, W, d, dtype=torch.bfloat16, device="cuda")
    K, V = (torch.empty(B, L, Hkv, N, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def project(rows):
        x = torch.randn(B, rows, H + 2 * Hkv, d, generator=g, device="cuda").to(torch.bfloat16)
        return x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]

    for l in range(L):
        for first, rows in ((0, 250), (250, 150)):
            skv.shotkv_norm_rope(ctx, dims, skv.make_rope(rows=rows, rot=d, first=first, layer=l), *project(rows), wq, wk, table, None,
                                 Qwin, K, V)
    M = skv.shotkv_kept_capacity(dims, pol, off)
    o = skv.alloc_prefill_outputs(dims, M)
    K4, V4 = skv.alloc_kv4(dims, M)
    skv.shotkv_prefill_compress_kv4(ctx, dims, pol, Qwin, K, V, off, o["shot_scores"], o["keep"], o["kept_idx"], o["kept_count"], M, K4, V4,
                                    None, 0, o["ws"])
    # a layer's own state, stepped layer after layer
    one = skv.make_dims(B, 1, H, Hkv, d, 1, 1, 0)
    Dcap = skv.shotkv_decode_capacity(pol, steps)
    states, tensors = [], []
    for l in range(L):
        t = [torch.zeros(B, 1, Hkv, Dcap, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        t += [torch.zeros(B, 1, Dcap, device="cuda"), torch.zeros(B, 1, Dcap, dtype=torch.int32, device="cuda"),
              torch.empty(skv.shotkv_decode_workspace_bytes(one, Dcap), dtype=torch.uint8, device="cuda")]
        tensors.append(t)
        states.append(skv.shotkv_decode_init(ctx, one, pol, Dcap, M, *t))
    q, k, v = (torch.empty(B, 1, h, 1, d, dtype=torch.bfloat16, device="cuda") for h in (H, Hkv, Hkv))
    out = torch.empty(B, 1, H, d, device="cuda")
    K4l, V4l, counts = ([x[:, l].contiguous() for l in range(L)] for x in (K4, V4, o["kept_count"]))
    oracles, prompt = {}, {}
    for b in range(B):
        for l in range(L):
            ref = O.prefill_compress(wl.bf16_to_f64(Qwin[b, l]), wl.bf16_to_f64(K[b, l]), wl.bf16_bits(V[b, l]), off[b], r_p)
            n = int(counts[l][b])
            assert np.array_equal(o["kept_idx"][b, l, :n].cpu().numpy(), ref["kept_idx"])
            kept = [wl.bf16_to_f64(x[b, l])[:, ref["kept_idx"]] for x in (K, V)]
            rows = [R.values_of(x, i == 0) for i, x in enumerate(kept)]
            oracles[b, l] = O.DecodeOracle(rows[0], H, r_d, every, Vc=rows[1])
            prompt[b, l] = kept
    for i in range(steps):
        at = torch.full((B, 1), N + i, dtype=torch.int32, device="cuda")
        for l in range(L):
            skv.shotkv_norm_rope(ctx, one, skv.make_rope(rows=1, rot=d), *project(1), wq, wk, table, at, q, k, v)
            skv.shotkv_decode_step_attend_kv4(ctx, states[l], q[:, :, :, 0], k[:, :, :, 0], v[:, :, :, 0], K4l[l], V4l[l], counts[l], out)
            for b in range(B):
                orc = oracles[b, l]
                orc.accumulate(wl.bf16_to_f64(q[b, 0, :, 0]), wl.bf16_to_f64(k[b, 0, :, 0]), wl.bf16_bits(v[b, 0, :, 0]), wl.bf16_to_f64(v[b, 0, :, 0]))
                # sums in 32 bits of some 200 rows: 2^-12 of the head's largest component is 100 times what they come to
                assert np.abs(out[b, 0].cpu().numpy() - orc.last_out).max() <= 2.0 ** -12 * np.abs(orc.last_out).max()
                if orc.eviction_due():
                    orc.apply_keep(orc.choose_keep())
                n = states[l].n_dec
                assert tensors[l][3][b, 0, :n].tolist() == orc.born
                np.testing.assert_allclose(tensors[l][2][b, 0, :n].cpu().numpy(), np.array(orc.acc), rtol=1e-4, atol=1e-6)
