"""Norm and rotation of prompts long enough for every way of dealing rows to warps, and of tensors past 2^31 elements."""
import pytest
import torch

import paper_2502_01941_b200 as skv
from test_norm_rope_gpu import Layer

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2502_01941_b200.build import build_library
    build_library()
    c = skv.Context(0)
    yield c
    c.close()


CASES = [  # B, L, H, Hkv, d, N, W, first, rows, rot, more
    (1, 1, 32, 8, 128, 1201, 1201, 0, 1201, 128, dict(all_q=True)),
    (1, 1, 20, 5, 128, 701, 64, 0, 701, 128, dict(all_q=True, interleaved=True)),       # a last section and a last piece in part
    (1, 1, 36, 9, 128, 650, 33, 0, 650, 96, dict(all_q=True, given=True)),
    (2, 1, 8, 8, 128, 1301, 40, 0, 1301, 64, dict(all_q=True)),                         # two rows of queries a warp, the last alone
    (2, 1, 7, 7, 128, 1301, 1000, 3, 1297, 64, dict(norm=False)),
    (1, 2, 18, 9, 64, 1250, 50, 0, 1250, 64, dict(layer=1, all_q=True, interleaved=True)),
    (1, 1, 72, 36, 64, 640, 20, 0, 640, 32, dict(all_q=True, given=True, norm=False)),
    (3, 1, 12, 3, 64, 2003, 16, 1, 2001, 48, dict(all_q=True, given=True)),
    (1, 1, 16, 16, 64, 1207, 700, 0, 1207, 64, dict(fused=False)),
    (2, 1, 6, 2, 128, 2399, 77, 0, 2399, 128, dict(all_q=True, interleaved=True)),
]


def pieces(heads, rows, B, d, ahead, sms):
    """Pieces a lane that the call chooses for a row's heads: as many as a warp has in flight, fewer for few heads or little to do."""
    a_piece = 32 // (d // 8)
    all_ = -(-heads // a_piece)
    most = ahead
    while True:
        vectors = 1
        while vectors < all_ and vectors < most:
            vectors *= 2
        warps = -(-rows // (ahead // vectors)) * -(-all_ // vectors)
        if most <= 2 or warps * B >= 4 * sms:
            return vectors
        most //= 2


def test_the_cases_reach_every_way():
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    keys, queries = set(), set()
    for B, L, H, Hkv, d, N, W, first, rows, rot, more in CASES:
        keys.add((d, pieces(Hkv, rows, B, d, 4, sms)))
        skip = 0 if more.get("all_q") else min(max(N - W - first, 0), rows)
        queries.add((d, pieces(H, rows - skip, B, d, 8, sms)))
    assert {(64, 4), (128, 4), (64, 1), (128, 1)} <= keys
    assert {(64, 4), (128, 4), (64, 8), (128, 8)} <= queries


@pytest.mark.parametrize("B,L,H,Hkv,d,N,W,first,rows,rot,more", CASES)
def test_long_prompts_are_the_definition_s(ctx, B, L, H, Hkv, d, N, W, first, rows, rot, more):
    s = Layer(B, L, H, Hkv, d, N, W, first, rows, rot, seed=H + N, **more)
    s.run(ctx)
    s.check()


def test_strides_past_two_to_the_31_elements(ctx):
    """From prompt to prompt, and from a prompt's first row to its last."""
    B, H, Hkv, d, rows = 2, 4, 2, 64, 10
    s = Layer(B, 1, H, Hkv, d, rows, 4, 0, rows, 64, given=True)
    row = (1 << 28) + 8
    prompt = rows * row + 16
    assert (rows - 1) * row > 1 << 31 and prompt > 1 << 31
    big = torch.empty(B * prompt, dtype=torch.bfloat16, device="cuda")               # 10.7 GB
    x = big.as_strided((B, rows, H + 2 * Hkv, d), (prompt, row, d, 1))
    x.copy_(torch.cat([s.q, s.k, s.v], 2))
    s.q, s.k, s.v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
    s.run(ctx)
    s.check()


def test_caches_past_two_to_the_31_elements(ctx):
    s = Layer(1, 4, 8, 8, 128, 540000, 4, 539994, 6, 128, layer=3, given=True)
    assert s.K.numel() > 1 << 31
    s.run(ctx)
    s.check()
    assert (s.K[0, 0, 0, -6:] == 7).all()
