"""The 4-bit form's definition and sizes, and the norm and rotation's arguments, without a GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

import kv4_reference as R
import paper_2502_01941_b200 as skv
from paper_2502_01941_b200 import binding
from paper_2502_01941_b200.build import build_library


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16).float().numpy().astype(np.float64)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("keys", [True, False])
def test_every_element_has_a_place_of_its_own(d, keys):
    word, nibble, group = R.places(d, keys)
    assert sorted((8 * word + nibble).ravel().tolist()) == list(range(32 * d))
    assert group.max() * 4 + 4 == R.tile_bytes(d, keys) and R.tile_bytes(d, keys) % 128 == 0
    rows = bf16(np.random.default_rng(d).standard_normal((2, 64, d)) * 3)
    tiles = R.write_tiles(rows, keys)
    assert tiles.shape == (2, 2, R.tile_bytes(d, keys))
    c, s, z = R.read_tiles(tiles, d, keys)
    assert np.array_equal(s * (c + z), R.values_of(rows, keys))


@pytest.mark.parametrize("group", [32, 64, 128])
def test_an_element_is_off_by_half_a_step(group):
    rng = np.random.default_rng(group)
    for scale, mean in [(1, 0), (1e-20, 0), (1e20, 0), (1, 30), (0.01, -5), (0, 2.5), (0, 0), (1e-39, 0)]:
        x = bf16(rng.standard_normal((50, group)) * scale + mean)
        c, s, z = R.quantise(x)
        assert c.min() >= -8 and c.max() <= 7
        assert (np.abs(s[:, None] * (c + z[:, None]) - x) <= s[:, None] / 2).all()
        exact = s[:, None].astype(np.float32) * (c + z[:, None]).astype(np.float32)
        assert np.array_equal(exact.astype(np.float64), s[:, None] * (c + z[:, None])), "s (c + z) is exact in 32 bits"


@pytest.mark.parametrize("d", [64, 128])
def test_sizes(d):
    for B, L, Hkv, M in [(1, 1, 1, 1), (2, 3, 4, 32), (1, 2, 8, 33), (8, 32, 8, 3276), (4, 32, 8, 131072)]:
        dims = skv.make_dims(B, L, Hkv, Hkv, d, 1, 1, 0)
        tiles = -(-M // 32)
        assert skv.shotkv_kv4_key_bytes(dims, M) == B * L * Hkv * tiles * R.tile_bytes(d, True)
        assert skv.shotkv_kv4_value_bytes(dims, M) == B * L * Hkv * tiles * R.tile_bytes(d, False)
    for bad in [skv.make_dims(1, 1, 2, 2, 96, 1, 1, 0), skv.make_dims(0, 1, 2, 2, d, 1, 1, 0), skv.make_dims(1, 70000, 2, 2, d, 1, 1, 0)]:
        assert skv.shotkv_kv4_key_bytes(bad, 10) == 0 and skv.shotkv_kv4_value_bytes(bad, 10) == 0
    good = skv.make_dims(1, 1, 2, 2, d, 1, 1, 0)
    assert skv.shotkv_kv4_key_bytes(good, 0) == 0 and skv.shotkv_kv4_key_bytes(good, 2 ** 31 - 1) == 0
    k, v = skv.alloc_kv4(skv.make_dims(2, 3, 4, 2, d, 1, 1, 0), 33, device="cpu")
    assert k.shape == (2, 3, 2, 2, R.tile_bytes(d, True)) and v.shape == (2, 3, 2, 2, R.tile_bytes(d, False))


def test_calls_without_a_context_are_refused():
    L = skv.lib()
    dims, rope, st = skv.make_dims(1, 1, 4, 2, 64, 8, 2, 0), skv.make_rope(), skv.DecodeState()
    assert L.shotkv_norm_rope(None, C.byref(dims), C.byref(rope), *[None] * 12) == skv.ERR_INVALID_ARG
    assert L.shotkv_compact_kv4(None, C.byref(dims), None, None, None, None, 8, None, None, None) == skv.ERR_INVALID_ARG
    assert L.shotkv_unpack_kv4(None, C.byref(dims), None, None, None, 8, None, None, None) == skv.ERR_INVALID_ARG
    assert L.shotkv_decode_step_kv4(None, C.byref(st), *[None] * 6) == skv.ERR_INVALID_ARG
    assert L.shotkv_decode_step_attend_kv4(None, C.byref(st), *[None] * 8) == skv.ERR_INVALID_ARG


def test_rope_structure_is_the_header_s():
    assert C.sizeof(skv.Rope) == 7 * 4 + 4 + 6 * 8
    r = skv.make_rope(rows=3, rot=32, first=5, layer=1, interleaved=True, eps=0.25)
    assert (r.layer, r.first, r.rows, r.rot, r.interleaved, r.table_rows, r.eps) == (1, 5, 3, 32, 1, 0, 0.25)


@pytest.mark.parametrize("t,error", [(torch.zeros(1, 3, 4, 64), TypeError), (torch.zeros(1, 3, 4, 64, dtype=torch.bfloat16), ValueError),
                                     ([1.0], TypeError)])
def test_projected_heads_are_cuda_bf16(t, error):
    with pytest.raises(error, match="q"):
        binding._heads(t, 3, 4, 64, 1, "q")
