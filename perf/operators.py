"""The operators around a compressed cache that is held in 4 bits, as cases that can be timed.

A case is a dict of plain sizes and options; `prepare` makes what the calling program holds before the call (seeded
inputs on the GPU, output buffers, packed caches), `run` makes one pass and returns all of its outputs, `work` counts
the bytes and operations the pass cannot do without, `exact` says what the outputs are in 64-bit floating point.

Three kinds of pass:
  rope   shotkv_norm_rope: a layer's projected queries, keys and values, normed per head and rotated by position, into
         the layouts that the other calls take
  pack   shotkv_compact_kv4, the gather of the kept rows into 4 bits, and shotkv_unpack_kv4, the way back
  step   one step of shotkv_decode_step_kv4 (or of shotkv_decode_step_attend_kv4) over a prompt's cache in 4 bits

With `own` false the same is computed by elementary torch operations in 32 bits.

A row is held in 4 bits as x = s (c + z): whole c of -8 to 7, a scale s and a whole z for each group, which is 32 elements of a
key and all of a value.  s is the least bf16 number that is no less than a 15th of the group's range, a 240th of its
greatest magnitude and 2^-100; c + z is x / s rounded to the nearest whole number (ties up), and z is 8 more than the least
of them.  A unit's rows lie in tiles of 32 (a last, partly filled tile ends in rows of zeros): the codes, then the
groups' words with s in the high half and z in the low half, both bf16.
"""
import functools
import math

import torch

own = False


# ------------------------------------------------------------------------------------------------ cases
def _rope(name, B, L, H, Hkv, d, N, W, first, rows, rot, layer=0, interleaved=False, norm=True, all_q=False, given=False):
    return dict(name=name, kind="rope", B=B, L=L, H=H, Hkv=Hkv, d=d, N=N, W=W, first=first, rows=rows, rot=rot, layer=layer,
                interleaved=interleaved, norm=norm, all_q=all_q, given=given)


def _pack(name, B, L, Hkv, d, N, M, ragged=True):
    return dict(name=name, kind="pack", B=B, L=L, Hkv=Hkv, d=d, N=N, M=M, ragged=ragged)


def _step(name, B, L, H, Hkv, d, M, n0, attend, ragged=True):
    return dict(name=name, kind="step", B=B, L=L, H=H, Hkv=Hkv, d=d, M=M, n0=n0, attend=attend, ragged=ragged)


def listed():
    return [
        # one layer's token of eight sequences, each at a position of its own: what precedes every decode step
        _rope("rope_token_b8", 8, 1, 32, 8, 128, 1, 1, 0, 1, 128, given=True),
        # one layer of a 4K prompt, all queries wanted too: the model's own attention takes them
        _rope("rope_prompt_4k", 1, 1, 32, 8, 128, 4096, 32, 0, 4096, 128, all_q=True),
        # the largest: one layer of four 32K prompts, of the queries the window alone
        _rope("rope_prompt_32k_b4", 4, 1, 32, 8, 128, 32768, 64, 0, 32768, 128),
        # a later part of a prompt, odd sizes, neighbouring pairs, half of a small head rotated, no norms, second of two layers
        _rope("rope_chunk_ragged", 3, 2, 24, 8, 64, 5003, 33, 1777, 3001, 32, layer=1, interleaved=True, norm=False, given=True),
        # the smallest cache: one layer, two heads, a few shots of a 512-token prompt
        _pack("pack_tiny", 1, 1, 2, 64, 512, 204, ragged=False),
        # all layers of a 16K prompt compressed to a fifth
        _pack("pack_model_16k", 1, 32, 8, 128, 16384, 3276),
        # odd sizes, kept counts that differ from layer to layer
        _pack("pack_ragged", 3, 4, 8, 128, 5003, 1751),
        # the smallest step: one small layer, scores only
        _step("step_tiny", 1, 1, 4, 2, 64, 204, 128, False, ragged=False),
        # one layer of four sequences: a model calls the step layer after layer
        _step("step_attend_layer_b4", 4, 1, 32, 8, 128, 3276, 127, True),
        # all layers of eight sequences, scores only
        _step("step_model_b8", 8, 32, 32, 8, 128, 3276, 144, False),
        # the largest: the same with the attention output
        _step("step_attend_model_b8", 8, 32, 32, 8, 128, 3276, 144, True),
        # three query heads to a KV head, small heads, odd lengths, caches from empty to full
        _step("step_attend_ragged", 5, 3, 24, 8, 64, 1009, 301, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "pack", "step", "step"])
    d = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8, 8])
    G = rng.choice([1, 2, 3, 4, 4, 7, 8])
    if kind == "rope":
        B = _log_int(rng, 1, 8)
        N = rng.choice([1, _log_int(rng, 2, 32768), _log_int(rng, 512, 32768)])
        while B * N > 4 * 32768 or B * N * (G + 2) * Hkv * d > 32768 * 48 * 128:
            B, N = (B + 1) // 2, (N + 1) // 2
        W = min(rng.randint(1, 64), N, 256 // G)
        first = rng.choice([0, rng.randint(0, N - 1)])
        rows = rng.choice([N - first, rng.randint(1, N - first)])
        rot = rng.choice([d, d, d // 2, d // 4])
        L = rng.choice([1, 1, 2])
        c = _rope("", B, L, G * Hkv, Hkv, d, N, W, first, rows, rot, rng.randint(0, L - 1), rng.random() < 0.4, rng.random() < 0.6,
                  rng.random() < 0.5, rng.random() < 0.5)
    elif kind == "pack":
        B, L = _log_int(rng, 1, 4), rng.choice([1, _log_int(rng, 1, 32)])
        N = _log_int(rng, 512, 32768)
        while B * L * Hkv * N * d > 32 * 8 * 16384 * 128:
            B, L, N = (B + 1) // 2, (L + 1) // 2, max(512, N // 2)
        M = rng.randint(max(1, N // 16), N // 4)
        c = _pack("", B, L, Hkv, d, N, M, rng.random() < 0.7)
    else:
        B, L, M = _log_int(rng, 1, 8), rng.choice([1, 1, _log_int(rng, 1, 32)]), _log_int(rng, 1, 16384)
        n0 = rng.choice([0, _log_int(rng, 1, 1000), _log_int(rng, 32, 400)])
        while B * L * Hkv * (M + 4 * n0) * d > 8 * 32 * 8 * (3276 + 4 * 144) * 128:
            B, L = (B + 1) // 2, (L + 1) // 2
        c = _step("", B, L, G * Hkv, Hkv, d, M, n0, rng.random() < 0.65, rng.random() < 0.7)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ inputs
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _keys(g, *shape):
    """Keys as models have them: channels of very different sizes, some of them far from zero."""
    lead, d = shape[:-2], shape[-1]
    gain = torch.exp(0.5 * _normal(g, *lead, 1, d))
    return (_normal(g, *shape) * gain + 0.7 * _normal(g, *lead, 1, d)).to(torch.bfloat16)


def _tile_bytes(d):
    """Bytes of 32 rows of keys, and of values."""
    return 32 * (d // 2 + d // 8), 32 * (d // 2 + 4)


def _scale(x):
    """[..., group] float32 -> the group's scale; in 64 bits, as a quotient may lie next to a bf16 number."""
    top, low = x.amax(-1, keepdim=True).double(), x.amin(-1, keepdim=True).double()
    s = torch.maximum((top - low) / 15, torch.maximum(top.abs(), low.abs()) / 240).clamp_min(2.0**-100).float()
    return ((s.view(torch.int32) + 0xFFFF) & -65536).view(torch.float32)            # up to bf16


def _quantise(x):
    """[..., group] float32 -> codes -8..7, scale, z, as float32."""
    s = _scale(x)
    c = torch.floor(x / s + 0.5)
    z = c.amin(-1, keepdim=True) + 8
    return c - z, s, z


def _words(s, z):
    """Scale and z of a group as one 32-bit word."""
    lo = z.to(torch.bfloat16).float().view(torch.int32)
    return s.view(torch.int32) | ((lo >> 16) & 0xFFFF)


def _rows_to_tiles(x, axes, shape, order, words):
    """Packs codes [U, T * 32, d] (0..15) and the groups' words into tiles."""
    U, R, _ = x.shape
    n = x.to(torch.int32).reshape(U, R // 32, *shape).permute(0, 1, *[2 + axes.index(a) for a in order])
    n = n.reshape(U, R // 32, -1, 8)
    shift = 4 * torch.arange(8, device=x.device, dtype=torch.int32)
    w = (n << shift).sum(-1, dtype=torch.int64)
    w = torch.where(w > 0x7FFFFFFF, w - (1 << 32), w).to(torch.int32)
    return torch.cat([w, words.reshape(U, R // 32, -1)], -1).view(torch.uint8)


# the axes of a tile of keys: 16-row half, 8-row half, row | 64 dims, 32 dims, 8, 4, 2, 1; and in the order in which their codes
# lie, the last three within a word, least significant last.  For values the rows are cut otherwise.
_KEY_ROWS, _KEY_CODES = "hrgqjtlke", "hqgtjlekr"
_VALUE_ROWS, _VALUE_CODES = "hktEqgid", "hqgtiEkd"


def _key_shape(d):
    return 2, 2, 8, d // 64, 2, 4, 2, 2, 2


def _value_shape(d):
    return 2, 2, 4, 2, d // 64, 8, 4, 2


def _pack_rows(x, keys):
    """[U, T * 32, d] float32 -> tiles [U, T, bytes]."""
    U, R, d = x.shape
    c, s, z = _quantise(x.reshape(U, R, -1, 32) if keys else x.reshape(U, R, 1, d))
    args = (_KEY_ROWS, _key_shape(d), _KEY_CODES) if keys else (_VALUE_ROWS, _value_shape(d), _VALUE_CODES)
    return _rows_to_tiles(c.reshape(U, R, d) + 8, *args, _words(s, z))


def _packed_cache(g, c, keys):
    """A prompt's cache in 4 bits, [B, L, Hkv, tiles, bytes]; made a few units at a time."""
    U, T, d = c["B"] * c["L"] * c["Hkv"], (c["M"] + 31) // 32, c["d"]
    out = torch.empty(U, T, _tile_bytes(d)[0 if keys else 1], dtype=torch.uint8, device="cuda")
    each = max(1, (1 << 26) // (T * 32 * d))
    for u in range(0, U, each):
        n = min(each, U - u)
        x = _keys(g, n, T * 32, d) if keys else _normal(g, n, T * 32, d).to(torch.bfloat16)
        out[u:u + n] = _pack_rows(x.float(), keys)
    return out.reshape(c["B"], c["L"], c["Hkv"], T, -1)


def _counts(g, c):
    """Kept rows of every (sequence, layer): all of them, or any number; one of the first is the cap and one is none."""
    B, L, M = c["B"], c["L"], c["M"]
    n = torch.full((B, L), M, dtype=torch.int32, device="cuda")
    if c["ragged"]:
        low = 0 if c["kind"] == "step" and c["L"] < 32 else M - M // 8
        n = torch.randint(low, M + 1, (B, L), generator=g, device="cuda", dtype=torch.int32)
        n[0, 0] = M
        if low == 0 and B * L > 1:
            n[-1, -1] = 0
    return n


def _prepare_rope(c, g):
    B, L, H, Hkv, d, N, W, rows = (c[k] for k in ("B", "L", "H", "Hkv", "d", "N", "W", "rows"))
    # the projection's rows, of a width of their own for each head and channel
    x = _normal(g, B, rows, H + 2 * Hkv, d).to(torch.bfloat16)
    x *= torch.exp(0.4 * _normal(g, H + 2 * Hkv, d)).to(torch.bfloat16)
    q, k, v = x.split([H, Hkv, Hkv], 2)
    positions, end = None, N
    if c["given"]:
        start = torch.randint(0, 16384, (B, 1), generator=g, device="cuda")
        positions = (start + torch.arange(c["first"], c["first"] + rows, device="cuda")).to(torch.int32)
        end = 16384 + N
    angle = torch.arange(end, device="cuda", dtype=torch.float64)[:, None] * \
        500000.0 ** (-torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64) / c["rot"])
    s = dict(case=c, q=q, k=k, v=v, positions=positions, table=torch.stack([angle.cos(), angle.sin()], -1).float(),
             q_weight=None, k_weight=None, q_out=None)
    if c["norm"]:
        s["q_weight"], s["k_weight"] = ((1 + 0.2 * _normal(g, d)).to(torch.bfloat16) for _ in range(2))
    if c["all_q"]:
        s["q_out"] = torch.zeros(B, rows, H, d, dtype=torch.bfloat16, device="cuda")
    s["Qwin"] = torch.zeros(B, L, H, W, d, dtype=torch.bfloat16, device="cuda")
    s["K"], s["V"] = (torch.zeros(B, L, Hkv, N, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return s


def _prepare_pack(c, g):
    B, L, Hkv, d, N, M = (c[k] for k in ("B", "L", "Hkv", "d", "N", "M"))
    count = _counts(g, c)
    # whole runs of tokens are kept, as shots are
    run = max(1, N // 48)
    rank = torch.rand(B, L, -(-N // run), generator=g, device="cuda").repeat_interleave(run, 2)[..., :N].argsort(dim=-1, stable=True)
    idx = torch.where(torch.arange(M, device="cuda") < count[..., None], rank[..., :M], N).sort(-1).values
    idx = torch.where(idx < N, idx, -1).to(torch.int32)
    T, (kb, vb) = (M + 31) // 32, _tile_bytes(d)
    s = dict(case=c, K=_keys(g, B, L, Hkv, N, d), V=_normal(g, B, L, Hkv, N, d).to(torch.bfloat16), kept_idx=idx, kept_count=count)
    s["K4"], s["V4"] = (torch.zeros(B, L, Hkv, T, n, dtype=torch.uint8, device="cuda") for n in (kb, vb))
    s["Kc"], s["Vc"] = (torch.zeros(B, L, Hkv, M, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return s


def _prepare_step(c, g):
    """A generation that holds n0 entries since its last eviction, and the next token's queries, key and value."""
    B, L, H, Hkv, d, n0 = (c[k] for k in ("B", "L", "H", "Hkv", "d", "n0"))
    cap = n0 + 8
    s = dict(case=c, kept_count=_counts(g, c), K4=_packed_cache(g, c, True), V4=_packed_cache(g, c, False) if c["attend"] else None,
             q=_normal(g, B, L, H, d).to(torch.bfloat16), k=_keys(g, B, L, Hkv, 1, d)[:, :, :, 0].contiguous(),
             v=_normal(g, B, L, Hkv, d).to(torch.bfloat16), Kd=_keys(g, B, L, Hkv, cap, d),
             Vd=_normal(g, B, L, Hkv, cap, d).to(torch.bfloat16))
    s["born"] = torch.zeros(B, L, cap, dtype=torch.int32, device="cuda")
    s["born"][:, :, :n0] = torch.arange(n0, device="cuda")
    s["acc"] = torch.rand(B, L, cap, generator=g, device="cuda") * H / (c["M"] + n0)
    s["ws"] = torch.empty(B * L * (Hkv + 1) * cap * 4 + 1024, dtype=torch.uint8, device="cuda")
    if c["attend"]:
        s["out"] = torch.zeros(B, L, H, d, device="cuda")
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"rope": _prepare_rope, "pack": _prepare_pack, "step": _prepare_step}[case["kind"]](case, g)


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_turn(x, weight, table, rot, interleaved, eps):
    """Rows [B, t, heads, d] normed and rotated, in float32; table [B or 1, t, rot / 2, 2]."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * weight.float()
    cos, sin = table[..., 0].unsqueeze(2), table[..., 1].unsqueeze(2)
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., rot:]], -1)


EPS = 1e-6


def _plain_rope(s):
    c = s["case"]
    first, rows, layer, N, W = c["first"], c["rows"], c["layer"], c["N"], c["W"]
    at = s["positions"].long() if s["positions"] is not None else torch.arange(first, first + rows, device="cuda")[None]
    table = s["table"][at]
    win = max(0, N - W - first)                                      # the chunk's first window row
    q = _plain_turn(s["q"] if c["all_q"] else s["q"][:, win:], s["q_weight"], table if c["all_q"] else table[:, win:], c["rot"], c["interleaved"], EPS)
    s["K"][:, layer, :, first:first + rows] = _plain_turn(s["k"], s["k_weight"], table, c["rot"], c["interleaved"], EPS).transpose(1, 2)
    s["V"][:, layer, :, first:first + rows] = s["v"].transpose(1, 2)
    if win < rows:
        to = first + win - (N - W)
        s["Qwin"][:, layer, :, to:to + rows - win] = (q[:, win:] if c["all_q"] else q).transpose(1, 2)
    if c["all_q"]:
        s["q_out"].copy_(q)


def _plain_pack(s):
    M = s["case"]["M"]
    held = (torch.arange(M, device="cuda") < s["kept_count"][..., None])[:, :, None, :, None]
    at = s["kept_idx"].clamp_min(0).long()[:, :, None, :, None]
    for name, group in (("K", 32), ("V", s["case"]["d"])):
        x = s[name].gather(3, at.expand(*s[name].shape[:3], M, s[name].shape[4])).float()
        c, scale, z = _quantise(x.unflatten(-1, (-1, group)))
        s[name + "c"].copy_(torch.where(held, ((c + z) * scale).flatten(-2), s[name + "c"].float()))


def _plain_rows(tiles, d, keys):
    """Tiles [..., T, bytes] -> rows [..., T * 32, d] in float32."""
    words = tiles.view(torch.int32)
    lead, n = words.shape[:-1], 32 * d // 8
    rows, codes, shape = (_KEY_ROWS, _KEY_CODES, _key_shape(d)) if keys else (_VALUE_ROWS, _VALUE_CODES, _value_shape(d))
    x = ((words[..., :n, None] >> (4 * torch.arange(8, device="cuda", dtype=torch.int32))) & 15).to(torch.float32) - 8
    x = x.reshape(-1, *[shape[rows.index(a)] for a in codes]).permute(0, *[1 + codes.index(a) for a in rows])
    meta = words[..., n:].reshape(-1, 32, d // 32 if keys else 1, 1)
    scale, z = (meta & -65536).view(torch.float32), (meta << 16).view(torch.float32)
    x = (x.reshape(-1, 32, meta.shape[2], d // meta.shape[2]) + z) * scale
    return x.reshape(*lead[:-1], lead[-1] * 32, d)


def _plain_step(s):
    c = s["case"]
    B, L, H, Hkv, d, M, n0 = (c[k] for k in ("B", "L", "H", "Hkv", "d", "M", "n0"))
    n = n0 + 1
    s["Kd"][:, :, :, n0], s["Vd"][:, :, :, n0] = s["k"], s["v"]
    s["acc"][:, :, n0] = 0
    s["born"][:, :, n0] = n0
    q = s["q"].float().reshape(B, L, Hkv, H // Hkv, d)
    keys = torch.cat([_plain_rows(s["K4"], d, True)[:, :, :, :M], s["Kd"][:, :, :, :n].float()], 3)
    x = torch.matmul(q, keys.transpose(-1, -2)) / math.sqrt(d)
    gone = torch.arange(M, device="cuda") >= s["kept_count"][..., None]
    x[..., :M] = x[..., :M].masked_fill(gone[:, :, None, None], -math.inf)
    p = torch.exp(x - x.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    s["acc"][:, :, :n] += p[..., M:].sum((2, 3))
    if c["attend"]:
        values = torch.cat([_plain_rows(s["V4"], d, False)[:, :, :, :M], s["Vd"][:, :, :, :n].float()], 3)
        s["out"].copy_(torch.matmul(p, values).reshape(B, L, H, d))


# ------------------------------------------------------------------------------------------------ the framework's calls
@functools.lru_cache(maxsize=1)
def _context():
    """One context for the process, as a program that serves one GPU keeps."""
    import paper_2502_01941_b200 as skv
    return skv, skv.Context(0)


def _own_rope(s):
    skv, ctx = _context()
    c = s["case"]
    if "args" not in s:                                              # what a program makes once
        s["dims"] = skv.make_dims(c["B"], c["L"], c["H"], c["Hkv"], c["d"], c["N"], c["W"], 0)
        s["args"] = skv.make_rope(rows=c["rows"], rot=c["rot"], first=c["first"], layer=c["layer"], interleaved=c["interleaved"], eps=EPS)
    skv.shotkv_norm_rope(ctx, s["dims"], s["args"], s["q"], s["k"], s["v"], s["q_weight"], s["k_weight"], s["table"], s["positions"],
                         s["Qwin"], s["K"], s["V"], s["q_out"])


def _own_pack(s):
    skv, ctx = _context()
    c = s["case"]
    if "dims" not in s:
        s["dims"] = skv.make_dims(c["B"], c["L"], c["Hkv"], c["Hkv"], c["d"], c["N"], 1, 0)
    skv.shotkv_compact_kv4(ctx, s["dims"], s["K"], s["V"], s["kept_idx"], s["kept_count"], c["M"], s["K4"], s["V4"])
    skv.shotkv_unpack_kv4(ctx, s["dims"], s["K4"], s["V4"], s["kept_count"], c["M"], s["Kc"], s["Vc"])


def _own_step(s):
    skv, ctx = _context()
    c = s["case"]
    if "st" not in s:
        s["st"] = skv.shotkv_decode_init(ctx, skv.make_dims(c["B"], c["L"], c["H"], c["Hkv"], c["d"], 1, 1, 0),
                                         skv.make_policy(r_d=1.0, recompress_every=1 << 20), c["n0"] + 8, c["M"], s["Kd"], s["Vd"],
                                         s["acc"], s["born"], s["ws"])
    st = s["st"]
    st.T = st.n_dec = c["n0"]                                        # the same step again
    if c["attend"]:
        skv.shotkv_decode_step_attend_kv4(ctx, st, s["q"], s["k"], s["v"], s["K4"], s["V4"], s["kept_count"], s["out"])
    else:
        skv.shotkv_decode_step_kv4(ctx, st, s["q"], s["k"], s["v"], s["K4"], s["kept_count"])


def _outputs(s):
    c = s["case"]
    if c["kind"] == "rope":
        names = ("Qwin", "K", "V") + (("q_out",) if c["all_q"] else ())
    elif c["kind"] == "pack":
        names = ("Kc", "Vc")
    else:
        n = c["n0"] + 1
        out = dict(acc=s["acc"][:, :, :n], born=s["born"][:, :, :n], Kd=s["Kd"][:, :, :, :n], Vd=s["Vd"][:, :, :, :n])
        return {**out, "out": s["out"]} if c["attend"] else out
    return {k: s[k] for k in names}


def run(state):
    if own:
        {"rope": _own_rope, "pack": _own_pack, "step": _own_step}[state["case"]["kind"]](state)
    else:
        {"rope": _plain_rope, "pack": _plain_pack, "step": _plain_step}[state["case"]["kind"]](state)
    return _outputs(state)


# ------------------------------------------------------------------------------------------------ the least work
def work(case):
    c = case
    B, L, Hkv, d = (c[k] for k in ("B", "L", "Hkv", "d"))
    if c["kind"] == "rope":
        rows, H = c["rows"], c["H"]
        window = max(0, min(rows, c["first"] + rows - (c["N"] - c["W"])))
        read = rows * H if c["all_q"] else window * H
        written = window * H + (rows * H if c["all_q"] else 0)
        table = (B if c["given"] else 1) * rows * c["rot"] * 4
        return dict(bytes=2 * d * B * (read + written + 4 * rows * Hkv) + table + (4 * B * rows if c["given"] else 0),
                    flops=B * (read + rows * Hkv) * (3 * c["rot"] + (4 * d if c["norm"] else 0)))
    if c["kind"] == "pack":
        rows = B * L * Hkv * (c["M"] - (c["M"] // 16 if c["ragged"] else 0))
        packed = sum(_tile_bytes(d)) / 32
        return dict(bytes=rows * (4 * d + 2 * packed + 4 * d) + rows // Hkv * 4, flops=rows * 2 * d * 6)
    kept, n = c["M"], c["n0"] + 1
    if c["ragged"]:
        kept = c["M"] // 2 if L < 32 else c["M"] - c["M"] // 16
    kb, vb = (b / 32 for b in _tile_bytes(d))
    U, both = B * L * Hkv, 2 if c["attend"] else 1
    nbytes = U * (kept * (kb + (vb if c["attend"] else 0)) + n * 2 * d * both + 6 * d) + B * L * n * 8
    nbytes += B * L * c["H"] * d * (6 if c["attend"] else 2)
    return dict(bytes=nbytes, flops=2 * B * L * c["H"] * d * (kept + n) * both)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_rope(s):
    c = s["case"]
    B, H, Hkv, d, rows, first, rot = (c[k] for k in ("B", "H", "Hkv", "d", "rows", "first", "rot"))
    i = torch.arange(rot, device="cuda")
    pair = i // 2 if c["interleaved"] else i % (rot // 2)
    mate = (i ^ 1) if c["interleaved"] else (i + rot // 2) % rot
    sign = torch.where(i < mate, -1.0, 1.0).double()
    pos = s["positions"].long() if s["positions"] is not None else first + torch.arange(rows, device="cuda").expand(B, rows)
    cs = s["table"].double()[pos][:, :, None]                        # [B, rows, 1, rot / 2, 2]

    def turn(x, w):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * w.double()
        y = x.clone()
        y[..., :rot] = x[..., :rot] * cs[..., pair, 0] + sign * x[..., mate] * cs[..., pair, 1]
        return y

    out = {n: s[n].double() for n in ("Qwin", "K", "V")}
    q, k = turn(s["q"], s["q_weight"]), turn(s["k"], s["k_weight"])
    out["K"][:, c["layer"], :, first:first + rows] = k.transpose(1, 2)
    out["V"][:, c["layer"], :, first:first + rows] = s["v"].double().transpose(1, 2)
    start = c["N"] - c["W"]
    t0 = max(first, start)
    if t0 < first + rows:
        out["Qwin"][:, c["layer"], :, t0 - start:first + rows - start] = q[:, t0 - first:].transpose(1, 2)
    if c["all_q"]:
        out["q_out"] = q
    return out


def _exact_pack(s):
    """Group by group from the definition: a bf16 number up is the bf16 nearest to it, or the next one."""
    out = {}
    M, d = s["case"]["M"], s["case"]["d"]
    for name, groups in (("K", d // 32), ("V", 1)):
        x = torch.take_along_dim(s[name], s["kept_idx"].long().clamp_min(0)[:, :, None, :, None], 3).double()
        x = x.reshape(*x.shape[:-1], groups, d // groups)
        wide, high = x.amax(-1) - x.amin(-1), x.abs().amax(-1)
        s64 = torch.maximum(wide / 15, high / 240).clamp_min(2.0**-100).float().to(torch.bfloat16)
        # a product of bf16 numbers and 15 or 240 is exact, their quotient is not: no less than, by the products
        short = (s64.double() * 15 < wide) | (s64.double() * 240 < high)
        s64 = torch.where(short, (s64.view(torch.int16) + 1).view(torch.bfloat16), s64).double()[..., None]
        y = (torch.floor(x / s64 + 0.5) * s64).reshape(*x.shape[:-2], d)
        beyond = torch.arange(M, device="cuda")[None, None] >= s["kept_count"][..., None]
        out[name + "c"] = y.masked_fill_(beyond[:, :, None, :, None], 0.0)
    return out


def _exact_rows(tiles, d, keys):
    """Every element's code by its own place: word and nibble of row r, dimension i of a tile."""
    r, i = torch.arange(32, device="cuda")[:, None], torch.arange(d, device="cuda")[None]
    if keys:
        lane, j = 4 * (r % 8) + i // 8 % 4, 2 * (i // 32) + i // 4 % 2
        nibble = (r // 8 % 2) + 2 * (i // 2 % 2) + 4 * (i % 2)
    else:
        lane, j = 4 * (i // 8 % 8) + r // 2 % 4, 4 * (i // 64) + i // 2 % 4
        nibble = (i % 2) + 2 * (r // 8 % 2) + 4 * (r % 2)
    word = ((r // 16 * (d // 64) + j // 4) * 32 + lane) * 4 + j % 4
    w = tiles.contiguous().view(torch.int32).flatten(0, -2)
    code = ((w[:, word.flatten()] >> (4 * nibble).flatten().to(torch.int32)) & 15).reshape(-1, 32, d)
    group = (4 * d + r * (d // 32) + i // 32 if keys else 4 * d + r + 0 * i).flatten()
    meta = w[:, group].reshape(-1, 32, d)
    halves = meta.view(torch.bfloat16).reshape(-1, 32, d, 2)         # the low half comes first
    rows = (code.double() - 8 + halves[..., 0].double()) * halves[..., 1].double()
    return rows.reshape(*tiles.shape[:-2], tiles.shape[-2] * 32, d)


def _exact_step(s):
    """A few sequences at a time: 64-bit keys and values of all of them take much memory."""
    c = s["case"]
    B, L, H, Hkv, d, M, n0 = (c[k] for k in ("B", "L", "H", "Hkv", "d", "M", "n0"))
    out = dict(acc=s["acc"][:, :, :n0 + 1].double(), born=None, Kd=s["Kd"][:, :, :, :n0 + 1].double(), Vd=s["Vd"][:, :, :, :n0 + 1].double())
    out["acc"][:, :, n0] = 0
    out["Kd"][:, :, :, n0], out["Vd"][:, :, :, n0] = s["k"].double(), s["v"].double()
    if c["attend"]:
        out["out"] = torch.empty(B, L, H, d, dtype=torch.float64, device="cuda")
    for b in range(B):
        q = s["q"][b].double().reshape(L, Hkv, H // Hkv, d)
        masked = torch.arange(M, device="cuda")[None] >= s["kept_count"][b][:, None]
        prompt = torch.einsum("lhgd,lhtd->lhgt", q, _exact_rows(s["K4"][b], d, True)[:, :, :M]).masked_fill(masked[:, None, None], -math.inf)
        x = torch.cat([prompt, torch.einsum("lhgd,lhtd->lhgt", q, out["Kd"][b])], -1) * d ** -0.5
        p = torch.softmax(x, -1)
        out["acc"][b] += p[..., M:].sum((1, 2))
        if c["attend"]:
            o = torch.einsum("lhgt,lhtd->lhgd", p[..., :M], _exact_rows(s["V4"][b], d, False)[:, :, :M])
            out["out"][b] = (o + torch.einsum("lhgt,lhtd->lhgd", p[..., M:], out["Vd"][b])).reshape(L, H, d)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "pack": _exact_pack, "step": _exact_step}[case["kind"]](s)
