"""What drafted trees of tokens, windows with sinks, rows at positions of their own and the keeping of accepted rows are
measured at: calls as a decoder makes them, over the range of sizes they are used at, and the same in elementary torch
operations.

A case is one attention layer of a model at one point of its decoding (`keep`: all layers at the end of a step).  The pools
are made here in the layouts that the library documents, so that both forms work on the same bytes:

  bf16   per (block, kv head), in groups of 32 slots; keys: 16-byte units (dims 32s + 8c .. +7 of slot
         16*tile + row) in the order [tile][s][c][row]; values: units (dim 16dt + n of the slots
         4c..4c+3, 16+4c..16+4c+3) in the order [dt][c][n].
  e4m3   first the codes of all (block, kv head) tiles, then the scale bytes of all of them.  Codes:
         keys, 16-byte units (dims 64w + 8c .. +7 and 64w + 32 + 8c .. +7 of slot 16*tile + row) in the
         order [tile][w][c][row]; values, units (dims 32w + n and 32w + 16 + n of the slots above) in
         the order [w][c][n].  Scale bytes of a group: keys, of the slots row, 16 + row for row = 0..15;
         values, of the slots 4c..4c+3, 16+4c..16+4c+3 for c = 0..3.  A byte E is the scale 2^(E-127).
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"

# Attention-layer shapes: (query heads, kv heads, head_dim), as the library's own benchmark has them.
LLAMA = (24, 8, 128)
NARROW = (32, 8, 64)
WIDE_GROUP = (32, 4, 128)
ONE_EACH = (16, 16, 64)
TINY = (8, 2, 64)


def _case(name, kind, shape, **more):
    c = {"kind": kind, "store": "bf16", "q_heads": shape[0], "kv_heads": shape[1], "head_dim": shape[2], "block": 64,
         "batch": 1, "t": 0, "count": 1, "window": 0, "sinks": 0, "ragged": False, "axes": 1, "spread": False, "layers": 1}
    if name:
        c["name"] = name
    c.update(more)
    return c


def listed():
    return [
        # One user, a small draft: 8 drafted tokens behind 300 cached ones.  Latency counts.
        _case("tree_small", "tree", LLAMA, t=300, count=8),
        # A serving batch, every sequence at its own step and with a tree of its own size.
        _case("tree_batch", "tree", LLAMA, batch=16, t=4000, count=32, ragged=True, block=256),
        # One sequence with a very long context, on the 8-bit store.
        _case("tree_long", "tree", LLAMA, store="e4m3", t=65000, count=60, block=256),
        # Large trees under a wide group: as much product as memory.
        _case("tree_wide", "tree", WIDE_GROUP, batch=8, t=6007, count=63),
        # One user in an endless conversation: a step, its row written, on blocks that are used in turn.
        _case("sinks_step", "step", LLAMA, t=20000, window=1000, sinks=4),
        # A batch of endless conversations on 8-bit stores, three steps each, every one at its own place.
        _case("sinks_batch", "block", NARROW, store="e4m3", batch=48, t=100000, count=3, window=4095, sinks=4, ragged=True),
        # Prompts with a window and sinks.
        _case("sinks_prompt", "prompt", LLAMA, batch=4, count=4096, window=1024, sinks=4, block=256),
        # A stretch of a long document behind what is cached, 8 bits.
        _case("sinks_chunk", "prompt", NARROW, store="e4m3", batch=2, t=9001, count=777, window=2000, sinks=33),
        # The rows of a batch of trees: each rotated to its depth's position and written to its own slot.
        _case("place_tree", "place", LLAMA, batch=16, t=4000, count=32, ragged=True),
        # Images and video: rows with a position in time, height and width.
        _case("place_video", "place", WIDE_GROUP, batch=2, t=17, count=5000, axes=3),
        # The accepted path of one user's tree, one layer.
        _case("keep_one", "keep", LLAMA, store="e4m3", t=300, count=8),
        # The accepted paths of a batch, all layers of a model.
        _case("keep_batch", "keep", LLAMA, batch=16, t=1000, count=32, ragged=True, layers=28),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "step", "block", "block", "prompt", "prompt", "place", "place", "keep"])
    shape = rng.choice([LLAMA, LLAMA, NARROW, WIDE_GROUP, ONE_EACH, TINY])
    row = shape[1] * shape[2]                       # elements of one step's keys
    block = rng.choice([32, 64, 256])
    store = rng.choice(["bf16", "bf16", "e4m3"])
    ragged = rng.random() < 0.4
    if kind == "keep":
        layers = rng.choice([1, _log(rng, 1, 32)])
        batch = _log(rng, 1, 16)
        return _case("", kind, shape, store=store, block=block, batch=batch, layers=layers, ragged=ragged, count=_log(rng, 2, 64),
                     t=_log(rng, 1, max(2, min(2000, 500000000 // (row * batch * layers)))))
    if kind == "place":
        axes = rng.choice([1, 1, 2, 3])
        batch = _log(rng, 1, 32)
        count = _log(rng, 1, max(2, min(8000, 16000000 // (row * batch))))
        return _case("", kind, shape, store=store, block=block, batch=batch, t=rng.randrange(0, 3000), count=count, axes=axes,
                     spread=rng.random() < 0.4, ragged=ragged and store == "bf16" and count < 300)
    if kind == "prompt":
        batch = _log(rng, 1, 8)
        count = _log(rng, 20, max(21, min(6000, 16000 // batch)))
        return _case("", kind, shape, store=store, block=block, batch=batch, t=rng.choice([0, 0, _log(rng, 1, 5000)]), count=count,
                     window=_log(rng, 32, 2048), sinks=rng.choice([1, 4, _log(rng, 1, 200)]))
    batch = _log(rng, 1, 64)
    if kind in ("step", "block"):
        count = 1 if kind == "step" else rng.choice([1, _log(rng, 1, 24)])
        return _case("", kind, shape, store=store, block=block, batch=batch, t=_log(rng, 1, 200000), count=count, ragged=ragged,
                     window=_log(rng, 32, max(33, min(8192, 40000000 // (row * batch)))), sinks=rng.choice([1, 4, _log(rng, 1, 200)]))
    count = _log(rng, 1, 128)
    batch = min(batch, max(1, 1024 // count))
    most = min(67000000 // (row * batch), 12000000000 // (shape[0] * shape[2] * batch * count))
    window = rng.choice([0, 0, _log(rng, 64, 4096)])
    return _case("", kind, shape, store=store, block=block, batch=batch, t=_log(rng, 20, min(65536, most)), count=count,
                 ragged=ragged, window=window, sinks=rng.choice([0, 4, 40]) if window else 0)


# ---- layouts ------------------------------------------------------------------------------------


def _to_tiles_bf16(keys, x):
    """x [..., Z, D] to the element order of a tile, [..., Z * D]."""
    lead, (Z, D) = x.shape[:-2], x.shape[-2:]
    n = len(lead)
    if keys:  # [grp][tile][row][s][c][e] -> [grp][tile][s][c][row][e]
        y = x.reshape(*lead, Z // 32, 2, 16, D // 32, 4, 8).permute(*range(n), n, n + 1, n + 3, n + 4, n + 2, n + 5)
    else:     # [grp][half][c][r][dt][n] -> [grp][dt][c][n][half][r]
        y = x.reshape(*lead, Z // 32, 2, 4, 4, D // 16, 16).permute(*range(n), n, n + 4, n + 2, n + 5, n + 1, n + 3)
    return y.reshape(*lead, Z * D)


def _from_tiles_bf16(keys, x, D):
    lead, Z = x.shape[:-1], x.shape[-1] // D
    n = len(lead)
    if keys:
        y = x.reshape(*lead, Z // 32, 2, D // 32, 4, 16, 8).permute(*range(n), n, n + 1, n + 4, n + 2, n + 3, n + 5)
    else:
        y = x.reshape(*lead, Z // 32, D // 16, 4, 16, 2, 4).permute(*range(n), n, n + 4, n + 2, n + 5, n + 1, n + 3)
    return y.reshape(*lead, Z, D)


def _to_tiles_e4m3(keys, x):
    lead, (Z, D) = x.shape[:-2], x.shape[-2:]
    n = len(lead)
    if keys:  # [grp][tile][row][w][h][c][e] -> [grp][tile][w][c][row][h][e]
        y = x.reshape(*lead, Z // 32, 2, 16, D // 64, 2, 4, 8).permute(*range(n), n, n + 1, n + 3, n + 5, n + 2, n + 4, n + 6)
    else:     # [grp][half][c][r][w][h][n] -> [grp][w][c][n][h][half][r]
        y = x.reshape(*lead, Z // 32, 2, 4, 4, D // 32, 2, 16).permute(*range(n), n, n + 4, n + 2, n + 6, n + 5, n + 1, n + 3)
    return y.reshape(*lead, Z * D)


def _from_tiles_e4m3(keys, x, D):
    lead, Z = x.shape[:-1], x.shape[-1] // D
    n = len(lead)
    if keys:
        y = x.reshape(*lead, Z // 32, 2, D // 64, 4, 16, 2, 8).permute(*range(n), n, n + 1, n + 4, n + 2, n + 5, n + 3, n + 6)
    else:
        y = x.reshape(*lead, Z // 32, D // 32, 4, 16, 2, 2, 4).permute(*range(n), n, n + 5, n + 2, n + 6, n + 1, n + 4, n + 3)
    return y.reshape(*lead, Z, D)


def _to_scales(keys, x):
    """x [..., Z] to the order of a tile's scale bytes."""
    lead, Z = x.shape[:-1], x.shape[-1]
    n = len(lead)
    if keys:
        return x.reshape(*lead, Z // 32, 2, 16).transpose(-1, -2).reshape(*lead, Z)
    return x.reshape(*lead, Z // 32, 2, 4, 4).permute(*range(n), n, n + 2, n + 1, n + 3).reshape(*lead, Z)


def _from_scales(keys, x):
    lead, Z = x.shape[:-1], x.shape[-1]
    n = len(lead)
    if keys:
        return x.reshape(*lead, Z // 32, 16, 2).transpose(-1, -2).reshape(*lead, Z)
    return x.reshape(*lead, Z // 32, 4, 2, 4).permute(*range(n), n, n + 2, n + 1, n + 3).reshape(*lead, Z)


def _power(e):
    """2^e in 32 bits, e whole, -126 to 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(x):
    """Rows x [..., D]: (codes, scale bytes), both uint8."""
    x = x.float()
    m, e = torch.frexp(x.abs().amax(-1))                      # top = m 2^e, m in [0.5, 1): at most 448 2^(e-9) if m <= 0.875
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-111)
    return (x * _power(-e)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _values(codes, scales):
    """What codes [..., D] with scale bytes [...] stand for, in 32 bits."""
    return codes.view(torch.float8_e4m3fn).float() * _power(scales.to(torch.int32) - 127)[..., None]


# ---- inputs -------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _normal(shape, g):
    return torch.empty(shape, dtype=torch.bfloat16, device=DEVICE).normal_(0.0, 1.0, generator=g)


def _keys(shape, g):
    """Keys have a few channels larger than the others."""
    x = _normal(shape, g)
    x[..., 5::40] *= 4
    return x


def _per_sequence(c, most, salt):
    """Whole numbers up to `most` for the sequences: the same set for every seed, so that every seed is the same work."""
    if not c["ragged"]:
        return [most] * c["batch"]
    r = random.Random(c["batch"] * 65536 + most + salt)
    return [r.randrange(1, most + 1) for _ in range(c["batch"])]


def _shuffled(values, g):
    x = torch.tensor(values, dtype=torch.int32, device=DEVICE)
    return x[torch.randperm(len(values), generator=g, device=DEVICE)].contiguous()


def _trees(c, g):
    """parents [B][N]: of node i one of -1 .. i-1 (-1: the last cached token), nodes near the root preferred."""
    i = torch.arange(c["count"], device=DEVICE)
    u = torch.rand((c["batch"], c["count"]), generator=g, device=DEVICE)
    return (torch.floor(u * (0.7 * i + 1)) - 1).clamp(min=-1).minimum((i - 1).float()).to(torch.int32)


def _columns(c):
    return (c["t"] + c["count"] - 1) // c["block"] + 1


def _table(c, g):
    """(block table, number of blocks).  Steps and blocks of steps with a window use the blocks behind the sinks' in turn."""
    B, Z, columns = c["batch"], c["block"], _columns(c)
    first = -(-c["sinks"] // Z)
    turn = (c["window"] + c["count"] - 1) // Z + 2                     # blocks that the keys of one call can touch, and one more
    own_blocks = columns
    n = torch.arange(columns, device=DEVICE)
    if c["window"] and c["kind"] in ("step", "block") and first + turn < columns:
        own_blocks = first + turn
        n = torch.where(n < first, n, first + (n - first) % turn)
    blocks = torch.randperm(B * own_blocks, generator=g, device=DEVICE).to(torch.int32).reshape(B, own_blocks)
    return blocks[:, n].contiguous(), B * own_blocks


def _axes(c):
    """The axis of each of the D/2 rotated pairs: the axes' pairs in a row, or in turn."""
    half, n = c["head_dim"] // 2, c["axes"]
    if c["spread"]:
        return [i % n for i in range(half)]
    cuts = {1: [half], 2: [half // 2, half // 2], 3: [half // 4, 3 * half // 8, half - half // 4 - 3 * half // 8]}[n]
    return [a for a, k in enumerate(cuts) for _ in range(k)]


POSITIONS = 16384


def prepare(case, seed):
    c = case
    g = _generator(seed)
    B, Hq, Hkv, D, Z, C, L = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["block"], c["count"], c["layers"]
    s = {"case": c, "axis_of_pair": _axes(c)}
    s["table"], s["blocks"] = _table(c, g)
    s["steps"] = _shuffled(_per_sequence(c, c["t"], 0), g) if c["ragged"] else None
    for name, keys in (("k_pool", True), ("v_pool", False)):
        x = (_keys if keys else _normal)((L, s["blocks"], Hkv, Z, D), g)
        if c["store"] == "bf16":
            s[name] = _to_tiles_bf16(keys, x).contiguous()
        else:
            codes, scales = _quantise(x)
            s[name] = torch.cat([_to_tiles_e4m3(keys, codes).reshape(L, -1), _to_scales(keys, scales).reshape(L, -1)], dim=1)
    if c["kind"] in ("step", "prompt", "place"):
        s["k"], s["v"] = _keys((B, C, Hkv, D), g), _normal((B, C, Hkv, D), g)
    if c["kind"] != "keep":
        s["q"] = _normal((B, C, Hq, D), g)
    if c["kind"] == "tree":
        s["parents"] = _trees(c, g)
        s["nodes"] = _shuffled(_per_sequence(c, C, 1), g) if c["ragged"] else None
    if c["kind"] == "place":
        angle = torch.arange(POSITIONS, dtype=torch.float64, device=DEVICE)[:, None] * \
            10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device=DEVICE) * 2 / D)
        s["cos"], s["sin"] = torch.cos(angle).float().contiguous(), torch.sin(angle).float().contiguous()
        base = torch.randint(0, 4000, (B, 1), generator=g, device=DEVICE)
        i = torch.arange(C, device=DEVICE)
        if c["axes"] == 1:  # a tree's rows: its depths
            p = (base + torch.floor(torch.log2(i + 1.0)).long())[..., None]
        else:               # frames of 24 by 30 patches
            p = base[..., None] + torch.stack([i // 720, i % 720 // 30, i % 30], dim=-1)[:, :c["axes"]]
        s["positions"] = p.to(torch.int32).contiguous()
    if c["kind"] == "keep":  # an ascending path through the nodes, -1 behind its last one
        kept = torch.rand((B, C), generator=g, device=DEVICE) < 5.0 / C
        order = torch.where(kept, torch.arange(C, device=DEVICE), C).sort(dim=-1)[0][:, :min(C, 16)]
        s["path"] = torch.where(order == C, -1, order).to(torch.int32).contiguous()
    return s


# ---- one pass: the library's calls ----------------------------------------------------------------

def _kept(state):
    """What a program keeps between calls: the stores' descriptors, the workspace, buffers for answers."""
    from paper_2501_05408_amd import tempo as T

    c = state["case"]
    B, Hq, Hkv, D, C = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["count"]
    dtype = T.TEMPO_E4M3 if c["store"] == "e4m3" else T.TEMPO_BF16
    table = state["table"]
    kvs = [T.make_kv(state["k_pool"][i], state["v_pool"][i], table, state["blocks"], table.shape[1], c["block"], Hkv, D, dtype)
           for i in range(c["layers"])]
    need = {"tree": lambda: T.tempo_attn_tree_workspace_bytes(kvs[0], B, Hq, C, c["t"], c["window"], c["sinks"]),
            "step": lambda: T.tempo_attn_sinks_workspace_bytes(kvs[0], B, Hq, 1, c["t"], c["window"], c["sinks"]),
            "block": lambda: T.tempo_attn_sinks_workspace_bytes(kvs[0], B, Hq, C, c["t"], c["window"], c["sinks"]),
            "prompt": lambda: T.tempo_prefill_sinks_workspace_bytes(kvs[0], B, Hq, c["t"] + C - 1)}
    nbytes = need[c["kind"]]() if c["kind"] in need else 0
    new = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device=DEVICE)  # noqa: E731
    return {"T": T, "kv": kvs[0], "kvs": T.make_kv_layers(kvs), "bytes": nbytes,
            "workspace": torch.empty(max(nbytes, 1), dtype=torch.uint8, device=DEVICE),
            "out": torch.zeros_like(state["q"]) if "q" in state else None, "k_back": new(B, C, Hkv, D), "v_back": new(B, C, Hkv, D),
            "rope": T.make_rope(state["cos"], state["sin"], D) if "cos" in state else None,
            "axes": T.make_rope_axes(state["axis_of_pair"]) if c["axes"] > 1 else None}


def _own(state):
    if "kept" not in state:
        state["kept"] = _kept(state)
    h, c = state["kept"], state["case"]
    T, kv, out, ws, nb, steps = h["T"], h["kv"], h["out"], h["workspace"], h["bytes"], state["steps"]
    B, Hq, C, t, window, sinks = c["batch"], c["q_heads"], c["count"], c["t"], c["window"], c["sinks"]
    scale = 1.0 / math.sqrt(c["head_dim"])
    kind = c["kind"]
    if kind == "tree":
        T.tempo_attn_tree(kv, state["q"], out, state["parents"], state["nodes"], B, Hq, C, t, steps, window, sinks, scale, ws, nb)
        return [out]
    if kind == "block":
        T.tempo_attn_sinks(kv, state["q"], out, B, Hq, C, t, steps, window, sinks, scale, ws, nb)
        return [out]
    if kind == "step":
        T.tempo_decode_step_sinks(kv, state["q"], state["k"], state["v"], out, B, Hq, t, steps, window, sinks, scale, ws, nb)
        return [out] + _stored(state)
    if kind == "prompt":
        T.tempo_prefill_sinks(kv, state["q"], state["k"], state["v"], out, B, Hq, t, C, None, window, sinks, scale, ws, nb)
        return [out] + _stored(state)
    if kind == "place":
        T.tempo_rope_kv_append_at(kv, h["rope"], h["axes"], state["positions"], state["k"], state["v"], state["q"], out, B, Hq, t, steps,
                                  C, None)
        if c["store"] == "bf16":
            return [out] + _stored(state)
        T.tempo_kv_gather(kv, h["k_back"], h["v_back"], B, t, C)
        return [out, h["k_back"], h["v_back"]]
    T.tempo_kv_keep(h["kvs"], c["layers"], B, t, steps, C, state["path"], state["path"].shape[1])
    return _stored(state)


# ---- one pass: the plain form -----------------------------------------------------------------------

def _code_bytes(state):
    c = state["case"]
    return state["blocks"] * c["kv_heads"] * c["block"] * c["head_dim"]


def _stored(state):
    """The pools; of an 8-bit store the codes as numbers, and the scale bytes."""
    pools = [state["k_pool"], state["v_pool"]]
    if state["case"]["store"] == "bf16":
        return pools
    n = _code_bytes(state)
    return [y for x in pools for y in (x[:, :n].view(torch.float8_e4m3fn), x[:, n:])]


def _rows(state, keys, tiles):
    """Rows of the physical blocks tiles [B][n] of the first layer, in 32 bits: [B][n][Hkv][Z][D]."""
    c = state["case"]
    pool, D = state["k_pool" if keys else "v_pool"][0], c["head_dim"]
    if c["store"] == "bf16":
        return _from_tiles_bf16(keys, pool[tiles], D).float()
    n = _code_bytes(state)
    codes, scales = (x.reshape(state["blocks"], c["kv_heads"], -1) for x in (pool[:n], pool[n:]))
    return _values(_from_tiles_e4m3(keys, codes[tiles], D), _from_scales(keys, scales[tiles]))


def _first_steps(state):
    c = state["case"]
    return state["steps"].long() if state["steps"] is not None else torch.full((c["batch"],), c["t"], dtype=torch.int64, device=DEVICE)


def _places(state, keys):
    """(offset of (slot, d) inside a tile [Z][D], place of a slot's scale byte [Z])."""
    c = state["case"]
    Z, D = c["block"], c["head_dim"]
    order = torch.arange(Z * D, device=DEVICE).reshape(Z, D)
    place, spot = torch.empty_like(order), torch.empty(Z, dtype=torch.int64, device=DEVICE)
    place.view(-1)[(_to_tiles_bf16 if c["store"] == "bf16" else _to_tiles_e4m3)(keys, order)] = torch.arange(Z * D, device=DEVICE)
    spot[_to_scales(keys, torch.arange(Z, device=DEVICE))] = torch.arange(Z, device=DEVICE)
    return place, spot


def _slots(state, at):
    """Steps at [B][n]: (tile number [B][n][Hkv] among the store's, slot [B][n][Hkv])."""
    c = state["case"]
    Hkv, Z = c["kv_heads"], c["block"]
    phys = torch.gather(state["table"].long(), 1, at // Z)[..., None]
    tile = phys * Hkv + torch.arange(Hkv, device=DEVICE)
    return tile, (at % Z)[..., None].expand_as(tile)


def _steps_of_rows(state):
    return _first_steps(state)[:, None] + torch.arange(state["case"]["count"], device=DEVICE)


def _write(state, k, v):
    """Rows k, v [B][C][Hkv][D] into the first layer's pools."""
    c = state["case"]
    Z, D = c["block"], c["head_dim"]
    tile, slot = _slots(state, _steps_of_rows(state))
    for x, pool, keys in ((k, state["k_pool"][0], True), (v, state["v_pool"][0], False)):
        place, spot = _places(state, keys)
        to = (tile * (Z * D))[..., None] + place[slot]
        if c["store"] == "bf16":
            pool.view(-1)[to] = x
        else:
            codes, scales = _quantise(x)
            pool[to] = codes
            pool[_code_bytes(state) + tile * Z + spot[slot]] = scales


def _read(state):
    """The rows of the call's steps as bf16, [B][C][Hkv][D] of keys and of values."""
    c = state["case"]
    Z, D = c["block"], c["head_dim"]
    tile, slot = _slots(state, _steps_of_rows(state))
    got = []
    for keys, pool in ((True, state["k_pool"][0]), (False, state["v_pool"][0])):
        place, spot = _places(state, keys)
        got.append(_values(pool[(tile * (Z * D))[..., None] + place[slot]], pool[_code_bytes(state) + tile * Z + spot[slot]]).to(torch.bfloat16))
    return got


def _softmax_product(q, k, v, seen, scale):
    """q [B][Hkv][M][D], k, v [B][Hkv][N][D], seen [B][1][M][N], in 32 bits."""
    x = torch.matmul(q, k.transpose(-1, -2).contiguous()) * scale
    x = x.masked_fill(~seen, float("-inf"))
    w = torch.exp(x - x.amax(-1, keepdim=True))
    return torch.matmul(w, v) / w.sum(-1, keepdim=True)


def _ancestors(state):
    """[B][N][N]: node i is below node j, or is it."""
    p = state["parents"].long()
    N = p.shape[1]
    step = torch.eye(N, dtype=torch.float64, device=DEVICE) + (p[..., None] == torch.arange(N, device=DEVICE)).double()
    return torch.matrix_power(step, max(1, N - 1)) > 0.5


def _attend(state):
    c = state["case"]
    B, Hq, Hkv, D, Z, C, window, sinks = (c[x] for x in ("batch", "q_heads", "kv_heads", "head_dim", "block", "count", "window", "sinks"))
    G, columns = Hq // Hkv, state["table"].shape[1]
    t0 = _first_steps(state)
    # the tiles that some row sees: the sinks' and, per sequence, those from the first row's window on
    first = -(-sinks // Z) if window else 0
    lo = ((t0 - window + 1).clamp(min=0) // Z if window else torch.zeros_like(t0))[:, None]
    wide = min(columns, (window + C - 2) // Z + 2) if window else columns
    tiles = lo + torch.arange(wide, device=DEVICE)
    there = (tiles >= first) & (tiles <= (t0[:, None] + C - 1) // Z)
    tiles = torch.cat([torch.arange(first, device=DEVICE).expand(B, first), tiles], dim=1)
    there = torch.cat([(torch.arange(first, device=DEVICE) <= (t0[:, None] + C - 1) // Z), there], dim=1)
    phys = torch.gather(state["table"].long(), 1, tiles.clamp(max=columns - 1))
    k, v = (_rows(state, keys, phys).transpose(1, 2).reshape(B, Hkv, -1, D) for keys in (True, False))
    j = (tiles[..., None] * Z + torch.arange(Z, device=DEVICE)).reshape(B, 1, -1)
    there = there[..., None].expand(B, tiles.shape[1], Z).reshape(B, 1, -1)
    if c["kind"] == "tree":
        up = _ancestors(state)
        step = t0[:, None] + up.sum(-1) - 1                                                  # [B][C]: positions
        node = (j - t0[:, None, None]).clamp(0, C - 1)
        at = torch.gather(step, 1, node[:, 0])[:, None]                                      # a node's position, where j is one
        in_tree = torch.gather(up, 2, node.expand(B, C, j.shape[2]))
        cached = j < t0[:, None, None]
        seen = cached | (in_tree & (j < (t0 + C)[:, None, None]))
        at = torch.where(cached, j, at)
    else:
        step = _steps_of_rows(state)
        seen, at = j <= step[..., None], j
    if window:
        seen = seen & ((at > step[..., None] - window) | (at < sinks))
    seen = (seen & there)[:, None, :, None, :].expand(B, 1, C, G, -1).reshape(B, 1, C * G, -1)
    v = torch.where(seen.any(2)[..., None], v, torch.zeros_like(v))
    q = state["q"].float().reshape(B, C, Hkv, G, D).transpose(1, 2).reshape(B, Hkv, C * G, D)
    out = _softmax_product(q, k, v, seen, 1.0 / math.sqrt(D))
    out = out.reshape(B, Hkv, C, G, D).transpose(1, 2).reshape(B, C, Hq, D).to(torch.bfloat16)
    if state.get("nodes") is not None:  # rows behind a sequence's last node stay as they were: 0
        out = torch.where((torch.arange(C, device=DEVICE) < state["nodes"][:, None])[..., None, None], out, torch.zeros_like(out))
    return out


def _rotated(state, x):
    """Rows x [B][C][heads][D], each pair turned to its axis' position."""
    c = state["case"]
    D, axis = c["head_dim"], torch.tensor(state["axis_of_pair"], device=DEVICE)
    at, i = state["positions"].long()[..., axis], torch.arange(D // 2, device=DEVICE)        # [B][C][D/2]
    cos, sin = (state[n][at, i][:, :, None] for n in ("cos", "sin"))
    lo, hi = x.float()[..., :D // 2], x.float()[..., D // 2:]
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1).to(torch.bfloat16)


def _keep(state):
    c = state["case"]
    Z, D, L = c["block"], c["head_dim"], c["layers"]
    path = state["path"].long()
    i = torch.arange(path.shape[1], device=DEVICE)
    t0 = _first_steps(state)[:, None]
    (a, a_slot), (b, b_slot) = (_slots(state, t0 + x) for x in (torch.where(path >= 0, path, i), i.expand_as(path)))
    for pool, keys in ((state["k_pool"], True), (state["v_pool"], False)):
        place, spot = _places(state, keys)
        at, to = ((tile * (Z * D))[..., None] + place[slot] for tile, slot in ((a, a_slot), (b, b_slot)))
        flat = pool.view(L, -1)
        flat[:, to] = flat[:, at]
        if c["store"] != "bf16":
            n = _code_bytes(state)
            flat[:, n + b * Z + spot[b_slot]] = flat[:, n + a * Z + spot[a_slot]]


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "keep":
        _keep(state)
        return _stored(state)
    if kind == "place":
        q = _rotated(state, state["q"])
        _write(state, _rotated(state, state["k"]), state["v"])
        return [q] + (_stored(state) if state["case"]["store"] == "bf16" else _read(state))
    if kind in ("step", "prompt"):
        _write(state, state["k"], state["v"])
        return [_attend(state)] + _stored(state)
    return [_attend(state)]


# ---- what a pass cannot do without -------------------------------------------------------------------

def work(case):
    c = case
    B, Hq, Hkv, D, C, window, sinks, L = (c[x] for x in ("batch", "q_heads", "kv_heads", "head_dim", "count", "window", "sinks", "layers"))
    row = Hkv * (D + 1 if c["store"] == "e4m3" else 2 * D)          # bytes of one step's keys, or values, in the store
    new = Hkv * 2 * D                                               # ... as the caller's bf16 rows
    kind, steps = c["kind"], _per_sequence(c, c["t"], 0)
    if kind == "keep":
        rows = B * min(C, 5)                                        # about 5 are accepted, the first often where it belongs
        return {"bytes": rows * L * 4 * row, "flops": rows * L}
    if kind == "place":
        back = 2 * B * C * (row + new) if c["store"] == "e4m3" else 0
        return {"bytes": B * C * (4 * Hq * D + 2 * (new + row)) + back, "flops": 3 * B * C * (Hq + Hkv) * D}
    counts = _per_sequence(c, C, 1) if kind == "tree" else [C] * B
    answers = sum(counts) * Hq * D * 4                              # q in, out out
    keys = pairs = 0
    for t, n in zip(steps, counts):
        if kind == "tree":  # a node sees itself; how many of its ancestors there are is the draft's
            seen = min(t, window - 1 + min(sinks, max(0, t - window + 1))) if window else t
            keys += seen + n
            pairs += n * (seen + 1)
        elif n == 1 or not window:
            keys += min(t + 1, window + sinks) if window else t + n
            pairs += min(t + 1, window + sinks) if window else t + 1
        else:
            keys += min(t + n, window + n - 1 + sinks)
            pairs += sum(min(t + i + 1, window + sinks) for i in range(n))
    extra = 2 * B * C * (new + row) if kind in ("step", "prompt") else 0
    return {"bytes": 2 * keys * row + answers + extra, "flops": 4 * pairs * Hq * D}


# ---- the same in 64 bits, from the definitions ---------------------------------------------------------

def _exact_power(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_rows(x):
    """What the 8-bit store holds for rows x [..., D]: (codes' values, e) with the least e >= -111 that keeps the row within
    448 2^e; 3 bits after the leading one, steps of 2^-9 below 2^-6, ties to even."""
    x = x.double()
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True) / 448.0)
    e = torch.where(m == 0.5, e - 1, e).clamp(min=-111)
    y = x / _exact_power(e)
    step = _exact_power(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(y / step) * step, e[..., 0]


def _exact_index(c, keys):
    """(slot, dim) of every element of a 32-slot group, by the documented order; and of every scale byte its slot."""
    D = c["head_dim"]
    i = torch.arange(32 * D, device=DEVICE)
    b = torch.arange(32, device=DEVICE)
    spot = 16 * (b % 2) + b // 2 if keys else 16 * (b // 4 % 2) + 4 * (b // 8) + b % 4
    if c["store"] == "bf16":
        unit, e = i // 8, i % 8
        if keys:
            row, cc, s, tile = unit % 16, unit // 16 % 4, unit // 64 % (D // 32), unit // 64 // (D // 32)
            return 16 * tile + row, 32 * s + 8 * cc + e, spot
        n, cc, dt = unit % 16, unit // 16 % 4, unit // 64
        return 16 * (e // 4) + 4 * cc + e % 4, 16 * dt + n, spot
    unit, byte = i // 16, i % 16
    if keys:
        row, cc, w, tile = unit % 16, unit // 16 % 4, unit // 64 % (D // 64), unit // 64 // (D // 64)
        return 16 * tile + row, 64 * w + 32 * (byte // 8) + 8 * cc + byte % 8, spot
    n, cc, w = unit % 16, unit // 16 % 4, unit // 64
    return 16 * (byte // 4 % 2) + 4 * cc + byte % 4, 32 * w + 16 * (byte // 8) + n, spot


def _unpacked(s, keys):
    """All rows of a store: (what an element's bits stand for [L][blocks][Hkv][Z][D] in 64 bits, e [L][blocks][Hkv][Z])."""
    c = s["case"]
    L, Hkv, Z, D = c["layers"], c["kv_heads"], c["block"], c["head_dim"]
    slot, dim, spot = _exact_index(c, keys)
    x = s["k_pool" if keys else "v_pool"]
    out = torch.empty((L, s["blocks"], Hkv, Z // 32, 32, D), dtype=torch.float64, device=DEVICE)
    e = torch.zeros((L, s["blocks"], Hkv, Z // 32, 32), dtype=torch.int64, device=DEVICE)
    if c["store"] == "bf16":
        out[..., slot, dim] = x.reshape(L, s["blocks"], Hkv, Z // 32, 32 * D).double()
    else:
        n = _code_bytes(s)
        b = x[:, :n].reshape(L, s["blocks"], Hkv, Z // 32, 32 * D).to(torch.int64)
        power, frac = b >> 3 & 15, b & 7
        value = torch.where(power == 0, frac * 2.0 ** -9, (8 + frac).double() * _exact_power(power - 10))
        out[..., slot, dim] = torch.where(b > 127, -value, value)
        e[..., spot] = x[:, n:].reshape(L, s["blocks"], Hkv, Z // 32, 32).long() - 127
    return out.reshape(L, s["blocks"], Hkv, Z, D), e.reshape(L, s["blocks"], Hkv, Z)


def _packed(s, keys, x):
    """Rows as _unpacked() gives them, back in the order of the pool's elements and its shape in _stored()."""
    c = s["case"]
    L, Hkv, Z, D = c["layers"], c["kv_heads"], c["block"], c["head_dim"]
    slot, dim, _ = _exact_index(c, keys)
    y = x.reshape(L, s["blocks"], Hkv, Z // 32, 32, D)[..., slot, dim]
    return y.reshape(L, s["blocks"], Hkv, Z * D) if c["store"] == "bf16" else y.reshape(L, -1)


def _exact_stored(s, rows):
    """What _stored() is of rows [keys', values'] (scale bytes, whole numbers, are left out)."""
    got = [_packed(s, keys, rows[i]) for i, keys in enumerate((True, False))]
    return got if s["case"]["store"] == "bf16" else [got[0], None, got[1], None]


def _exact_seen(c, t, n, parents):
    """For each of the n rows of a sequence the steps that it sees."""
    window, sinks = c["window"], c["sinks"]
    got = []
    for i in range(n):
        if c["kind"] == "tree":
            path, a = [], i
            while a >= 0:
                path.append(a)
                a = parents[a]
            path.reverse()
            here = t + len(path) - 1
            own_steps = [t + a for d, a in enumerate(path) if not window or len(path) - 1 - d < window or t + d < sinks]
        else:
            here, own_steps = t + i, []
        past = t if c["kind"] == "tree" else here + 1                # steps below are seen by their number
        lo = max(0, here - window + 1) if window else 0
        steps = list(range(min(sinks, lo, past))) + list(range(min(lo, past), past)) + own_steps
        got.append(torch.tensor(steps, device=DEVICE))
    return got


def _exact_attend(s, rows):
    """rows: [(keys, values)] of every (sequence, kv head) by step, from a function of (b, h, steps)."""
    c = s["case"]
    B, Hq, Hkv, D, C = c["batch"], c["q_heads"], c["kv_heads"], c["head_dim"], c["count"]
    G, steps = Hq // Hkv, s["steps"].tolist() if s["steps"] is not None else [c["t"]] * B
    nodes = s["nodes"].tolist() if s.get("nodes") is not None else [C] * B
    out = torch.zeros((B, C, Hq, D), dtype=torch.float64, device=DEVICE)
    for b in range(B):
        parents = s["parents"][b].tolist() if "parents" in s else None
        seen = _exact_seen(c, steps[b], nodes[b], parents)
        some = torch.unique(torch.cat(seen))                         # sorted
        mask = torch.zeros((nodes[b], some.numel()), dtype=torch.bool, device=DEVICE)
        for i, x in enumerate(seen):
            mask[i, torch.searchsorted(some, x)] = True
        for h in range(Hkv):
            k, v = (rows(x, b, h, some) for x in (0, 1))
            q = s["q"][b, :nodes[b], h * G:(h + 1) * G].double()     # [n][G][D]
            x = (q.reshape(-1, D) @ k.t()).reshape(nodes[b], G, -1) / math.sqrt(D)
            x = torch.where(mask[:, None], x, torch.full_like(x, -math.inf))
            w = torch.exp(x - x.max(dim=-1, keepdim=True)[0])
            y = (w / w.sum(dim=-1, keepdim=True)).reshape(-1, some.numel()) @ v
            out[b, :nodes[b], h * G:(h + 1) * G] = y.reshape(nodes[b], G, D)
    return out


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    B, Z, C, D, kind = c["batch"], c["block"], c["count"], c["head_dim"], c["kind"]
    steps = s["steps"].tolist() if s["steps"] is not None else [c["t"]] * B
    table = s["table"].tolist()
    if kind == "keep":
        got = [_unpacked(s, keys)[0] for keys in (True, False)]
        for x in got:
            for b in range(B):
                path = [p for p in s["path"][b].tolist() if p >= 0]
                old = [x[:, table[b][(steps[b] + p) // Z], :, (steps[b] + p) % Z].clone() for p in path]
                for i, r in enumerate(old):
                    x[:, table[b][(steps[b] + i) // Z], :, (steps[b] + i) % Z] = r
        return _exact_stored(s, got)
    at = torch.tensor(steps, device=DEVICE)[:, None] + torch.arange(C, device=DEVICE)
    phys = s["table"].long()[torch.arange(B, device=DEVICE)[:, None], at // Z]               # [B][C]
    if kind == "place":
        axis = torch.tensor(s["axis_of_pair"], device=DEVICE)
        spot = s["positions"].long()[:, :, axis]
        pair = torch.arange(D // 2, device=DEVICE)
        turn = torch.complex(s["cos"][spot, pair].double(), s["sin"][spot, pair].double())[:, :, None]
        q, k = (torch.complex(x.double()[..., :D // 2], x.double()[..., D // 2:]) * turn for x in (s["q"], s["k"]))
        q, k = (torch.cat([x.real, x.imag], dim=-1) for x in (q, k))
        if c["store"] == "bf16":
            got = [_unpacked(s, keys)[0] for keys in (True, False)]
            got[0][0, phys, :, at % Z], got[1][0, phys, :, at % Z] = k, s["v"].double()
            return [q] + _exact_stored(s, got)
        code, e = _exact_rows(s["v"])  # the rotated keys are rounded to bf16 and then to their codes
        return [q, None, code * _exact_power(e)[..., None]]
    if kind == "tree" or kind == "block":
        rows = [_unpacked(s, keys) for keys in (True, False)]
    else:
        rows = [_unpacked(s, keys) for keys in (True, False)]
        for i, x in enumerate((s["k"], s["v"])):
            code, e = _exact_rows(x) if c["store"] == "e4m3" else (x.double(), torch.zeros(x.shape[:-1], dtype=torch.int64, device=DEVICE))
            rows[i][0][0, phys, :, at % Z], rows[i][1][0, phys, :, at % Z] = code, e.long()

    def of(i, b, h, which):
        tile, slot = s["table"][b].long()[which // Z], which % Z
        return rows[i][0][0, tile, h, slot] * _exact_power(rows[i][1][0, tile, h, slot])[:, None]

    out = _exact_attend(s, of)
    return [out] if kind in ("tree", "block") else [out] + _exact_stored(s, [x[0] for x in rows])
