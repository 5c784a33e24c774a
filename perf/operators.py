"""A key/value cache held in 4 or 8 bits, as measurable cases: written (`kv_append`), read back (`kv_read`), attended over (`kv_attn`).

A program that serves a decoder model keeps the keys and values of its live sequences in a pool of pages.  A prompt's tokens, or the one
token that each live sequence decodes, are rotated and quantized into the pages, and their queries attend over everything that the pages hold of their own
sequence.  Now and then a sequence is read back (to hand it to code that wants 16 bits, or to move it elsewhere).

Formats are the blocks of the weights: levels of 4 or 8 bits, a scale and an offset in 16 bits for every 32 or 64 components of a head.  A page holds
`page` positions of all key/value heads, head after head, in tiles of 32 positions.  A tile is [key codes][value codes][key headers][value headers]:

  codes    as 16-byte pieces [n][g: 4][i: 16]; the pieces n = 0, 1, .. of one (g, i) are one run of bits, little-endian.  Keys: for h = 0, 1 the components
           g D/4 .. (g + 1) D/4 - 1 of position 16 h + i.  Values: for c = 0 .. D/16 - 1 component 16 c + i of the positions 4 g, .. 4 g + 3, 16 + 4 g, .. 16 + 4 g + 3.
           8 bits: a byte each.  4 bits: eight in a 32-bit word, v0 v2 v4 v6 v1 v3 v5 v7 from the lowest nibble.
  headers  keys: [block][i][h] pairs (scale, offset) of position 16 h + i.  Values: [block][g] eight scales, then eight offsets, of the positions in the order above.

Sizes are those of the repository's benchmark and tests: 32 query heads over 8 or 32 key/value heads and 64 over 8 (7B and 70B layers) with 128 components,
many heads over one or eight with 64, contexts from one token to 16 thousand and one.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
TILE = 32
ROPE_BASE = 10000.0
HALVES = 1                                  # the pairing of components (i, i + D/2)
FORMAT = {"Q4_B32": (4, 32), "Q4_B64": (4, 64), "Q8_B32": (8, 32), "Q8_B64": (8, 64)}       # bits of a level, components of a block
MAX_PAIRS = 64 * 128 * 2500 * 2500 * 3 // 4  # heads x components x (token, position) pairs of the largest listed case, roughly


def listed():
    return [
        # the smallest call: one sequence's next token goes into the cache (latency and host work count)
        {"name": "append_token", "kind": "append", "format": "Q4_B64", "heads": 32, "kv_heads": 8, "dim": 128, "seqs": 1, "longest": 512, "tokens": 1, "page": 64, "ragged": 1},
        # dynamic batching: the next token of 64 live sequences of any length
        {"name": "append_batch64", "kind": "append", "format": "Q4_B64", "heads": 64, "kv_heads": 8, "dim": 128, "seqs": 64, "longest": 2047, "tokens": 1, "page": 64, "ragged": 2},
        # prompts of four sequences at once, chunks that begin and end inside a tile
        {"name": "append_prompts", "kind": "append", "format": "Q4_B32", "heads": 32, "kv_heads": 8, "dim": 128, "seqs": 4, "longest": 4001, "tokens": 2000, "page": 128, "ragged": 3},
        # one long sequence read back
        {"name": "read_16k", "kind": "read", "format": "Q4_B64", "heads": 64, "kv_heads": 8, "dim": 128, "seqs": 1, "longest": 16001, "tokens": 16001, "page": 256, "ragged": 4},
        # a batch of short ones, 8 bits, 64 components
        {"name": "read_batch", "kind": "read", "format": "Q8_B32", "heads": 128, "kv_heads": 8, "dim": 64, "seqs": 12, "longest": 777, "tokens": 777, "page": 32, "ragged": 5},
        # a decode step's attention, one sequence at a short context
        {"name": "decode_short", "kind": "attn", "format": "Q4_B64", "heads": 32, "kv_heads": 8, "dim": 128, "seqs": 1, "longest": 512, "tokens": 1, "page": 64, "ragged": 6},
        # ... eight query heads per key/value head over a long context
        {"name": "decode_16k", "kind": "attn", "format": "Q4_B64", "heads": 64, "kv_heads": 8, "dim": 128, "seqs": 1, "longest": 16001, "tokens": 1, "page": 256, "ragged": 7},
        # ... 32 live sequences of any length up to 8 thousand
        {"name": "decode_batch32", "kind": "attn", "format": "Q4_B64", "heads": 32, "kv_heads": 8, "dim": 128, "seqs": 32, "longest": 8001, "tokens": 1, "page": 128, "ragged": 8},
        # ... as many key/value heads as query heads, 8 bits
        {"name": "decode_mha_8bit", "kind": "attn", "format": "Q8_B64", "heads": 32, "kv_heads": 32, "dim": 128, "seqs": 8, "longest": 3001, "tokens": 1, "page": 64, "ragged": 9},
        # a few drafted tokens per sequence are checked at once, every head over one key/value head of 64 components
        {"name": "draft_mqa_64", "kind": "attn", "format": "Q4_B32", "heads": 71, "kv_heads": 1, "dim": 64, "seqs": 16, "longest": 2000, "tokens": 4, "page": 64, "ragged": 10},
        # a prompt's chunk of 512 tokens behind what the cache holds of it
        {"name": "chunk_512", "kind": "attn", "format": "Q4_B64", "heads": 32, "kv_heads": 8, "dim": 128, "seqs": 1, "longest": 4400, "tokens": 512, "page": 128, "ragged": 11},
        # the largest: whole prompts of a large model
        {"name": "prompts_2500", "kind": "attn", "format": "Q4_B64", "heads": 64, "kv_heads": 8, "dim": 128, "seqs": 3, "longest": 2500, "tokens": 2500, "page": 64, "ragged": 12},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ones' ranges: any format, head dimension, group, page, number of sequences and tokens, odd lengths."""
    kind = rng.choice(["append", "read", "attn", "attn", "attn"])
    kv = rng.choice([1, 2, 4, 8, 8, 16, 32])
    case = {"kind": kind, "format": rng.choice(sorted(FORMAT)), "heads": kv * rng.choice([g for g in (1, 2, 3, 4, 8, 16, 71) if g * kv <= 128]), "kv_heads": kv,
            "dim": rng.choice([64, 128, 128]), "page": 32 * rng.choice([1, 2, 3, 4, 8]), "ragged": rng.randrange(1, 1 << 20)}
    tokens = rng.choice([1, 1, rng.randrange(2, 9), _log_int(rng, 9, 2500)]) if kind != "read" else 0
    if tokens > 8:
        seqs, longest = rng.randrange(1, 4), tokens + rng.choice([0, rng.randrange(1, 2000)])
        if kind == "attn":                                   # (no more work than the largest listed case)
            tokens = max(9, min(tokens, MAX_PAIRS // (case["heads"] * case["dim"] * seqs * longest)))
    else:
        seqs = _log_int(rng, 1, 64)
        longest = max(tokens, _log_int(rng, 1, min(16001, 2000000 // (seqs * kv))))
    case.update(seqs=seqs, longest=longest, tokens=tokens or longest)
    return case


# ---- a case's lengths (the same for every seed) ------------------------------------------------------------------------------

def _lengths(case):
    """(length, new tokens) of every sequence; the first is the longest and has the most tokens."""
    r, longest, most = random.Random(case["ragged"]), case["longest"], case["tokens"]
    both = [(longest, most)]
    while len(both) < case["seqs"]:
        n = r.randint(max(1, longest // 8), longest)
        both.append((n, n if most == longest else 1 if most == 1 else r.randint(1, min(most, n))))
    return both


def _tile_words(case):
    """32-bit words of a tile's codes (of the keys, and as many of the values) and of the whole tile."""
    w, block = FORMAT[case["format"]]
    codes = TILE * case["dim"] * w // 32
    return codes, 2 * codes + 2 * TILE * (case["dim"] // block)


# ---- inputs ------------------------------------------------------------------------------------------------------------------

def _normal(g, shape):
    return torch.empty(shape, dtype=torch.float32, device=DEVICE).normal_(0.0, 1.0, generator=g)


def _blocks_quantized(x, case):
    """x [..., D] in 16 bits -> levels [..., D] int32, scales and offsets [..., D / block] in 16 bits (each step in 32 bits, divisions exactly rounded)."""
    w, block = FORMAT[case["format"]]
    steps = torch.full((), float(2 ** w - 1), device=x.device)
    b = x.float().unflatten(-1, (-1, block))
    low, high = b.amin(-1) + 0.0, b.amax(-1) + 0.0
    scale, offset = ((high - low) / steps).half(), low.half()
    s = scale.float().unsqueeze(-1)
    t = (b - offset.float().unsqueeze(-1)) / torch.where(s == 0, torch.ones_like(s), s)
    down = t.floor()
    level = torch.where(t - down >= 0.5, down + 1, down).clamp(0, 2 ** w - 1)
    return torch.where(s == 0, torch.zeros_like(level), level).flatten(-2).int(), scale, offset


def _code_places(case):
    """For the elements [position of a tile][component]: the word of the key codes and the bit in it; the same for the value codes."""
    w, d = FORMAT[case["format"]][0], case["dim"]
    r = torch.arange(TILE, device=DEVICE).unsqueeze(1)
    c = torch.arange(d, device=DEVICE).unsqueeze(0)
    per = 32 // w                                            # elements of a word
    nibble = lambda e: e // 2 * 4 + e % 2 * 16               # noqa: E731
    g, x = c // (d // 4), c % (d // 4)
    at = r // 16 * (d // 4 // per) + x // per                # word of the run of (g, i)
    key = (at // 4 * 64 + g * 16 + r % 16) * 4 + at % 4
    key_bit = (nibble(x % 8) if w == 4 else x % 4 * 8) + 0 * r
    g, k = r % 16 // 4, r // 16 * 4 + r % 4
    at = c // 16 * (8 // per) + k // per
    value = (at // 4 * 64 + g * 16 + c % 16) * 4 + at % 4
    value_bit = (nibble(k) if w == 4 else k % 4 * 8) + 0 * c
    return key, key_bit, value, value_bit


def _header_places(case):
    """For [position of a tile][block]: where in the tile, in 16-bit units, the key's scale, the key's offset, the value's scale, the value's offset are."""
    codes, words = _tile_words(case)
    blocks = case["dim"] // FORMAT[case["format"]][1]
    r = torch.arange(TILE, device=DEVICE).unsqueeze(1)
    b = torch.arange(blocks, device=DEVICE).unsqueeze(0)
    key = 4 * codes + ((b * 16 + r % 16) * 2 + r // 16) * 2
    value = 4 * codes + 2 * TILE * blocks + (b * 4 + r % 16 // 4) * 16 + r // 16 * 4 + r % 4
    return key, key + 1, value, value + 8


def _packed_tiles(x, case, places, bits):
    """x [kv][positions][D] in 16 bits -> code words [kv][tile][..] of tiles of 32 positions, scales and offsets [kv][tile][position][block]."""
    level, scale, offset = _blocks_quantized(x, case)
    order = (places.flatten() * 64 + bits.flatten()).argsort().view(_tile_words(case)[0], -1)          # the elements of each word, lowest bits first
    flat = level.unflatten(1, (-1, TILE)).flatten(2)
    words = (flat[..., order] << bits.flatten()[order].int()).sum(-1, dtype=torch.int32)
    return words, scale.unflatten(1, (-1, TILE)), offset.unflatten(1, (-1, TILE))


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    both = _lengths(case)
    kv, d, page = case["kv_heads"], case["dim"], case["page"]
    codes, words = _tile_words(case)
    per_page = page // TILE
    need = [-(-n // page) for n, _ in both]
    most = max(need)
    pages = sum(need) + 3
    # pages in any order, as sequences came and went; what no sequence has written holds anything
    order = torch.randperm(pages, generator=g, device=DEVICE, dtype=torch.int64).int()
    table = torch.full((len(both), most), -1, dtype=torch.int32, device=DEVICE)
    pool = torch.randint(-2 ** 31, 2 ** 31, (pages, kv, per_page, words), dtype=torch.int32, device=DEVICE, generator=g)
    key, key_bit, value, value_bit = _code_places(case)
    headers = _header_places(case)
    used = 0
    channel = 1.0 + 4.0 * (torch.rand((kv, 1, d), device=DEVICE, generator=g) < 0.04)                  # a few components of the keys are much larger
    for b, (n, _) in enumerate(both):
        mine = order[used:used + need[b]]
        used += need[b]
        table[b, :need[b]] = mine
        tiles = -(-n // TILE)
        new = torch.randint(-2 ** 31, 2 ** 31, (kv, need[b] * per_page, words), dtype=torch.int32, device=DEVICE, generator=g)
        half = new.view(torch.float16)
        for which, x in enumerate(((_normal(g, (kv, tiles * TILE, d)) * channel).half(), _normal(g, (kv, tiles * TILE, d)).half())):
            w, scale, offset = _packed_tiles(x, case, *((key, key_bit) if which == 0 else (value, value_bit)))
            new[:, :tiles, which * codes:(which + 1) * codes] = w
            half[:, :tiles, headers[2 * which].flatten()] = scale.flatten(2)
            half[:, :tiles, headers[2 * which + 1].flatten()] = offset.flatten(2)
        if n % TILE:                                         # behind the sequence's last position: headers that are no numbers
            behind = torch.cat([h[n % TILE:].flatten() for h in headers])
            half[:, tiles - 1, behind] = float("nan")
        pool[mine.long()] = new.view(kv, need[b], per_page, words).transpose(0, 1)
    counts = [t for _, t in both]
    first = torch.tensor([0] + [sum(counts[:i + 1]) for i in range(len(counts))], dtype=torch.int32, device=DEVICE)
    lens = torch.tensor([n for n, _ in both], dtype=torch.int32, device=DEVICE)
    rows = sum(counts)
    state = {"case": case, "pool": pool, "table": table, "lens": lens, "first": first, "rows": rows}
    if case["kind"] in ("append", "attn"):
        state["q"] = _normal(g, (rows, case["heads"], d)).half()
        state["q_out"] = torch.empty_like(state["q"])
    if case["kind"] == "append":
        state["k"] = (_normal(g, (rows, kv, d)) * channel[:, 0]).half()
        state["v"] = _normal(g, (rows, kv, d)).half()
    if case["kind"] in ("append", "read"):
        state["k_out"] = torch.empty((rows, kv, d), dtype=torch.float16, device=DEVICE)
        state["v_out"] = torch.empty_like(state["k_out"])
    return state


# ---- the framework's calls -----------------------------------------------------------------------------------------------------

def _handles(state):
    """The cache's and the batch's descriptions and the attention's workspace, which a program makes once and keeps."""
    if "handles" not in state:
        from paper_2401_08294_amd import iflow
        case = state["case"]
        cache = iflow.kv_cache(iflow.FORMATS[case["format"]], case["kv_heads"], case["dim"], case["page"], state["pool"].shape[0], state["pool"])
        batch = iflow.kv_batch(state["table"].shape[0], state["table"].shape[1], state["table"], state["lens"], case["longest"], first_token=state["first"] if case["tokens"] > 1 else None,
                               n_tokens=state["rows"], max_tokens=case["tokens"])
        room = iflow.kv_attn_workspace_bytes(cache, batch, case["heads"]) if case["kind"] == "attn" else 0
        state["handles"] = iflow, cache, batch, torch.empty((max(room, 16),), dtype=torch.uint8, device=DEVICE), room
    return state["handles"]


def _run_own(state):
    iflow, cache, batch, workspace, room = _handles(state)
    case = state["case"]
    if case["kind"] == "attn":
        iflow.kv_attn(cache, batch, state["q"], case["heads"], 1.0 / math.sqrt(case["dim"]), state["q_out"], workspace, room)
        return state["q_out"]
    if case["kind"] == "append":
        iflow.kv_append(cache, batch, state["q"], state["k"], state["v"], case["heads"], ROPE_BASE, HALVES, state["q_out"])
    iflow.kv_read(cache, batch, state["k_out"], state["v_out"])
    return {"k": state["k_out"], "v": state["v_out"], "q": state["q_out"]} if case["kind"] == "append" else {"k": state["k_out"], "v": state["v_out"]}


# ---- the plain form --------------------------------------------------------------------------------------------------------------

def _half_once(x):
    """64 bits to 16, rounded once (through 32 bits that are cut off and made odd where something was cut)."""
    f = x.float()
    bits = f.view(torch.int32)
    cut = torch.where(f.double().abs() > x.abs(), bits - 1, bits) | (f.double() != x).int()
    return cut.view(torch.float32).half()


def _rotated(x, positions):
    """x [rows][heads][D] in 16 bits, rotated by its row's position; 64 bits."""
    d = x.shape[-1]
    turn = ROPE_BASE ** (-2.0 * torch.arange(d // 2, device=x.device, dtype=torch.float64) / d)
    angle = (positions.double().unsqueeze(1) * turn).unsqueeze(1)
    a, b = x.double().chunk(2, -1)
    return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1)


def _rows(state):
    """The sequence and the position of every row of the new tokens."""
    row = torch.arange(state["rows"], device=DEVICE)
    seq = (row.unsqueeze(1) >= state["first"][1:].unsqueeze(0)).sum(1)
    return seq, row - state["first"][seq + 1] + state["lens"][seq]


def _row_tiles(state):
    """Where every row's position lies: the number of its tile at key/value head 0, and the position in the tile."""
    case = state["case"]
    seq, position = _rows(state)
    page = state["table"][seq, position // case["page"]].long()
    per_page = case["page"] // TILE
    return page * (case["kv_heads"] * per_page) + position % case["page"] // TILE, position % TILE, per_page


def _values(words, bits, levels, scale, offset, block):
    """What codes stand for: fp16(level scale + offset), in 16 bits."""
    level = ((words >> bits) & levels).float()
    return (level * scale.float().repeat_interleave(block, -1) + offset.float().repeat_interleave(block, -1)).half()


def _plain_append_read(state):
    case = state["case"]
    w, block = FORMAT[case["format"]]
    codes, words = _tile_words(case)
    tile, r, per_page = _row_tiles(state)
    head = torch.arange(case["kv_heads"], device=DEVICE) * per_page
    base = (tile.unsqueeze(1) + head) * words                # [row][kv head]: first word of the tile
    key, key_bit, value, value_bit = _code_places(case)
    headers = _header_places(case)
    pool, half = state["pool"].view(-1), state["pool"].view(torch.float16).view(-1)
    out = {}
    if case["kind"] == "append":
        q = _half_once(_rotated(state["q"], _rows(state)[1]))
        k = _half_once(_rotated(state["k"], _rows(state)[1]))
        out["q"] = q
    k_at = base.unsqueeze(2) + key[r].unsqueeze(1)           # [row][kv head][component]
    v_at = base.unsqueeze(2) + codes + value[r].unsqueeze(1)
    k_bit, v_bit = key_bit[r].unsqueeze(1).int(), value_bit[r].unsqueeze(1).int()
    ks, ko, vs, vo = [base.unsqueeze(2) * 2 + h[r].unsqueeze(1) for h in headers]
    if case["kind"] == "append":
        k_level, half[ks], half[ko] = _blocks_quantized(k, case)
        v_level, half[vs], half[vo] = _blocks_quantized(state["v"], case)
        mask = 2 ** w - 1                                    # (several positions share a word: each adds what its own bits change)
        pool.index_add_(0, k_at.flatten(), ((k_level - ((pool[k_at] >> k_bit) & mask)) << k_bit).flatten())
        pool.index_add_(0, v_at.flatten(), ((v_level - ((pool[v_at] >> v_bit) & mask)) << v_bit).flatten())
    out["k"] = _values(pool[k_at], k_bit, 2 ** w - 1, half[ks], half[ko], block)
    out["v"] = _values(pool[v_at], v_bit, 2 ** w - 1, half[vs], half[vo], block)
    return out


def _plain_attn(state):
    case = state["case"]
    w, block = FORMAT[case["format"]]
    codes, words = _tile_words(case)
    kv, d, n_seqs = case["kv_heads"], case["dim"], case["seqs"]
    tiles = state["pool"][state["table"].clamp_min(0).long()].transpose(1, 2).flatten(2, 3)            # [sequence][kv head][tile][words]
    half = tiles.view(torch.float16)
    key, key_bit, value, value_bit = _code_places(case)
    ks, ko, vs, vo = _header_places(case)
    blocks = lambda at: half[..., at.flatten()].unflatten(-1, (TILE, -1))                              # noqa: E731
    k = _values(tiles[..., key.flatten()].unflatten(-1, (TILE, d)), key_bit.int(), 2 ** w - 1, blocks(ks), blocks(ko), block).float().flatten(2, 3)
    v = _values(tiles[..., codes + value.flatten()].unflatten(-1, (TILE, d)), value_bit.int(), 2 ** w - 1, blocks(vs), blocks(vo), block).float().flatten(2, 3)
    place = torch.arange(k.shape[2], device=DEVICE)
    there = place < state["lens"].unsqueeze(1)               # what lies behind a sequence holds anything
    k, v = [torch.where(there[:, None, :, None], x, torch.zeros((), device=DEVICE)) for x in (k, v)]
    # queries as [sequence][kv head][token x head of the group][D], padded to the most tokens
    seq, position = _rows(state)
    token = torch.arange(state["rows"], device=DEVICE) - state["first"][seq]
    q = torch.zeros((n_seqs, case["tokens"], case["heads"], d), device=DEVICE)
    q[seq, token] = state["q"].float()
    group = case["heads"] // kv
    q = q.view(n_seqs, case["tokens"], kv, group, d).transpose(1, 2).reshape(n_seqs, kv, -1, d)
    score = torch.matmul(q * (1.0 / math.sqrt(d)), k.transpose(2, 3).contiguous())
    counts = state["first"][1:] - state["first"][:-1]
    last = state["lens"].unsqueeze(1) - counts.unsqueeze(1) + torch.arange(case["tokens"], device=DEVICE)      # the position of each token
    seen = place <= last.clamp_min(0).repeat_interleave(group, 1).unsqueeze(2)
    score = score.masked_fill_(~seen.unsqueeze(1), float("-inf"))
    score = score.sub_(score.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(score, v) / score.sum(-1, keepdim=True)
    o = o.view(n_seqs, kv, case["tokens"], group, d).transpose(1, 2).reshape(n_seqs, case["tokens"], case["heads"], d)
    return o[seq, token].half()


def run(state):
    if own:
        return _run_own(state)
    return _plain_attn(state) if state["case"]["kind"] == "attn" else _plain_append_read(state)


# ---- the floor -------------------------------------------------------------------------------------------------------------------

def work(case):
    both = _lengths(case)
    w, block = FORMAT[case["format"]]
    per_position = case["kv_heads"] * (2 * case["dim"] * w // 8 + 2 * 4 * case["dim"] // block)
    rows = sum(t for _, t in both)
    q_bytes, kv_bytes = 2 * rows * case["heads"] * case["dim"], 2 * 2 * rows * case["kv_heads"] * case["dim"]
    if case["kind"] == "append":                             # queries in and out, keys and values in, codes out, values out
        return {"bytes": 2 * q_bytes + kv_bytes + rows * per_position + kv_bytes, "flops": 6 * rows * (case["heads"] + case["kv_heads"]) * case["dim"] // 2}
    if case["kind"] == "read":
        return {"bytes": rows * per_position + kv_bytes, "flops": 2 * rows * 2 * case["kv_heads"] * case["dim"]}
    pairs = sum(t * (n - t) + t * (t + 1) // 2 for n, t in both)
    return {"bytes": sum(n for n, _ in both) * per_position + 2 * q_bytes, "flops": 4 * case["heads"] * case["dim"] * pairs}


# ---- 64 bits ---------------------------------------------------------------------------------------------------------------------

def _runs(region, w, d):
    """Code bytes of tiles [..., bytes] -> the run of every (g, i) as levels [..., g, i, elements]."""
    x = region.unflatten(-1, (-1, 4, 16, 16))
    lead = list(range(x.dim() - 4))
    n = len(lead)
    x = x.permute(*lead, n + 1, n + 2, n, n + 3).flatten(-2).long()
    if w == 8:
        return x
    # bytes 0, 1, 2, 3 of a word hold v0 v2, v4 v6, v1 v3, v5 v7
    x = x.unflatten(-1, (-1, 4))
    low, high = x & 15, x >> 4
    return torch.stack([low[..., 0], low[..., 2], high[..., 0], high[..., 2], low[..., 1], low[..., 3], high[..., 1], high[..., 3]], -1).flatten(-2)


def _stand_for(tiles, case):
    """Tiles [..., bytes] -> keys and values [..., 32, D] that they stand for, in 64 bits and not rounded."""
    w, block = FORMAT[case["format"]]
    d = case["dim"]
    codes = TILE * d * w // 8
    blocks = d // block
    lead = tiles.shape[:-1]
    n = len(lead)
    keys = _runs(tiles[..., :codes], w, d).view(*lead, 4, 16, 2, d // 4).permute(*range(n), n + 2, n + 1, n, n + 3).reshape(*lead, TILE, d)
    values = _runs(tiles[..., codes:2 * codes], w, d).view(*lead, 4, 16, d // 16, 2, 4).permute(*range(n), n + 3, n, n + 4, n + 2, n + 1).reshape(*lead, TILE, d)
    head = tiles[..., 2 * codes:].contiguous().view(torch.float16).double()
    kh = head[..., :TILE * blocks * 2].reshape(*lead, blocks, 16, 2, 2).permute(*range(n), n + 2, n + 1, n, n + 3).reshape(*lead, TILE, blocks, 2)
    vh = head[..., TILE * blocks * 2:].reshape(*lead, blocks, 4, 2, 2, 4).permute(*range(n), n + 3, n + 1, n + 4, n, n + 2).reshape(*lead, TILE, blocks, 2)
    both = []
    for level, h in ((keys, kh), (values, vh)):
        x = level.double().unflatten(-1, (blocks, block)) * h[..., :1] + h[..., 1:]
        both.append(x.flatten(-2))
    return both


def _sequence(state, b, length):
    """Keys and values [kv head][position][D] of a sequence, in 64 bits."""
    case = state["case"]
    need = -(-length // case["page"])
    tiles = state["pool"][state["table"][b, :need].long()].transpose(0, 1).reshape(case["kv_heads"], -1, state["pool"].shape[-1]).contiguous()
    k, v = _stand_for(tiles.view(torch.uint8), case)
    return k.flatten(1, 2)[:, :length], v.flatten(1, 2)[:, :length]


def _to16(x):
    """64 bits rounded to what 16 bits hold (to the nearest, ties to even), still in 64."""
    unit = torch.ldexp(torch.ones_like(x), (torch.frexp(x).exponent - 1).clamp_min(-14) - 10)
    return (x / unit).round() * unit


def _written(x, case):
    """x [row][kv head][D] in 16 bits as the cache will stand for it, in 64 bits: the quantizer's roundings are part of what it is."""
    w, block = FORMAT[case["format"]]
    b = x.unflatten(-1, (-1, block)).float()
    low, high = b.min(-1, keepdim=True).values, b.max(-1, keepdim=True).values
    scale = ((high - low).double() / (2 ** w - 1)).float().half().double()
    offset = low.half().double()
    quotient = ((b.double() - offset).float().double() / scale).float().double()
    level = (quotient + 0.5).floor().clamp(0, 2 ** w - 1)
    level = torch.where(scale == 0, torch.zeros_like(level), level)
    return (level * scale + offset).flatten(-2)


def exact(case, seed):
    state = prepare(case, seed)
    both = _lengths(case)
    starts = state["first"].tolist()
    parts = []
    for b, (length, count) in enumerate(both):
        rows = slice(starts[b], starts[b + 1])
        places = torch.arange(length - count, length, device=DEVICE, dtype=torch.float64)
        if case["kind"] == "read":
            k, v = _sequence(state, b, length)
            parts.append({"k": k[:, length - count:].transpose(0, 1), "v": v[:, length - count:].transpose(0, 1)})
        elif case["kind"] == "append":
            d = case["dim"]
            i = torch.arange(d // 2, device=DEVICE, dtype=torch.float64)
            turn = torch.polar(torch.ones((count, d // 2), dtype=torch.float64, device=DEVICE), places[:, None] * torch.exp(-2.0 * i / d * math.log(ROPE_BASE)))
            spin = lambda x: torch.view_as_real(torch.complex(x[..., :d // 2].double(), x[..., d // 2:].double()) * turn[:, None]).transpose(-1, -2).flatten(-2)   # noqa: E731
            parts.append({"k": _written(_to16(spin(state["k"][rows])), case), "v": _written(state["v"][rows], case), "q": spin(state["q"][rows])})
        else:
            k, v = [_to16(x) for x in _sequence(state, b, length)]
            group = case["heads"] // case["kv_heads"]
            q = state["q"][rows].double().transpose(0, 1)    # [head][token][D]
            out = []
            for h in range(case["heads"]):
                score = q[h] @ k[h // group].T.contiguous() / math.sqrt(case["dim"])
                score = score.masked_fill(torch.arange(length, device=DEVICE)[None, :] > places[:, None], float("-inf"))
                out.append(torch.softmax(score, -1) @ v[h // group])
            parts.append(torch.stack(out, 1))
    if case["kind"] == "attn":
        return torch.cat(parts)
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}
