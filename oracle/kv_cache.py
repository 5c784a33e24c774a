"""A key/value cache held in 4 or 8 bits, in pages: the plain definition, element by element from the layout's description in include/iflow.h.

TEST INFRASTRUCTURE ONLY: imported by ``tests/`` (and nothing in the GPU package); this module imports nothing from
the GPU package either.

arXiv 2401.08294 quantizes weights; the same blocks (Table 3, Eq.1 and Eq.2) are applied to a head's components here.  Quantizer, dequantizer and rotary
embedding are the oracle's own for weights and for the fp16 cache; what is new is where a position's codes lie and which positions a token sees.
All fp16 inputs and outputs are uint16 bit patterns, like everywhere else in the oracle.
"""
from __future__ import annotations

import numpy as np

from . import oracle, rope

TILE = 32
BITS = {oracle.Q4_B32: 4, oracle.Q4_B64: 4, oracle.Q8_B32: 8, oracle.Q8_B64: 8}


def tile_bytes(fmt: int, d: int) -> int:
    return 2 * (TILE * d * BITS[fmt] // 8 + TILE * (d // oracle.block_size(fmt)) * 4)


def code_place(fmt: int, d: int, value: bool, position: int, component: int):
    """(byte of the tile, bit of the byte) where the code of a component of a position begins."""
    w = BITS[fmt]
    if not value:
        h, i = divmod(position, 16)
        g, x = divmod(component, d // 4)
        element = h * (d // 4) + x                             # in the run of (g, i)
    else:
        c, i = divmod(component, 16)
        y, r = divmod(position, 16)
        g, k = r // 4, y * 4 + r % 4
        element = c * 8 + k
    if w == 8:
        byte, bit = element, 0
    else:
        word, e = divmod(element, 8)
        nibble = [0, 4, 1, 5, 2, 6, 3, 7][e]                   # of v0 .. v7 in the order v0 v2 v4 v6 v1 v3 v5 v7
        byte, bit = word * 4 + nibble // 2, 4 * (nibble % 2)
    n, within = divmod(byte, 16)
    return (TILE * d * w // 8 if value else 0) + (n * 64 + g * 16 + i) * 16 + within, bit


def header_places(fmt: int, d: int, value: bool, position: int, block: int):
    """(byte of the scale, byte of the offset)."""
    nb = d // oracle.block_size(fmt)
    at = 2 * (TILE * d * BITS[fmt] // 8)
    if not value:
        h, i = divmod(position, 16)
        at += ((block * 16 + i) * 2 + h) * 4
        return at, at + 2
    y, r = divmod(position, 16)
    at += TILE * nb * 4 + (block * 4 + r // 4) * 32 + (y * 4 + r % 4) * 2
    return at, at + 16


class Cache:
    """pages: uint8 [n_pages][page bytes] (modified in place by append)."""

    def __init__(self, fmt: int, n_kv: int, d: int, page_positions: int, pages: np.ndarray):
        self.fmt, self.n_kv, self.d, self.page_positions, self.pages = fmt, n_kv, d, page_positions, pages
        self.block, self.bits = oracle.block_size(fmt), BITS[fmt]
        self.tile = tile_bytes(fmt, d)
        nb = d // self.block
        self.code = [np.array([[code_place(fmt, d, v, r, c) for c in range(d)] for r in range(TILE)]) for v in (False, True)]          # [position][component][byte, bit]
        self.header = [np.array([[header_places(fmt, d, v, r, b) for b in range(nb)] for r in range(TILE)]) for v in (False, True)]
        assert pages.shape[1] == n_kv * (page_positions // TILE) * self.tile

    def page(self, table_row, position: int):
        """The page that holds a position, or None."""
        p = int(table_row[position // self.page_positions])
        return p if 0 <= p < self.pages.shape[0] else None

    def _at(self, table_row, position: int, head: int):
        p = self.page(table_row, position)
        if p is None:
            return None, 0
        t = head * (self.page_positions // TILE) + position % self.page_positions // TILE
        return self.pages[p, t * self.tile:(t + 1) * self.tile], position % TILE

    def store(self, table_row, position: int, k16, v16):
        """k16, v16 [n_kv][d]: quantized into their places (nothing else changes)."""
        for which, x in enumerate((k16, v16)):
            q, s, o = oracle.quantize(self.fmt, np.ascontiguousarray(x, np.uint16).view(np.float16).astype(np.float32))
            q, s, o = q.reshape(self.n_kv, self.d), s.reshape(self.n_kv, -1), o.reshape(self.n_kv, -1)
            for j in range(self.n_kv):
                tile, r = self._at(table_row, position, j)
                if tile is None:
                    return
                byte, bit = self.code[which][r, :, 0], self.code[which][r, :, 1]
                if self.bits == 8:
                    tile[byte] = q[j]
                else:
                    for b in (0, 4):                           # (both nibbles of a byte may be this position's)
                        at = byte[bit == b]
                        tile[at] = (tile[at] & (0xF0 if b == 0 else 0x0F)) | (q[j][bit == b].astype(np.uint8) << b)
                for n in range(s.shape[1]):
                    a, c = self.header[which][r, n]
                    tile[a:a + 2] = np.array([s[j, n]], np.uint16).view(np.uint8)
                    tile[c:c + 2] = np.array([o[j, n]], np.uint16).view(np.uint8)

    def load(self, table_row, position: int):
        """(k16, v16) [n_kv][d] that a position stands for; zeros where its page is none."""
        out = np.zeros((2, self.n_kv, self.d), np.uint16)
        for j in range(self.n_kv):
            tile, r = self._at(table_row, position, j)
            if tile is None:
                break
            for which in (0, 1):
                q = (tile[self.code[which][r, :, 0]] >> self.code[which][r, :, 1]) & (2 ** self.bits - 1)
                h = self.header[which][r]
                s, o = [np.array([tile[a:a + 2].copy().view(np.uint16)[0] for a in h[:, x]], np.uint16) for x in (0, 1)]
                level = q.astype(np.float64).reshape(-1, self.block)
                with np.errstate(invalid="ignore", over="ignore"):             # (headers that nobody wrote)
                    value = level * s.view(np.float16).astype(np.float64)[:, None] + o.view(np.float16).astype(np.float64)[:, None]       # exact
                    out[which, j] = value.reshape(-1).astype(np.float16).view(np.uint16)
        return out[0], out[1]


def tokens(lens, first, n_tokens: int, max_tokens: int, max_seq: int):
    """The batch's tokens: (sequence, row, position, has a place in the cache) of each that has a row."""
    for b, length in enumerate(lens):
        a, z = (b, b + 1) if first is None else (int(first[b]), int(first[b + 1]))
        for i in range(min(z - a, max_tokens)):
            position = int(length) - (z - a) + i
            if 0 <= a + i < n_tokens:
                yield b, a + i, position, 0 <= position < max_seq


def append(cache: Cache, table, lens, first, max_tokens: int, max_seq: int, q16, k16, v16, base: float, mode: int, q_out16):
    """Writes the tokens' keys and values into the cache and their rotated queries into q_out16."""
    for b, row, position, there in tokens(lens, first, q16.shape[0], max_tokens, max_seq):
        if there:
            q_out16[row] = rope.rope(q16[row], position, base, mode)
            cache.store(table[b], position, rope.rope(k16[row], position, base, mode), v16[row])


def read(cache: Cache, table, lens, first, max_tokens: int, max_seq: int, k_out16, v_out16):
    for b, row, position, there in tokens(lens, first, k_out16.shape[0], max_tokens, max_seq):
        k_out16[row], v_out16[row] = cache.load(table[b], position) if there else (0, 0)


def attend(cache: Cache, table, lens, first, max_tokens: int, max_seq: int, q16, scale: float, out, window=None, sinks: int = 0):
    """out [n_tokens][n_heads][d] in fp64, rows of no token as they were.  With a window a token sees the last `window` positions up to its own, and the first `sinks`."""
    held = {}
    group = q16.shape[1] // cache.n_kv
    for b, row, position, _ in tokens(lens, first, q16.shape[0], max_tokens, max_seq):
        n = max(0, min(position + 1, max_seq))
        if b not in held or len(held[b][2]) < n:
            most = max([0] + [min(p + 1, max_seq) for c, _, p, _ in tokens(lens, first, q16.shape[0], max_tokens, max_seq) if c == b])
            kv = [cache.load(table[b], p) for p in range(most)]
            there = np.array([cache.page(table[b], p) is not None for p in range(most)], bool)
            held[b] = [np.array([x[w] for x in kv], np.uint16).reshape(most, cache.n_kv, cache.d).view(np.float16).astype(np.float64) for w in (0, 1)] + [there]
        k, v, there = [x[:n] for x in held[b]]
        if window is not None:
            p = np.arange(n)
            there = there & ((p >= n - window) | (p < sinks))
        out[row] = 0.0
        if not there.any():
            continue
        for h in range(q16.shape[1]):
            j = h // group
            s = scale * (k[there, j] @ q16[row, h].view(np.float16).astype(np.float64))
            e = np.exp(s - s.max())
            out[row, h] = (e / e.sum()) @ v[there, j]


def tables(lens, new, held, free, ring, table, shared, page: int, n_pages: int, n_tokens: int, max_tokens: int, max_seq: int, slots):
    """Page table, first tokens and slots of a step, one sequence and one page after another (include/iflow.h: iflow_kv_tables).  new None: one token each.  ring, table and slots are
    modified in place; returns held, {first free, how many, missing} and first_token as they are then."""
    n_shared = len(shared)
    start, count = int(free[0]), int(free[1])
    front, end, missing, row = start, start + count, 0, 0
    held, first = [int(h) for h in held], [0]
    for b in range(len(lens)):
        n = min(max(int(lens[b]), 0), max_seq)
        if n > 0:
            table[b, :n_shared] = shared
        need, had = max(0, -(-n // page) - n_shared), held[b]
        held[b] = min(need, had)
        for j in range(need, had):
            ring[end % n_pages] = table[b, n_shared + j]
            end += 1
        for j in range(had, need):
            there = front < start + count
            table[b, n_shared + j] = ring[front % n_pages] if there else -1
            front, held[b], missing = (front + 1, held[b] + 1, missing) if there else (front, held[b], missing + 1)
        tokens = 1 if new is None else min(max(int(new[b]), 0), max_tokens)
        for i in range(tokens):
            p = int(lens[b]) - tokens + i
            at = int(table[b, p // page]) if 0 <= p < max_seq else -1
            if row < n_tokens:
                slots[row] = at * page + p % page if 0 <= at < n_pages else -1
            row += 1
        first.append(row)
    return held, [front % n_pages, end - front, missing], first
