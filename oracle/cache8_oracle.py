"""Float64 CPU oracle of the cache held in 8 bits: numbers, blocks with their powers and bounds, rows turned by positions, the choice of blocks, attention.

THIS IS TEST INFRASTRUCTURE, NOT THE PRODUCT: plain numpy and Python loops, written from the format's description in the library's header, sharing no
code with the HIP path.  Pages that are handed out, shared and given back are those of the cache held in 4 bits (cache_oracle.Cache).
"""
from __future__ import annotations

import numpy as np

from oracle import cache_oracle


def _grid():
    """The values of the codes 0 .. 126, ascending."""
    out = []
    for code in range(127):
        e, m = code >> 3, code & 7
        out.append(m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(out)


GRID = _grid()


def value(codes):
    codes = np.asarray(codes).astype(np.int64)
    x = np.concatenate([GRID, [np.nan]])[codes & 127]
    return np.where(codes >= 128, -x, x)


def encode(x):
    """The nearest codes, ties to the even one; more than 464, infinities and NaN: 0x7f (with the sign)."""
    x = np.asarray(x, dtype=np.float64)
    m = np.abs(x)
    hi = np.clip(np.searchsorted(GRID, np.where(np.isnan(m), 0, m)), 1, 126)
    lo = hi - 1
    below, above = m - GRID[lo], GRID[hi] - m
    code = np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(m <= 464, code, 127)                                       # (NaN compares false)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def power(x):
    """The smallest e from -100 to 119 with max|x| <= 448 * 2^e, over the finite numbers"""
    x = np.abs(x[np.isfinite(x)])
    top, e = (x.max() if x.size else 0.0), -100
    while e < 119 and top > 448 * 2.0 ** e:
        e += 1
    return e


def turn(x, positions, freqs, dims, interleaved):
    """x [rows, heads, d] turned by the rows' positions; freqs as the fp32 numbers that they are"""
    x = np.array(x, dtype=np.float64)
    for i in range(dims // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + dims // 2)
        angle = np.asarray(positions, dtype=np.longdouble) * np.longdouble(freqs[i])
        c, s = np.cos(angle).astype(np.float64)[:, None], np.sin(angle).astype(np.float64)[:, None]
        x[..., a], x[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return x


def places(d):
    """The bytes of K's and V's code of token t < 32 and channel c: [32, d] each, inside a block's 64 d bytes"""
    k, v = np.zeros((32, d), dtype=np.int64), np.zeros((32, d), dtype=np.int64)
    for half in range(2):
        for s in range(d // 64):
            for j in range(4):
                for t in range(16):
                    for byte in range(16):
                        k[16 * half + t, 64 * s + 16 * j + byte] = (((half * (d // 64) + s) * 4 + j) * 16 + t) * 16 + byte
    for g in range(d // 32):
        for j in range(4):
            for r in range(16):
                for p in range(2):
                    for e in range(8):
                        v[16 * (e // 4) + 4 * j + e % 4, 32 * g + 16 * p + r] = 32 * d + (((g * 4 + j) * 16 + r) * 2 + p) * 8 + e
    return k, v


class Cache8(cache_oracle.Cache):
    def __init__(self, n_pages, page_tokens, n_slots, max_pages, n_kv_heads, d, fill=0):
        super().__init__(n_pages, page_tokens, n_slots, max_pages, 1, 64)
        self.hkv, self.d, self.T = n_kv_heads, d, page_tokens // 32
        blocks = n_kv_heads * self.T
        self.at = (blocks * 64 * d, blocks * 66 * d)
        self.pages = np.full((n_pages, -(-blocks * (66 * d + 2) // 256) * 256), fill, dtype=np.uint8)
        self.places = places(d)

    def block(self, page, head, tile):
        """Views of a block: codes [64 d], bounds int8 [2, d], powers [2]"""
        p, i = self.pages[page], head * self.T + tile % self.T
        return (p[i * 64 * self.d:(i + 1) * 64 * self.d], p[self.at[0] + i * 2 * self.d:][:2 * self.d].view(np.int8).reshape(2, self.d), p[self.at[1] + 2 * i:][:2])

    def _copy_token(self, src, src_token, dst, dst_token):
        self.pages[dst] = self.pages[src]

    def append(self, k, v, row_idx, offsets, slots, start, max_new=1 << 40):
        """k, v float64 [rows, hkv, d], turned already"""
        listed = np.arange(len(k)) if row_idx is None else row_idx
        for i, s in enumerate(slots):
            if not 0 <= s < len(self.lens) or start[i] < 0 or s in list(slots)[:i]:
                continue
            end = min(start[i] + min(int(offsets[i + 1]) - int(offsets[i]), max_new), self.lens[s])
            for tile in range(start[i] // 32, -(-end // 32)):
                first, last = max(start[i], 32 * tile), min(end, 32 * tile + 32)
                page = self.table[s, 32 * tile // self.page]
                if last <= first or not 0 <= page < len(self.refs):
                    continue
                rows = []
                for t in range(first, last):
                    at = int(offsets[i]) + t - start[i]
                    row = listed[at] if 0 <= at < len(listed) else -1
                    rows.append((k[row], v[row]) if 0 <= row < len(k) else (np.full(k.shape[1:], np.nan),) * 2)
                new = np.array(rows)                                               # [tokens, 2, hkv, d]
                for h in range(self.hkv):
                    self._put_tokens(self.block(page, h, tile), new[:, 0, h], new[:, 1, h], first - 32 * tile)

    def _put_tokens(self, block, k, v, first):
        codes, bounds, powers = block
        shift = [0, 0]
        for n, x in enumerate((k, v)):
            e = power(x)
            if first > 0:
                old = int(powers[n]) - 127
                if e > old:
                    shift[n] = min(e - old, 100)
                    at = self.places[n]
                    codes[at] = encode(value(codes[at]) * 2.0 ** -shift[n])
                e = max(e, old)
            powers[n] = e + 127
            codes[self.places[n][first:first + len(x)]] = encode(x / 2.0 ** e)
        stored = value(codes[self.places[0][first:first + len(k)]])
        none = np.isnan(stored).any(axis=0)
        up, down = np.ceil(np.nan_to_num(stored).max(axis=0) / 4), np.floor(np.nan_to_num(stored).min(axis=0) / 4)
        up, down = np.where(none, 127, up), np.where(none, -127, down)
        if first > 0:
            up = np.maximum(up, np.ceil(bounds[0] / 2.0 ** shift[0]))
            down = np.minimum(down, np.floor(bounds[1] / 2.0 ** shift[0]))
        bounds[0], bounds[1] = up.astype(np.int8), down.astype(np.int8)

    def read(self, slot, first=0):
        """float64 K, V [len - first, hkv, d]"""
        n = max(int(self.lens[slot]) - first, 0)
        k, v = np.zeros((n, self.hkv, self.d)), np.zeros((n, self.hkv, self.d))
        for tile in range(first // 32, self.pages_for(0) + -(-int(self.lens[slot]) // 32)):
            a, b = max(first, 32 * tile), min(int(self.lens[slot]), 32 * tile + 32)
            for h in range(self.hkv):
                codes, _, powers = self.block(self.table[slot, 32 * tile // self.page], h, tile)
                for x, n in ((k, 0), (v, 1)):
                    x[a - first:b - first, h] = value(codes[self.places[n][a - 32 * tile:b - 32 * tile]]) * 2.0 ** (int(powers[n]) - 127)
        return k, v

    def select(self, q, slot, n_first, n_recent, n_best, max_len=1 << 40):
        """q float64 [tokens, hq, d] -> blocks [tokens, hkv, n_first + n_recent + n_best]"""
        tokens, hq, d = q.shape
        g, width = hq // self.hkv, n_first + n_recent + n_best
        out = np.full((tokens, self.hkv, width), -1, dtype=np.int64)
        length = 0 if slot < 0 else int(self.lens[slot])
        for i in range(tokens):
            count = -(-max(length - tokens + i + 1, 0) // 32)
            low = min(n_first, count)
            tail = max(low, count - n_recent)
            high = max(low, min(tail, -(-max_len // 32)))
            for h in range(self.hkv):
                score = [max(self._score(q[i, h * g + x], self.block(self.table[slot, 32 * c // self.page], h, c)) for x in range(g)) for c in range(low, high)]
                best = sorted(range(len(score)), key=lambda c: (-score[c], c))[:n_best]
                chosen = list(range(low)) + sorted(low + c for c in best) + list(range(tail, count))
                out[i, h, :len(chosen)] = chosen
        return out

    def _score(self, q, block):
        _, bounds, powers = block
        finite = np.abs(q[np.isfinite(q)])
        top, e = (finite.max() if finite.size else 0.0), -100
        while top > 127 * 2.0 ** e:
            e += 1
        u = np.where(np.isnan(q), 0, np.clip(np.round(q / 2.0 ** e), -127, 127))
        total = np.where(u > 0, u * bounds[0], u * bounds[1]).sum()
        return total * 2.0 ** min(max(e + 2 + int(powers[0]) - 127, -120), 100)


def attention(q, k, v, scale=None, blocks=None):
    """As cache_oracle.attention; blocks [tokens, hkv, n]: those that a token attends to, an entry that it does not see left out"""
    if blocks is None:
        return cache_oracle.attention(q, k, v, scale)
    tokens, hq, d = q.shape
    S, hkv = k.shape[0], k.shape[1]
    out, lse = np.zeros((tokens, hq, d)), np.full((tokens, hq), -np.inf)
    for i in range(tokens):
        seen = S - tokens + i + 1
        for h in range(hq):
            mine = [t for c in blocks[i, h // (hq // hkv)] if c >= 0 for t in range(32 * c, min(32 * c + 32, seen))]
            if mine:
                o, l = cache_oracle.attention(q[i:i + 1, h:h + 1], k[mine][:, h // (hq // hkv)][:, None], v[mine][:, h // (hq // hkv)][:, None], scale)
                out[i, h], lse[i, h] = o[0, 0], l[0, 0]
    return out, lse
