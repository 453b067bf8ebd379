"""Float64 CPU oracle of the cache held in 4 bits: numbers, pages, attention over them.

THIS IS TEST INFRASTRUCTURE, NOT THE PRODUCT: plain numpy and Python loops, written from the format's description in the library's
header, one byte and one number at a time, sharing no code with the HIP path.

A number is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, times 2^e, one e for 32 channels of a head of a token.  2^e is the smallest power of
two with max|x| <= 7 * 2^e, within 2^-126 .. 2^125; the nearest number, ties to the one with the even code; a block that holds
an infinity or a NaN is NaN.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """[..., 32 * blocks] float64 -> codes uint8 of the same shape, scale bytes uint8 [..., blocks]"""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(x.shape[:-1] + (-1, 32))
    codes = np.zeros(blocks.shape, dtype=np.uint8)
    scales = np.zeros(blocks.shape[:-1], dtype=np.uint8)
    for at in np.ndindex(scales.shape):
        block = blocks[at]
        if not np.isfinite(block).all():
            scales[at] = 255
            continue
        top, e = np.abs(block).max(), -126
        while e < 125 and top > 7 * 2.0 ** e:
            e += 1
        scales[at] = e + 127
        gap = np.abs(np.abs(block / 2.0 ** e)[:, None] - GRID)                  # [32, 8]
        nearest = gap == gap.min(axis=1, keepdims=True)
        for c in range(32):
            hits = np.flatnonzero(nearest[c])
            code = hits[0] if len(hits) == 1 else [h for h in hits if h % 2 == 0][0]
            codes[at + (c,)] = code + (8 if np.signbit(block[c]) else 0)
    return codes.reshape(x.shape), scales


def values(codes, scales):
    """float64 of codes [..., 32 * blocks] and scale bytes [..., blocks]; 255: NaN"""
    sign = np.where(codes >= 8, -1.0, 1.0)
    power = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return sign * GRID[codes % 8] * np.repeat(power, 32, axis=-1)


def tile_places(d):
    """For token t < 32 and channel c < d of a tile of 34 * d bytes: (byte, high) of K's code, of V's code, byte of K's scale, of V's."""
    nb = d // 32
    kb, vb = np.zeros((32, d, 2), dtype=np.int64), np.zeros((32, d, 2), dtype=np.int64)
    ks, vs = np.zeros((32, nb), dtype=np.int64), np.zeros((32, nb), dtype=np.int64)
    for half in range(2):
        for block in range(nb):
            for token in range(16):
                for byte in range(16):
                    for high in range(2):
                        kb[16 * half + token, 32 * block + 2 * byte + high] = (((half * nb + block) * 16 + token) * 16 + byte, high)
                ks[16 * half + token, block] = 32 * d + (block * 16 + token) * 2 + half
    for h in range(d // 64):
        for j in range(4):
            for r in range(16):
                for p in range(2):
                    for q in range(2):
                        for byte in range(4):
                            for high in range(2):
                                token = 16 * (byte // 2) + 4 * j + 2 * (byte % 2) + high
                                vb[token, 64 * h + 32 * p + 2 * r + q] = (16 * d + ((((h * 4 + j) * 16 + r) * 2 + p) * 2 + q) * 4 + byte, high)
    for j in range(4):
        for block in range(nb):
            for half in range(2):
                for s in range(4):
                    vs[16 * half + 4 * j + s, block] = 33 * d + ((j * nb + block) * 2 + half) * 4 + s
    return kb, vb, ks, vs


class Cache:
    """Pages, counts, table and lengths as numpy arrays; every operation as the header says, row by row."""

    def __init__(self, n_pages, page_tokens, n_slots, max_pages, n_kv_heads, d, fill=0):
        self.page, self.hkv, self.d = page_tokens, n_kv_heads, d
        self.pages = np.zeros((n_pages, n_kv_heads, page_tokens // 32, 34 * d), dtype=np.uint8) + np.uint8(fill)
        self.refs = np.zeros(n_pages, dtype=np.int32)
        self.table = np.full((n_slots, max_pages), -1, dtype=np.int32)
        self.lens = np.zeros(n_slots, dtype=np.int32)
        self.places = tile_places(d)

    def pages_for(self, tokens):
        return -(-tokens // self.page)

    def _take(self, count):
        free = np.flatnonzero(self.refs == 0)
        if len(free) < count:
            return None, count - len(free)
        self.refs[free[:count]] = 1
        return list(free[:count]), 0

    def _bad_slots(self, slots):
        named = [s for s in slots if s != -1]
        return any(s < 0 or s >= len(self.lens) for s in named) or len(set(named)) < len(named)

    def reserve(self, slots, n_new):
        n = len(slots)
        start, none = np.full(n, -1, dtype=np.int32), np.full(n, -1, dtype=np.int32)
        most = self.table.shape[1] * self.page
        status = 0
        if self._bad_slots(slots):
            status = -1
        if any(s != -1 and 0 <= s < len(self.lens) and (m < 0 or self.lens[s] + m > most) for s, m in zip(slots, n_new)):
            status = -2
        if status:
            return none, status
        need = [0 if s == -1 else self.pages_for(self.lens[s] + m) - self.pages_for(self.lens[s]) for s, m in zip(slots, n_new)]
        got, lacking = self._take(sum(need))
        if lacking:
            return none, lacking
        for i, s in enumerate(slots):
            if s == -1:
                continue
            start[i] = self.lens[s]
            first = self.pages_for(self.lens[s])
            for c in range(need[i]):
                self.table[s, first + c] = got.pop(0)
            self.lens[s] += n_new[i]
        return start, 0

    def fork(self, parents, children):
        pairs = [(a, c) for a, c in zip(parents, children) if (a, c) != (-1, -1)]
        inside = lambda s: 0 <= s < len(self.lens)  # noqa: E731
        if any(not inside(a) or not inside(c) or self.lens[c] != 0 for a, c in pairs) or len({c for _, c in pairs}) < len(pairs) or \
                {a for a, _ in pairs} & {c for _, c in pairs}:
            return -1
        got, lacking = self._take(sum(self.lens[a] % self.page != 0 for a, _ in pairs))
        if lacking:
            return lacking
        for a, c in pairs:
            full = self.lens[a] // self.page
            self.table[c, :full] = self.table[a, :full]
            self.refs[self.table[a, :full]] += 1
            if self.lens[a] % self.page:
                self.table[c, full] = got.pop(0)
                for t in range(full * self.page, self.lens[a]):
                    self._copy_token(self.table[a, full], t, self.table[c, full], t)
            self.lens[c] = self.lens[a]
        return 0

    def release(self, slots):
        for s in slots:
            if 0 <= s < len(self.lens):
                for i in range(self.pages_for(self.lens[s])):
                    self.refs[self.table[s, i]] -= 1
                    self.table[s, i] = -1
                self.lens[s] = 0

    def compact(self, slots, kept, seq_offsets, out_offsets, max_keep):
        keep = [int(out_offsets[i + 1] - out_offsets[i]) for i in range(len(slots))]
        status = 0
        if self._bad_slots(slots):
            status = -1
        if any(s != -1 and 0 <= s < len(self.lens) and (k < 0 or out_offsets[i] < 0 or out_offsets[i + 1] > len(kept) or k > max_keep or
                                                        k > self.table.shape[1] * self.page) for i, (s, k) in enumerate(zip(slots, keep))):
            status = -2
        if status:
            return status
        got, lacking = self._take(sum(self.pages_for(k) for s, k in zip(slots, keep) if s != -1))
        if lacking:
            return lacking
        for i, s in enumerate(slots):
            if s == -1:
                continue
            fresh = [got.pop(0) for _ in range(self.pages_for(keep[i]))]
            for j in range(keep[i]):
                old = int(kept[out_offsets[i] + j]) - int(seq_offsets[i])
                if 0 <= old < self.lens[s]:
                    self._copy_token(self.table[s, old // self.page], old, fresh[j // self.page], j)
                else:
                    self._put(fresh[j // self.page], j, np.zeros((self.hkv, self.d), np.uint8), np.full((self.hkv, self.d // 32), 255, np.uint8),
                              np.zeros((self.hkv, self.d), np.uint8), np.full((self.hkv, self.d // 32), 255, np.uint8))
            self.release([s])
            self.table[s, :len(fresh)] = fresh
            self.lens[s] = keep[i]
        return 0

    # a token's codes and scale bytes, [hkv, d] and [hkv, d / 32]
    def _get(self, page, token):
        t = token % self.page
        tile = self.pages[page, :, t // 32]
        kb, vb, ks, vs = (x[t % 32] for x in self.places)
        return (tile[:, kb[:, 0]] >> (4 * kb[:, 1]).astype(np.uint8) & 15, tile[:, ks], tile[:, vb[:, 0]] >> (4 * vb[:, 1]).astype(np.uint8) & 15, tile[:, vs])

    def _put(self, page, token, kc, ksc, vc, vsc):
        t = token % self.page
        tile = self.pages[page, :, t // 32]
        kb, vb, ks, vs = (x[t % 32] for x in self.places)
        for places, codes in ((kb, kc), (vb, vc)):
            for c, (byte, high) in enumerate(places):
                tile[:, byte] = (tile[:, byte] & (0x0F if high else 0xF0)) | (codes[:, c].astype(np.uint8) << np.uint8(4 * high))
        tile[:, ks] = ksc
        tile[:, vs] = vsc

    def _copy_token(self, src, src_token, dst, dst_token):
        self._put(dst, dst_token, *self._get(src, src_token))

    def store(self, k, v, row_idx, offsets, slots, start):
        """k, v float64 [rows, hkv, d]"""
        for i, s in enumerate(slots):
            if not 0 <= s < len(self.lens) or start[i] < 0 or s in list(slots)[:i]:
                continue
            for j in range(int(offsets[i + 1] - offsets[i])):
                row = offsets[i] + j if row_idx is None else row_idx[offsets[i] + j]
                token = start[i] + j
                if token >= self.lens[s] or not 0 <= row < len(k) or not 0 <= self.table[s, token // self.page] < len(self.refs):
                    continue
                self._put(self.table[s, token // self.page], token, *quantise(k[row]), *quantise(v[row]))

    def read(self, slot):
        """float64 K, V [len, hkv, d]"""
        k, v = np.zeros((self.lens[slot], self.hkv, self.d)), np.zeros((self.lens[slot], self.hkv, self.d))
        for t in range(self.lens[slot]):
            kc, ks, vc, vs = self._get(self.table[slot, t // self.page], t)
            k[t], v[t] = values(kc, ks), values(vc, vs)
        return k, v


def attention(q, k, v, scale=None):
    """q float64 [tokens, hq, d], the newest of the tokens of k, v [len, hkv, d] -> out [tokens, hq, d], lse [tokens, hq] (base 2)"""
    tokens, hq, d = q.shape
    S, hkv = k.shape[0], k.shape[1]
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out, lse = np.zeros((tokens, hq, d)), np.full((tokens, hq), -np.inf)
    for i in range(tokens):
        seen = S - tokens + i + 1
        if seen <= 0:
            continue
        for h in range(hq):
            x = scale * (k[:seen, h // (hq // hkv)] @ q[i, h])
            p = np.exp(x - x.max())
            out[i, h] = p @ v[:seen, h // (hq // hkv)] / p.sum()
            lse[i, h] = (x.max() + np.log(p.sum())) / np.log(2.0)
    return out, lse
