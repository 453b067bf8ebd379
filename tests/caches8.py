"""A cache held in 8 bits on the GPU beside its oracle, for the tests of the operators on it."""
import numpy as np
import torch

from oracle import cache8_oracle as orc
from tests.caches import bf16, dev  # noqa: F401


class Pair8:
    """lens: tokens of the first slots, pages in random order, random codes (none of them NaN) under powers drawn from `powers`, bounds that fit them; every
    other byte is `fill`, which as a code and as a power is NaN."""

    def __init__(self, lib, lens, hkv, d, page=64, n_slots=None, max_pages=None, spare=4, fill=0xFF, seed=0, powers=(115, 122)):
        self.lib, self.rng = lib, np.random.default_rng(seed)
        pages = [-(-S // page) for S in lens]
        n_slots = len(lens) if n_slots is None else n_slots
        max_pages = max(pages + [1]) if max_pages is None else max_pages
        c = self.o = orc.Cache8(sum(pages) + spare, page, n_slots, max_pages, hkv, d, fill=fill)
        order = list(self.rng.permutation(len(c.refs)))
        for s, (S, n) in enumerate(zip(lens, pages)):
            for i in range(n):
                c.table[s, i] = order.pop()
                c.refs[c.table[s, i]] = 1
            c.lens[s] = S
            for tile in range(-(-S // 32)):
                for h in range(hkv):
                    codes, bounds, p = c.block(c.table[s, 32 * tile // page], h, tile)
                    there = min(S - 32 * tile, 32)
                    p[:] = self.rng.integers(*powers, 2)
                    drawn = (self.rng.integers(0, 127, (2, there, d)) + 128 * self.rng.integers(0, 2, (2, there, d))).astype(np.uint8)
                    drawn[:, :, ::3] &= 0xBF                                          # (some channels far below the others)
                    for n in range(2):
                        codes[c.places[n][:there]] = drawn[n]
                    y = orc.value(drawn[0])
                    bounds[0], bounds[1] = np.ceil(y.max(axis=0) / 4), np.floor(y.min(axis=0) / 4)
        self.up()

    def up(self):
        c = self.o
        self.pages, self.refs, self.table, self.lens = (torch.from_numpy(x.copy()).cuda() for x in (c.pages, c.refs, c.table, c.lens))
        self.cache = self.lib.make_cache8(self.pages, self.refs, self.table, self.lens, c.page, c.hkv, c.d)
        self.status = torch.full((1,), 12345, dtype=torch.int32, device="cuda")

    def check_pages(self):
        """Every byte; a code that is no number may have either sign."""
        got, want = self.pages.cpu().numpy(), self.o.pages.copy()
        codes = self.o.at[0]
        for x in (got, want):
            x[:, :codes][(x[:, :codes] & 127) == 127] = 127
        wrong = np.argwhere(got != want)
        assert len(wrong) == 0, (wrong[:5].tolist(), codes, self.o.at[1], got[tuple(wrong[0])], want[tuple(wrong[0])])

    def check_rows(self):
        torch.cuda.synchronize()
        c, table = self.o, self.table.cpu().numpy()
        assert self.lens.cpu().tolist() == c.lens.tolist() and self.refs.cpu().tolist() == c.refs.tolist()
        for s in range(len(c.lens)):
            n = c.pages_for(int(c.lens[s]))
            assert table[s, :n].tolist() == c.table[s, :n].tolist(), s


def append(pair, kt, vt, n_rows, row_idx, offsets, slots, start, max_new, rotation=None, q=None, q_out=None, stream=None, strides=(0, 0, 0)):
    n_list = n_rows if row_idx is None else len(row_idx)
    pair.lib.cache8_append(pair.cache, kt, vt, strides[0], strides[1], n_rows, None if row_idx is None else dev(row_idx), n_list, dev(offsets), dev(slots),
                           dev(start), len(slots), max_new, rotation, q, strides[2], 0 if q is None else q.shape[1], q_out, stream)


def attend(pair, q, slots, n_tokens, max_len, blocks=None, scale=0.0, want_lse=True, stream=None, ws=None):
    """q: bf16 tensor [n, tokens, hq, d]"""
    lib, n, hq = pair.lib, q.shape[0], q.shape[2]
    width = 0 if blocks is None else blocks.shape[3]
    size = lib.cache8_attention_workspace_bytes(pair.cache, n, n_tokens, hq, max_len, width)
    if ws is None:
        ws = torch.full((max(size, 256),), 0xFF, dtype=torch.uint8, device="cuda")      # (NaN: nothing may be taken from it)
    out = torch.full_like(q, float("nan"))
    lse = torch.full((n, n_tokens, hq), float("nan"), dtype=torch.float32, device="cuda") if want_lse else None
    lib.cache8_attention(pair.cache, q, dev(slots), n, n_tokens, hq, max_len, scale, blocks, width, out, lse, ws, size, stream)
    return out, lse


def select(pair, q, slots, n_tokens, max_len, n_first, n_recent, n_best, stream=None):
    lib, n, hq = pair.lib, q.shape[0], q.shape[2]
    size = lib.cache8_select_workspace_bytes(pair.cache, n, n_tokens, hq, max_len)
    ws = torch.full((max(size, 256),), 0xFF, dtype=torch.uint8, device="cuda")
    blocks = torch.full((n, n_tokens, pair.o.hkv, n_first + n_recent + n_best), -7, dtype=torch.int32, device="cuda")
    lib.cache8_select(pair.cache, q, dev(slots), n, n_tokens, hq, max_len, n_first, n_recent, n_best, blocks, ws, size, stream)
    return blocks


def check_attention(pair, q64, slots, out, lse, scale=None, reads=None, blocks=None):
    """Element by element against the oracle.  With u = 2^-24, logits x in base e: a product's operands are exact, so |dx| <= (d + 4) u * scale * |q|.|k|, and
    a weight is off by |dx| + 2^-20 (exp2, its argument's rounding at |x| < 8192 / log2(e) units of the reference's distance) on either side of the quotient.
    P is rounded to bf16, by 2^-8 at most and divided by the sum of the rounded (2^-8 more of what is summed, at most), the output by 2^-8."""
    out, lse = out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
    d, hq = q64.shape[3], q64.shape[2]
    s = 1.0 / np.sqrt(d) if scale is None else scale
    for b, slot in enumerate(slots):
        if slot < 0 or pair.o.lens[slot] == 0:
            assert not out[b].any() and (lse is None or np.isneginf(lse[b]).all())
            continue
        k, v = pair.o.read(slot) if reads is None else reads[slot]
        mine = None if blocks is None else blocks[b]
        ref, ref_lse = orc.attention(q64[b], k, v, scale, mine)
        size, _ = orc.attention(q64[b], k, np.abs(v), scale, mine)                 # sum of p |v|
        g = hq // k.shape[1]
        top = np.stack([(np.abs(np.nan_to_num(k[:, h // g])) @ np.abs(q64[b, :, h].T)).max(axis=0) for h in range(hq)], axis=1) * s      # [tokens, hq]
        dx = (d + 4) * 2.0 ** -24 * top + 2.0 ** -20 + 2.0 ** -23 * top
        bound = (2.0 ** -7 + 2 * dx[..., None]) * size * 1.01 + 2.0 ** -8 * np.abs(ref) + 1e-30
        assert np.array_equal(np.isnan(out[b]), np.isnan(ref))
        fine = ~np.isnan(ref)
        assert (np.abs(out[b] - ref)[fine] <= bound[fine]).all(), (b, slot, np.nanmax(np.abs(out[b] - ref) / bound))
        if lse is not None:
            finite = np.isfinite(ref_lse)
            assert np.array_equal(np.isnan(lse[b]), np.isnan(ref_lse)) and np.array_equal(np.isneginf(lse[b]), np.isneginf(ref_lse))
            assert (np.abs(lse[b][finite] - ref_lse[finite]) <= (2 * dx + 2.0 ** -22 * np.abs(ref_lse))[finite]).all()
