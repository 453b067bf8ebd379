"""A cache held in 4 bits on the GPU beside its oracle, for the tests of the operators on it."""
import numpy as np
import torch

from oracle import cache_oracle as orc


def dev(values, dtype=torch.int32):
    return torch.from_numpy(np.array(values)).to(dtype).cuda()


def bf16(x):
    """float64 array -> the bf16 tensor nearest to it and that tensor's float64 values"""
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


class Pair:
    """lens: tokens of the first slots, pages in random order; every byte outside them is `fill`."""

    def __init__(self, lib, lens, hkv, d, page=64, n_slots=None, max_pages=None, spare=4, fill=0xFF, seed=0, scales=(118, 132)):
        self.lib, self.rng = lib, np.random.default_rng(seed)
        pages = [-(-S // page) for S in lens]
        n_slots = len(lens) if n_slots is None else n_slots
        max_pages = max(pages + [1]) if max_pages is None else max_pages
        c = self.o = orc.Cache(sum(pages) + spare, page, n_slots, max_pages, hkv, d, fill=fill)
        order = list(self.rng.permutation(len(c.refs)))
        for s, (S, n) in enumerate(zip(lens, pages)):
            for i in range(n):
                c.table[s, i] = order.pop()
                c.refs[c.table[s, i]] = 1
            c.lens[s] = S
            for t in range(S):
                c._put(c.table[s, t // page], t, *self.token(scales))
        self.up()

    def token(self, scales):
        c, rng = self.o, self.rng
        return (rng.integers(0, 16, (c.hkv, c.d)).astype(np.uint8), rng.integers(*scales, (c.hkv, c.d // 32)).astype(np.uint8),
                rng.integers(0, 16, (c.hkv, c.d)).astype(np.uint8), rng.integers(*scales, (c.hkv, c.d // 32)).astype(np.uint8))

    def up(self):
        c = self.o
        self.pages, self.refs, self.table, self.lens = (torch.from_numpy(x.copy()).cuda() for x in (c.pages, c.refs, c.table, c.lens))
        self.cache = self.lib.make_cache(self.pages, self.refs, self.table, self.lens, c.page, c.hkv, c.d)
        self.status = torch.full((1,), 12345, dtype=torch.int32, device="cuda")

    def check(self):
        """Table rows as far as they are in use, counts, lengths, and every bit of the tokens held."""
        torch.cuda.synchronize()
        c = self.o
        lens, table, pages = self.lens.cpu().numpy(), self.table.cpu().numpy(), self.pages.cpu().numpy()
        assert lens.tolist() == c.lens.tolist()
        assert self.refs.cpu().tolist() == c.refs.tolist()
        mine = orc.Cache(1, c.page, 1, 1, c.hkv, c.d)
        mine.pages = pages
        for s in range(len(lens)):
            n = c.pages_for(int(c.lens[s]))
            assert table[s, :n].tolist() == c.table[s, :n].tolist(), s
            for t in range(int(c.lens[s])):
                for a, b in zip(mine._get(table[s, t // c.page], t), c._get(c.table[s, t // c.page], t)):
                    assert np.array_equal(a, b), (s, t)


def attend(pair, q, slots, n_tokens, max_len, scale=0.0, want_lse=True, stream=None, ws=None):
    """q: bf16 tensor [n, tokens, hq, d]"""
    lib = pair.lib
    n, hq = q.shape[0], q.shape[2]
    size = lib.cache_attention_workspace_bytes(pair.cache, n, n_tokens, hq, max_len)
    if ws is None:
        ws = torch.full((max(size, 256),), 0xFF, dtype=torch.uint8, device="cuda")      # (NaN: nothing may be taken from it)
    out = torch.full_like(q, float("nan"))
    lse = torch.full((n, n_tokens, hq), float("nan"), dtype=torch.float32, device="cuda") if want_lse else None
    lib.cache_attention(pair.cache, q, dev(slots), n, n_tokens, hq, max_len, scale, out, lse, ws, size, stream)
    return out, lse


def check_attention(pair, q64, slots, out, lse, scale=None, reads=None):
    """Element by element against the oracle.  With u = 2^-24, logits x in base e: a product's operands are exact, so |dx| <= (d + 4) u * scale * |q|.|k|, and
    a weight is off by |dx| + 2^-20 (exp2, its argument's rounding at |x| < 8192 / log2(e) units of the reference's distance) on either side of the quotient.
    P * 2^e is rounded to bf16 (2^-8), the output too."""
    out, lse = out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
    d, hq = q64.shape[3], q64.shape[2]
    s = 1.0 / np.sqrt(d) if scale is None else scale
    for b, slot in enumerate(slots):
        if slot < 0 or pair.o.lens[slot] == 0:
            assert not out[b].any() and (lse is None or np.isneginf(lse[b]).all())
            continue
        k, v = pair.o.read(slot) if reads is None else reads[slot]
        ref, ref_lse = orc.attention(q64[b], k, v, scale)
        size, _ = orc.attention(q64[b], k, np.abs(v), scale)                       # sum of p |v|
        g = hq // k.shape[1]
        top = np.stack([(np.abs(np.nan_to_num(k[:, h // g])) @ np.abs(q64[b, :, h].T)).max(axis=0) for h in range(hq)], axis=1) * s      # [tokens, hq]
        dx = (d + 4) * 2.0 ** -24 * top + 2.0 ** -20 + 2.0 ** -23 * top
        bound = (2.0 ** -8 + 2 * dx[..., None]) * size * 1.01 + 2.0 ** -8 * np.abs(ref) + 1e-30
        assert np.array_equal(np.isnan(out[b]), np.isnan(ref))
        fine = ~np.isnan(ref)
        assert (np.abs(out[b] - ref)[fine] <= bound[fine]).all(), (b, slot, np.nanmax(np.abs(out[b] - ref) / bound))
        if lse is not None:
            finite = np.isfinite(ref_lse)                                       # (a key that is NaN makes no bound: rows that see it are NaN)
            assert np.array_equal(np.isnan(lse[b]), np.isnan(ref_lse)) and np.array_equal(np.isneginf(lse[b]), np.isneginf(ref_lse))
            assert (np.abs(lse[b][finite] - ref_lse[finite]) <= (2 * dx + 2.0 ** -22 * np.abs(ref_lse))[finite]).all()
