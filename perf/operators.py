"""The operators on a cache held in 4 bits, as cases that can be timed and compared.

A cache is a pool of pages that the slots of a table share: K and V of a token are 4-bit floating-point numbers (e2m1: sign, two
exponent bits, one mantissa bit; 0, 0.5, 1, 1.5, 2, 3, 4, 6) with a power of two for every 32 channels of a head.  A case is what a
serving program does with it:

  attend   attention of the newest token of every sequence, or of its newest few, over the sequence's cache
  store    rows of K and V, chosen by a list of kept rows or all of them, go into the cache, and the cache is read back as bf16
  step     a branch of every sequence grows: the branches of the last pass are given back, the sequences are forked, get room for
           their new tokens, the tokens' K and V are stored, and the tokens attend to the branch
  evict    a branch of every sequence is cut to its pivotal tokens: give back, fork, keep the listed tokens, read them as bf16
  turn     sequences end and others begin: pages are given back and handed out

Lengths come from the case itself ("lens": a seed), so every input seed has the same shapes.  What is held in 4 bits is returned as the
values it stands for.

The pages, [n_pages, n_kv_heads, page_tokens / 32] tiles of 34 * d bytes, a tile being 32 tokens of one head, nb = d / 32:
  16 * d bytes  K's codes   [half][block nb][token 16][16 bytes]: token 16 * half + token, channel 32 * block + 2 * byte + high nibble
  16 * d bytes  V's codes   [d / 64][j 4][r 16][2][2][4 bytes]: with indexes h, j, r, p, q, byte and nibble: channel
                            64 * h + 32 * p + 2 * r + q, token 16 * (byte / 2) + 4 * j + 2 * (byte % 2) + high nibble
       d bytes  K's scales  [block nb][token 16][half]: 2^(byte - 127), 255: not a number
       d bytes  V's scales  [j 4][block nb][half][s 4]: token 16 * half + 4 * j + s
"""
import math
import random

import torch

own = False                                         # False: plain torch operations; True: the library's entry points


def listed():
    return [
        # the smallest decode: one short conversation on a small model, launches and latency are all there is
        dict(name="attend-1x256-d64", kind="attend", n=1, lo=256, hi=256, hq=8, hkv=8, d=64, page=64, tokens=1),
        # one long document, half of its tokens kept, many query heads on few key/value heads: the work has to be split along the cache
        dict(name="attend-1x16384-gqa", kind="attend", n=1, lo=16384, hi=16384, hq=64, hkv=8, d=128, page=64, tokens=1),
        # a serving batch of 2k tokens on a 7B-shaped layer: bound by the cache's bytes
        dict(name="attend-64x2048", kind="attend", n=64, lo=2048, hi=2048, hq=32, hkv=32, d=128, page=64, tokens=1),
        # a ragged batch on a 13B-shaped layer, 60 % of the tokens kept, four drafted tokens to verify
        dict(name="attend-ragged32-4tokens", kind="attend", n=32, lo=307, hi=4915, lens=4, hq=40, hkv=40, d=128, page=128, tokens=4),
        # the prompt's pivotal tokens go into the cache right after their selection: 70 % of 8 prompts of 2k tokens
        dict(name="store-8x2048-kept", kind="store", n=8, lo=2048, hi=2048, hq=32, hkv=32, d=128, page=64, keep=70, base=0),
        # pieces of ragged prompts behind what the cache holds already, beginning and ending inside a tile
        dict(name="store-ragged7-d64", kind="store", n=7, lo=100, hi=3000, lens=7, hq=32, hkv=8, d=64, page=32, keep=100, base=77),
        # generation, one conversation
        dict(name="step-1x1434", kind="step", n=1, lo=1434, hi=1434, hq=32, hkv=32, d=128, page=64, tokens=1),
        # generation, a serving batch with grouped heads
        dict(name="step-64x1337-gqa", kind="step", n=64, lo=1337, hi=1337, hq=32, hkv=8, d=128, page=64, tokens=1),
        # a batch cut to 70 %
        dict(name="evict-8x2048", kind="evict", n=8, lo=2048, hi=2048, hq=32, hkv=32, d=128, page=64, keep=70),
        # long inputs cut to one half
        dict(name="evict-4x32768-gqa", kind="evict", n=4, lo=32768, hi=32768, hq=64, hkv=8, d=128, page=128, keep=50),
        # 64 sequences of 2k tokens end, 64 others begin
        dict(name="turn-64x2048", kind="turn", n=64, lo=2048, hi=2048, hq=32, hkv=32, d=128, page=64),
        # many ragged sequences in a large pool
        dict(name="turn-ragged200", kind="turn", n=200, lo=100, hi=8000, lens=3, hq=32, hkv=8, d=64, page=32),
    ]


_HEADS = [(8, 8, 64), (32, 8, 64), (12, 12, 64), (32, 32, 128), (40, 40, 128), (32, 8, 128), (64, 8, 128), (24, 24, 128)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "store", "step", "step", "evict", "turn"])
    hq, hkv, d = rng.choice(_HEADS)
    n = _log_int(rng, 1, 128)
    tokens = 1 if rng.random() < 0.6 else rng.randint(2, 9)
    # values of K in the cache, so that a drawn case costs no more than the largest listed one: a branch copies pages, rows in bf16 are
    # four times the cache's, and more than 16 query rows on a head of K cost products
    most = (64 * 2048 * 32 * 128) // dict(attend=1, step=3, store=10, evict=10, turn=1)[kind]
    if kind in ("attend", "step"):
        most //= -(-tokens * (hq // hkv) // 16)
    top = max(1, min(_log_int(rng, 1, 65536), most // (hkv * d * n)))
    low = top if rng.random() < 0.5 else max(1, int(top * rng.uniform(0.1, 0.9)))
    case = dict(kind=kind, n=n, lo=low, hi=top, hq=hq, hkv=hkv, d=d, page=rng.choice([32, 64, 128, 256]))
    if low < top:
        case["lens"] = rng.randrange(1000)
    if kind in ("attend", "step"):
        case["tokens"] = tokens
    if kind == "attend":
        case["pad"] = 0 if rng.random() < 0.7 else rng.randint(1, n)       # rows of a padded batch at its end
    if kind in ("store", "evict"):
        case["keep"] = rng.randint(30, 100)
    if kind == "store":
        case["base"] = 0 if rng.random() < 0.5 else rng.randint(1, min(200, top))
    return case


def _lengths(case):
    if case["lo"] == case["hi"]:
        return [case["lo"]] * case["n"]
    rng = random.Random(case["lens"])
    return [rng.randint(case["lo"], case["hi"]) for _ in range(case["n"])]


def _keeps(case, lens):
    return [max(1, (case["keep"] * S + 50) // 100) for S in lens]


def _offsets(lens):
    off = [0]
    for S in lens:
        off.append(off[-1] + S)
    return off


# ------------------------------------------------------------------------------------------------ inputs
def _ints(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


class _Pool:
    """The cache of a case: pages in an order that a long-running server leaves, free ones among them, all bytes of what is not
    held at random.  held: tokens in the first slots; spare: pages that stay free."""

    def __init__(self, case, held, n_slots, spare, longest, gen):
        self.hkv, self.d, self.page, self.tiles = case["hkv"], case["d"], case["page"], case["page"] // 32
        self.n_slots = n_slots
        pages = [-(-S // self.page) for S in held]
        self.max_pages = max(1, -(-longest // self.page))
        self.n_pages = sum(pages) + spare
        order = torch.randperm(self.n_pages, generator=gen, device="cuda").to(torch.int32)
        self.table = torch.full((n_slots, self.max_pages), -1, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(self.n_pages, dtype=torch.int32, device="cuda")
        first = _offsets(pages)
        at = torch.arange(self.max_pages, device="cuda")
        count = torch.tensor(pages, device="cuda")
        there = at[None, :] < count[:, None]
        rank = torch.tensor(first[:-1], device="cuda")[:, None] + at[None, :]
        rows = order[rank.clamp(max=self.n_pages - 1)]
        self.table[:len(held)] = torch.where(there, rows, torch.full_like(rows, -1))
        self.refs[order[:first[-1]].long()] = 1
        self.lens = torch.zeros(n_slots, dtype=torch.int32, device="cuda")
        self.lens[:len(held)] = _ints(held)
        size = self.n_pages * self.hkv * self.tiles * 34 * self.d
        self.pages = torch.randint(0, 256, (size,), generator=gen, device="cuda", dtype=torch.uint8)
        self.pages = self.pages.view(self.n_pages, self.hkv, self.tiles, 34 * self.d)


def _rows(gen, count, hkv, d, u, spread):
    """bf16 rows [count, hkv, d]: normal numbers along a direction u per head that tokens have to a degree of their own (so that they
    differ in importance by orders of magnitude, as in a trained model); spread == 0: plain ones."""
    x = torch.randn((count, hkv, d), generator=gen, device="cuda")
    if spread:
        x += (spread * torch.randn(count, generator=gen, device="cuda"))[:, None, None] * u[None]
    return x.to(torch.bfloat16)


def _fill(pool, held, gen, u):
    """Every held token's K and V, a piece of the batch at a time."""
    step = max(1, (1 << 27) // (pool.hkv * pool.d * max(max(held), 1)))
    for b in range(0, len(held), step):
        part = held[b:b + step]
        off = _offsets(part)
        k, v = _rows(gen, off[-1], pool.hkv, pool.d, u, 3.0), _rows(gen, off[-1], pool.hkv, pool.d, u, 0.0)
        _plain_store(pool, k, v, None, _ints(off), _ints(list(range(b, b + len(part)))), _ints([0] * len(part)), max(part))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, lens, n, page = case["kind"], _lengths(case), case["n"], case["page"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    u = torch.randn((hkv, d), generator=gen, device="cuda")
    u /= u.norm(dim=1, keepdim=True)
    s = dict(kind=kind, n=n, hq=hq, tokens=case.get("tokens", 0), slots=_ints(list(range(n))), status=_ints([0]))
    parts = sum(-(-S // page) for S in lens)

    def queries(tokens):
        q = torch.randn((n * tokens, hkv, hq // hkv, d), generator=gen, device="cuda")
        q += (0.35 * math.sqrt(d)) * u[None, :, None, :]
        s["q"] = q.reshape(n, tokens, hq, d).to(torch.bfloat16)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((n, tokens, hq), dtype=torch.float32, device="cuda")

    if kind == "attend":
        pad = min(case.get("pad", 0), n)
        s["pool"] = _Pool(case, lens, n, 1 + n // 8, max(lens), gen)
        _fill(s["pool"], lens, gen, u)
        s["slots"] = _ints(list(range(n - pad)) + [-1] * pad)
        s["max_len"] = max(lens)
        queries(case["tokens"])
    elif kind == "store":
        # what the cache holds already has been put there; the new rows' pages are reserved
        base = case["base"]
        keeps = _keeps(case, lens)
        held = [base + k for k in keeps]
        s["pool"] = _Pool(case, held, n, 1 + n // 8, max(held), gen)
        if base:
            _fill(s["pool"], [base] * n, gen, u)
        off, koff = _offsets(lens), _offsets(keeps)
        s["k"], s["v"] = _rows(gen, off[-1], hkv, d, u, 3.0), _rows(gen, off[-1], hkv, d, u, 0.0)
        s["row_idx"] = _choose(gen, lens, keeps) if case["keep"] < 100 else None
        s["offsets"], s["start"], s["max_new"] = _ints(koff), _ints([base] * n), max(keeps)
        s["read_off"], s["max_len"], total = _ints(_offsets(held)), max(held), sum(held)
        s["k_out"] = torch.empty((total, hkv, d), dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.empty_like(s["k_out"])
    elif kind == "step":
        t = case["tokens"]
        s["pool"] = _Pool(case, lens, 2 * n, sum(-(-(S + t) // page) - S // page for S in lens) + 1 + n // 4, max(lens) + t, gen)
        _fill(s["pool"], lens, gen, u)
        s["children"], s["n_new"], s["start"] = _ints(list(range(n, 2 * n))), _ints([t] * n), _ints([0] * n)
        s["k"], s["v"] = _rows(gen, n * t, hkv, d, u, 3.0), _rows(gen, n * t, hkv, d, u, 0.0)
        s["offsets"], s["max_new"], s["max_len"] = _ints(_offsets([t] * n)), t, max(lens) + t
        queries(t)
    elif kind == "evict":
        keeps = _keeps(case, lens)
        s["pool"] = _Pool(case, lens, 2 * n, sum(-(-k // page) for k in keeps) + n + 1, max(lens), gen)
        _fill(s["pool"], lens, gen, u)
        s["children"] = _ints(list(range(n, 2 * n)))
        s["kept"], s["offsets"], s["koffsets"] = _choose(gen, lens, keeps), _ints(_offsets(lens)), _ints(_offsets(keeps))
        s["max_keep"] = max(keeps)
        s["k_out"] = torch.empty((sum(keeps), hkv, d), dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.empty_like(s["k_out"])
    else:
        # as many slots again hold sequences of the same lengths that stay; (a small head: no page's bytes are touched)
        s["pool"] = _Pool(dict(case, hkv=1, d=64, page=page), lens + lens, 2 * n, 1 + parts // 8, max(lens), gen)
        s["n_new"], s["start"] = _ints(lens), _ints([0] * n)
    return s


def _choose(gen, lens, keeps):
    """keeps[b] rows of every sequence, ascending, as row numbers of the packed batch."""
    chosen, at = [], 0
    for S, k in zip(lens, keeps):
        chosen.append(torch.randperm(S, generator=gen, device="cuda")[:k].sort().values.to(torch.int32) + at)
        at += S
    return torch.cat(chosen)


# ------------------------------------------------------------------------------------------------ the plain form
def _unpack_codes(tiles, d):
    """[..., 34 * d] bytes -> codes of K and V [..., 32, d] and scale bytes [..., 32, d / 32]"""
    lead, nb = tiles.shape[:-1], d // 32
    dims = tuple(range(len(lead)))
    m = len(lead)

    def nibbles(x):
        return torch.stack((x & 15, x >> 4), dim=-1)

    k = nibbles(tiles[..., :16 * d].reshape(*lead, 2, nb, 16, 16))                     # half block token byte nibble
    k = k.permute(*dims, m, m + 2, m + 1, m + 3, m + 4).reshape(*lead, 32, d)
    v = nibbles(tiles[..., 16 * d:32 * d].reshape(*lead, d // 64, 4, 16, 2, 2, 2, 2))  # h j r p q byte/2 byte%2 nibble
    v = v.permute(*dims, m + 5, m + 1, m + 6, m + 7, m, m + 3, m + 2, m + 4).reshape(*lead, 32, d)
    ks = tiles[..., 32 * d:33 * d].reshape(*lead, nb, 16, 2).permute(*dims, m + 2, m + 1, m).reshape(*lead, 32, nb)
    vs = tiles[..., 33 * d:].reshape(*lead, 4, nb, 2, 4).permute(*dims, m + 2, m, m + 3, m + 1).reshape(*lead, 32, nb)
    return k, v, ks, vs


def _pack_codes(k, v, ks, vs):
    lead, d = k.shape[:-2], k.shape[-1]
    nb, m, dims = d // 32, len(k.shape) - 2, tuple(range(len(k.shape) - 2))
    k = k.reshape(*lead, 2, 16, nb, 16, 2).permute(*dims, m, m + 2, m + 1, m + 3, m + 4)
    v = v.reshape(*lead, 2, 4, 2, 2, d // 64, 2, 16, 2).permute(*dims, m + 4, m + 1, m + 6, m + 5, m + 7, m, m + 2, m + 3)
    ks = ks.reshape(*lead, 2, 16, nb).permute(*dims, m + 2, m + 1, m)
    vs = vs.reshape(*lead, 2, 4, 4, nb).permute(*dims, m + 1, m + 3, m, m + 2)
    return torch.cat([(k[..., 0] | k[..., 1] << 4).reshape(*lead, 16 * d), (v[..., 0] | v[..., 1] << 4).reshape(*lead, 16 * d),
                      ks.reshape(*lead, d), vs.reshape(*lead, d)], dim=-1)


def _powers(e):
    """2^(e - 127) in fp32 for e in 1 .. 254, by its bits"""
    return (e.int() << 23).view(torch.float32)


def _values(codes, scales):
    """fp32 values of codes [..., d] with scale bytes [..., d / 32]"""
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float32, device=codes.device)
    power = _powers(torch.arange(256, device=codes.device))
    power[0], power[255] = 2.0 ** -127, math.nan
    x = grid[codes.int()].unflatten(-1, (-1, 32)) * power[scales.int()].unsqueeze(-1)
    return x.flatten(-2)


def _quantise(x):
    """bf16 [..., d] -> codes uint8 [..., d], scale bytes uint8 [..., d / 32].  The power of two is the smallest that brings the block's
    largest magnitude to 7 or less (7 is rounded to 6, the largest value), between 2^-126 and 2^125; the nearest value, ties to the even
    code."""
    b = x.float().unflatten(-1, (-1, 32))
    top = b.abs().amax(dim=-1)
    bits = top.view(torch.int32)
    e = ((bits >> 23) - 2 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(1, 252)
    bad = ~torch.isfinite(b).all(dim=-1)
    y = b * _powers(254 - e).unsqueeze(-1)
    m = y.abs()
    code = ((m > 0.25).int() + (m >= 0.75).int() + (m > 1.25).int() + (m >= 1.75).int() + (m > 2.5).int() + (m >= 3.5).int() + (m > 5.0).int())
    code = torch.where(torch.signbit(b), code + 8, code)
    code = torch.where(bad.unsqueeze(-1), torch.zeros_like(code), code)
    return code.to(torch.uint8).flatten(-2), torch.where(bad, torch.full_like(e, 255), e).to(torch.uint8)


def _plain_store(pool, k, v, row_idx, offsets, slots, start, max_new):
    """Tokens start[b] .. of slots[b] become the quantised rows offsets[b] .. offsets[b + 1] - 1 (of row_idx)."""
    off, slot, start = offsets.long(), slots.long(), start.long()
    count = off[1:] - off[:-1]
    tile = start[:, None] // 32 + torch.arange((max_new + 31) // 32 + 1, device="cuda")        # [n, tiles] of a slot
    token = tile[:, :, None] * 32 + torch.arange(32, device="cuda")                            # [n, tiles, 32]
    mine = (token >= start[:, None, None]) & (token < (start + count)[:, None, None])
    b, c = torch.nonzero(mine.any(dim=2), as_tuple=True)
    tile, token, mine = tile[b, c], token[b, c], mine[b, c]
    at = (pool.table[slot[b], tile // pool.tiles].long(), tile % pool.tiles)
    row = (off[b] - start[b])[:, None] + token
    row = torch.where(mine, row, torch.zeros_like(row))
    row = row if row_idx is None else row_idx[row].long()
    old = _unpack_codes(pool.pages[at[0], :, at[1]], pool.d)
    new = _quantise(k[row].permute(0, 2, 1, 3)), _quantise(v[row].permute(0, 2, 1, 3))          # [tiles, hkv, 32, .]
    new = new[0][0], new[1][0], new[0][1], new[1][1]
    pool.pages[at[0], :, at[1]] = _pack_codes(*(torch.where(mine[:, None, :, None], x, y) for x, y in zip(new, old)))


def _plain_read(pool, slots, tokens):
    """K and V in fp32 [n, hkv, tokens rounded up to pages, d] of slots, tokens that a slot does not hold are zero; the lengths [n]"""
    slot = slots.long()
    held = torch.where(slot >= 0, pool.lens[slot.clamp(min=0)].long(), torch.zeros_like(slot))
    table = pool.table[slot.clamp(min=0), :max(1, -(-tokens // pool.page))].long()
    codes = _unpack_codes(pool.pages[table.clamp(min=0)], pool.d)                               # [n, pages, hkv, tiles, 32, .]
    codes = [x.permute(0, 2, 1, 3, 4, 5).flatten(2, 4) for x in codes]
    there = (torch.arange(codes[0].shape[2], device="cuda") < held[:, None])[:, None, :, None]
    k, v = _values(codes[0], codes[2]), _values(codes[1], codes[3])
    zero = torch.zeros((), device="cuda")
    return torch.where(there, k, zero), torch.where(there, v, zero), held


def _plain_load(s, slots, offsets, max_len):
    k, v, held = _plain_read(s["pool"], slots, max_len)
    there = torch.arange(k.shape[2], device="cuda") < torch.minimum(held, (offsets[1:] - offsets[:-1]).long())[:, None]
    b, t = torch.nonzero(there, as_tuple=True)
    row = offsets.long()[b] + t
    s["k_out"][row] = k[b, :, t].to(torch.bfloat16)
    s["v_out"][row] = v[b, :, t].to(torch.bfloat16)


def _plain_attend(s, slots):
    q, (n, tokens, hq, d) = s["q"].float(), s["q"].shape
    k, v, held = _plain_read(s["pool"], slots, s["max_len"])
    hkv = k.shape[1]
    q = q.reshape(n, tokens, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(n * hkv, -1, d)
    x = torch.bmm(q, k.flatten(0, 1).transpose(1, 2).contiguous()) / math.sqrt(d)
    x = x.reshape(n, hq, tokens, -1)
    seen = held[:, None] - tokens + 1 + torch.arange(tokens, device="cuda")                     # [n, tokens] keys that a token sees
    x = x.masked_fill(torch.arange(x.shape[3], device="cuda") >= seen[:, None, :, None], -math.inf)
    top = x.amax(dim=3, keepdim=True)
    p = torch.exp(x - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = p.sum(dim=3, keepdim=True)
    out = torch.bmm(p.reshape(n * hkv, -1, p.shape[3]), v.flatten(0, 1)).reshape(n, hq, tokens, d)
    out = out / torch.where(total > 0, total, torch.ones_like(total))
    s["out"].copy_(out.permute(0, 2, 1, 3).to(torch.bfloat16))
    s["lse"].copy_(((top + torch.log(total)) / math.log(2.0))[..., 0].permute(0, 2, 1))


def _free_pages(pool, ranks):
    """The free pages of these ranks, the lowest page first; n_pages where there are not so many."""
    return torch.searchsorted(torch.cumsum((pool.refs == 0).int(), 0), ranks + 1)


def _plain_grow(pool, slots, before, after, ok_extra=None):
    """Pages before[b] .. after[b] - 1 of the table's rows become fresh ones, in the order of the rows; how many are lacking (then nothing is done)."""
    fresh = after - before
    first = torch.cumsum(fresh, 0) - fresh
    lacking = (fresh.sum() - (pool.refs == 0).sum()).clamp(min=0)
    at = torch.arange(pool.max_pages, device="cuda")
    mine = (at >= before[:, None]) & (at < after[:, None]) & (lacking == 0)
    page = _free_pages(pool, torch.where(mine, first[:, None] + at - before[:, None], torch.zeros_like(mine, dtype=torch.long)))
    pool.table[slots] = torch.where(mine, page.int(), pool.table[slots])
    pool.refs.index_add_(0, page.flatten().clamp(max=pool.n_pages - 1), mine.flatten().int())
    return lacking


def _plain_reserve(s, slots):
    pool, slot, new = s["pool"], slots.long(), s["n_new"].long()
    old = pool.lens[slot].long()
    lacking = _plain_grow(pool, slot, -(-old // pool.page), -(-(old + new) // pool.page))
    s["start"].copy_(torch.where(lacking == 0, old, torch.full_like(old, -1)))
    pool.lens[slot] = torch.where(lacking == 0, old + new, old).int()
    s["status"].copy_(lacking.reshape(1))


def _plain_release(pool, slots):
    slot = slots.long()
    rows = pool.table[slot]
    held = torch.arange(pool.max_pages, device="cuda") < (-(-pool.lens[slot] // pool.page))[:, None]
    pool.refs.index_add_(0, rows.clamp(min=0).flatten().long(), -held.flatten().int())
    pool.table[slot] = torch.where(held, torch.full_like(rows, -1), rows)
    pool.lens[slot] = 0


def _plain_fork(s, parents, children):
    pool, a, c = s["pool"], parents.long(), children.long()
    held = pool.lens[a].long()
    full, all_ = held // pool.page, -(-held // pool.page)
    lacking = _plain_grow(pool, c, full, all_)
    at = torch.arange(pool.max_pages, device="cuda")
    shared = (at < full[:, None]) & (lacking == 0)
    rows = pool.table[a]
    pool.table[c] = torch.where(shared, rows, pool.table[c])
    pool.refs.index_add_(0, rows.clamp(min=0).flatten().long(), shared.flatten().int())
    last = torch.nonzero((all_ > full) & (lacking == 0))[:, 0]
    pool.pages[pool.table[c[last], full[last]].long()] = pool.pages[pool.table[a[last], full[last]].long()]
    pool.lens[c] = torch.where(lacking == 0, held, torch.zeros_like(held)).int()
    s["status"].copy_(lacking.reshape(1))


def _plain_compact(s, slots):
    """Token j of a slot becomes its token kept[koffsets[b] + j] - offsets[b], in fresh pages; the old ones are given back."""
    pool, slot = s["pool"], slots.long()
    off, koff, page = s["offsets"].long(), s["koffsets"].long(), pool.page
    keep = koff[1:] - koff[:-1]
    old_rows = pool.table[slot].clone()
    old_pages = -(-pool.lens[slot].long() // page)
    lacking = _plain_grow(pool, slot, torch.zeros_like(keep), -(-keep // page))
    # the kept tokens' codes and scales [n, hkv, tokens rounded up to tiles, .], zero behind the last, go into the new pages tile by tile
    token = torch.arange(-(-s["max_keep"] // 32) * 32, device="cuda")
    there = token < keep[:, None]
    src = s["kept"][torch.where(there, koff[:-1, None] + token, torch.zeros_like(there, dtype=torch.long))].long()
    src = torch.where(there, src - off[:-1, None], torch.zeros_like(src))
    codes = _unpack_codes(pool.pages[old_rows.clamp(min=0).long()], pool.d)                     # [n, pages, hkv, tiles, 32, .]
    codes = [x.permute(0, 1, 3, 4, 2, 5).flatten(1, 3) for x in codes]                          # [n, tokens, hkv, .]
    each = torch.arange(len(slot), device="cuda")[:, None]
    codes = [torch.where(there[:, :, None, None], x[each, src], torch.zeros((), dtype=torch.uint8, device="cuda")) for x in codes]
    tiles = _pack_codes(*(x.unflatten(1, (-1, 32)).transpose(2, 3) for x in codes))             # [n, tiles, hkv, bytes]
    b, c = torch.nonzero(there[:, ::32] & (lacking == 0), as_tuple=True)
    pool.pages[pool.table[slot[b], c // pool.tiles].long(), :, c % pool.tiles] = tiles[b, c]
    at = torch.arange(pool.max_pages, device="cuda")
    gone = (at < old_pages[:, None]) & (lacking == 0)
    pool.refs.index_add_(0, old_rows.clamp(min=0).flatten().long(), -gone.flatten().int())
    rest = gone & (at >= (-(-keep // page))[:, None])
    pool.table[slot] = torch.where(rest, torch.full_like(old_rows, -1), pool.table[slot])
    pool.lens[slot] = torch.where(lacking == 0, keep, pool.lens[slot].long()).int()
    s["status"].copy_(lacking.reshape(1))


# ------------------------------------------------------------------------------------------------ a pass
def _handle(s, lib):
    """What a program makes once for its cache and keeps: the description of the cache, a workspace."""
    if "cache" not in s:
        p, size = s["pool"], 0
        s["cache"] = lib.make_cache(p.pages, p.refs, p.table, p.lens, p.page, p.hkv, p.d)
        if "q" in s:
            size = lib.cache_attention_workspace_bytes(s["cache"], s["n"], s["tokens"], s["hq"], s["max_len"])
        elif "max_keep" in s:
            size = lib.cache_compact_workspace_bytes(s["cache"], s["n"])
        s["ws_bytes"], s["ws"] = size, torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    return s["cache"]


def _run_own(s):
    from paper_2405_12532_amd import binding as lib
    cache, n, kind = _handle(s, lib), s["n"], s["kind"]
    who = s["slots"] if kind in ("attend", "store", "turn") else s["children"]
    if kind in ("step", "evict"):
        lib.cache_release(cache, who, n)
        lib.cache_fork(cache, s["slots"], who, n, s["status"])
    if kind == "turn":
        lib.cache_release(cache, who, n)
    if kind in ("step", "turn"):
        lib.cache_reserve(cache, who, s["n_new"], n, s["start"], s["status"])
    if kind in ("step", "store"):
        idx = s.get("row_idx")
        rows = s["k"].shape[0]
        lib.cache_store(cache, s["k"], s["v"], rows, idx, rows if idx is None else idx.shape[0], s["offsets"], who, s["start"], n, s["max_new"])
    if kind == "evict":
        lib.cache_compact(cache, who, n, s["kept"], s["kept"].shape[0], s["offsets"], s["koffsets"], s["max_keep"], s["status"], s["ws"], s["ws_bytes"])
        lib.cache_load(cache, who, s["koffsets"], n, s["max_keep"], s["k_out"], s["v_out"], s["k_out"].shape[0])
    if kind == "store":
        lib.cache_load(cache, who, s["read_off"], n, s["max_len"], s["k_out"], s["v_out"], s["k_out"].shape[0])
    if kind in ("attend", "step"):
        lib.cache_attention(cache, s["q"], who, n, s["tokens"], s["hq"], s["max_len"], 0.0, s["out"], s["lse"], s["ws"], s["ws_bytes"])


def _run_plain(s):
    pool, kind = s["pool"], s["kind"]
    who = s["slots"] if kind in ("attend", "store", "turn") else s["children"]
    if kind in ("step", "evict"):
        _plain_release(pool, who)
        _plain_fork(s, s["slots"], who)
    if kind == "turn":
        _plain_release(pool, who)
    if kind in ("step", "turn"):
        _plain_reserve(s, who)
    if kind in ("step", "store"):
        _plain_store(pool, s["k"], s["v"], s.get("row_idx"), s["offsets"], who, s["start"], s["max_new"])
    if kind == "evict":
        _plain_compact(s, who)
        _plain_load(s, who, s["koffsets"], s["max_keep"])
    if kind == "store":
        _plain_load(s, who, s["read_off"], s["max_len"])
    if kind in ("attend", "step"):
        _plain_attend(s, who)


def run(s):
    if own:
        _run_own(s)
    else:
        _run_plain(s)
    kind, pool = s["kind"], s["pool"]
    r = {}
    if kind in ("attend", "step"):
        r.update(out=s["out"], lse=s["lse"])
    if kind in ("store", "evict"):
        r.update(k=s["k_out"], v=s["v_out"])
    if kind in ("step", "evict", "turn"):
        r.update(table=pool.table, refs=pool.refs, lens=pool.lens, status=s["status"])
    if kind in ("step", "turn"):
        r.update(start=s["start"])
    return r


def work(case):
    lens, kind, page = _lengths(case), case["kind"], case["page"]
    hq, hkv, d, t = case["hq"], case["hkv"], case["d"], case.get("tokens", 0)
    token4, token16 = hkv * d * 34 // 32, hkv * d * 4                                          # bytes of a token, K and V
    n, entries = case["n"], sum(-(-S // page) for S in lens)
    branch = 2 * token4 * sum(S % page for S in lens) + 16 * entries                            # fork: the last page's tokens, the rows' entries and counts
    if kind == "attend":
        live = lens[:n - min(case.get("pad", 0), n)]
        return dict(bytes=sum(live) * token4 + 4 * n * t * hq * (d + 1) + 4 * entries, flops=4.0 * d * hq * t * sum(live))
    if kind == "store":
        keeps = _keeps(case, lens)
        rows = sum(keeps) + n * case["base"]
        return dict(bytes=sum(keeps) * (token16 + token4) + rows * (token4 + token16) + (4 * sum(keeps) if case["keep"] < 100 else 0), flops=0)
    if kind == "step":
        total = sum(lens) + n * t
        return dict(bytes=branch + total * token4 + n * t * (token16 + token4) + 4 * n * t * hq * (d + 1), flops=4.0 * d * hq * t * total)
    if kind == "evict":
        kept = sum(_keeps(case, lens))
        return dict(bytes=branch + kept * (3 * token4 + token16 + 4), flops=0)
    return dict(bytes=40 * entries + 24 * n, flops=0)                                           # given back and handed out: entries and counts, read and written


# ------------------------------------------------------------------------------------------------ 64 bits
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_powers(e):
    return (e.long() + 1023 << 52).view(torch.float64)


def _exact_rows(x):
    """The values that bf16 rows [rows, hkv, d] have in the cache: the nearest points of the block's grid, in 64 bits."""
    x = x.double().unflatten(-1, (-1, 32))
    part, e = torch.frexp(x.abs().amax(dim=-1, keepdim=True))                                                # part in [1/2, 1): 7 is 7/8 * 2^3
    step = _exact_powers((e - torch.where(part > 0.875, 2, 3)).clamp(-126, 125))
    m = x.abs() / step
    best, gap = torch.zeros_like(m), m.clone()
    for i, g in enumerate(_GRID[1:], 1):
        closer = ((m - g).abs() < gap) | (((m - g).abs() == gap) & (i % 2 == 0))
        best, gap = torch.where(closer, torch.full_like(m, g), best), torch.minimum((m - g).abs(), gap)
    return (torch.copysign(best, x) * step).flatten(-2)


def _exact_held(pool, b, count):
    """K and V [tokens, hkv, d] in 64 bits of a slot's first tokens, byte by byte from the pages' description."""
    d, dev = pool.d, "cuda"
    t = torch.arange(count, device=dev)
    base = pool.table[b].long()[t // pool.page] * pool.hkv * pool.tiles + (t % pool.page) // 32
    base = (base[:, None] + torch.arange(pool.hkv, device=dev) * pool.tiles)[:, :, None] * (34 * d)         # [tokens, hkv, 1]
    i, c, flat = (t % 32)[:, None, None], torch.arange(d, device=dev), pool.pages.flatten()
    half, low, j = i // 16, i % 16, i % 16 // 4
    kbyte = base + ((half * (d // 32) + c // 32) * 16 + low) * 16 + c % 32 // 2
    vword = ((c // 64 * 4 + j) * 16 + c % 32 // 2) * 4 + c % 64 // 32 * 2 + c % 2
    vbyte = base + 16 * d + vword * 4 + half * 2 + i % 4 // 2
    kscale, vscale = base + 32 * d + (c // 32 * 16 + low) * 2 + half, base + 33 * d + ((j * (d // 32) + c // 32) * 2 + half) * 4 + i % 4
    grid = torch.tensor(_GRID, dtype=torch.float64, device=dev)

    def value(byte, high, scale):
        code = flat[byte].long() >> (4 * high) & 15
        return torch.where(code >= 8, -1.0, 1.0) * grid[code % 8] * _exact_powers(flat[scale].long() - 127)
    return value(kbyte, c % 2, kscale), value(vbyte, i % 2, vscale)


def _exact_attend(s, b, k, v, out, lse):
    q = s["q"][b].double()                                                                                   # [tokens, hq, d]
    tokens, hq, d = q.shape
    S, hkv = k.shape[0], k.shape[1]
    qh = q.reshape(tokens, hkv, hq // hkv, d).permute(1, 2, 0, 3).reshape(hkv, -1, d)
    x = torch.bmm(qh, k.permute(1, 2, 0).contiguous()).reshape(hq, tokens, S) / math.sqrt(d)
    x.masked_fill_(torch.arange(S, device="cuda") > torch.arange(S - tokens, S, device="cuda")[:, None], -math.inf)
    norm = torch.logsumexp(x, dim=2, keepdim=True)
    p = torch.where(norm > -math.inf, torch.exp(x - norm), torch.zeros_like(x)).reshape(hkv, -1, S)
    out[b] = torch.bmm(p, v.permute(1, 0, 2).contiguous()).reshape(hq, tokens, d).permute(1, 0, 2)
    lse[b] = norm[..., 0].t() / math.log(2.0)


def exact(case, seed):
    kind, lens = case["kind"], _lengths(case)
    if kind == "turn":
        return None
    s = prepare(case, seed)
    pool, n = s["pool"], case["n"]
    none = dict(table=None, refs=None, lens=None, status=None)
    if kind in ("attend", "step"):
        out, lse = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda"), torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
        for b in range(n - (min(case.get("pad", 0), n) if kind == "attend" else 0)):
            k, v = _exact_held(pool, b, lens[b])
            if kind == "step":
                t = case["tokens"]
                k, v = torch.cat([k, _exact_rows(s["k"][b * t:b * t + t])]), torch.cat([v, _exact_rows(s["v"][b * t:b * t + t])])
            _exact_attend(s, b, k, v, out, lse)
        return dict(out=out, lse=lse) if kind == "attend" else dict(out=out, lse=lse, start=None, **none)
    ks, vs = [], []
    keeps = _keeps(case, lens)
    off, koff = _offsets(lens), _offsets(keeps)
    for b in range(n):
        if kind == "store":
            rows = torch.arange(off[b], off[b + 1], device="cuda") if s["row_idx"] is None else s["row_idx"][koff[b]:koff[b + 1]].long()
            k, v = _exact_rows(s["k"][rows]), _exact_rows(s["v"][rows])
            if case["base"]:
                before = _exact_held(pool, b, case["base"])
                k, v = torch.cat([before[0], k]), torch.cat([before[1], v])
        else:
            at = s["kept"][koff[b]:koff[b + 1]].long() - off[b]
            k, v = (x[at] for x in _exact_held(pool, b, lens[b]))
        ks.append(k)
        vs.append(v)
    r = dict(k=torch.cat(ks), v=torch.cat(vs))
    return r if kind == "store" else dict(r, **none)
