"""Attention over the cache held in 8 bits within what its roundings leave, close enough that every block of V shows.

With u = 2^-24, logits x in base e: a product's operands are exact, so |dx| <= (d + 4) u * scale * |q|.|k|, and a weight is off by |dx| + 2^-20 (exp2, its argument's
rounding, 2^-23 |x|) on either side of the quotient.  P is two bf16 numbers, each the nearest one: off by 2^-8 * 2^-8.  A block of V goes into O by two matrix
instructions of 32 products, 66 sums of fp32, each rounded by u (2 u, should it be cut off) of what is there: what the wavefront's blocks have added up to, and the block's p |v| at most.
Wavefronts and parts are added up likewise.  The output is rounded to bf16, by 2^-8."""
import numpy as np


def weights(q, k, blocks=None):
    """q float64 [tokens, hq, d], k [S, hkv, d], blocks [tokens, hkv, n] or None -> softmax weights [tokens, hq, S], lse (base 2), |q|.|k| at most"""
    tokens, hq, d = q.shape
    S, hkv = k.shape[:2]
    g = hq // hkv
    x, size = np.empty((tokens, hq, S)), np.empty((tokens, hq))
    for h in range(hq):
        x[:, h] = q[:, h] @ k[:, h // g].T / np.sqrt(d)
        size[:, h] = (np.abs(q[:, h]) @ np.abs(k[:, h // g]).T / np.sqrt(d)).max(axis=1)
    seen = np.arange(S) <= (S - tokens + np.arange(tokens))[:, None]
    times = np.repeat(seen[:, None], hq, axis=1).astype(np.float64)
    if blocks is not None:
        for i in range(tokens):
            for h in range(hq):
                mine = blocks[i, h // g]
                count = np.bincount(mine[(mine >= 0) & (mine < -(-S // 32))], minlength=-(-S // 32))
                times[i, h] *= np.repeat(count, 32)[:S]
    top = np.where(times > 0, x, -np.inf).max(axis=2, keepdims=True)
    p = np.where(times > 0, np.exp(x - top), 0) * times
    total = p.sum(axis=2, keepdims=True)
    return p / total, ((top + np.log(total)) / np.log(2))[..., 0], size


def of_blocks(p, v):
    """What every block adds to the output, and the sum of its p |v|: [tokens, hq, blocks, d]"""
    n, g = -(-len(v) // 32), p.shape[1] // v.shape[1]
    p = np.pad(p, ((0, 0), (0, 0), (0, 32 * n - len(v)))).reshape(*p.shape[:2], n, 32)
    v = np.pad(v, ((0, 32 * n - len(v)), (0, 0), (0, 0))).reshape(n, 32, *v.shape[1:])
    return [np.stack([(p[:, h, :, None] @ y[:, :, h // g])[:, :, 0] for h in range(p.shape[1])], axis=1) for y in (v, np.abs(v))]


def bounds(p, lse, size, v, route, blocks=None):
    """The output, how far it may be off, and lse; route: how the call is cut up."""
    parts, all_parts = of_blocks(p, v)
    tokens, hq, n, d = parts.shape
    g, sums = hq // v.shape[1], np.zeros((tokens, hq, d))
    for i in range(tokens):
        for h in range(hq):
            order = np.arange(n) if blocks is None else blocks[i, h // g][blocks[i, h // g] < n]
            for first in range(0, len(order), route.chunk):
                for w in range(route.waves):
                    mine = order[first:first + route.chunk][w::route.waves]
                    sums[i, h] += (np.abs(np.cumsum(parts[i, h, mine], axis=0)) + all_parts[i, h, mine]).sum(axis=0)
    dx = (d + 4) * 2.0 ** -24 * size + 2.0 ** -20 + 2.0 ** -23 * size
    joins = (route.waves + route.splits + 16) * 2.0 ** -23
    ref = parts.sum(axis=2)
    off = (2.0 ** -16 + joins + 2 * dx[..., None]) * all_parts.sum(axis=2) + 66 * 2.0 ** -23 * sums + 2.0 ** -8 * np.abs(ref)
    # (a sum of weights: 16 roundings a block, of what is there)
    return ref, off * 1.01 + 1e-30, 2 * dx + 2.0 ** -22 * np.abs(lse) + (16 * -(-route.chunk // route.waves)) * 2.0 ** -24 + joins


# lengths, rows of the call (slots), query heads, KV heads, channels, tokens, blocks of a list (0: none).  Short ones; split along the cache, into more parts than a join takes at
# once; wavefronts with more than 64 blocks, by eight and by four, of one and of two groups of 16 rows; lists likewise.
CASES = [([100, 33, 64], [2, 0, 1], 8, 2, 128, 3, 0), ([300, 129], [0, 1], 12, 1, 64, 3, 0), ([5000, 1, 700], [0, 1, 2], 4, 2, 128, 1, 0), ([4097, 4096], [1, 0], 8, 1, 64, 3, 0),
         ([9000], [0], 2, 1, 64, 1, 0), ([3000, 2999], [0, 1], 24, 1, 128, 2, 0), ([9000], [0], 2, 1, 128, 1, 0), ([20000], [0], 2, 1, 64, 1, 0), ([20000], [0] * 130, 2, 1, 64, 1, 0),
         ([9000], [0] * 256, 2, 1, 128, 1, 0), ([9000], [0] * 130, 20, 1, 64, 1, 0), ([700, 300], [0, 1], 8, 2, 128, 2, 9), ([9000], [0], 4, 2, 64, 1, 200), ([20000], [0] * 130, 2, 1, 64, 1, 600),
         ([9000], [0] * 64, 20, 1, 128, 4, 280)]


def inputs(make, case):
    """make: as Pair8 -> pair, q float64 of bf16 numbers, lists or None, the rows that are looked at"""
    lens, slots, hq, hkv, d, tokens, width = case
    pair = make(lens, hkv, d, seed=len(slots) + hq, powers=(120, 121))
    q = (pair.rng.normal(size=(len(slots), tokens, hq, d)) * 0.5).astype(np.float32)
    q = (np.round(q.view(np.uint32) / 65536).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    lists = None
    if width:
        lists = np.stack([[[pair.rng.permutation(max(width, -(-lens[s] // 32)))[:width] for _ in range(hkv)] for _ in range(tokens)] for s in slots]).astype(np.int32)
    rows = range(len(slots)) if len(slots) < 4 else (0, len(slots) // 2, len(slots) - 1)
    return pair, q, lists, rows
