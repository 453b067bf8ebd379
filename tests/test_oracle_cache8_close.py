"""The bounds that the attention over the cache held in 8 bits is compared within: no block of V that a row attends to could be left out, or have its tokens in another order,
and stay inside them."""
import numpy as np
import pytest

from tests import close8

torch = pytest.importorskip("torch")
from paper_2405_12532_amd import binding  # noqa: E402
from tests.caches8 import Pair8  # noqa: E402


class OnHost(Pair8):
    def up(self):
        pass


@pytest.mark.parametrize("case", close8.CASES)
def test_every_block_of_v_shows(case):
    lens, slots, hq, hkv, d, tokens, width = case
    pair, q, lists, rows = close8.inputs(lambda *a, **k: OnHost(None, *a, **k), case)
    o = pair.o
    cache = binding.PyrCache8(binding.PyrCache(n_pages=len(o.refs), page_tokens=o.page, n_slots=len(o.lens), max_pages=o.table.shape[1], n_kv_heads=hkv, head_dim=d))
    route = binding.diag_cache8_attention(cache, len(slots), tokens, hq, max(lens), width)
    reads = {s: o.read(s) for s in set(slots)}
    for b in rows:
        k, v = reads[slots[b]]
        p, lse, size = close8.weights(q[b], k, None if lists is None else lists[b])
        _, off, _ = close8.bounds(p, lse, size, v, route, None if lists is None else lists[b])
        lost, _ = close8.of_blocks(p, v)
        n = lost.shape[2]
        turned = np.pad(v, ((0, 32 * n - len(v)), (0, 0), (0, 0)))
        for c in range(n):
            mine = slice(32 * c, min(32 * c + 32, len(v)))
            turned[mine] = v[mine][::-1]
        turned = lost - close8.of_blocks(p, turned[:len(v)])[0]
        there = close8.of_blocks(p, np.ones_like(v))[0].reshape(tokens, hkv, -1, n, d)[..., 0].any(axis=(0, 2))      # [hkv, blocks] that a row attends to
        for change, held in ((lost, 1), (turned, 2)):
            shows = (np.abs(change) > 2 * off[:, :, None]).reshape(tokens, hkv, -1, n, d).any(axis=(0, 2, 4))
            alone = np.arange(n) * 32 + held > len(v)                              # (one token in any order)
            assert (shows | ~there | alone).all(), (b, held, np.argwhere(~(shows | ~there | alone))[:5])
