"""Attention over the cache held in 8 bits within bounds that a lost or misplaced block of V would leave (which the tests of the bounds themselves show, on the host)."""
import numpy as np
import pytest

from tests import close8

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests.caches8 import Pair8, attend, dev  # noqa: E402


@pytest.mark.parametrize("case", close8.CASES)
def test_attention_keeps_to_its_roundings(lib, case):
    lens, slots, hq, hkv, d, tokens, width = case
    pair, q, lists, rows = close8.inputs(lambda *a, **k: Pair8(lib, *a, **k), case)
    qt = torch.from_numpy(q).to(torch.bfloat16).cuda()
    assert np.array_equal(qt.double().cpu().numpy(), q)
    out, lse = attend(pair, qt, slots, tokens, max(lens), None if lists is None else dev(lists))
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    route = lib.diag_cache8_attention(pair.cache, len(slots), tokens, hq, max(lens), width)
    reads = {s: pair.o.read(s) for s in set(slots)}
    for b in rows:
        k, v = reads[slots[b]]
        p, ref_lse, size = close8.weights(q[b], k, None if lists is None else lists[b])
        ref, off, lse_off = close8.bounds(p, ref_lse, size, v, route, None if lists is None else lists[b])
        assert (np.abs(out[b] - ref) <= off).all(), (b, (np.abs(out[b] - ref) / off).max())
        assert (np.abs(lse[b] - ref_lse) <= lse_off).all(), b
