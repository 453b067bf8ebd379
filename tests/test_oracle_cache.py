"""Pins of the oracle of the cache held in 4 bits: exhaustive nearest numbers, the layout as a bijection, attention by the prefill oracle."""
import itertools

import numpy as np
import pytest

from oracle import cache_oracle as orc
from oracle import pyr_oracle


def test_quantise_is_the_nearest_number_of_the_grid():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(40, 32)) * 2.0 ** rng.integers(-20, 20, (40, 1))
    codes, scales = orc.quantise(x)
    got = orc.values(codes, scales)
    for row, e, y in zip(x, scales[:, 0].astype(int) - 127, got):
        grid = np.concatenate([orc.GRID, -orc.GRID]) * 2.0 ** e
        assert np.abs(row).max() <= 7 * 2.0 ** e and np.abs(row).max() > 3.5 * 2.0 ** e       # the smallest that holds it
        for a, b in zip(row, y):
            assert abs(a - b) == np.abs(grid - a).min()


def test_quantise_ties_borders_and_numbers_that_are_none():
    block = np.zeros(32)
    block[:15] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -1.25, -2.5, -5, 0.0, -0.0]
    codes, scales = orc.quantise(block)
    assert scales.tolist() == [127]
    assert orc.values(codes, scales)[:15].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, -0.0, -1, -1, -2, -4, 0.0, -0.0]
    for top, scale in ((7.0, 127), (7.03125, 128), (3.5, 126), (3.515625, 127), (0.0, 1), (2.0 ** -130, 1), (3.38e38, 252)):
        assert orc.quantise(np.full(32, top))[1].tolist() == [scale], top
    for bad in (np.inf, -np.inf, np.nan):
        block[7] = bad
        codes, scales = orc.quantise(np.concatenate([block, np.ones(32)]))
        assert scales.tolist() == [255, 125] and not codes[:32].any()
        assert np.isnan(orc.values(codes, scales)[:32]).all() and (orc.values(codes, scales)[32:] == 1).all()


def test_quantising_the_cache_again_changes_nothing():
    rng = np.random.default_rng(1)
    once = orc.values(*orc.quantise(rng.normal(size=(64, 64))))
    assert np.array_equal(orc.values(*orc.quantise(once)), once)


@pytest.mark.parametrize("d", [64, 128])
def test_every_bit_of_a_tile_has_one_place(d):
    kb, vb, ks, vs = orc.tile_places(d)
    halves = [tuple(p) for p in itertools.chain(kb.reshape(-1, 2), vb.reshape(-1, 2))]
    assert sorted(halves) == [(b, h) for b in range(32 * d) for h in range(2)]
    assert sorted(itertools.chain(ks.ravel(), vs.ravel())) == list(range(32 * d, 34 * d))


def test_a_token_comes_back_and_leaves_its_neighbours_alone():
    rng = np.random.default_rng(2)
    c = orc.Cache(3, 64, 2, 3, 2, 64, fill=0xA5)
    c.refs[1], c.table[0, 0], c.lens[0] = 1, 1, 64
    before = c.read(0)
    k, v = rng.normal(size=(2, 1, 2, 64))
    c.store(k, v, None, [0, 1], [0], [37])
    after = c.read(0)
    for old, new, x in zip(before, after, (k, v)):
        assert np.array_equal(new[37], orc.values(*orc.quantise(x[0])))
        assert np.array_equal(np.delete(new, 37, 0), np.delete(old, 37, 0))


def test_attention_is_the_prefill_oracles_on_the_last_rows():
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(20, 4, 64)), rng.normal(size=(20, 2, 64)), rng.normal(size=(20, 2, 64))
    out, lse = orc.attention(q[17:], k, v)
    ref = pyr_oracle.causal_attention(q, k, v)
    ref = ref[0] if isinstance(ref, tuple) else ref
    assert np.allclose(out, ref[17:], atol=1e-12)
    short = orc.attention(q[17:], k[:1], v[:1])                 # three tokens, one of them in the cache
    assert not short[0][:2].any() and np.isneginf(short[1][:2]).all() and np.allclose(short[0][2], np.repeat(v[0], 2, axis=0))


def test_pages_are_shared_counted_and_given_back():
    c = orc.Cache(8, 32, 4, 4, 1, 64)
    start, status = c.reserve([0, -1, 1], [70, 5, 32])
    assert status == 0 and start.tolist() == [0, -1, 0] and c.table[0].tolist() == [0, 1, 2, -1] and c.table[1, 0] == 3
    assert c.fork([0, 0], [2, 3]) == 0
    assert c.refs.tolist() == [3, 3, 1, 1, 1, 1, 0, 0] and c.table[2].tolist() == [0, 1, 4, -1]
    assert c.reserve([1, 2], [65, 58])[1] == 2 and c.lens.tolist() == [70, 32, 70, 70]       # 3 and 1 pages, 2 are free: nothing happens
    c.release([0, 0, 7, -1])
    assert c.refs.tolist() == [2, 2, 0, 1, 1, 1, 0, 0] and c.lens[0] == 0
    assert c.compact([2], np.array([69, 3, 3]) + 100, [100], [0, 3], 3) == 0
    assert c.table[2].tolist() == [2, -1, -1, -1] and c.refs.tolist() == [1, 1, 1, 1, 0, 1, 0, 0]
    assert c.fork([1], [1]) == -1 and c.fork([2], [1]) == -1 and c.reserve([0, 0], [1, 1])[1] == -1 and c.reserve([0], [129])[1] == -2
