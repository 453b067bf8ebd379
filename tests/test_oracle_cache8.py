"""Pins of the oracle of the cache held in 8 bits: nearest numbers, the layout as a bijection, turns, bounds, the choice of blocks."""

import numpy as np
import pytest

from oracle import cache8_oracle as orc
from oracle import cache_oracle


def test_codes_are_the_nearest_numbers():
    assert len(orc.GRID) == 127 and orc.GRID[-1] == 448 and orc.GRID[1] == 2.0 ** -9 and orc.GRID[8] == 2.0 ** -6
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(size=4000) * 2.0 ** rng.integers(-12, 9, 4000), orc.GRID, (orc.GRID[1:] + orc.GRID[:-1]) / 2, [464.0, 449.0]])
    x = np.concatenate([x, -x])
    x = x[np.abs(x) <= 464]
    got = orc.value(orc.encode(x))
    for a, b, code in zip(x, got, orc.encode(x)):
        gap = np.abs(np.concatenate([orc.GRID, -orc.GRID]) - a)
        assert abs(a - b) == gap.min()
        if (gap == gap.min()).sum() > 1 and a != 0 and abs(a) < 448:
            assert code % 2 == 0
    assert np.isnan(orc.value(orc.encode([464.1, np.inf, -np.inf, np.nan, 1e300]))).all()
    assert np.array_equal(orc.encode(orc.value(np.arange(127))), np.arange(127))




def test_torch_agrees_on_what_a_code_is():
    torch = pytest.importorskip("torch")
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(orc.value(codes.numpy()), want, equal_nan=True)


def test_the_power_is_the_smallest_that_holds_a_block():
    for top, e in ((448.0, 0), (448.1, 1), (224.0, -1), (0.0, -100), (2.0 ** -140, -100), (3.38e38, 119), (1.75 * 2.0 ** 127, 119)):
        assert orc.power(np.array([top, -top / 3])) == e, top
    assert orc.power(np.array([np.inf, np.nan, 7.0])) == orc.power(np.array([7.0])) and orc.power(np.array([np.nan])) == -100


@pytest.mark.parametrize("d", [64, 128])
def test_every_byte_of_a_block_is_one_code(d):
    k, v = orc.places(d)
    assert sorted(np.concatenate([k.ravel(), v.ravel()]).tolist()) == list(range(64 * d))


def test_turns_keep_lengths_and_add_up():
    rng = np.random.default_rng(1)
    x, freqs = rng.normal(size=(3, 2, 64)), (10000.0 ** (-np.arange(16) / 16)).astype(np.float32)
    for pairs in (0, 1):
        once = orc.turn(x, [7, 100000, -3], freqs, 32, pairs)
        assert np.array_equal(once[..., 32:], x[..., 32:]) and np.allclose((once ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-13)
        twice = orc.turn(once, [5, 1, 3], freqs, 32, pairs)
        assert np.allclose(twice, orc.turn(x, [12, 100001, 0], freqs, 32, pairs), atol=1e-9)
        assert np.allclose(twice[2], x[2], atol=1e-12)
    y = orc.turn(np.eye(64)[None, :1], [1], freqs, 32, 1)                            # a pair by hand: frequency 1, position 1
    assert np.allclose(y[0, 0, :2], [np.cos(1), np.sin(1)]) and not y[0, 0, 2:].any()


def test_appending_in_pieces_keeps_powers_and_bounds_of_all():
    rng = np.random.default_rng(2)
    k, v = rng.normal(size=(40, 2, 64)) * 2.0 ** rng.integers(-3, 4, (40, 1, 1)), rng.normal(size=(40, 2, 64))
    caches = []
    for cut in ([0, 40], [0, 13, 40], list(range(41))):
        c = orc.Cache8(2, 32, 1, 2, 2, 64, fill=0xFF)
        c.table[0], c.lens[0] = [1, 0], 40
        for a, b in zip(cut[:-1], cut[1:]):
            c.append(k, v, None, [a, b], [0], [a])
        caches.append(c)
    for c in caches:
        for tile in range(2):
            for h in range(2):
                codes, bounds, powers = c.block(c.table[0, tile], h, tile)
                first = caches[0].block(c.table[0, tile], h, tile)
                assert np.array_equal(powers, first[2])
                x, bounds = orc.value(codes[c.places[0][:32 if tile == 0 else 8]]), bounds.astype(int)
                assert (bounds[0] * 4 >= x.max(axis=0)).all() and (bounds[1] * 4 <= x.min(axis=0)).all() and np.abs(bounds).max() <= 112
                assert (np.abs(bounds - first[1]) <= 1).all()
        got = c.read(0)[0]
        # half a step of the largest power's grid, and another half for a code that was rounded before its power grew
        e = np.repeat([[orc.power(k[32 * t:32 * t + 32, h]) for h in range(2)] for t in range(2)], [32, 8], axis=0)
        step = np.maximum(2.0 ** (np.floor(np.log2(np.abs(k))) - 3), 2.0 ** (e[..., None] - 9))
        assert (np.abs(got - k) <= step).all()
    assert np.array_equal(caches[0].read(0)[1].shape, (40, 2, 64))


def test_a_score_is_at_least_every_logit_of_its_block():
    rng = np.random.default_rng(3)
    c = orc.Cache8(3, 32, 1, 3, 1, 64)
    c.table[0], c.lens[0] = [2, 0, 1], 90
    k = rng.normal(size=(90, 1, 64))
    c.append(k, k, None, [0, 90], [0], [0])
    q = rng.integers(-127, 128, 64) * 2.0 ** -5                                     # whole numbers of a power: nothing is rounded
    q[0] = 127 * 2.0 ** -5
    held = c.read(0)[0]
    for tile in range(3):
        score = c._score(q, c.block(c.table[0, tile], 0, tile))
        assert score >= (held[32 * tile:32 * tile + 32, 0] @ q).max()


def test_the_choice_of_blocks():
    rng = np.random.default_rng(4)
    c = orc.Cache8(8, 32, 2, 8, 2, 64)
    c.table[0], c.lens[0] = rng.permutation(8), 250
    k = rng.normal(size=(250, 2, 64))
    c.append(k, k, None, [0, 250], [0], [0])
    q = rng.normal(size=(2, 4, 64))
    assert (c.select(q, 0, 1, 2, 9)[:, :, :8] == np.arange(8)).all()                # enough for all of them
    assert c.select(q, 0, 1, 2, 0)[1].tolist() == [[0, 6, 7]] * 2
    assert (c.select(q, 1, 1, 2, 3) == -1).all() and (c.select(q, -1, 1, 2, 3) == -1).all()
    got = c.select(q, 0, 0, 1, 3)
    for i in range(2):
        for h in range(2):
            score = [max(c._score(q[i, x], c.block(c.table[0, t], h, t)) for x in (2 * h, 2 * h + 1)) for t in range(7)]
            assert set(got[i, h, :3].tolist()) == set(np.argsort(-np.array(score), kind="stable")[:3].tolist()) and got[i, h, 3] == 7
    # ties: bounds of two blocks alike
    a, b = (c.block(c.table[0, t], 0, t) for t in (2, 4))
    b[1][:], b[2][:] = a[1], a[2]
    ranks = [c._score(q[0, 0], c.block(c.table[0, t], 0, t)) for t in range(7)]
    assert ranks[2] == ranks[4]
    assert c.select(q, 0, 0, 1, 7, max_len=64)[0, 0].tolist() == [0, 1, 7] + [-1] * 5


def test_attention_over_blocks_is_attention_over_their_tokens():
    rng = np.random.default_rng(5)
    q, k, v = rng.normal(size=(2, 4, 64)), rng.normal(size=(100, 2, 64)), rng.normal(size=(100, 2, 64))
    every = np.tile(np.arange(4), (2, 2, 1))
    for a, b in zip(orc.attention(q, k, v, None, every), cache_oracle.attention(q, k, v)):
        assert np.allclose(a, b, rtol=1e-12)
    one = np.full((2, 2, 3), -1)
    one[1, 0, 1] = 2
    out, lse = orc.attention(q, k, v, None, one)
    assert not out[0].any() and np.isneginf(lse[0]).all() and np.isneginf(lse[1, 2:]).all()
    x = k[64:96, 0] @ q[1, 1] / 8
    p = np.exp(x) / np.exp(x).sum()
    assert np.allclose(out[1, 1], p @ v[64:96, 0]) and np.isclose(lse[1, 1], np.log2(np.exp(x).sum()))
