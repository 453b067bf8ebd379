"""The operators on a cache held in 8 bits against the float64 oracle: pages and lists bit for bit, turned rows and attention within the bounds their
roundings give."""
import numpy as np
import pytest

from oracle import cache8_oracle as orc
from paper_2405_12532_amd import synth

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
from tests.caches8 import Pair8, append, attend, bf16, check_attention, dev, select  # noqa: E402


# ------------------------------------------------------------------------------------------------ rows in and out
def special_rows(rng, rows, hkv, d):
    """Rows with what a conversion can trip over: ties, borders of the power of two, the ends of bf16's range, numbers that are none."""
    x = rng.normal(size=(rows, hkv, d)) * 2.0 ** rng.integers(-30, 30, (rows, hkv, 1)) if rows % 2 else rng.normal(size=(rows, hkv, d))
    flat = x.reshape(-1, 32)
    n = len(flat)
    ties = np.concatenate([orc.GRID[8:24], (orc.GRID[8:16] + orc.GRID[9:17]) / 2, (orc.GRID[1:9] + orc.GRID[:8]) / 2])
    for i in range(0, n, 7):
        flat[i] = ties * rng.choice([-1, 1], 32) * 2.0 ** float(rng.integers(-3, 3))
    for i, top in zip(range(1, n, 31), [448.0, 450.0, 224.0, 225.0, 2.0 ** -100, 2.0 ** -92, 2.0 ** -130, 3.38e38, 2.9e38, 1.7e38, 0.0] * n):
        flat[i] = rng.choice([-1, 1, 0.5, 0.25, 0], 32) * top
    for i, bad in zip(range(3, n, 41), [np.inf, -np.inf, np.nan] * n):
        flat[i, rng.integers(32)] = bad
    return flat.reshape(rows, hkv, d)


@pytest.mark.parametrize("hkv,d,page", [(1, 128, 32), (3, 64, 64), (5, 128, 256), (8, 64, 32)])
def test_append_writes_the_nearest_numbers_and_nothing_else(lib, hkv, d, page):
    # pieces that begin and end inside a block, one token, none, whole blocks, across pages; one in a padded row, one without room
    lens = [100, 70, 64, 33, 200, 40, 40, 96, 33]
    start, count, slots = [37, 69, 0, 31, 5, 3, -1, 20, 32], [50, 1, 64, 0, 190, 7, 9, 40, 1], [0, 1, 2, 3, 4, -1, 6, 7, 8]
    pair = Pair8(lib, lens, hkv, d, page, seed=d + hkv)
    rows = sum(count)
    kt, k = bf16(special_rows(pair.rng, rows, hkv, d))
    vt, v = bf16(special_rows(pair.rng, rows, hkv, d))
    offsets = np.concatenate([[0], np.cumsum(count)])
    append(pair, kt, vt, rows, None, offsets, slots, start, max(count))
    pair.o.append(k, v, None, offsets, slots, start)
    pair.check_pages()
    # again: nothing changes
    append(pair, kt, vt, rows, None, offsets, slots, start, max(count))
    pair.check_pages()


@pytest.mark.parametrize("hkv,d", [(3, 128), (2, 64)])
@pytest.mark.parametrize("count", [1, 4, 5, 20])
def test_a_larger_power_rounds_what_the_block_holds(lib, hkv, d, count):
    """Powers that stay, grow by one, by many and from the least to the most, of K and V apart, of some heads."""
    pair = Pair8(lib, [64] * 6, hkv, d, 32, powers=(100, 101))
    starts = [3, 10, 7, 43, 1, 32]
    kx, vx = pair.rng.normal(size=(6, count, hkv, d)), pair.rng.normal(size=(6, count, hkv, d))
    for i, (ks, vs) in enumerate([(2.0 ** -24, 2.0 ** -22), (2.0 ** -17, 2.0 ** -30), (2.0 ** -30, 2.0 ** -15), (2.0 ** 100, 2.0 ** 3), (1, 2.0 ** 90), (1, 1)]):
        kx[i] *= ks
        vx[i] *= vs
    kx[0, 0, 0] *= 64
    kt, k = bf16(kx.reshape(-1, hkv, d))
    vt, v = bf16(vx.reshape(-1, hkv, d))
    offsets = np.arange(7) * count
    append(pair, kt, vt, 6 * count, None, offsets, np.arange(6), starts, count)
    pair.o.append(k, v, None, offsets, np.arange(6), starts)
    pair.check_pages()


def test_a_block_in_pieces_of_every_size(lib):
    """Tokens one by one, and in pieces of 2 to 9: powers and bounds follow."""
    hkv, d = 2, 128
    for sizes in ([1] * 40, [2, 3, 4, 5, 6, 7, 9, 4], [40]):
        pair = Pair8(lib, [], hkv, d, 32, n_slots=2, max_pages=2, spare=4, fill=0xA7)
        pair.o.table[1], pair.o.lens[1] = [3, 1], 40
        pair.up()
        x = pair.rng.normal(size=(40, hkv, d)) * 2.0 ** pair.rng.integers(-4, 5, (40, hkv, 1))
        kt, k = bf16(x)
        vt, v = bf16(x[::-1])
        at = 0
        for n in sizes:
            append(pair, kt, vt, 40, None, [at, at + n], [1], [at], n)
            pair.o.append(k, v, None, [at, at + n], [1], [at])
            at += n
        pair.check_pages()


def test_append_through_an_index_list_and_rows_that_are_not_there(lib):
    """An index outside k and v, a place outside the list: tokens of NaN."""
    pair = Pair8(lib, [90, 64, 50, 50], 4, 128, 32)
    kt, k = bf16(pair.rng.normal(size=(200, 4, 128)))
    vt, v = bf16(pair.rng.normal(size=(200, 4, 128)))
    idx = pair.rng.integers(0, 200, 60).astype(np.int32)
    idx[[5, 41]], idx[17] = 200, -1
    least = -2 ** 31
    for offsets, slots, start, most in (([0, 40, 60], [0, 1], [50, 44], 40), ([-5, 20], [2], [3], 25), ([50, 70], [3], [10], 20), ([least, least + 7], [3], [40], 7), ([30, 20, 60], [0, 1], [5, 2], 99)):
        append(pair, kt, vt, 200, idx, offsets, slots, start, most)
        pair.o.append(k, v, idx, offsets, slots, start, most)
        pair.check_pages()
    append(pair, kt[:10], vt[:10], 10, None, [4, 14], [2], [20], 10)
    pair.o.append(k[:10], v[:10], None, [4, 14], [2], [20])
    pair.check_pages()


def test_append_of_strided_rows(lib):
    """K and V side by side in the rows of a fused projection, and rows further apart than they are long."""
    hkv, d = 3, 64
    pair = Pair8(lib, [70], hkv, d, 32)
    fused, x = bf16(pair.rng.normal(size=(60, 8 * hkv, d)))
    kt, vt = fused[:, 2 * hkv:3 * hkv], fused[:, 5 * hkv:6 * hkv]
    append(pair, kt, vt, 60, None, [0, 60], [0], [7], 60, strides=(kt.stride(0), vt.stride(0), 0))
    pair.o.append(x[:, 2 * hkv:3 * hkv], x[:, 5 * hkv:6 * hkv], None, [0, 60], [0], [7])
    pair.check_pages()


def test_append_takes_the_first_row_of_a_slot_and_stops_at_its_limits(lib):
    pair = Pair8(lib, [64] * 4 + [40, 64], 2, 64, 32, max_pages=4)
    pair.o.table[4, 2:], pair.o.table[5, 1] = pair.o.table[0, 0], len(pair.o.refs)          # anything behind the length; a page outside the pool
    pair.up()
    n = 150
    slots = [0, 1, 0, 1, 2] + [-1] * 139 + [5, 2, 3, 0, 3, 4]
    start = [0, 7, 10, 7, 40] + [0] * 139 + [20, 50, 1, 0, 20, 33]
    kt, k = bf16(pair.rng.normal(size=(20 * n, 2, 64)))
    offsets = np.arange(n + 1) * 20
    for most in (20, 13, 2 ** 31 - 1):
        append(pair, kt, kt, 20 * n, None, offsets, slots, start, most)
        pair.o.append(k, k, None, offsets, slots, start, most)
        pair.check_pages()


@pytest.mark.parametrize("d,hq,hkv,dims,pairs,far", [(128, 8, 2, 128, 0, 0), (128, 4, 4, 128, 1, 100000), (64, 6, 2, 64, 0, 2 ** 31 - 200), (64, 8, 8, 32, 1, 5000),
                                                     (128, 5, 1, 48, 0, 1000000), (128, 4, 2, 112, 0, 77), (64, 2, 1, 16, 0, -300), (64, 3, 3, 48, 1, 9)])
def test_append_turns_rows_by_their_positions(lib, d, hq, hkv, dims, pairs, far):
    """K as the codes say within half a step and what fp32 loses; Q within half a step of bf16; both strided.  An angle is off by far * 2^-51 in 64
    bits, a sine by its rounding to fp32 besides, a product and the sum by theirs, so that a turned number is by 2^-21 (|a| + |b|) at most."""
    lens, start, count = [90, 40, 33, 64], [10, 39, 0, 31], [70, 1, 33, 0]
    pair = Pair8(lib, lens, hkv, d, 32, powers=(113, 114))
    rows = sum(count)
    fused, x = bf16(pair.rng.normal(size=(rows, hq + 2 * hkv, d)))
    qt, kt, vt = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    positions = (far + pair.rng.integers(0, 190, rows)).astype(np.int32)
    freqs = (10000.0 ** (-np.arange(dims // 2) * 2 / dims)).astype(np.float32)
    rotation = lib.make_rotation(torch.from_numpy(freqs).cuda(), torch.from_numpy(positions).cuda(), dims, pairs)
    q_out = torch.full((rows + 1, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    offsets = np.concatenate([[0], np.cumsum(count)])
    stride = fused.stride(0)
    append(pair, kt, vt, rows, None, offsets, np.arange(4), start, max(count), rotation, qt, q_out, strides=(stride, stride, stride))
    q, k, v = orc.turn(x[:, :hq], positions, freqs, dims, pairs), orc.turn(x[:, hq:hq + hkv], positions, freqs, dims, pairs), x[:, hq + hkv:]
    i = np.arange(d)
    other = np.where(i < dims, np.where(i % 2 == 0, i + 1, i - 1) if pairs else np.where(i < dims // 2, i + dims // 2, i - dims // 2), i)
    fine = lambda y: (2.0 ** -21 + abs(far) * 2.0 ** -50) * (np.abs(y) + np.abs(y[..., other])) * (i < dims)  # noqa: E731
    got = q_out.double().cpu().numpy()
    assert (got[rows] == 7).all()
    assert (np.abs(got[:rows] - q) <= 2.0 ** -8 * np.abs(q) * 1.001 + fine(x[:, :hq])).all()
    before = {s: pair.o.read(s) for s in range(4)}
    pair.o.pages = pair.pages.cpu().numpy()
    for s in range(3):
        if count[s] == 0:
            continue
        mine = slice(offsets[s], offsets[s + 1])
        gk, gv = pair.o.read(s)
        span = slice(start[s], start[s] + count[s])
        for tile in range(start[s] // 32, -(-(start[s] + count[s]) // 32)):
            for h in range(hkv):
                codes, bounds, powers = pair.o.block(pair.o.table[s, tile], h, tile)
                a, b = max(start[s], 32 * tile), min(start[s] + count[s], 32 * tile + 32)
                new = k[mine][a - start[s]:b - start[s], h]
                want = max(orc.power(new), 113 - 127 if start[s] > 32 * tile else -100)
                assert int(powers[0]) - 127 == want or abs(np.abs(new).max() / (448 * 2.0 ** min(want, int(powers[0]) - 127)) - 1) < 1e-6
                y = orc.value(codes[pair.o.places[0][:b - 32 * tile]])              # (what a block held behind the new tokens is not theirs)
                assert (bounds[0].astype(int) * 4 >= y.max(axis=0)).all() and (bounds[1].astype(int) * 4 <= y.min(axis=0)).all()
                if start[s] <= 32 * tile and b == min(lens[s], 32 * tile + 32):
                    assert np.array_equal(bounds[0], np.ceil(y.max(axis=0) / 4)) and np.array_equal(bounds[1], np.floor(y.min(axis=0) / 4))
                step = 2.0 ** (int(powers[0]) - 127) * 2.0 ** np.maximum(np.floor(np.log2(np.abs(new / 2.0 ** (int(powers[0]) - 127)) + 1e-300)) - 3, -9)
                assert (np.abs(gk[a:b, h] - new) <= step / 2 * 1.001 + fine(x[:, hq:hq + hkv])[mine][a - start[s]:b - start[s], h]).all()
        assert np.array_equal(gv[:start[s] // 32 * 32], before[s][1][:start[s] // 32 * 32])
        step = 2.0 ** (np.floor(np.log2(np.abs(v[mine]) + 1e-300)) - 4)
        # half a step of a number's own, or half of the least, 2^-9 times the power: of numbers up to 448 * 2^-6 that is 2^-6 at most
        assert np.abs(v[mine]).max() <= 7 and (np.abs(gv[span] - v[mine]) <= np.maximum(step, 2.0 ** -9 * 2.0 ** -6 / 2)).all()


@pytest.mark.parametrize("d,dims,pairs", [(128, 128, 0), (128, 128, 1), (64, 64, 0), (64, 32, 0)])
def test_turned_keys_get_the_nearest_codes(lib, d, dims, pairs):
    """Where the two products of a turn do not cancel, fp32's result is by 2^-24 (2 |x| + |x|) off at most (sine and cosine, a product, the sum), three units of its last place, and
    what is so near to a border is turned again: millions of numbers, of which fp32 alone gives some the wrong code, and those of 64 bits, by 2^-33, hardly one in 10^9."""
    hkv, tokens = 16, 4096
    pair = Pair8(lib, [], hkv, d, 1024, n_slots=1, max_pages=4, spare=4, fill=0)
    pair.o.table[0], pair.o.lens[0] = [2, 0, 3, 1], tokens
    pair.up()
    gen = torch.Generator("cuda").manual_seed(d + dims + pairs)
    k = torch.randn((tokens, hkv, d), generator=gen, device="cuda").to(torch.bfloat16)
    freqs = torch.logspace(0, -4, dims // 2, device="cuda")
    positions = torch.randint(1, 100000, (tokens,), generator=gen, device="cuda", dtype=torch.int32)
    append(pair, k, k, tokens, None, [0, tokens], [0], [0], tokens, lib.make_rotation(freqs, positions, dims, pairs))
    got = torch.empty_like(k)
    lib.cache8_load(pair.cache, torch.zeros(1, dtype=torch.int32, device="cuda"), None, torch.tensor([0, tokens], dtype=torch.int32, device="cuda"), 1, tokens, got, None, tokens)
    pair.o.pages = pair.pages.cpu().numpy()
    powers = torch.tensor([[pair.o.block(pair.o.table[0, t // 32], h, t)[2][0] for h in range(hkv)] for t in range(tokens // 32)]).repeat_interleave(32, 0).double().cuda() - 127
    angle = positions.double()[:, None] * freqs.double()
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    first, second = (slice(0, dims, 2), slice(1, dims, 2)) if pairs else (slice(0, dims // 2), slice(dims // 2, dims))
    for part, own, other in ((first, c, -s), (second, c, s)):
        x, y = k[..., part].double() * own, k[..., second if part == first else first].double() * other
        want, same = x + y, x * y >= 0
        unit = torch.exp2(torch.floor(torch.log2(want.abs() + 1e-300)) - 3)
        sure = same & (unit >= torch.exp2(powers)[..., None] * 2.0 ** -9)
        assert sure.double().mean() > 0.45
        assert torch.equal(got[..., part].double()[sure], ((want / unit).round() * unit)[sure])


@pytest.mark.parametrize("d,dims,pairs", [(128, 128, 0), (128, 128, 1), (64, 64, 0)])
@pytest.mark.parametrize("far", [2 ** 21, 2 ** 24, 2 ** 31 - 4096, -2 ** 31])
def test_turned_keys_get_the_nearest_codes_at_far_positions(lib, d, dims, pairs, far):
    """As above, where an angle has more bits than a number of 64 bits holds, or its quarters of a turn take most of them: against angles, sines and cosines of 80 bits, in which a
    position times a frequency (31 and 24 bits) is exact."""
    hkv, tokens = 16, 4096
    pair = Pair8(lib, [], hkv, d, 1024, n_slots=1, max_pages=4, spare=4, fill=0)
    pair.o.table[0], pair.o.lens[0] = [2, 0, 3, 1], tokens
    pair.up()
    gen = torch.Generator("cuda").manual_seed(d + dims + pairs)
    k = torch.randn((tokens, hkv, d), generator=gen, device="cuda").to(torch.bfloat16)
    freqs = torch.linspace(1, 0.5, dims // 2, device="cuda")
    positions = torch.arange(far, far + tokens, device="cuda").to(torch.int32)
    append(pair, k, k, tokens, None, [0, tokens], [0], [0], tokens, lib.make_rotation(freqs, positions, dims, pairs))
    got = torch.empty_like(k)
    lib.cache8_load(pair.cache, dev([0]), None, dev([0, tokens]), 1, tokens, got, None, tokens)
    pair.o.pages = pair.pages.cpu().numpy()
    powers = torch.tensor([[pair.o.block(pair.o.table[0, t // 32], h, t)[2][0] for h in range(hkv)] for t in range(tokens // 32)]).repeat_interleave(32, 0).double().cuda() - 127
    angle = positions.cpu().numpy().astype(np.longdouble)[:, None] * freqs.cpu().numpy().astype(np.longdouble)
    c, s = (torch.from_numpy(f(angle).astype(np.float64)).cuda()[:, None] for f in (np.cos, np.sin))
    first, second = (slice(0, dims, 2), slice(1, dims, 2)) if pairs else (slice(0, dims // 2), slice(dims // 2, dims))
    for part, own, other in ((first, c, -s), (second, c, s)):
        x, y = k[..., part].double() * own, k[..., second if part == first else first].double() * other
        want, same = x + y, x * y >= 0
        unit = torch.exp2(torch.floor(torch.log2(want.abs() + 1e-300)) - 3)
        sure = same & (unit >= torch.exp2(powers)[..., None] * 2.0 ** -9)
        assert sure.double().mean() > 0.45
        assert torch.equal(got[..., part].double()[sure], ((want / unit).round() * unit)[sure])


def test_angles_that_64_bits_do_not_hold_turn_all_the_same(lib):
    """Frequencies up to fp32's largest: a turn by some angle, which leaves a pair's length (within half a step of bf16 a number, 2^-8, and 2^-20 besides)."""
    pair = Pair8(lib, [60], 2, 128, 64)
    qt, q = bf16(pair.rng.normal(size=(50, 4, 128)))
    kt, _ = bf16(pair.rng.normal(size=(50, 2, 128)))
    positions = dev(pair.rng.integers(-2 ** 31, 2 ** 31, 50).astype(np.int32))
    q_out = torch.empty_like(qt)
    append(pair, kt, kt, 50, None, [0, 50], [0], [5], 50, lib.make_rotation(torch.logspace(3, 38.5, 64, device="cuda"), positions, 128), qt, q_out)
    got = q_out.double().cpu().numpy()
    want = np.hypot(q[..., :64], q[..., 64:])
    assert (np.abs(np.hypot(got[..., :64], got[..., 64:]) - want) <= (2.0 ** -8 + 2.0 ** -20) * want).all()


@pytest.mark.parametrize("d,dims,pairs", [(128, 128, 0), (128, 64, 1), (64, 64, 0), (64, 32, 0)])
@pytest.mark.parametrize("tokens", [1, 7, 50])
def test_turns_by_nothing_change_nothing(lib, d, dims, pairs, tokens):
    """A position or frequencies of 0: what rows without a turn leave."""
    left = []
    zeros, ones = torch.zeros(64, dtype=torch.int32, device="cuda"), torch.ones(64, device="cuda")
    for rotation in (None, lib.make_rotation(ones[:dims // 2], zeros[:tokens], dims, pairs), lib.make_rotation(0 * ones[:dims // 2], zeros[:tokens] + 12345, dims, pairs)):
        pair = Pair8(lib, [60], 3, d, 64, powers=(115, 118))
        kt, _ = bf16(pair.rng.normal(size=(tokens, 3, d)))
        append(pair, kt, kt, tokens, None, [0, tokens], [0], [9], tokens, rotation)
        left.append(pair.pages.clone())
    assert torch.equal(left[0], left[1]) and torch.equal(left[0], left[2])


@pytest.mark.parametrize("d,hq,hkv,dims,pairs", [(128, 8, 2, 128, 0), (128, 5, 5, 128, 1), (64, 6, 2, 64, 0), (64, 24, 3, 64, 1), (64, 8, 8, 32, 1), (128, 5, 1, 48, 0), (64, 2, 1, 16, 0)])
def test_turns_of_pieces_of_every_size(lib, d, hq, hkv, dims, pairs):
    """Tokens behind others in a block whose power holds them: one by one, up to nine at a time and all at once leave the same bytes and turn Q alike."""
    left, out = [], []
    for sizes in ([1] * 29, [2, 9, 5, 7, 6], [29]):
        pair = Pair8(lib, [32], hkv, d, 32, powers=(124, 125))
        qt, _ = bf16(pair.rng.normal(size=(29, hq, d)))
        kt, _ = bf16(pair.rng.normal(size=(29, hkv, d)))
        rotation = lib.make_rotation(torch.logspace(0, -3, dims // 2, device="cuda"), torch.arange(900, 929, dtype=torch.int32, device="cuda"), dims, pairs)
        q_out, at = torch.zeros_like(qt), 0
        for n in sizes:
            append(pair, kt, kt, 29, None, [at, at + n], [0], [3 + at], n, rotation, qt, q_out)
            at += n
        left.append(pair.pages.clone())
        out.append(q_out)
    for i in (0, 1):
        assert torch.equal(left[i], left[2]) and torch.equal(out[i], out[2]), i


def test_queries_turn_in_place_and_of_stored_tokens_alone(lib):
    pair = Pair8(lib, [40, 40], 2, 128, 32)
    qt, q = bf16(pair.rng.normal(size=(30, 4, 128)))
    kt, _ = bf16(pair.rng.normal(size=(30, 2, 128)))
    freqs, positions = torch.full((64,), 0.5, device="cuda"), torch.arange(30, dtype=torch.int32, device="cuda")
    rotation = lib.make_rotation(freqs, positions, 128)
    before = qt.clone()
    # slot 1's piece runs over its length, the third row is padded, the fourth found no room
    append(pair, kt, kt, 30, None, [0, 5, 12, 20, 30], [0, 1, -1, 0], [3, 36, 0, -1], 10, rotation, qt, qt)
    got = qt.double().cpu().numpy()
    want = orc.turn(q, np.arange(30), np.full(64, 0.5, np.float32), 128, 0)
    stored = np.r_[0:5, 5:9]
    assert (np.abs(got - want)[stored] <= 2.0 ** -8 * np.abs(want[stored]) + 2.0 ** -18).all()
    left = np.setdiff1d(np.arange(30), stored)
    assert torch.equal(qt[left], before[left])
    # without a rotation q is copied
    out = torch.empty_like(before)
    append(pair, kt, kt, 30, None, [0, 30], [0], [0], 30, None, before, out)
    assert torch.equal(out, before)


@pytest.mark.parametrize("hkv,d,page", [(1, 128, 32), (6, 64, 128), (5, 128, 64), (8, 64, 32)])
@pytest.mark.parametrize("max_len", [1, 33, 200, 2 ** 31 - 1])
def test_load_gives_the_exact_values(lib, hkv, d, page, max_len):
    lens = [0, 1, 33, 64, 200, 31, 90, 64]
    pair = Pair8(lib, lens, hkv, d, page, powers=(27, 247))
    pair.o.block(pair.o.table[4, 0], 0, 0)[0][77] = 0x7F                                 # a number that is none
    pair.o.table[7, 0] = -5                                                              # a page below the pool
    pair.up()
    room = [3, 1, 33, 70, 150, 31, 9, 64]                                                # rows for them: more than there are, fewer than there are
    slots, first = [0, 1, 2, 3, 4, -1, 6, 7], [0, 0, 31, 5, 37, 0, 64, 0]
    offsets = np.concatenate([[0], np.cumsum(room)])
    n_rows = int(offsets[-1]) - 2                                                        # the last two have no rows
    for given in (first, None):
        out = [torch.full((n_rows + 5, hkv, d), 77.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        lib.cache8_load(pair.cache, dev(slots), None if given is None else dev(given), dev(offsets), 8, max_len, out[0], out[1], n_rows)
        want = [np.full((n_rows + 5, hkv, d), 77.0) for _ in range(2)]
        for i, s in enumerate(slots):
            at = 0 if given is None else given[i]
            n = min(lens[i] - at, room[i], max_len, n_rows - offsets[i]) if s >= 0 and s != 7 else 0
            for x, y in zip(want, pair.o.read(s, at) if n > 0 else want):
                if n > 0:
                    x[offsets[i]:offsets[i] + n] = y[:n]
            if s == 7 and pair.o.page == 32 and min(64, max_len, n_rows - offsets[i]) > 32:      # (its second page is in the pool)
                n = min(64, max_len, n_rows - offsets[i])
                for x, which in zip(want, (0, 1)):
                    for h in range(hkv):
                        codes, _, powers = pair.o.block(pair.o.table[7, 1], h, 1)
                        x[offsets[i] + 32:offsets[i] + n, h] = orc.value(codes[pair.o.places[which]])[:n - 32] * 2.0 ** (int(powers[which]) - 127)
        for x, y in zip(out, want):
            assert np.array_equal(x.double().cpu().numpy(), y, equal_nan=True)
    only = torch.empty((n_rows + 5, hkv, d), dtype=torch.bfloat16, device="cuda")
    lib.cache8_load(pair.cache, dev(slots), None, dev(offsets), 8, max_len, None, only.fill_(77), n_rows)
    assert torch.equal(only.view(torch.int16), out[1].view(torch.int16))


def test_load_takes_offsets_and_first_tokens_that_cannot_be(lib):
    pair = Pair8(lib, [40, 40], 2, 64, 32)
    out = torch.full((40, 2, 64), 77.0, dtype=torch.bfloat16, device="cuda")
    least = -2 ** 31
    for slots, first, offsets in (([0, 1], [0, 0], [30, 20, 10]), ([0], [0], [-5, 30]), ([0], [-1], [0, 30]), ([0], [least], [0, 30]), ([0], [0], [least, 2 ** 31 - 1]),
                                  ([0], [40], [0, 30]), ([0], [2 ** 31 - 1], [0, 40]), ([2], [0], [0, 30])):
        lib.cache8_load(pair.cache, dev(slots), dev(first), dev(offsets), len(slots), 40, out, out, 40)
    assert (out == 77).all()


# ------------------------------------------------------------------------------------------------ attention
ATTEND = [([100, 1, 0, 33, 64], 8, 8, 128, 32, 1), ([100, 31, 0, 33, 65], 8, 2, 64, 64, 1), ([300, 2, 5, 129], 12, 1, 128, 32, 3), ([77, 500], 40, 8, 64, 32, 4),
          ([40, 3, 64], 16, 1, 128, 64, 5), ([256, 255], 34, 2, 64, 128, 2), ([1, 2, 3], 4, 4, 128, 32, 9)]


@pytest.mark.parametrize("lens,hq,hkv,d,page,tokens", ATTEND)
def test_attention(lib, lens, hq, hkv, d, page, tokens):
    pair = Pair8(lib, lens, hkv, d, page, seed=hq)
    slots = list(range(len(lens)))[::-1] + [-1, len(lens)]
    qt, q = bf16(pair.rng.normal(size=(len(slots), tokens, hq, d)) * 0.05)
    out, lse = attend(pair, qt, slots, tokens, max(lens))
    check_attention(pair, q, [s if s < len(lens) else -1 for s in slots], out, lse)
    for scale, most in ((0.3, max(lens)), (0.0, 0)):                                     # another scale, a limit that is too short
        out, _ = attend(pair, qt, slots, tokens, most, scale=scale, want_lse=False)
        check_attention(pair, q, [s if s < len(lens) else -1 for s in slots], out, None, scale or None)


@pytest.mark.parametrize("lens,hq,hkv,d,tokens", [([5000, 1, 700, 0], 4, 2, 128, 1), ([4097, 4096], 8, 1, 64, 3), ([9000], 2, 1, 64, 1), ([3000, 2999], 24, 1, 128, 2)])
def test_attention_split_along_the_cache(lib, lens, hq, hkv, d, tokens):
    pair = Pair8(lib, lens, hkv, d, 64, seed=hq)
    qt, q = bf16(pair.rng.normal(size=(len(lens), tokens, hq, d)) * 0.05)
    slots = list(range(len(lens)))
    assert lib.diag_cache8_attention(pair.cache, len(lens), tokens, hq, max(lens), 0).splits > 1
    check_attention(pair, q, slots, *attend(pair, qt, slots, tokens, max(lens)))
    check_attention(pair, q, slots, *attend(pair, qt, slots, tokens, 40 * 32))           # sequences longer than the limit


def test_attention_of_many_rows_by_workgroups_of_four_wavefronts(lib):
    lens = [37 * (i % 7) for i in range(600)]
    pair = Pair8(lib, lens, 1, 64, 32)
    qt, q = bf16(pair.rng.normal(size=(600, 1, 3, 64)) * 0.05)
    assert lib.diag_cache8_attention(pair.cache, 600, 1, 3, 222, 0).waves == 4
    check_attention(pair, q, range(600), *attend(pair, qt, list(range(600)), 1, 222))


@pytest.mark.parametrize("d", [64, 128])
def test_attention_with_large_and_growing_logits(lib, d):
    """Logits that grow along the sequence by hundreds, fall, and are all alike."""
    pair = Pair8(lib, [0] * 3, 1, d, 32, n_slots=3, max_pages=20, spare=60)
    order = pair.rng.permutation(60)
    for s in range(3):
        pair.o.table[s], pair.o.lens[s] = order[20 * s:20 * s + 20], 600
    pair.up()
    u = pair.rng.normal(size=d)
    u /= np.linalg.norm(u)
    ramp = np.linspace(-1, 1, 600)
    k = np.concatenate([8 * f[:, None] * u + 0.1 * pair.rng.normal(size=(600, d)) for f in (ramp, -ramp, 0 * ramp)])[:, None]
    kt, k = bf16(k)
    vt, v = bf16(pair.rng.normal(size=(1800, 1, d)))
    off = np.array([0, 600, 1200, 1800])
    append(pair, kt, vt, 1800, None, off, [0, 1, 2], [0, 0, 0], 600)
    pair.o.append(k, v, None, off, [0, 1, 2], [0, 0, 0])
    qt, q = bf16(np.tile(u * 40, (3, 2, 3, 1)) * np.array([1, 0.5, -1])[None, None, :, None])
    check_attention(pair, q, [0, 1, 2], *attend(pair, qt, [0, 1, 2], 2, 600, scale=1.0), scale=1.0)


@pytest.mark.parametrize("d,hq,tokens", [(128, 8, 1), (64, 8, 3), (128, 24, 2)])
@pytest.mark.parametrize("lens", [[500, 1, 33], [2000, 64, 7]])
def test_attention_over_the_largest_and_the_smallest_numbers(lib, d, hq, tokens, lens):
    """V up to where a sum of its numbers times the weights may still be taken: finite and right; beyond it a number or NaN, never an infinity.  V down to the
    least: every product keeps to fp32's normal range, as P is not below 2^-20 here."""
    for power, scale in ((127 + 97, 0.02), (27, 0.02)):
        pair = Pair8(lib, lens, 2, d, 32, powers=(118, 119))
        for s, S in enumerate(lens):
            for c in range(-(-S // 32)):
                for h in range(2):
                    pair.o.block(pair.o.table[s, c], h, c)[2][1] = power
        pair.up()
        qt, q = bf16(pair.rng.normal(size=(3, tokens, hq, d)) * scale)
        out, lse = attend(pair, qt, [0, 1, 2], tokens, max(lens))
        up = 2.0 ** (127 - power)                                                        # (the bounds have an absolute part)
        reads = {s: (k, v * up) for s, (k, v) in ((s, pair.o.read(s)) for s in range(3))}
        check_attention(pair, q, [0, 1, 2], out.double() * up, lse, reads=reads)
    for s, S in enumerate(lens):
        for c in range(-(-S // 32)):
            for h in range(2):
                pair.o.block(pair.o.table[s, c], h, c)[2][1] = 246
    pair.up()
    out, _ = attend(pair, qt, [0, 1, 2], tokens, max(lens))
    assert not torch.isinf(out.float()).any()


@pytest.mark.parametrize("d,hq,tokens", [(128, 2, 1), (64, 4, 3), (128, 24, 2)])
def test_numbers_that_are_none_reach_the_rows_that_see_them_alone(lib, d, hq, tokens):
    """V's: one channel of the rows that see the token, whatever their weights; K's: all of those rows.  Behind the last token every byte is a NaN."""
    lens = [100, 100, 100, 64, 2000]
    pair = Pair8(lib, lens, 2, d, 32)

    def spoil(slot, token, channel, which):
        codes = pair.o.block(pair.o.table[slot, token // 32], 1, token // 32)[0]
        codes[pair.o.places[which][token % 32, channel]] = 0xFF
    spoil(0, 99, 5, 1)                                                                   # seen by the newest token alone
    spoil(0, 98, d - 1, 1)
    spoil(1, 98, 3, 0)
    spoil(2, 40, 17, 1)
    spoil(3, 63, 33, 1)
    spoil(4, 1234, 9, 1)
    pair.up()
    qt, q = bf16(pair.rng.normal(size=(5, tokens, hq, d)) * 0.05)
    out, lse = attend(pair, qt, list(range(5)), tokens, 2000)
    got = out.float().cpu().numpy()
    assert np.isnan(got[0, -1, hq // 2:, 5]).all() and not np.isnan(got[:, :, :hq // 2]).any()
    check_attention(pair, q, range(5), out, lse)
    every = torch.arange(63, dtype=torch.int32, device="cuda").repeat(5, tokens, 2, 1).contiguous()
    check_attention(pair, q, range(5), *attend(pair, qt, list(range(5)), tokens, 2000, every))


def test_a_page_outside_the_pool_gives_nan(lib):
    for page in (-3, 10 ** 9):
        pair = Pair8(lib, [100, 100, 90], 2, 64, 32)
        pair.o.table[1, 2] = page
        pair.up()
        qt, q = bf16(pair.rng.normal(size=(3, 1, 4, 64)) * 0.1)
        out, lse = attend(pair, qt, [0, 1, 2], 1, 100)
        assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all()
        check_attention(pair, q[[0, 2]], [0, 2], out[[0, 2]], lse[[0, 2]])
        lists = dev([[[[0, 1], [0, 2]]]] * 3)
        out, lse = attend(pair, qt, [0, 1, 2], 1, 100, lists)
        assert torch.isnan(out[1, 0, 2:]).all() and not torch.isnan(out[1, 0, :2]).any() and not torch.isnan(out[[0, 2]]).any()
        append(pair, qt[:, 0, :2], qt[:, 0, :2], 3, None, [0, 3], [1], [70], 3, strides=(4 * 64, 4 * 64, 0))       # nowhere to go
        assert not select(pair, qt, [0, 1, 2], 1, 100, 1, 1, 1).eq(-7).any()
        pair.check_pages()


def test_queries_that_are_no_numbers(lib):
    pair = Pair8(lib, [300], 2, 64, 32)
    q = pair.rng.normal(size=(1, 1, 8, 64)) * 0.1
    q[0, 0, 1, 3], q[0, 0, 5, 9], q[0, 0, 6] = np.nan, np.inf, 0
    qt, q = bf16(q)
    out, _ = attend(pair, qt, [0], 1, 300)
    bad = torch.isnan(out[0, 0].float()).any(dim=1).cpu().tolist()
    assert bad == [False, True, False, False, False, True, False, False]
    got = select(pair, qt, [0], 1, 300, 1, 1, 3)
    assert np.array_equal(got.cpu().numpy()[0], pair.o.select(q[0], 0, 1, 1, 3))


# ------------------------------------------------------------------------------------------------ the choice of blocks
@pytest.mark.parametrize("lens,hq,hkv,d,page,tokens", [([100, 1, 0, 900, 64], 8, 8, 128, 32, 1), ([1000, 31, 0, 33, 650], 8, 2, 64, 64, 2), ([700, 2, 2500], 20, 1, 128, 32, 3),
                                                       ([77, 1500], 40, 8, 64, 32, 4), ([1200], 34, 2, 64, 128, 1), ([9000, 33], 4, 2, 64, 64, 1), ([20000], 2, 1, 128, 256, 2)])
def test_select(lib, lens, hq, hkv, d, page, tokens):
    pair = Pair8(lib, lens, hkv, d, page, seed=hq, powers=(115, 118))
    slots = list(range(len(lens)))[::-1] + [-1, len(lens)]
    qt, q = bf16(pair.rng.normal(size=(len(slots), tokens, hq, d)) * 2.0 ** pair.rng.integers(-3, 3, (len(slots), 1, hq, 1)))
    for first, recent, best, most in ((1, 2, 5, max(lens)), (0, 1, 1, max(lens)), (2, 3, 0, max(lens)), (3, 1, 17, 2 ** 31 - 1), (0, 1, 3, 170), (40, 40, 40, max(lens)), (0, 1, 100, max(lens))):
        got = select(pair, qt, slots, tokens, most, first, recent, best).cpu().numpy()
        for b, s in enumerate(slots):
            want = pair.o.select(q[b], s if s < len(lens) else -1, first, recent, best, most)
            assert np.array_equal(got[b], want), (b, first, recent, best, most)


def test_select_of_more_blocks_than_a_workgroup_holds(lib):
    """140000 tokens: 4375 blocks, whose keys are looked through in two passes; and the attention over what is chosen."""
    pair = Pair8(lib, [140000, 50], 1, 64, 1024, powers=(117, 119))
    qt, q = bf16(pair.rng.normal(size=(2, 1, 2, 64)) * 0.1)
    for first, recent, best, most in ((1, 2, 5, 140000), (0, 1, 300, 140000), (5, 1, 4100, 140000), (0, 1, 4374, 2 ** 31 - 1), (3, 3, 4000, 135000), (4200, 1, 20, 140000), (9999, 1, 20, 140000)):
        got = select(pair, qt, [0, 1], 1, most, first, recent, best)
        for b in (0, 1):
            assert np.array_equal(got[b].cpu().numpy(), pair.o.select(q[b], b, first, recent, best, most)), (first, recent, best, most, b)
    blocks = select(pair, qt, [0, 1], 1, 140000, 1, 2, 120)
    check_attention(pair, q, [0, 1], *attend(pair, qt, [0, 1], 1, 140000, blocks), blocks=blocks.cpu().numpy())


@pytest.mark.parametrize("rows,hkv,d,length", [(48, 2, 64, 20000), (100, 1, 128, 32768), (256, 1, 64, 32760), (257, 1, 64, 20000), (65, 3, 64, 49152), (96, 1, 64, 49200), (30, 1, 64, 16390)])
def test_select_of_many_rows_and_blocks(lib, rows, hkv, d, length):
    """One sequence asked for by many rows: blocks scored by sixteen wavefronts, in parts, and through memory."""
    pair = Pair8(lib, [length], hkv, d, 1024, powers=(116, 118))
    qt, q = bf16(pair.rng.normal(size=(rows, 1, 2 * hkv, d)) * 2.0 ** pair.rng.integers(-3, 3, (rows, 1, 2 * hkv, 1)))
    for first, recent, best, most in ((1, 2, 60, length), (0, 1, 1, length), (0, 1, 500, length), (7, 5, length // 32 - 20, 2 ** 31 - 1), (2, 1, 33, length - 100)):
        got = select(pair, qt, [0] * rows, 1, most, first, recent, best).cpu().numpy()
        for b in (0, rows // 2, rows - 1):
            assert np.array_equal(got[b], pair.o.select(q[b], 0, first, recent, best, most)), (b, first, recent, best, most)


@pytest.mark.parametrize("n", [1, 200])
def test_select_of_thousands_of_ties(lib, n):
    """Blocks that score alike by the hundred, in one workgroup's lanes and through memory."""
    pair = Pair8(lib, [64], 1, 64, 64, n_slots=n, max_pages=1100, powers=(115, 116))
    pair.o.table[:], pair.o.lens[:] = pair.o.table[0, 0], 64 * 1100 - 5                  # (the one page again and again)
    pair.up()
    qt, q = bf16(pair.rng.normal(size=(n, 1, 1, 64)))
    few = pair.o.select(q[0], 0, 0, 1, 1)                                                # which of the page's two blocks scores higher
    for best in (1, 700, 1100, 1101, 2000):
        got = select(pair, qt, list(range(n)), 1, 64 * 1100, 0, 1, best).cpu().numpy()
        even = int(few[0, 0, 0]) % 2 == 0
        order = list(range(0 if even else 1, 2199, 2)) + list(range(1 if even else 0, 2199, 2))
        assert got[0, 0, 0, :best + 1].tolist() == sorted(order[:best]) + [2199], best
        if n > 1:
            scores = [pair.o._score(q[7, 0, 0], pair.o.block(pair.o.table[0, 0], 0, c)) for c in (0, 1)]
            even = scores[0] >= scores[1]
            order = list(range(0 if even else 1, 2199, 2)) + list(range(1 if even else 0, 2199, 2)) if scores[0] != scores[1] else list(range(2199))
            assert got[7, 0, 0, :best + 1].tolist() == sorted(order[:best]) + [2199], best


@pytest.mark.parametrize("n,d", [(1, 64), (40, 128)])
def test_select_breaks_ties_by_number(lib, n, d):
    """Few different bounds and powers, so that many blocks score alike; a query of zeros scores all of them alike."""
    pair = Pair8(lib, [2000] * n, 4, d, 64, powers=(115, 116))
    for s in range(n):
        for c in range(63):
            for h in range(4):
                pair.o.block(pair.o.table[s, c // 2], h, c)[1][:] = np.array([[3], [-3]]) + (c % 3)
    pair.up()
    q = pair.rng.normal(size=(n, 1, 4, d))
    q[:, :, 2] = 0
    qt, q = bf16(q)
    for best in (1, 7, 20, 21, 22, 59, 60):
        got = select(pair, qt, list(range(n)), 1, 2000, 1, 2, best).cpu().numpy()
        for b in (0, n - 1):
            assert np.array_equal(got[b], pair.o.select(q[b], b, 1, 2, best)), best
        assert got[0, 0, 2, :best + 3].tolist() == list(range(best + 1)) + [61, 62]


def test_select_with_powers_and_queries_at_their_ends(lib):
    """Exponents that meet the limits of a score, the largest and the smallest queries."""
    pair = Pair8(lib, [640] * 3, 1, 64, 32, powers=(27, 247))
    for b, scale in enumerate((1e38, 1e-38, 1.0)):
        qt, q = bf16(pair.rng.normal(size=(3, 1, 2, 64)) * scale)
        got = select(pair, qt, [0, 1, 2], 1, 640, 0, 1, 5).cpu().numpy()
        for s in range(3):
            assert np.array_equal(got[s], pair.o.select(q[s], s, 0, 1, 5))


@pytest.mark.parametrize("lens,hq,hkv,d,page,tokens", [([100, 1, 0, 900, 64], 8, 8, 128, 32, 1), ([1000, 31, 0, 33, 650], 8, 2, 64, 64, 2), ([700, 2, 2500], 20, 1, 128, 32, 3),
                                                       ([77, 1500], 40, 8, 64, 32, 4), ([5000], 34, 1, 128, 128, 1)])
def test_attention_over_chosen_blocks(lib, lens, hq, hkv, d, page, tokens):
    pair = Pair8(lib, lens, hkv, d, page, seed=hq)
    slots = list(range(len(lens)))[::-1] + [-1]
    qt, q = bf16(pair.rng.normal(size=(len(slots), tokens, hq, d)) * 0.05)
    for first, recent, best in ((1, 2, 5), (0, 1, 0), (0, 1, 60)):
        blocks = select(pair, qt, slots, tokens, max(lens), first, recent, best)
        out, lse = attend(pair, qt, slots, tokens, max(lens), blocks)
        check_attention(pair, q, slots, out, lse, blocks=blocks.cpu().numpy())
    # all blocks: the result without a list, up to the order of sums
    every = torch.arange(-(-max(lens) // 32), dtype=torch.int32, device="cuda").repeat(len(slots), tokens, hkv, 1).contiguous()
    out, lse = attend(pair, qt, slots, tokens, max(lens), every)
    check_attention(pair, q, slots, out, lse)


def test_lists_of_any_entries(lib):
    """Any order, gaps, blocks that a token does not see, numbers that are no block, one block twice, a list of nothing."""
    pair = Pair8(lib, [200, 70], 2, 128, 32, n_slots=3, max_pages=8, spare=9)
    tokens = 3
    qt, q = bf16(pair.rng.normal(size=(3, tokens, 4, 128)) * 0.05)
    lists = np.full((3, tokens, 2, 9), -1, dtype=np.int32)
    lists[0, :, 0] = [5, -1, 3, 100, 0, -2 ** 31, 2 ** 31 - 1, 6, 7]
    lists[0, 1, 1] = [2] * 9
    lists[1, :, :] = [2, 1, 0, 3, 4, 5, 6, 7, 8]
    lists[2] = 0
    out, lse = attend(pair, qt, [0, 1, 2], tokens, 200, dev(lists))
    seen = np.where((lists < 0) | (lists > 6), -1, lists)
    check_attention(pair, q, [0, 1, -1], out, lse, blocks=seen)
    assert torch.isneginf(lse[0, 0, 2:]).all() and not out[0, 2, 2:].any()


# ------------------------------------------------------------------------------------------------ pages, streams, graphs, together
@pytest.mark.parametrize("hkv,d,page", [(1, 64, 32), (3, 128, 64), (2, 64, 1024)])
def test_pages_through_a_life(lib, hkv, d, page):
    """Reserve, append, fork, grow the branches, give back: pages, counts and bytes as the oracle's; what a branch gets does not show in its parent."""
    pair = Pair8(lib, [70, 64, 5], hkv, d, page, n_slots=7, max_pages=8, spare=20)
    o = pair.o
    lib.cache8_fork(pair.cache, dev([0, 1, 0, 2]), dev([3, 4, 5, 6]), 4, pair.status)
    assert o.fork([0, 1, 0, 2], [3, 4, 5, 6]) == 0 and int(pair.status) == 0
    pair.check_rows()
    pair.check_pages()
    start = dev([9] * 5)
    lib.cache_reserve(pair.cache.pool, dev([3, 4, -1, 5, 6]), dev([1, 40, 9, 3, 33]), 5, start, pair.status)
    want, status = o.reserve([3, 4, -1, 5, 6], [1, 40, 9, 3, 33])
    assert status == 0 and start.cpu().tolist() == want.tolist()
    kt, k = bf16(pair.rng.normal(size=(77, hkv, d)))
    offsets = [0, 1, 41, 41, 44, 77]
    lib.cache8_append(pair.cache, kt, kt, 0, 0, 77, None, 77, dev(offsets), dev([3, 4, -1, 5, 6]), start, 5, 40)
    o.append(k, k, None, offsets, [3, 4, -1, 5, 6], want)
    pair.check_rows()
    pair.check_pages()
    lib.cache8_fork(pair.cache, dev([3]), dev([0]), 1, pair.status)
    assert int(pair.status) == -1                                                        # slot 0 holds tokens
    lib.cache_release(pair.cache.pool, dev([0, 3, 1, 4, 2, 5, 6, 6, -1]), 9)
    o.release([0, 3, 1, 4, 2, 5, 6])
    pair.check_rows()
    assert not pair.refs.any()


def test_a_fork_of_pages_outside_the_pool(lib):
    pair = Pair8(lib, [70], 2, 64, 64, n_slots=2, max_pages=2)
    pair.o.table[0, 1] = 10 ** 8
    pair.up()
    before = pair.pages.clone()
    lib.cache8_fork(pair.cache, dev([0]), dev([1]), 1, pair.status)
    assert int(pair.status) == 0 and torch.equal(pair.pages, before) and int(pair.table[1, 0]) == int(pair.table[0, 0])


def test_offsets_past_32_bits(lib):
    """A pool of 5 GB and rows of 2^31 numbers and more: the same calls on their last pages and rows as on a small pool and few rows, bit for bit."""
    hkv, d, page, many, rows = 32, 128, 1024, 600, 530000
    one = lib.cache8_page_bytes(page, hkv, d)
    assert many * one > 1 << 32 and rows * hkv * d > 1 << 31
    gen = torch.Generator(device="cuda").manual_seed(5)
    near = [torch.randn((1500, hkv, d), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
    far = [torch.empty((rows, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for x, y in zip(near, far):
        y[rows - 1500:] = x
    q = torch.randn((1, 1, 32, d), generator=gen, device="cuda").to(torch.bfloat16)
    results = []
    for n_pages, k, v in ((6, *near), (many, *far)):
        n_rows, lift, shift = k.shape[0], n_pages - 6, k.shape[0] - 1500
        pages = torch.empty(n_pages * one, dtype=torch.uint8, device="cuda")
        refs, table, lens = torch.ones(n_pages, dtype=torch.int32, device="cuda"), torch.full((2, 3), -1, dtype=torch.int32, device="cuda"), dev([0, 0])
        refs[lift:] = 0
        pages[-6 * one:] = 0
        c = lib.make_cache8(pages, refs, table, lens, page, hkv, d)
        status, start, idx = dev([9]), dev([9]), torch.arange(shift, n_rows, dtype=torch.int32, device="cuda")
        positions = torch.zeros(n_rows, dtype=torch.int32, device="cuda")
        positions[shift:] = torch.arange(1500, dtype=torch.int32, device="cuda")
        rotation = lib.make_rotation(torch.full((64,), 0.3, device="cuda"), positions, 128)
        lib.cache_reserve(c.pool, dev([0]), dev([1500]), 1, start, status)
        q_out = torch.empty_like(k)
        lib.cache8_append(c, k, v, 0, 0, n_rows, idx, 1500, dev([0, 1500]), dev([0]), start, 1, 1500, rotation, k, 0, 32, q_out)
        lib.cache8_fork(c, dev([0]), dev([1]), 1, status)
        k_out, v_out = torch.empty_like(k), torch.empty_like(k)
        lib.cache8_load(c, dev([1]), dev([750]), dev([n_rows - 750, n_rows]), 1, 750, k_out, v_out, n_rows)
        blocks = torch.empty((1, 1, 32, 10), dtype=torch.int32, device="cuda")
        lib.cache8_select(c, q, dev([1]), 1, 1, 32, 1500, 1, 2, 7, blocks, torch.empty(256, dtype=torch.uint8, device="cuda"), 256)
        outs = []
        for lists in (None, blocks):
            out = torch.empty_like(q)
            width = 0 if lists is None else 10
            size = lib.cache8_attention_workspace_bytes(c, 1, 1, 32, 1500, width)
            ws = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
            lib.cache8_attention(c, q, dev([0]), 1, 1, 32, 1500, 0.0, lists, width, out, None, ws, size)
            outs.append(out.view(torch.int16))
        torch.cuda.synchronize()
        assert int(status) == 0 and int(start) == 0 and lens.cpu().tolist() == [1500, 1500]
        results.append((table.cpu() - lift * (table.cpu() >= 0), refs[lift:].cpu(), pages[-6 * one:].clone(), k_out[n_rows - 750:].view(torch.int16).clone(),
                        v_out[n_rows - 750:].view(torch.int16).clone(), q_out[shift:].view(torch.int16).clone(), blocks, *outs))
        del pages, k_out, v_out, q_out
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_another_stream_than_the_current_one(lib):
    pair = Pair8(lib, [900, 330], 4, 128, 32, n_slots=4, max_pages=30, spare=8)
    qt, q = bf16(pair.rng.normal(size=(2, 1, 8, 128)) * 0.05)
    kt, k = bf16(pair.rng.normal(size=(2, 4, 128)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    parents, children = dev([0, 1]), dev([2, 3])
    torch.cuda.synchronize()
    lib.cache8_fork(pair.cache, parents, children, 2, pair.status, stream=side)
    append(pair, kt, kt, 2, None, [0, 1, 2], [2, 3], [899, 329], 1, stream=side)
    blocks = select(pair, qt, [2, 3], 1, 900, 1, 1, 4, stream=side)
    out, lse = attend(pair, qt, [2, 3], 1, 900, blocks, stream=side)
    side.synchronize()
    pair.o.fork([0, 1], [2, 3])
    pair.o.append(k, k, None, [0, 1, 2], [2, 3], [899, 329])
    pair.check_pages()
    assert np.array_equal(blocks.cpu().numpy()[0], pair.o.select(q[0], 2, 1, 1, 4))
    check_attention(pair, q, [2, 3], out, lse, blocks=blocks.cpu().numpy())


def test_captured_steps_grow_the_sequences_on_every_replay(lib):
    """reserve, append with its turns, select and both attentions in a graph: every replay is a step, and what it leaves is what eager calls leave.  The program's
    own work goes on between replays; two graphs share the workspaces."""
    lens, hq, hkv, d, page, steps = [30, 1500, 63, 0], 8, 2, 128, 64, 6
    pairs = [Pair8(lib, lens, hkv, d, page, n_slots=5, max_pages=30, spare=30, seed=4) for _ in range(2)]
    rows = [bf16(pairs[0].rng.normal(size=(4, hq + 2 * hkv, d)))[0] for _ in range(steps)]
    slots, n_new, offsets = dev([2, 0, 1, 3, -1]), dev([1, 1, 1, 1, 1]), dev([0, 1, 2, 3, 4, 4])
    freqs = torch.from_numpy((10000.0 ** (-np.arange(64) / 64)).astype(np.float32)).cuda()
    most = page * 30
    sizes = [max(lib.cache8_attention_workspace_bytes(pairs[0].cache, 5, 1, hq, most, w) for w in (0, 9)), lib.cache8_select_workspace_bytes(pairs[0].cache, 5, 1, hq, most)]
    ws = [torch.empty(max(s, 256), dtype=torch.uint8, device="cuda") for s in sizes]
    bufs = []
    for pair in pairs:
        b = dict(x=torch.empty_like(rows[0]), q=torch.zeros((5, 1, hq, d), dtype=torch.bfloat16, device="cuda"), start=torch.empty(5, dtype=torch.int32, device="cuda"),
                 blocks=torch.empty((5, 1, hkv, 9), dtype=torch.int32, device="cuda"), positions=dev([2000, 30, 1500, 0]))
        for name in ("out", "sparse"):
            b[name] = torch.empty_like(b["q"])
            b[name + "_lse"] = torch.empty(5, 1, hq, dtype=torch.float32, device="cuda")
        b["rotation"] = lib.make_rotation(freqs, b["positions"], d)
        bufs.append(b)

    def step(pair, b):
        c, x = pair.cache, b["x"]
        lib.cache_reserve(c.pool, slots, n_new, 5, b["start"], pair.status)
        k, v = x[:, hq:hq + hkv], x[:, hq + hkv:]
        lib.cache8_append(c, k, v, x.stride(0), x.stride(0), 4, None, 4, offsets, slots, b["start"], 5, 1, b["rotation"], x, x.stride(0), hq, b["q"])
        lib.cache8_select(c, b["q"], slots, 5, 1, hq, most, 1, 2, 6, b["blocks"], ws[1], sizes[1])
        lib.cache8_attention(c, b["q"], slots, 5, 1, hq, most, 0.0, b["blocks"], 9, b["sparse"], b["sparse_lse"], ws[0], sizes[0])
        lib.cache8_attention(c, b["q"], slots, 5, 1, hq, most, 0.0, None, 0, b["out"], b["out_lse"], ws[0], sizes[0])
        b["positions"].add_(1)

    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(pairs[0], bufs[0])
        graphs.append(g)
    torch.cuda.synchronize()
    for i in range(steps):
        for b in bufs:
            b["x"].copy_(rows[i])
        graphs[i % 2].replay()
        step(pairs[1], bufs[1])
        torch.cuda.synchronize()
        for name in ("q", "out", "out_lse", "sparse", "sparse_lse", "start", "blocks", "positions"):
            assert torch.equal(bufs[0][name], bufs[1][name]), (i, name)
        for name in ("pages", "table", "refs", "lens"):
            assert torch.equal(getattr(pairs[0], name), getattr(pairs[1], name)), (i, name)
        o = pairs[0].o
        o.reserve([2, 0, 1, 3, -1], [1] * 5)
        o.pages, o.table = pairs[0].pages.cpu().numpy(), pairs[0].table.cpu().numpy()
        q = bufs[0]["q"].double().cpu().numpy()
        lists = bufs[0]["blocks"].cpu().numpy()
        assert np.array_equal(lists[2], o.select(q[2], 1, 1, 2, 6))
        check_attention(pairs[0], q, [2, 0, 1, 3, -1], bufs[0]["out"], bufs[0]["out_lse"])
        check_attention(pairs[0], q, [2, 0, 1, 3, -1], bufs[0]["sparse"], bufs[0]["sparse_lse"], blocks=lists)
    pairs[0].check_rows()


def test_two_calls_at_once(lib):
    """Two streams read one cache, each with its own workspaces."""
    pair = Pair8(lib, [9000, 500], 2, 128, 64)
    qs = [bf16(pair.rng.normal(size=(2, 1, 8, 128)) * 0.05) for _ in range(2)]
    reads = {s: pair.o.read(s) for s in range(2)}
    sizes = [lib.cache8_attention_workspace_bytes(pair.cache, 2, 1, 8, 9000, 0), lib.cache8_select_workspace_bytes(pair.cache, 2, 1, 8, 9000)]
    streams, slots = [torch.cuda.Stream() for _ in range(2)], dev([0, 1])
    bufs = [([torch.empty(max(s, 256), dtype=torch.uint8, device="cuda") for s in sizes], torch.empty_like(q[0]), torch.empty(2, 1, 8, dtype=torch.float32, device="cuda"),
             torch.empty((2, 1, 2, 20), dtype=torch.int32, device="cuda")) for q in qs]
    torch.cuda.synchronize()
    for _ in range(10):
        for st, q, (ws, out, lse, blocks) in zip(streams, qs, bufs):
            lib.cache8_attention(pair.cache, q[0], slots, 2, 1, 8, 9000, 0.0, None, 0, out, lse, ws[0], sizes[0], stream=st)
            lib.cache8_select(pair.cache, q[0], slots, 2, 1, 8, 9000, 1, 2, 17, blocks, ws[1], sizes[1], stream=st)
    torch.cuda.synchronize()
    for q, (ws, out, lse, blocks) in zip(qs, bufs):
        check_attention(pair, q[1], [0, 1], out, lse, reads=reads)
        assert np.array_equal(blocks.cpu().numpy()[0], pair.o.select(q[1][0], 0, 1, 2, 17))


def test_from_a_prompt_to_the_cache_and_through_its_updates(lib):
    """What a serving program does with the whole of it: a layer's prefill step chooses rows, they go into the cache, a branch takes new tokens turned by their places in
    the text and attends to chosen blocks, the cache is read back for the generation-phase update, and its choice becomes a cache of its own."""
    wl = synth.shrunk(synth.workload("cfg2"), (150, 97), n_q_heads=8, n_kv_heads=2, head_dim=128, w=16, hidden_dim=0)
    x = synth.make_inputs(wl)
    keep = np.array([90, 60], dtype=np.int32)
    x["keep_len"] = keep
    res = lib.prefill_layer_from_numpy(x, wl.w)
    F = synth.bf16_bits_to_f64
    pair = Pair8(lib, [], 2, 128, 32, n_slots=4, max_pages=6, spare=24, fill=0x5A)
    o = pair.o
    k, v = lib.to_device_bf16(x["k"]), lib.to_device_bf16(x["v"])
    start, koff = torch.empty(2, dtype=torch.int32, device="cuda"), np.array([0, 90, 150])
    lib.cache_reserve(pair.cache.pool, dev([0, 1]), dev(keep), 2, start, pair.status)
    lib.cache8_append(pair.cache, k, v, 0, 0, k.shape[0], dev(res["kept_idx"]), 150, dev(koff), dev([0, 1]), start, 2, 90)
    o.reserve([0, 1], keep)
    o.append(F(x["k"]), F(x["v"]), res["kept_idx"], koff, [0, 1], [0, 0])
    pair.check_rows()
    pair.check_pages()
    # a branch of both grows by two tokens, whose places are those in the text
    lib.cache8_fork(pair.cache, dev([0, 1]), dev([2, 3]), 2, pair.status)
    o.fork([0, 1], [2, 3])
    lib.cache_reserve(pair.cache.pool, dev([2, 3]), dev([2, 2]), 2, start, pair.status)
    o.reserve([2, 3], [2, 2])
    fused, new = bf16(pair.rng.normal(size=(4, 12, 128)) * 0.3)
    positions, freqs = dev([150, 151, 97, 98]), (10000.0 ** (-np.arange(64) / 64)).astype(np.float32)
    rotation = lib.make_rotation(torch.from_numpy(freqs).cuda(), positions, 128)
    q = torch.empty((2, 2, 8, 128), dtype=torch.bfloat16, device="cuda")
    lib.cache8_append(pair.cache, fused[:, 8:10], fused[:, 10:], 12 * 128, 12 * 128, 4, None, 4, dev([0, 2, 4]), dev([2, 3]), start, 2, 2, rotation, fused, 12 * 128, 8, q)
    pair.check_rows()
    turned = orc.turn(new[:, :10], [150, 151, 97, 98], freqs, 128, 0)
    o.pages = pair.pages.cpu().numpy()
    for s, rows in ((2, slice(0, 2)), (3, slice(2, 4))):
        held = o.read(s, int(keep[s - 2]))[0]
        # half a step of a number's own, or of the least that the block's power holds; the block's largest is at most 2^5 here: 2^-4 * 2^-14
        assert (np.abs(held - turned[rows, 8:]) <= 2.0 ** -4 * np.abs(turned[rows, 8:]) * 1.001 + 2.0 ** -12).all()
    assert (np.abs(q.double().cpu().numpy().reshape(4, 8, 128) - turned[:, :8]) <= 2.0 ** -8 * np.abs(turned[:, :8]) + 2.0 ** -18).all()
    blocks = select(pair, q, [2, 3], 2, 92, 1, 1, 1)
    q64 = q.double().cpu().numpy()
    for b in range(2):
        assert np.array_equal(blocks.cpu().numpy()[b], o.select(q64[b], 2 + b, 1, 1, 1))
    check_attention(pair, q64, [2, 3], *attend(pair, q, [2, 3], 2, 92, blocks), blocks=blocks.cpu().numpy())
    check_attention(pair, q64, [2, 3], *attend(pair, q, [2, 3], 2, 92))
    # read back, updated, what is kept stored anew: numbers of the cache are numbers of the cache again
    off = np.array([0, 92, 154], dtype=np.int32)
    kb, vb = (torch.empty((154, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lib.cache8_load(pair.cache, dev([2, 3]), None, dev(off), 2, 92, kb, vb, 154)
    q_win = pair.rng.normal(size=(2, 16, 8, 128)).astype(np.float32)
    q_bits = torch.from_numpy(q_win).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
    upd = lib.decode_update_from_numpy(q_bits, lib.to_host_bits(kb), lib.to_host_bits(vb), off, [70, 40], 16)
    lib.cache_release(pair.cache.pool, dev([2, 3]), 2)
    lib.cache_reserve(pair.cache.pool, dev([2, 3]), dev([70, 40]), 2, start, pair.status)
    lib.cache8_append(pair.cache, kb, vb, 0, 0, 154, dev(upd["kept_idx"]), 110, dev([0, 70, 110]), dev([2, 3]), start, 2, 70)
    o.release([2, 3])
    o.reserve([2, 3], [70, 40])
    o.append(kb.double().cpu().numpy(), vb.double().cpu().numpy(), upd["kept_idx"], [0, 70, 110], [2, 3], [0, 0])
    pair.check_rows()
    pair.check_pages()
    check_attention(pair, q64, [2, 3], *attend(pair, q, [2, 3], 2, 70))
    lib.cache_release(pair.cache.pool, dev([0, 1, 2, 3]), 4)
    assert not pair.refs.any()
