"""CPU-only checks of the entry points on a cache held in 8 bits: sizes, and arguments that have to be refused before anything is launched."""
import ctypes

import pytest

from paper_2405_12532_amd import binding

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3, -6


def cache(**change):
    fields = dict(pages=0x10000, refs=0x20000, table=0x30000, lens=0x40000, n_pages=100, page_tokens=64, n_slots=8, max_pages=16, n_kv_heads=4, head_dim=128)
    return binding.PyrCache8(binding.PyrCache(**dict(fields, **change)))


BAD_CACHES = [(dict(pages=None), NULL), (dict(refs=None), NULL), (dict(table=None), NULL), (dict(lens=None), NULL), (dict(pages=0x10080), UNSUPPORTED),
              (dict(head_dim=96), UNSUPPORTED), (dict(page_tokens=48), UNSUPPORTED), (dict(page_tokens=16), UNSUPPORTED), (dict(page_tokens=2048), UNSUPPORTED),
              (dict(page_tokens=0), SHAPE), (dict(n_pages=0), SHAPE), (dict(n_slots=0), SHAPE), (dict(n_slots=262145), SHAPE), (dict(max_pages=0), SHAPE),
              (dict(n_kv_heads=0), SHAPE), (dict(n_pages=1 << 25), UNSUPPORTED), (dict(max_pages=1 << 25), UNSUPPORTED), (dict(n_kv_heads=40000), UNSUPPORTED),
              (dict(n_kv_heads=30000, page_tokens=1024), UNSUPPORTED)]


def call(name, *args):
    return getattr(binding.load(), name)(*args)


def calls(c, n):
    """Every call that launches, with arguments that pass but for the cache and the number of rows."""
    ref = None if c is None else ctypes.byref(c)
    return dict(
        fork=call("pyr_cache8_fork", ref, 0x1000, 0x2000, n, 0x4000, None),
        append=call("pyr_cache8_append", ref, 0x1000, 0x2000, 0, 0, 5, None, 5, 0x3000, 0x4000, 0x5000, n, 5, None, None, 0, 0, None, None),
        load=call("pyr_cache8_load", ref, 0x1000, None, 0x2000, n, 5, 0x3000, 0x4000, 5, None),
        select=call("pyr_cache8_select", ref, 0x1000, 0x2000, n, 1, 4 if c is None else max(c.pool.n_kv_heads, 1), 64, 1, 1, 1, 0x3000, 0x100, 1 << 20, None),
        attention=call("pyr_cache8_attention", ref, 0x1000, 0x2000, n, 1, 4 if c is None else max(c.pool.n_kv_heads, 1), 64, 0.0, None, 0, 0x3000, None, 0x100, 1 << 20, None))


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_a_cache_that_cannot_be(change, status):
    assert set(calls(cache(**change), 2).values()) == {status}


def test_no_cache_and_negative_rows():
    assert set(calls(None, 2).values()) == {NULL}
    assert set(calls(cache(), -1).values()) == {SHAPE}
    assert set(v for k, v in calls(cache(), 0).items() if k != "fork") == {OK}


def test_sizes():
    for page, heads, d in ((64, 32, 128), (32, 1, 64), (1024, 8, 128)):
        exact = heads * page // 32 * (66 * d + 2)
        size = binding.cache8_page_bytes(page, heads, d)
        assert size % 256 == 0 and exact <= size < exact + 256
    for bad in ((48, 1, 64), (64, 1, 80), (1024, 30000, 128)):
        with pytest.raises(binding.PyrError) as e:
            binding.cache8_page_bytes(*bad)
        assert e.value.status == UNSUPPORTED
    long = cache(n_pages=4096, max_pages=1024)
    assert binding.cache8_attention_workspace_bytes(long, 0, 1, 8, 64, 0) == 0
    assert binding.cache8_attention_workspace_bytes(long, 512, 1, 8, 1024, 0) == 0          # many sequences fill the chip by themselves; one long one is split
    size = binding.cache8_attention_workspace_bytes(long, 1, 1, 8, 65536, 0)
    assert size >= 2 * 8 * (128 + 2) * 4 and size % 256 == 0
    assert binding.cache8_attention_workspace_bytes(long, 1, 1, 8, 1 << 30, 0) == size      # (no more than a slot holds)
    assert binding.cache8_attention_workspace_bytes(long, 1, 1, 8, 65536, 4) == 0           # lists of four blocks
    assert binding.cache8_select_workspace_bytes(long, 200, 1, 8, 65536) == 0
    assert binding.cache8_select_workspace_bytes(long, 1, 1, 8, 65536) == 2048 * 4 * 4
    assert [binding.cache8_select_workspace_bytes(long, 24, 1, 8, 32 * b) for b in (1536, 1537)] == [0, (1537 * 96 * 4 + 255) // 256 * 256]
    assert [binding.cache8_select_workspace_bytes(long, 23, 1, 8, 32 * b) for b in (512, 513)] == [0, (513 * 92 * 4 + 255) // 256 * 256]
    r = binding.diag_cache8_attention(long, 1, 1, 8, 65536, 0)
    assert r.splits > 1 and r.chunk % r.waves == 0 and r.repeats == 1
    assert call("pyr_diag_cache8_attention", ctypes.byref(long), 1, 1, 8, 100, 0, None) == NULL


def test_descriptions_do_not_mix():
    """A cache in 4 bits is none in 8: ctypes refuses one for the other; handing out and giving back pages take the pool."""
    class Stream:
        cuda_stream = None
    with pytest.raises(ctypes.ArgumentError):
        binding.cache8_fork(binding.PyrCache(), None, None, 0, None, Stream)
    with pytest.raises(ctypes.ArgumentError):
        binding.cache_release(cache(), None, 0, Stream)
    with pytest.raises(ctypes.ArgumentError):
        binding.cache_fork(cache(), None, None, 0, None, Stream)
    binding.cache_release(cache().pool, None, 0, Stream)


def test_pages_of_8_bits_are_none_of_4():
    """What writes or reads numbers of 4 bits refuses the pool of a cache held in 8, before anything is launched; handing out and giving back its pages takes both."""
    class Stream:
        cuda_stream = None
    pool = cache().pool
    for call_4 in (lambda c: binding.cache_store(c, None, None, 0, None, 0, None, None, None, 0, 0, Stream),
                   lambda c: binding.cache_load(c, None, None, 0, 0, None, None, 0, Stream),
                   lambda c: binding.cache_fork(c, None, None, 0, None, Stream),
                   lambda c: binding.cache_compact(c, None, 0, None, 0, None, None, 0, None, None, 0, Stream),
                   lambda c: binding.cache_attention(c, None, None, 0, 1, 4, 0, 0.0, None, None, None, 0, Stream),
                   lambda c: binding.cache_compact_workspace_bytes(c, 1), lambda c: binding.cache_attention_workspace_bytes(c, 1, 1, 4, 64),
                   lambda c: binding.diag_cache_attention(c, 1, 1, 4, 64)):
        with pytest.raises(ctypes.ArgumentError):
            call_4(pool)
    four = binding.PyrCache(0x10000, 0x20000, 0x30000, 0x40000, 100, 64, 8, 16, 4, 128)
    for c in (pool, four):
        binding.cache_release(c, None, 0, Stream)
        with pytest.raises(binding.PyrError):
            binding.cache_reserve(c, None, None, 0, None, None, Stream)                  # (no status: refused by the library itself)
    assert (pool.n_pages, pool.page_tokens, pool.n_kv_heads) == (four.n_pages, four.page_tokens, four.n_kv_heads)


def test_tensors_that_do_not_belong_together():
    import torch
    size = binding.cache8_page_bytes(32, 2, 64)
    pages, refs, table, lens = torch.zeros(4 * size, dtype=torch.uint8), torch.zeros(4, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    c = binding.make_cache8(pages, refs, table, lens, 32, 2, 64).pool
    assert (c.n_pages, c.page_tokens, c.n_slots, c.max_pages, c.n_kv_heads, c.head_dim) == (4, 32, 3, 2, 2, 64)
    for bad in ((pages[1:], refs, table, lens), (pages, refs, table.t(), lens), (pages, refs, table, lens[1:]), (pages, torch.zeros(5, dtype=torch.int32), table, lens),
                (pages, refs.float(), table, lens), (pages, refs, table.long(), lens)):
        with pytest.raises(ValueError):
            binding.make_cache8(*bad, 32, 2, 64)
    freqs, positions = torch.zeros(32), torch.zeros(7, dtype=torch.int32)
    r = binding.make_rotation(freqs, positions, 64, True)
    assert (r.dims, r.interleaved) == (64, 1)
    for bad in ((freqs, positions, 66), (freqs.double(), positions, 64), (freqs, positions.long(), 64), (torch.zeros(64)[::2], positions, 64)):
        with pytest.raises(ValueError):
            binding.make_rotation(*bad)


def test_rows_without_a_position():
    """A rotation that is kept from a smaller batch: its positions would be read behind their end."""
    import torch

    class Stream:
        cuda_stream = None
    rows, ints, freqs, positions = torch.zeros((9, 4, 128), dtype=torch.bfloat16), torch.zeros(9, dtype=torch.int32), torch.zeros(64), torch.zeros(7, dtype=torch.int32)

    def append(n_rows, rotation):                                                        # (of no sequences: nothing is launched)
        binding.cache8_append(cache(), rows, rows, 0, 0, n_rows, None, n_rows, ints, ints, ints, 0, 9, rotation, stream=Stream)
    for pairs in (False, True):
        rotation = binding.make_rotation(freqs, positions, 128, pairs)
        append(7, rotation)
        append(0, rotation)
        for n_rows in (8, 9):
            with pytest.raises(ValueError):
                append(n_rows, rotation)
    append(9, binding.make_rotation(freqs, positions, 0))                                # nothing turns: none is read
    append(9, binding.PyrRotation(0x1000, 0x2000, 64, 0))                                # addresses: the caller's to know
    append(9, None)


def test_choices_that_one_launch_cannot_make():
    """A launch has fewer than 2^32 threads: 2^24 workgroups of up to four wavefronts, half of them of eight."""
    few, many = cache(n_kv_heads=1, max_pages=128), cache(n_kv_heads=1, max_pages=1024)
    for n, most, fine in (((1 << 24) - 1, 8192, True), (1 << 24, 8192, False), ((1 << 23) - 1, 8192 + 1, True), (1 << 23, 8192 + 1, False), (1 << 23, 16384, False),
                          ((1 << 23) - 1, 65536, True), (1 << 23, 65536, False), (1 << 23, 2 ** 31 - 1, False)):
        size, c = ctypes.c_size_t(0), ctypes.byref(many)
        assert call("pyr_cache8_select_workspace_bytes", c, n, 1, 1, most, ctypes.byref(size)) == (OK if fine else UNSUPPORTED), (n, most)
        if not fine:
            assert call("pyr_cache8_select", c, 0x1000, 0x2000, n, 1, 1, most, 1, 1, 1, 0x3000, 0x100, 1 << 62, None) == UNSUPPORTED
    size = ctypes.c_size_t(0)                                                            # (this one's slots hold 8192 tokens)
    assert call("pyr_cache8_select_workspace_bytes", ctypes.byref(few), (1 << 24) - 1, 1, 1, 2 ** 31 - 1, ctypes.byref(size)) == OK


def test_rows_and_sizes_that_cannot_be():
    c = ctypes.byref(cache())
    assert call("pyr_cache8_fork", c, 0x1000, None, 2, 0x4000, None) == NULL
    assert call("pyr_cache8_fork", c, 0x1000, 0x2000, 4097, 0x4000, None) == SHAPE
    assert call("pyr_cache8_fork", c, 0x1000, 0x2000, 2, None, None) == NULL

    def append(k=0x1000, ks=0, vs=0, rows=5, idx=None, listed=5, start=0x5000, n=2, most=5, turn=None, q=None, qs=0, hq=0, q_out=None):
        rotation = None if turn is None else ctypes.byref(binding.PyrRotation(*turn))
        return call("pyr_cache8_append", c, k, 0x2000, ks, vs, rows, idx, listed, 0x3000, 0x4000, start, n, most, rotation, q, qs, hq, q_out, None)
    assert append(k=None) == NULL and append(start=None) == NULL and append(k=0x1008) == UNSUPPORTED
    assert append(rows=-1) == SHAPE and append(listed=4) == SHAPE and append(idx=0x6000, listed=-1) == SHAPE and append(most=-1) == SHAPE
    assert append(ks=511) == UNSUPPORTED and append(vs=516) == UNSUPPORTED and append(ks=-512) == UNSUPPORTED and append(vs=1 << 40) == UNSUPPORTED
    assert append(turn=(0x1000, 0x2000, 24, 0)) == UNSUPPORTED and append(turn=(0x1000, 0x2000, 144, 0)) == SHAPE and append(turn=(0x1000, 0x2000, -16, 0)) == SHAPE
    assert append(turn=(None, 0x2000, 64, 0)) == NULL and append(turn=(0x1000, None, 64, 0)) == NULL
    assert append(q=0x7000, hq=8) == NULL and append(q=0x7000, q_out=0x8000, hq=0) == SHAPE and append(q=0x7000, q_out=0x8000, hq=6) == UNSUPPORTED
    assert append(q=0x7000, q_out=0x8008, hq=8) == UNSUPPORTED and append(q=0x7000, q_out=0x8000, hq=8, qs=1000) == UNSUPPORTED
    assert append(n=0) == OK and append(most=0) == OK and append(rows=0, listed=0) == OK and append(n=1 << 30, most=64) == UNSUPPORTED

    def load(k=0x3000, v=0x4000, rows=5, n=2, most=5, offsets=0x2000):
        return call("pyr_cache8_load", c, 0x1000, None, offsets, n, most, k, v, rows, None)
    assert load(k=None, v=None) == NULL and load(offsets=None) == NULL and load(k=0x3008) == UNSUPPORTED
    assert load(rows=-1) == SHAPE and load(most=-1) == SHAPE and load(rows=0) == OK and load(most=0) == OK
    assert load(n=1 << 30, rows=1 << 30, most=64) == UNSUPPORTED

    def select(q=0x1000, slots=0x2000, n=2, tokens=1, hq=8, most=64, first=1, recent=1, best=1, blocks=0x3000, ws=0x100, size=1 << 20, of=c):
        return call("pyr_cache8_select", of, q, slots, n, tokens, hq, most, first, recent, best, blocks, ws, size, None)
    assert select(q=None) == NULL and select(slots=None) == NULL and select(blocks=None) == NULL and select(q=0x1008) == UNSUPPORTED
    assert select(tokens=0) == SHAPE and select(most=-1) == SHAPE and select(first=-1) == SHAPE and select(recent=0) == SHAPE and select(best=-1) == SHAPE
    assert select(hq=6) == UNSUPPORTED and select(n=1 << 23, tokens=2) == UNSUPPORTED and select(first=1 << 30, best=1 << 30) == UNSUPPORTED and select(best=1 << 26) == UNSUPPORTED
    long = ctypes.byref(cache(n_pages=4096, max_pages=1024))
    assert select(of=long, n=1, most=65536, ws=None) == WORKSPACE and select(of=long, n=1, most=65536, size=100) == WORKSPACE and select(of=long, n=1, most=65536, ws=0x180) == WORKSPACE

    def attention(q=0x1000, n=2, tokens=1, hq=8, most=64, blocks=None, width=0, out=0x3000, ws=0x100, size=1 << 20, of=c):
        return call("pyr_cache8_attention", of, q, 0x2000, n, tokens, hq, most, 0.0, blocks, width, out, None, ws, size, None)
    assert attention(q=None) == NULL and attention(out=None) == NULL and attention(q=0x1008) == UNSUPPORTED
    assert attention(tokens=0) == SHAPE and attention(most=-1) == SHAPE and attention(width=-1) == SHAPE and attention(width=3) == SHAPE
    assert attention(blocks=0x4000) == SHAPE and attention(blocks=0x4000, width=(1 << 26) + 1) == UNSUPPORTED and attention(hq=6) == UNSUPPORTED and attention(n=1 << 23, tokens=1 << 9) == UNSUPPORTED
    assert attention(of=long, n=1, most=65536, ws=None) == WORKSPACE and attention(of=long, n=1, most=65536, size=100) == WORKSPACE
