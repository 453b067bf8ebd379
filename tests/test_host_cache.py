"""CPU-only checks of the cache's entry points: sizes, and arguments that have to be refused before anything is launched."""
import ctypes

import pytest

from paper_2405_12532_amd import binding

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3, -6


def cache(**change):
    fields = dict(pages=0x10000, refs=0x20000, table=0x30000, lens=0x40000, n_pages=100, page_tokens=64, n_slots=8, max_pages=16, n_kv_heads=4, head_dim=128)
    return binding.PyrCache(**dict(fields, **change))


BAD_CACHES = [(dict(pages=None), NULL), (dict(refs=None), NULL), (dict(table=None), NULL), (dict(lens=None), NULL), (dict(pages=0x10080), UNSUPPORTED),
              (dict(head_dim=96), UNSUPPORTED), (dict(page_tokens=48), UNSUPPORTED), (dict(page_tokens=16), UNSUPPORTED), (dict(page_tokens=2048), UNSUPPORTED),
              (dict(page_tokens=0), SHAPE), (dict(n_pages=0), SHAPE), (dict(n_slots=0), SHAPE), (dict(n_slots=262145), SHAPE), (dict(max_pages=0), SHAPE),
              (dict(n_kv_heads=0), SHAPE), (dict(n_pages=1 << 25), UNSUPPORTED), (dict(max_pages=1 << 25), UNSUPPORTED), (dict(n_kv_heads=40000), UNSUPPORTED)]


def call(name, *args):
    return getattr(binding.load(), name)(*args)


def calls(c):
    """Every call that launches, with arguments that pass but for the cache."""
    ref = None if c is None else ctypes.byref(c)
    return dict(
        reserve=call("pyr_cache_reserve", ref, 0x1000, 0x2000, -1 if c is not None and _fine(c) else 2, 0x3000, 0x4000, None),
        fork=call("pyr_cache_fork", ref, 0x1000, 0x2000, -1 if c is not None and _fine(c) else 2, 0x4000, None),
        release=call("pyr_cache_release", ref, 0x1000, -1 if c is not None and _fine(c) else 2, None),
        compact=call("pyr_cache_compact", ref, 0x1000, -1 if c is not None and _fine(c) else 2, 0x2000, 5, 0x3000, 0x4000, 5, 0x5000, 0x100, 1 << 20, None),
        store=call("pyr_cache_store", ref, 0x1000, 0x2000, 5, None, 5, 0x3000, 0x4000, 0x5000, -1 if c is not None and _fine(c) else 2, 5, None),
        load=call("pyr_cache_load", ref, 0x1000, 0x2000, -1 if c is not None and _fine(c) else 2, 5, 0x3000, 0x4000, 5, None),
        attention=call("pyr_cache_attention", ref, 0x1000, 0x2000, -1 if c is not None and _fine(c) else 2, 1, 8, 64, 0.0, 0x3000, None, 0x100, 1 << 20, None))


def _fine(c):
    return not any(bytes(c) == bytes(cache(**change)) for change, _ in BAD_CACHES)


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_a_cache_that_cannot_be(change, status):
    assert set(calls(cache(**change)).values()) == {status}


def test_no_cache_and_negative_rows():
    assert set(calls(None).values()) == {NULL}
    assert set(calls(cache()).values()) == {SHAPE}


def test_sizes():
    for page, heads, d in ((64, 32, 128), (32, 1, 64), (1024, 8, 128)):
        assert binding.cache_page_bytes(page, heads, d) == page * heads * d * 34 // 32
    for bad in ((48, 1, 64), (64, 1, 80)):
        with pytest.raises(binding.PyrError) as e:
            binding.cache_page_bytes(*bad)
        assert e.value.status == UNSUPPORTED
    c = cache()
    assert binding.cache_compact_workspace_bytes(c, 3) == 256 and binding.cache_compact_workspace_bytes(c, 0) == 0
    assert binding.cache_compact_workspace_bytes(cache(max_pages=100), 10) % 256 == 0
    assert binding.cache_compact_workspace_bytes(cache(max_pages=100), 10) >= 10 * 101 * 4
    assert binding.cache_attention_workspace_bytes(c, 0, 1, 8, 64) == 0
    # many sequences fill the chip by themselves; one long one is split
    assert binding.cache_attention_workspace_bytes(c, 512, 1, 8, 1024) == 0
    long = cache(n_pages=4096, max_pages=1024)
    size = binding.cache_attention_workspace_bytes(long, 1, 1, 8, 65536)
    assert size >= 2 * 8 * (128 + 2) * 4 and size % 256 == 0
    assert binding.cache_attention_workspace_bytes(long, 1, 1, 8, 1 << 30) == size          # (no more than a slot holds)


def test_a_cache_of_tensors_that_do_not_belong_together():
    import torch
    pages, refs, table, lens = torch.zeros(4 * 2176 * 2, dtype=torch.uint8), torch.zeros(4, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    c = binding.make_cache(pages, refs, table, lens, 32, 2, 64)
    assert (c.n_pages, c.page_tokens, c.n_slots, c.max_pages, c.n_kv_heads, c.head_dim) == (4, 32, 3, 2, 2, 64)
    for bad in ((pages[1:], refs, table, lens), (pages, refs, table.t(), lens), (pages, refs, table, lens[1:]), (pages, torch.zeros(5, dtype=torch.int32), table, lens)):
        with pytest.raises(ValueError):
            binding.make_cache(*bad, 32, 2, 64)


def test_how_an_attention_is_cut_up():
    c = cache(n_pages=1 << 15, max_pages=2048, n_slots=256, n_kv_heads=8)
    for n, tokens, hq, most, want in ((1, 1, 32, 1000, (1, 4, 8, 1, 1)), (1, 1, 32, 1537, (1, 4, 8, 1, 4)), (1, 1, 64, 1 << 16, (1, 2, 8, 1, 32)),
                                      (20, 1, 64, 8000, (1, 2, 4, 1, 4)), (64, 1, 32, 1 << 17, (1, 4, 4, 1, 1)), (33, 2, 64, 100, (1, 1, 4, 1, 1)),
                                      (1, 5, 64, 100, (2, 1, 4, 2, 1)), (4, 4, 64, 4096, (2, 1, 4, 1, 4)), (0, 1, 8, 100, (1, 4, 4, 1, 1)), (1, 1, 8, 0, (1, 4, 8, 1, 1))):
        r = binding.diag_cache_attention(c, n, tokens, hq, most)
        assert (r.col_tiles, r.repeats, r.waves, r.col_groups, r.splits) == want, (n, tokens, hq, most)
        assert r.chunk > 0 and r.chunk % r.waves == 0
    assert binding.diag_cache_attention(cache(head_dim=64), 1, 1, 16, 100).repeats == 2
    assert call("pyr_diag_cache_attention", ctypes.byref(c), 1, 1, 8, 100, None) == NULL
    with pytest.raises(binding.PyrError):
        binding.diag_cache_attention(c, 1, 0, 8, 100)


def test_rows_and_sizes_that_cannot_be():
    c = ctypes.byref(cache())
    assert call("pyr_cache_reserve", c, 0x1000, 0x2000, 4097, 0x3000, 0x4000, None) == SHAPE
    assert call("pyr_cache_reserve", c, 0x1000, 0x2000, 2, 0x3000, None, None) == NULL
    assert call("pyr_cache_reserve", c, None, 0x2000, 2, 0x3000, 0x4000, None) == NULL
    assert call("pyr_cache_reserve", c, 0x1000, 0x2000, 2, None, 0x4000, None) == NULL
    assert call("pyr_cache_reserve", ctypes.byref(cache(max_pages=1 << 20, page_tokens=32)), 0x1000, 0x2000, 4096, 0x3000, 0x4000, None) == UNSUPPORTED
    assert call("pyr_cache_fork", c, 0x1000, None, 2, 0x4000, None) == NULL
    assert call("pyr_cache_fork", c, 0x1000, 0x2000, 4097, 0x4000, None) == SHAPE
    assert call("pyr_cache_release", c, None, 2, None) == NULL
    assert call("pyr_cache_release", c, None, 0, None) == OK

    def compact(kept=0x2000, n_kept=5, out=0x4000, most=5, ws=0x100, size=1 << 20, n=2):
        return call("pyr_cache_compact", c, 0x1000, n, kept, n_kept, 0x3000, out, most, 0x5000, ws, size, None)
    assert compact(kept=None) == NULL and compact(out=None) == NULL
    assert compact(n_kept=-1) == SHAPE and compact(most=-1) == SHAPE and compact(n=4097) == SHAPE
    assert compact(ws=None) == WORKSPACE and compact(ws=0x180) == WORKSPACE and compact(size=100) == WORKSPACE

    def store(k=0x1000, rows=5, idx=None, listed=5, start=0x5000, n=2, most=5):
        return call("pyr_cache_store", c, k, 0x2000, rows, idx, listed, 0x3000, 0x4000, start, n, most, None)
    assert store(k=None) == NULL and store(start=None) == NULL and store(k=0x1008) == UNSUPPORTED
    assert store(rows=-1) == SHAPE and store(listed=4) == SHAPE and store(idx=0x6000, listed=-1) == SHAPE and store(most=-1) == SHAPE
    assert store(n=0) == OK and store(most=0) == OK and store(rows=0, listed=0) == OK and store(n=1 << 30, most=64) == UNSUPPORTED

    def load(k=0x3000, v=0x4000, rows=5, n=2, most=5):
        return call("pyr_cache_load", c, 0x1000, 0x2000, n, most, k, v, rows, None)
    assert load(k=None, v=None) == NULL and load(k=0x3008) == UNSUPPORTED and load(rows=-1) == SHAPE and load(most=-1) == SHAPE
    assert load(n=0) == OK and load(rows=0) == OK and load(most=0) == OK and load(n=1 << 30, most=64) == UNSUPPORTED


def test_attention_arguments_that_cannot_be():
    c = cache(n_pages=4096, max_pages=1024)

    def attend(q=0x1000, slots=0x2000, n=2, tokens=1, heads=8, most=65536, out=0x3000, ws=0x100, size=1 << 30):
        return call("pyr_cache_attention", ctypes.byref(c), q, slots, n, tokens, heads, most, 0.0, out, None, ws, size, None)
    assert attend(q=None) == NULL and attend(slots=None) == NULL and attend(out=None) == NULL
    assert attend(q=0x1008) == UNSUPPORTED and attend(out=0x3008) == UNSUPPORTED
    assert attend(tokens=0) == SHAPE and attend(heads=0) == SHAPE and attend(most=-1) == SHAPE
    assert attend(heads=6) == UNSUPPORTED and attend(heads=40000) == UNSUPPORTED and attend(n=1 << 30) == UNSUPPORTED
    assert attend(ws=None) == WORKSPACE and attend(ws=0x180) == WORKSPACE and attend(size=1000) == WORKSPACE
    assert attend(n=0) == OK


def test_calls_of_more_workgroups_than_a_launch_has():
    """2^24 of 256 threads; limits as large as an int32 are brought down to what a slot holds first."""
    most = 2 ** 31 - 1
    c = cache(n_slots=262144, page_tokens=1024, max_pages=256, n_pages=4096)                # 8192 tiles a slot
    ref = ctypes.byref(c)
    assert call("pyr_cache_release", ref, 0x1000, 1 << 24, None) == UNSUPPORTED
    assert call("pyr_cache_compact", ref, 0x1000, 2048, 0x2000, most, 0x3000, 0x4000, most, 0x5000, 0x100, 1 << 30, None) == UNSUPPORTED
    assert call("pyr_cache_store", ref, 0x1000, 0x2000, most, None, most, 0x3000, 0x4000, 0x5000, 2048, most, None) == UNSUPPORTED
    assert call("pyr_cache_load", ref, 0x1000, 0x2000, 2048, most, 0x3000, 0x4000, most, None) == UNSUPPORTED
    assert call("pyr_cache_attention", ref, 0x1000, 0x2000, 1 << 22, 1, 4, most, 0.0, 0x3000, None, 0x100, 1 << 30, None) == UNSUPPORTED
    binding.cache_attention_workspace_bytes(c, (1 << 22) - 1, 1, 4, most)
    assert call("pyr_cache_attention", ref, 0x1000, 0x2000, 0, 1 << 29, 8, most, 0.0, 0x3000, None, 0x100, 1 << 30, None) == UNSUPPORTED


@pytest.mark.parametrize("which,change", [(1, lambda t: t.long()), (2, lambda t: t.long()), (3, lambda t: t.short()), (1, lambda t: t.view(2, 2)), (2, lambda t: t.view(-1)),
                                          (3, lambda t: t.view(3, 1))])
def test_a_cache_of_tensors_of_another_type_or_shape(which, change):
    import torch
    tensors = [torch.zeros(4 * 2176 * 2, dtype=torch.uint8), torch.zeros(4, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)]
    binding.make_cache(*tensors, 32, 2, 64)
    tensors[which] = change(tensors[which])
    with pytest.raises(ValueError):
        binding.make_cache(*tensors, 32, 2, 64)


def test_an_attention_of_any_number_of_heads_is_cut_up():
    """Splits cover the cache, and their workgroups are no more than what a launch and its join are worth."""
    c = cache(n_pages=1 << 15, max_pages=2048, n_slots=4096, n_kv_heads=1)
    for d, g, tokens in ((128, 4, 1), (64, 8, 1), (128, 16, 1), (128, 8, 4)):
        c.head_dim = d
        for n in list(range(1, 1100, 7)) + [64, 65, 128, 129, 200, 256, 257, 384, 385, 512, 513, 768, 769]:
            for most in (0, 1, 1200, 1300, 1537, 2048, 2049, 100000):
                r = binding.diag_cache_attention(c, n, tokens, g, most)
                tiles = -(-most // 32)
                assert r.splits >= 1 and (r.splits - 1) * r.chunk < max(tiles, 1) <= r.splits * r.chunk
                assert r.splits == 1 or (n * r.splits < 1024 and r.chunk >= 16)
    c.head_dim = 128
    assert [binding.diag_cache_attention(c, n, 1, 4, 8000).splits for n in (160, 384, 385, 480, 769)] == [4, 2, 1, 1, 1]
    assert [binding.diag_cache_attention(c, n, 4, 8, 8000).splits for n in (160, 384, 385, 480, 769)] == [4, 2, 1, 1, 1]
    assert [binding.diag_cache_attention(c, n, 1, 4, 1536).splits for n in (1, 64, 160, 300)] == [1, 1, 1, 1]
    assert [binding.diag_cache_attention(c, n, 1, 4, 2048).splits > 1 for n in (1, 144, 145, 256)] == [True, True, False, False]


@pytest.mark.parametrize("which", [1, 2, 3])
def test_a_cache_of_other_tensors_of_four_bytes(which):
    import torch
    for other in (torch.float32, torch.uint32):
        tensors = [torch.zeros(4 * 2176 * 2, dtype=torch.uint8), torch.zeros(4, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)]
        tensors[which] = tensors[which].to(other)
        with pytest.raises(ValueError):
            binding.make_cache(*tensors, 32, 2, 64)


@pytest.mark.parametrize("which", [0, 1, 2, 3])
def test_a_cache_of_tensors_on_two_devices(which):
    import torch
    tensors = [torch.zeros(4 * 2176 * 2, dtype=torch.uint8), torch.zeros(4, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)]
    tensors[which] = tensors[which].to("meta")
    with pytest.raises(ValueError):
        binding.make_cache(*tensors, 32, 2, 64)
