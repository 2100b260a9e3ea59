"""What the calls of 8-bit caches, of pages and of adjusted logits refuse, and in which order: on the host, before anything is enqueued (no GPU needed)."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_1911_02150_amd", "libmqa_decode.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built (run __graft_entry__.build())")

vp, ci, cf, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
A = 0x10000                                                                # aligned, never dereferenced on these paths ...
U = 0x70004                                                                # ... and one that is not
NULL, SHAPE, ALIGN, WORKSPACE, DTYPE = 1, 2, 3, 4, 5
E4M3, INT8 = 2, 3


def entry(name, pointers, sizes, tail):
    fn = getattr(ctypes.CDLL(LIB), name)
    fn.argtypes = [vp] * pointers + [ci] * sizes + tail
    return fn


def places(count):
    return [A + 0x1000 * x for x in range(count)]


def but(ptrs, x, value):
    return [value if y == x else p for y, p in enumerate(ptrs)]


def bad_cache_sizes():
    return [dict(b=0), dict(h_kv=0), dict(num_pages=0), dict(page_size=-1), dict(max_pages=0), dict(k=24), dict(v=0), dict(k=272), dict(v=8), dict(v=1 << 20),
            dict(block=0), dict(block=-4), dict(block=3), dict(block=32),
            dict(page_size=1 << 20, max_pages=17), dict(b=1 << 12, h_kv=1 << 13), dict(b=1 << 12, max_pages=1 << 16), dict(num_pages=1 << 28),
            dict(num_pages=1 << 30, page_size=1, block=1)]


@pytest.mark.parametrize("dt", [E4M3, INT8])
def test_scaled_append_refuses(dt):
    fn = entry("mqa_paged_scaled_append_kv_rows", 10, 10, [vp])
    sizes = dict(b=2, n=3, h_kv=2, num_pages=8, page_size=16, block=8, max_pages=4, k=128, v=64, dt=dt)

    def call(ptrs=places(10), **kw):
        return fn(*ptrs, *{**sizes, **kw}.values(), None)

    for x in range(10):
        if x != 2:                                                             # (counts may be missing)
            assert call(but(places(10), x, None)) == NULL
        assert call(but(places(10), x, U)) == ALIGN
    for other in (0, 1, 4, -1):
        assert call(dt=other) == DTYPE
    for s in bad_cache_sizes() + [dict(n=0), dict(n=65), dict(b=1 << 20, n=64, h_kv=1, max_pages=1, page_size=64, block=8),
                                  dict(b=1 << 18, n=40, h_kv=1, page_size=16, block=1, k=16, v=16)]:
        assert call(**s) == SHAPE, s
    ptrs = places(10)
    assert call(but(ptrs, 9, ptrs[8])) == SHAPE and call(but(ptrs, 9, ptrs[2])) == SHAPE      # the lengths in place


@pytest.mark.parametrize("dt", [E4M3, INT8])
def test_scaled_decode_refuses(dt):
    fn = entry("mqa_paged_scaled_decode_step", 8, 11, [cf, vp, sz, vp])
    size = entry("mqa_paged_scaled_decode_workspace_bytes", 0, 9, [])
    size.restype = sz
    sizes = dict(b=2, n=3, h=4, h_kv=2, num_pages=64, page_size=16, block=16, max_pages=64, k=128, v=64, dt=dt)
    need = size(2, 3, 4, 2, 16, 64, 128, 64, dt)
    assert need > 0

    def call(ptrs=places(8), ws=A, nbytes=1 << 40, **kw):
        return fn(*ptrs, *{**sizes, **kw}.values(), 1.0, ws, nbytes, None)

    for x in range(8):
        assert call(but(places(8), x, None)) == NULL
        assert call(but(places(8), x, U)) == ALIGN
    for other in (0, 1, 4):
        assert call(dt=other) == DTYPE
    for s in bad_cache_sizes() + [dict(n=0), dict(h=0), dict(h=3), dict(n=513), dict(b=1 << 14, n=256, max_pages=1)]:
        assert call(**s) == SHAPE, s
    assert call(ws=None) == WORKSPACE and call(nbytes=need - 1) == WORKSPACE and call(ws=U) == ALIGN
    for s in ((0, 3, 4, 2, 16, 64, 128, 64, dt), (2, 3, 5, 2, 16, 64, 128, 64, dt), (2, 3, 4, 2, 16, 64, 136, 64, dt), (2, 3, 4, 2, 16, 64, 128, 64, 1)):
        assert size(*s) == 0


def bad_table_sizes():
    return [dict(b=0), dict(num_pages=0), dict(page_size=0), dict(max_pages=-1), dict(num_pages=(1 << 24) + 1), dict(page_size=1 << 20, max_pages=17),
            dict(b=1 << 20, max_pages=1 << 9)]


def test_fork_refuses():
    fn = entry("mqa_paged_fork_pages", 6, 5, [vp])
    sizes = dict(b=2, b_out=3, num_pages=64, page_size=16, max_pages=8)

    def call(ptrs=places(6), **kw):
        return fn(*ptrs, *{**sizes, **kw}.values(), None)

    ptrs = places(6)
    for x in range(6):
        assert call(but(ptrs, x, None)) == NULL
        assert call(but(ptrs, x, U)) == ALIGN
    for s in bad_table_sizes() + [dict(b_out=0), dict(b_out=1 << 20, max_pages=1 << 9)]:
        assert call(**s) == SHAPE, s
    for x, y in ((0, 3), (1, 4), (2, 4)):
        assert call(but(ptrs, y, ptrs[x])) == SHAPE


def test_free_refuses():
    fn = entry("mqa_paged_free_pages", 3, 4, [vp])
    sizes = dict(b=2, num_pages=64, page_size=16, max_pages=8)
    for x in range(3):
        assert fn(*but(places(3), x, None), *sizes.values(), None) == NULL
        assert fn(*but(places(3), x, U), *sizes.values(), None) == ALIGN
    for s in bad_table_sizes():
        assert fn(*places(3), *{**sizes, **s}.values(), None) == SHAPE, s


def test_reserve_refuses():
    fn = entry("mqa_paged_reserve_pages", 6, 5, [vp, sz, vp])
    size = entry("mqa_paged_reserve_workspace_bytes", 0, 5, [])
    size.restype = sz
    sizes = dict(b=2, n=3, num_pages=64, page_size=16, max_pages=8)
    need = size(*sizes.values())
    assert need > 0 and size(0, 3, 64, 16, 8) == size(2, 0, 64, 16, 8) == size(2, 129, 64, 16, 8) == 0

    def call(ptrs=places(6), ws=A, nbytes=1 << 30, **kw):
        return fn(*ptrs, *{**sizes, **kw}.values(), ws, nbytes, None)

    ptrs = places(6)
    for x in range(6):
        if x != 2:
            assert call(but(ptrs, x, None)) == NULL
        assert call(but(ptrs, x, U)) == ALIGN
    for s in bad_table_sizes() + [dict(n=0), dict(n=129), dict(b=(1 << 20) + 1)]:
        assert call(**s) == SHAPE, s
    assert call(but(ptrs, 4, ptrs[1])) == SHAPE and call(but(ptrs, 4, ptrs[2])) == SHAPE
    assert call(ws=None) == WORKSPACE and call(nbytes=need - 1) == WORKSPACE and call(ws=U) == ALIGN


def test_compact_refuses():
    fn = entry("mqa_paged_compact_pages", 6, 3, [vp, sz, vp])
    size = entry("mqa_paged_compact_workspace_bytes", 0, 3, [])
    size.restype = sz
    need = size(2, 64, 8)
    assert need > 0 and size(0, 64, 8) == size(2, 0, 8) == size(2, (1 << 24) + 1, 8) == 0

    def call(ptrs=places(6), b=2, num_pages=64, max_pages=8, ws=A, nbytes=1 << 30):
        return fn(*ptrs, b, num_pages, max_pages, ws, nbytes, None)

    ptrs = places(6)
    for x in range(6):
        assert call(but(ptrs, x, None)) == NULL
        assert call(but(ptrs, x, U)) == ALIGN
    for s in (dict(b=0), dict(num_pages=0), dict(max_pages=0), dict(num_pages=(1 << 24) + 1), dict(b=1 << 20, max_pages=1 << 9)):
        assert call(**s) == SHAPE, s
    assert call(but(ptrs, 2, ptrs[0])) == SHAPE and call(but(ptrs, 3, ptrs[1])) == SHAPE
    assert call(ws=None) == WORKSPACE and call(nbytes=need - 1) == WORKSPACE and call(ws=U) == ALIGN


def test_copy_refuses():
    fn = entry("mqa_paged_copy_pages", 2, 1, [vp, ci, ci, vp])

    def call(pools=(A, 2 * A), page_bytes=(4096, 64), num_pools=2, moves=A, m=5, num_pages=64):
        return fn((vp * len(pools))(*pools) if pools else None, (sz * len(page_bytes))(*page_bytes) if page_bytes else None, num_pools, moves, m, num_pages, None)

    assert call(pools=None) == NULL and call(page_bytes=None) == NULL and call(moves=None) == NULL and call(pools=(A, None)) == NULL
    for s in (dict(num_pools=0), dict(num_pools=4097), dict(m=0), dict(m=(1 << 28) + 1), dict(num_pages=0), dict(num_pages=(1 << 24) + 1),
              dict(page_bytes=(4096, 0)), dict(page_bytes=(4096, 66)), dict(page_bytes=(4096, (1 << 30) + 4))):
        assert call(**s) == SHAPE, s
    assert call(pools=(A, U)) == ALIGN and call(moves=U) == ALIGN


def test_adjust_refuses():
    fn = entry("mqa_stack_adjust_logits", 12, 5, [vp])
    sizes = dict(b=2, n=4, vocab=1000, cap=64, biases=8)

    def call(ptrs=places(12), **kw):
        return fn(*ptrs, *{**sizes, **kw}.values(), None)

    ptrs = places(12)
    for x in (0, 1, 2, 3, 5, 9, 10):                                            # (penalties, prompts and the mask may be missing)
        assert call(but(ptrs, x, None)) == NULL
    for x in range(12):
        assert call(but(ptrs, x, U)) == ALIGN
    for s in (dict(b=0), dict(n=-1), dict(n=(1 << 16) + 1), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(cap=-1), dict(cap=(1 << 24) + 1), dict(biases=-1),
              dict(biases=(1 << 24) + 1), dict(b=1 << 23, vocab=513), dict(b=1 << 10, cap=(1 << 21) + 1)):
        assert call(**s) == SHAPE, s


def test_the_calls_of_other_caches_refuse_8_bits():
    fn = entry("mqa_paged_append_kv_rows", 8, 9, [vp])
    for dt in (E4M3, INT8):
        assert fn(*places(8), 2, 3, 2, 8, 16, 4, 128, 64, dt, None) == DTYPE


def test_python_refuses_on_the_host():
    """Wrong tensors are named before the library is called."""
    import torch

    import paper_1911_02150_amd as m
    t, i = torch.zeros((2, 3, 16)), torch.zeros((2, 3), dtype=torch.int32)
    for call in (lambda: m.mqa_paged_scaled_append_kv_rows(t, t, t, t, t, t, t, t, t), lambda: m.mqa_paged_scaled_decode_step(t, t, t, t, t, t, t),
                 lambda: m.mqa_paged_fork_pages(i, i, i, i, i, i, 16), lambda: m.mqa_paged_free_pages(i, i, i, 16), lambda: m.mqa_paged_reserve_pages(i, i, i, 16, 1),
                 lambda: m.mqa_paged_compact_pages(i, i, i, i, i, i), lambda: m.mqa_paged_copy_pages([t], i), lambda: m.mqa_stack_adjust_logits(t, i, i)):
        with pytest.raises(ValueError, match="must be a device tensor"):
            call()
    with pytest.raises(ValueError, match="no pools"):
        m.mqa_paged_copy_pages([], i)
