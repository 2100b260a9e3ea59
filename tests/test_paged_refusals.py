"""What the paged calls and the verification of drafts refuse, and in which order: on the host, before anything is enqueued (no GPU needed)."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_1911_02150_amd", "libmqa_decode.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built (run __graft_entry__.build())")

vp, ci, cf, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
A, B, C, D, E, F, U = (0x10000 * x for x in (1, 2, 3, 4, 5, 6, 7))          # aligned, never dereferenced on these paths ...
U += 4                                                                     # ... and one that is not
NULL, SHAPE, ALIGN, WORKSPACE, DTYPE = 1, 2, 3, 4, 5


def entry(name, pointers, sizes, tail):
    fn = getattr(ctypes.CDLL(LIB), name)
    fn.argtypes = [vp] * pointers + [ci] * sizes + tail
    return fn


def with_(d, **kw):
    return {**d, **kw}


SIZES = dict(b=2, n=3, h_kv=2, num_pages=8, page_size=16, max_pages=4, k=128, v=64, dt=1)


def bad_cache_sizes():
    return [dict(b=0), dict(h_kv=0), dict(num_pages=0), dict(page_size=-1), dict(max_pages=0), dict(k=12), dict(v=0), dict(k=264), dict(v=1 << 20),
            dict(page_size=1 << 20, max_pages=17),                             # more than 2^24 positions
            dict(b=1 << 12, h_kv=1 << 13),                                     # more than 2^24 heads of sequences
            dict(b=1 << 12, max_pages=1 << 16),                                # b * h_kv * positions past 2^31
            dict(num_pages=1 << 28), dict(num_pages=1 << 30, page_size=1)]      # rows of the pool past 2^31


def test_append_refuses():
    fn = entry("mqa_paged_append_kv_rows", 8, 9, [vp])

    def call(ptrs=(A, B, None, C, D, E, A, F), **kw):
        return fn(*ptrs, *with_(SIZES, **kw).values(), None)

    for x in range(8):
        if x != 2:                                                             # (counts may be missing)
            assert call([None if y == x else A for y in range(8)]) == NULL
    assert call(dt=2) == DTYPE and call([None] + [A] * 7, dt=2) == NULL
    for sizes in bad_cache_sizes() + [dict(n=0), dict(n=65), dict(b=1 << 20, n=64, h_kv=1, max_pages=1, page_size=64)]:
        assert call(**sizes) == SHAPE, sizes
    assert call((A, B, None, C, D, E, F, F)) == SHAPE                          # the lengths in place
    for x in range(8):
        assert call([U if y == x else A + 0x1000 * y for y in range(8)]) == ALIGN


def test_decode_refuses():
    fn = entry("mqa_paged_decode_step", 8, 10, [cf, vp, sz, vp])
    size = entry("mqa_paged_decode_workspace_bytes", 0, 10, [])
    size.restype = sz
    sizes = dict(b=2, n=3, h=4, h_kv=2, num_pages=64, page_size=16, max_pages=64, k=128, v=64, dt=1)
    need = size(2, 3, 4, 2, 16, 64, 128, 64, 1, 0)
    scored = size(2, 3, 4, 2, 16, 64, 128, 64, 1, 1)
    assert 0 < need < scored

    def call(ptrs=(A, B, C, D, E, F, None, None), ws=A, nbytes=1 << 40, **kw):
        return fn(*ptrs, *with_(sizes, **kw).values(), 1.0, ws, nbytes, None)

    for x in range(6):
        assert call([None if y == x else A for y in range(6)] + [None, None]) == NULL
    assert call((A, B, C, D, E, F, A, None)) == NULL                           # scores to add to, and nowhere to put them
    assert call(dt=-1) == DTYPE
    for s in bad_cache_sizes() + [dict(n=0), dict(h=0), dict(h=3), dict(n=513), dict(b=1 << 14, n=256, max_pages=1)]:
        assert call(**s) == SHAPE, s
    for x in range(8):
        assert call([U if y == x else A for y in range(8)]) == ALIGN
    assert call(ws=None) == WORKSPACE and call(nbytes=need - 1) == WORKSPACE and call(ws=U) == ALIGN
    assert call((A, B, C, D, E, F, A, A), nbytes=scored - 1) == WORKSPACE
    for s in ((0, 3, 4, 2, 16, 64, 128, 64, 1, 0), (2, 3, 5, 2, 16, 64, 128, 64, 1, 0), (2, 3, 4, 2, 16, 64, 100, 64, 1, 0), (2, 3, 4, 2, 16, 64, 128, 64, 2, 0)):
        assert size(*s) == 0


def test_evict_refuses():
    fn = entry("mqa_paged_evict_kv", 9, 11, [vp])
    sizes = dict(b=2, h_kv=2, num_pages=64, page_size=16, max_pages=4, max_pages_out=2, k=128, v=64, dt=1, budget=32, recent=8)
    places = [A + 0x1000 * x for x in range(9)]

    def call(ptrs=places, **kw):
        return fn(*ptrs, *with_(sizes, **kw).values(), None)

    for x in range(9):
        assert call([None if y == x else p for y, p in enumerate(places)]) == NULL
        assert call([U if y == x else p for y, p in enumerate(places)]) == ALIGN
    assert call(dt=7) == DTYPE
    for s in bad_cache_sizes() + [dict(max_pages_out=0), dict(budget=0), dict(budget=33), dict(recent=-1), dict(recent=33), dict(max_pages_out=1 << 21),
                                 dict(b=1 << 21, max_pages=1), dict(b=1 << 20, max_pages=16, max_pages_out=16, budget=256)]:
        assert call(**s) == SHAPE, s
    for x, y in ((2, 5), (3, 6), (4, 7)):                                      # in place
        assert call([places[x] if z == y else p for z, p in enumerate(places)]) == SHAPE


def test_verify_refuses():
    fn = entry("mqa_stack_verify_drafts", 7, 3, [cf, vp, sz, vp])
    size = entry("mqa_stack_verify_workspace_bytes", 0, 3, [])
    size.restype = sz
    need = size(2, 4, 1000)
    assert need > 0 and size(0, 4, 1000) == size(2, -1, 1000) == size(2, 4, 0) == size(1, 1, (1 << 24) + 1) == size(1 << 20, 8, 8) == 0

    def call(ptrs=(A,) * 7, b=2, n=4, vocab=1000, temperature=1.0, ws=A, nbytes=1 << 30):
        return fn(*ptrs, b, n, vocab, temperature, ws, nbytes, None)

    for x in (0, 2, 4, 5, 6):                                                  # (draft logits and counts may be missing)
        assert call([None if y == x else A for y in range(7)]) == NULL
    for s in (dict(b=0), dict(n=-1), dict(vocab=0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf"))):
        assert call(**s) == SHAPE, s
    for x in range(7):
        assert call([U if y == x else A for y in range(7)]) == ALIGN
    assert call(ws=None) == WORKSPACE and call(nbytes=need - 1) == WORKSPACE and call(ws=U) == ALIGN


def test_python_refuses_on_the_host():
    """Wrong tensors are named before the library is called."""
    import torch

    import paper_1911_02150_amd as m
    t = torch.zeros((2, 3, 8))
    with pytest.raises(ValueError, match="must be a device tensor"):
        m.mqa_paged_decode_step(t, t, t, t, t)
    with pytest.raises(ValueError, match="must be a device tensor"):
        m.mqa_stack_verify_drafts(t, None, None)
    with pytest.raises(ValueError, match="must be a device tensor"):
        m.mqa_paged_append_kv_rows(t, t, t, t, t, t, t)
    with pytest.raises(ValueError, match="must be a device tensor"):
        m.mqa_paged_evict_kv(t, t, t, t, t, t, t, t, t, 0)


def test_append_refuses_counts_in_place():
    """The new lengths into the array of the counts: a sequence's other workgroups would read what the first one wrote."""
    fn = entry("mqa_paged_append_kv_rows", 8, 9, [vp])
    assert fn(A, B, F, C, D, E, A + 0x1000, F, *SIZES.values(), None) == SHAPE
