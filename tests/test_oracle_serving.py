"""The oracle of the 8-bit caches, of the pages and of the adjusted logits, held against what is known without it (no GPU needed)."""
import numpy as np
import pytest

from oracle import paged, serving

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_rounding(kind):
    """Every number of 8 bits is itself; halfway to the next one goes to the even one, a little less or more to the nearer."""
    if kind == "e4m3":
        every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
        every = np.unique(every[np.isfinite(every)])
    else:
        every = np.arange(-127.0, 128.0)
    assert np.array_equal(serving.rounded(every, kind), every) and every[-1] == serving.LARGEST[kind]
    middle = (every[1:] + every[:-1]) / 2
    got = serving.rounded(middle, kind)
    assert np.all((got == every[1:]) | (got == every[:-1]))
    if kind == "e4m3":
        assert np.array_equal(got, torch.from_numpy(middle).float().to(torch.float8_e4m3fn).double().numpy())
    else:
        assert np.array_equal(got % 2, np.zeros_like(got))
    for toward, want in ((1e-9, every[1:]), (-1e-9, every[:-1])):
        assert np.array_equal(serving.rounded(middle + toward * np.maximum(1e-3, np.abs(middle)), kind), want)
    odd = serving.rounded(np.array([np.inf, -np.inf, 1e30]), kind)
    assert np.array_equal(odd, np.array([1, -1, 1]) * serving.LARGEST[kind])
    assert np.isnan(serving.rounded(np.nan, kind)) if kind == "e4m3" else serving.rounded(np.nan, kind) == 0


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_scale(kind):
    top = serving.LARGEST[kind]
    for e in (-126, -3, 0, 40):
        assert serving.scale_of(top * 2.0 ** e, kind) == 2.0 ** e
        assert serving.scale_of(top * 2.0 ** e * (1 + 2.0 ** -23), kind) == 2.0 ** (e + 1)
    assert serving.scale_of(0.0, kind) == 2.0 ** -126


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_appending_bit_by_bit(kind):
    """A value is off by half a step of the scale that its block has in the end, and less than half a step more for the scales before it; all at once by half a step."""
    rng = np.random.default_rng(3)
    new = rng.standard_normal((2, 40, 1, 16)) * np.exp(rng.standard_normal((2, 40, 1, 1)))
    table = np.array([[3, 1, 5], [0, 4, 2]])
    caches = []
    for steps in ([40], [1] * 40, [3, 7, 13, 17]):
        K, Ks, V, Vs = np.zeros((6, 1, 16, 16)), np.zeros((6, 1, 2)), np.zeros((6, 1, 16, 16)), np.zeros((6, 1, 2))
        lens = np.zeros(2, dtype=np.int64)
        for n in steps:
            at = lens[0]
            lens = serving.append(K, Ks, V, Vs, table, new[:, at:at + n], -new[:, at:at + n], lens, kind=kind)
        assert (lens == 40).all() and np.array_equal(K, -V) and np.array_equal(Ks, Vs)
        caches.append((K, Ks))
        values = serving.whole(K, Ks)
        for i in range(2):
            for p in range(40):
                page, row = paged.where(table, i, p, 6, 16)
                s, x = Ks[page, 0, row // 8], new[i, p, 0]
                step = s if kind == "int8" else s * 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(x) / s, 1e-9))), -6) - 3)
                assert (np.abs(values[page, 0, row] - x) <= (0.5 if len(steps) == 1 else 1.0) * step * (1 + 1e-9)).all()
    for _, scales in caches:                                      # however the rows came: the largest of a block decides
        assert np.array_equal(scales[table.ravel()[[0, 1, 3, 4]]], caches[0][1][table.ravel()[[0, 1, 3, 4]]])


def test_pages_add_up():
    """Random turns of forks, reservations, ends and compactions: the counts stay those of the tables, nobody writes to a shared page."""
    rng = np.random.default_rng(11)
    page, pages, each, b = 4, 12, 6, 5
    refs, table, lens = np.zeros(pages, dtype=np.int64), np.full((b, each), -1), np.zeros(b, dtype=np.int64)
    seen = set()
    for turn in range(300):
        counts = rng.integers(0, 6, b)
        granted, moves = serving.reserve(table, lens, refs, page, 5, counts=counts)
        seen |= {("refused", bool((granted < counts).any())), ("copied", bool((moves >= 0).any()))}
        for i in range(b):
            for p in range(lens[i], lens[i] + granted[i]):
                at = paged.where(table, i, p, pages, page)
                assert at is not None and refs[at[0]] == 1
        lens = lens + granted
        assert np.array_equal(refs, np.bincount(table[table >= 0], minlength=pages))
        kept = np.where(rng.random(b) < 0.3, 0, np.maximum(lens - rng.integers(0, 4, b), 0))
        serving.free(table, kept, refs, page)
        lens = kept
        parents = rng.integers(-1, b + 1, b)
        if turn % 3 == 0:
            table_new, lens_new = serving.fork(table, lens, parents, refs, page)
            serving.free(table, np.zeros(b, dtype=np.int64), refs, page)
            table, lens = table_new, lens_new
        if turn % 7 == 0:
            table, refs, moves, used = serving.compact(table, refs)
            assert (refs[:used] > 0).all() and not refs[used:].any()
        assert np.array_equal(refs, np.bincount(table[table >= 0], minlength=pages))
    assert len(seen) == 4


def test_adjusted_logits_by_hand():
    x = np.array([[[1.0, -1.0, 2.0, 3.0, 0.5], [1.0, -1.0, 2.0, 3.0, 0.5]]])
    allowed = np.ones((1, 2, 5), dtype=bool)
    allowed[0, 1, 3] = False
    got = serving.adjust(x, np.array([[0, 1, 1, 7, 4]]), [4], drafts=np.array([[2]]), prompts=[1], repetition=[2.0], frequency=[0.25], presence=[1.0],
                         bias_tokens=np.array([[3, 3, 9]]), biases=np.array([[5.0, 0.5, 1.0]]), allowed=allowed)
    assert np.array_equal(got[0, 0], [0.5, -2 - 1.5, 2.0, 3.5, 0.5])
    assert np.array_equal(got[0, 1], [0.5, -2 - 1.5, 1 - 1.25, -np.inf, 0.5])
