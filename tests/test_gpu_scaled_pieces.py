"""Attention over pages of 8 bits: the work of more sequences than a wave looks through, with several K/V heads, found by all of a workgroup and from a list."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_gpu_scaled import attended, cache_of, f32, i32, tolerance  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def m():
    import paper_1911_02150_amd as mod
    mod.load_library()
    return mod


# lengths, K/V heads, heads: as many as a wave looks through and one more; a thread has one, two, three and four; long ones among short ones, whole and in pieces; a list
LENGTHS = [
    ([40, 700, 0, 31, 260] * 13, 2, 2),
    ([300, 31, 650] * 40, 2, 8),
    ([64, 0, 1100, 3, 90] * 60, 4, 4),
    ([9, 33, 900] * 100, 3, 60),
    ([33] * 199 + [2100], 8, 8),
    ([128, 5] * 260, 2, 36),
    ([20, 900, 64] * 170, 2, 4),
    ([1000, 31, 0, 64] * 200, 2, 2),
    ([31] * 1022 + [0, 1700], 2, 2),
    ([20, 33] * 515 + [900], 2, 2),
    ([64, 0, 300] * 400, 3, 3),
]


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("lens,h_kv,h", LENGTHS, ids=lambda x: str(len(x)) if isinstance(x, list) else str(x))
def test_pieces_of_many_sequences_and_heads(m, lens, h_kv, h, kind):
    """Sequences share pages; a table of a capacity that is cut."""
    b, k, page, scale, pages = len(lens), 32, 16, 0.25, 300
    rng = np.random.default_rng(b + h)
    each = -(-max(lens) // page)
    arrays, cache = cache_of(rng, 1, pages, h_kv, page, page, k, k, kind)
    table = rng.integers(0, pages, (b, each))
    order = rng.permutation(b)
    lens = np.array(lens)[order]
    q = rng.standard_normal((b, 1, h, k)).astype(np.float32)
    wide = np.concatenate([table, np.full((b, 1000 - each), -1)], 1)
    got = m.mqa_paged_scaled_decode_step(f32(q[:, 0]), *cache, i32(wide), i32(lens), scale=scale)
    want, size, K, top = attended(q, arrays, table, lens, scale)
    assert (np.abs(got.cpu().numpy().reshape(want.shape) - want) <= tolerance(q, K, size, scale, int(lens.max()), kind, top)).all()
    again = m.mqa_paged_scaled_decode_step(f32(q[:, 0]), *cache, i32(wide), i32(lens), scale=scale)
    assert torch.equal(got, again)
