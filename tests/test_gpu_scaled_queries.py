"""Attention over pages of 8 bits, query rows beside one another: what a row holds, and whether it sees anything, is nothing to the rows that share its workgroup."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_gpu_scaled import attended, cache_of, f32, i32, tables, tolerance  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = ["e4m3", "int8"]


@pytest.fixture(scope="module")
def m():
    import paper_1911_02150_amd as mod
    mod.load_library()
    return mod


def close(got, want, bound):
    """Equal where `want` is no finite number, else within the bound."""
    got, finite = got.astype(np.float64).reshape(want.shape), np.isfinite(want)
    assert np.array_equal(got[~finite], want[~finite], equal_nan=True)
    off = np.abs(got[finite] - want[finite])
    assert (off <= bound[finite]).all(), off.max()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("padding", [np.inf, -np.inf, 1e30, -3e38, np.nan])
@pytest.mark.parametrize("n,h,h_kv,k,times", [(5, 3, 1, 128, 1), (5, 8, 1, 128, 1), (3, 16, 2, 64, 1), (4, 8, 4, 48, 1), (6, 6, 1, 256, 1), (5, 8, 1, 128, 50), (7, 5, 1, 64, 45)])
def test_padded_queries_may_hold_anything(m, n, h, h_kv, k, times, padding, kind):
    """Sequences of fewer positions than there are new tokens, beside long ones: the queries that see nothing are padding, and their rows 0."""
    rng = np.random.default_rng(n * h + k)
    lens = np.array(list(range(n + 1)) * times + [700, n - 1])
    b, page = len(lens), 16
    each = -(-int(lens.max()) // page) + 1
    arrays, cache = cache_of(rng, b, each, h_kv, page, 16, k, k, kind)
    table = tables(rng, b, each)
    q = rng.standard_normal((b, n, h, k)).astype(np.float32)
    sees = lens[:, None] - (n - 1 - np.arange(n)) > 0
    clean = np.where(sees[:, :, None, None], q, 0).astype(np.float32)
    want, size, K, top = attended(clean, arrays, table, lens, 0.2)
    q[~sees] = padding
    got = m.mqa_paged_scaled_decode_step(f32(q), *cache, i32(table), i32(lens), scale=0.2).cpu().numpy()
    assert not got[~sees].any()
    close(got, want, tolerance(clean, K, size, 0.2, int(lens.max()), kind, top))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,h,length", [(500, 2, 1043), (256, 4, 1043), (128, 8, 1010), (33, 24, 4000)])
def test_an_infinite_query_is_its_own_row_s(m, n, h, length, kind):
    """Every eighth token's queries hold infinities, and what they see is NaN: the tokens after it see positions, and pieces of the work, that it does not."""
    rng = np.random.default_rng(n + h)
    page, k, scale = 16, 64, 0.1
    each = -(-length // page)
    arrays, cache = cache_of(rng, 1, each, 1, page, 16, k, k, kind)
    table, lens = tables(rng, 1, each), np.array([length])
    q = rng.standard_normal((1, n, h, k)).astype(np.float32)
    q[:, ::8, :, 5] = np.inf
    want, size, K, top = attended(q, arrays, table, lens, scale)
    assert np.isnan(want[:, ::8]).all() and np.isfinite(np.delete(want, np.s_[::8], axis=1)).all()
    got = m.mqa_paged_scaled_decode_step(f32(q), *cache, i32(table), i32(lens), scale=scale).cpu().numpy()
    close(got, want, tolerance(np.delete(q, np.s_[::8], axis=1), K, size, scale, length, kind, top))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("h,k", [(8, 128), (30, 128), (16, 64), (40, 48), (9, 256), (33, 208)])
@pytest.mark.parametrize("steps", [3, 7, 9, 20, 40, 63, 70, 100])
def test_queries_of_sizes_apart(m, h, k, steps, kind):
    """Rows whose numbers are 2^steps apart, twice that for the third of every four, and zeros: each is as exact as it is alone."""
    rng = np.random.default_rng(h + k + steps)
    arrays, cache = cache_of(rng, 2, 30, 1, 16, 16, k, k, kind)
    table, lens = tables(rng, 2, 30), np.array([470, 33])
    q = (0.3 * rng.standard_normal((2, 1, h, k))).astype(np.float32)
    for r in range(h):
        q[:, :, r] *= np.float32(2.0 ** min((0, steps, 2 * steps, 0)[r % 4], 100))
    q[:, :, 4] = 0
    want, size, K, top = attended(q, arrays, table, lens, 0.1)
    got = m.mqa_paged_scaled_decode_step(f32(q[:, 0]), *cache, i32(table), i32(lens), scale=0.1).cpu().numpy()
    for r in range(h):
        close(got[:, r], want[:, 0, r], tolerance(q[:, :, r], K, size[:, 0, r], 0.1, 470, kind, top[:, 0, r]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("padding", [np.inf, 1e30, np.nan])
@pytest.mark.parametrize("n,h,h_kv,k", [(5, 8, 1, 128), (4, 8, 4, 64), (6, 6, 1, 200)])
def test_padded_queries_over_wider_caches(m, n, h, h_kv, k, padding, dtype):
    """The same over pages of float32 and bfloat16."""
    from oracle import paged
    from test_gpu_paged import on_gpu, pool, tolerance as bound
    rng = np.random.default_rng(n * h + k)
    lens = np.array(list(range(n + 1)) + [700, n - 1])
    b, page, each = len(lens), 16, 45
    K, V = (pool(rng, b * each, h_kv, page, k, dtype) for _ in range(2))
    table = tables(rng, b, each)
    q = rng.standard_normal((b, n, h, k)).astype(np.float32)
    sees = lens[:, None] - (n - 1 - np.arange(n)) > 0
    clean = np.where(sees[:, :, None, None], q, 0).astype(np.float32)
    want, _, size = paged.attend(clean.astype(np.float64), K, V, table, lens, float(np.float32(0.2)))
    q[~sees] = padding
    one = h_kv == 1
    got = m.mqa_paged_decode_step(on_gpu(q), on_gpu(K, dtype, one), on_gpu(V, dtype, one), on_gpu(table), on_gpu(lens), scale=0.2).cpu().numpy()
    assert not got[~sees].any()
    close(got, want, bound(clean, K, size, 0.2, 700))
