"""Attention over pages of 8 bits whose scales are not what an append chooses."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_gpu_scaled import EPS, attended, bits, cache_of, f32, i32, tables, tolerance  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = ["e4m3", "int8"]


@pytest.fixture(scope="module")
def m():
    import paper_1911_02150_amd as mod
    mod.load_library()
    return mod


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("h,k,length", [(4, 128, 300), (20, 64, 40), (16, 48, 1500), (17, 256, 70), (32, 128, 20)])
def test_infinite_scales_of_k(m, h, k, length, kind):
    """A block's logits are infinities, or NaN where products of both signs meet: NaN rows, but for those whose logits there are all -infinity, which see the rest."""
    rng = np.random.default_rng(h + k)
    each = -(-length // 16)
    (K, Ks, V, Vs), _ = cache_of(rng, 1, each, 1, 16, 16, k, k, kind)
    table, lens = tables(rng, 1, each), np.array([length])
    Ks[table[0, 1]] = np.inf
    K[table[0, 1]] = np.maximum(np.abs(K[table[0, 1]]), 1)
    q = rng.standard_normal((1, 1, h, k)).astype(np.float32)
    q[0, 0, 0::4], q[0, 0, 1::4] = np.abs(q[0, 0, 0::4]), -np.abs(q[0, 0, 1::4])
    want, size, _, top = attended(q, (K, Ks, V, Vs), table, lens, 0.1)
    nan = np.arange(h) % 4 != 1
    assert np.isnan(want[0, 0, nan]).all() and np.isfinite(want[0, 0, ~nan]).all()
    got = m.mqa_paged_scaled_decode_step(f32(q[:, 0]), bits(K, kind, True), f32(Ks, True), bits(V, kind, True), f32(Vs, True), i32(table), i32(lens), scale=0.1).cpu().numpy()
    assert np.isnan(got[0, nan]).all()
    finite = np.where(np.isfinite(Ks), Ks, 0)
    bound = tolerance(q, K * np.repeat(finite, 16, axis=2)[..., None], size, 0.1, length, kind, top)
    assert (np.abs(got[0] - want[0, 0])[~nan] <= bound[0, 0][~nan]).all()


@pytest.mark.parametrize("kind", KINDS)
def test_logits_of_any_size_are_told_apart(m, kind):
    """K's scales of 2^120 and queries of 2^30 whose products are with zeros: the logits are -8 2^120 times 3, 1 and 2, and the one with the least takes all the weight."""
    (K, Ks, V, Vs), _ = cache_of(np.random.default_rng(3), 1, 1, 1, 3, 1, 64, 64, kind)
    K[:] = 0
    K[0, 0, :, 0] = 3, 1, 2
    Ks[:] = 2.0 ** 120
    q = np.full((1, 16, 64), 2.0 ** 30, dtype=np.float32)
    q[:, :, 0] = -8
    got = m.mqa_paged_scaled_decode_step(f32(q), bits(K, kind, True), f32(Ks, True), bits(V, kind, True), f32(Vs, True), i32([[0]]), i32([3])).cpu().numpy()
    want = V[0, 0, 1] * Vs[0, 0, 1]
    assert (np.abs(got - want) <= 2 * EPS * np.abs(want)).all()
