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


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lead", [5, 20, 40, 58, 90])
@pytest.mark.parametrize("h,k,each", [(8, 128, 7), (32, 128, 7), (16, 64, 40), (20, 48, 7), (9, 256, 30)])
def test_zeros_with_the_weight_leave_the_others_their_accuracy(m, h, k, each, lead, kind):
    """Two blocks of zeros, as an append leaves them, whose logits are 2^lead times the others' in weight: they count in the sum, and otherwise as if they had a scale of 2^-50."""
    rng = np.random.default_rng(h + k + lead)
    (K, Ks, V, Vs), _ = cache_of(rng, 1, each, 1, 16, 16, k, k, kind)
    table, lens = tables(rng, 1, each), np.array([16 * each - 3])
    direction = np.sign(rng.standard_normal(k))
    q = (direction * 0.5 + 0.05 * rng.standard_normal((1, 1, h, k))).astype(np.float32)
    zeros = table[0, [1, each - 2]]
    V[zeros], Vs[zeros] = 0, 2.0 ** -126
    K[zeros], Ks[zeros] = direction * 64, 2.0 ** -6                         # logits of about k / 2, times the scale
    scale = float(np.float32(lead / np.log2(np.e) / (k / 2)))
    counted = Vs.copy()
    counted[zeros] = 2.0 ** -50
    want, size, K_all, top = attended(q, (K, Ks, V, Vs), table, lens, scale)
    _, _, _, top = attended(q, (K, Ks, V, counted), table, lens, scale)
    got = m.mqa_paged_scaled_decode_step(f32(q[:, 0]), bits(K, kind, True), f32(Ks, True), bits(V, kind, True), f32(Vs, True), i32(table), i32(lens), scale=scale).cpu().numpy()
    bound = tolerance(q, K_all, size, scale, 16 * each, kind, top)
    off = np.abs(got - want[:, 0])
    assert (off <= bound[:, 0]).all(), (off / bound[:, 0]).max()


@pytest.mark.parametrize("kind", KINDS)
def test_logits_of_any_size_beside_larger_queries(m, kind):
    """The same with K's scales of 2^105 and every second row's queries 2^-20, 2^50 below the others', whose products are all with zeros: the others' mean is V's."""
    (K, Ks, V, Vs), _ = cache_of(np.random.default_rng(4), 1, 1, 1, 3, 1, 64, 64, kind)
    K[:] = 0
    K[0, 0, :, 0] = 3, 1, 2
    Ks[:] = 2.0 ** 105
    q = np.zeros((1, 16, 64), dtype=np.float32)
    q[:, 0::2, 1:] = 2.0 ** 30
    q[:, 1::2, 0] = -2.0 ** -20
    got = m.mqa_paged_scaled_decode_step(f32(q), bits(K, kind, True), f32(Ks, True), bits(V, kind, True), f32(Vs, True), i32([[0]]), i32([3])).cpu().numpy()
    held = V[0, 0] * Vs[0, 0][:, None]
    assert (np.abs(got[0, 1::2] - held[1]) <= 2 * EPS * np.abs(held[1])).all()
    assert (np.abs(got[0, 0::2] - held.mean(0)) <= 12 * EPS * np.abs(held).mean(0)).all()
