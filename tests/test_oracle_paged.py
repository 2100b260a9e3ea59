"""The paged oracle against the contiguous one and against itself where the answer is known (no GPU)."""
import numpy as np
import pytest

from oracle import mqa_oracle as orc
from oracle import paged


def cache(rng, b, h_kv, lens, page_size, k, v, spare=1):
    max_pages = max(-(-max(lens) // page_size), 1) + spare
    K, V = rng.standard_normal((b * max_pages, h_kv, page_size, k)), rng.standard_normal((b * max_pages, h_kv, page_size, v))
    return K, V, rng.permutation(b * max_pages).reshape(b, max_pages)


@pytest.mark.parametrize("page_size", [1, 3, 16])
def test_attention_is_the_contiguous_one(page_size):
    rng = np.random.default_rng(page_size)
    lens = np.array([0, 1, 17, 40])
    K, V, table = cache(rng, 4, 1, lens, page_size, 8, 16)
    q = rng.standard_normal((4, 1, 3, 8))
    o, total, _ = paged.attend(q, K, V, table, lens, 0.5)
    flat = [x[table].transpose(0, 2, 1, 3, 4).reshape(4, -1, x.shape[-1]) for x in (K, V)]
    assert np.allclose(o[:, 0], orc.mqa_decode(q[:, 0], *flat, lens, scale=0.5), rtol=1e-12, atol=1e-12)
    for i, n in enumerate(lens):
        assert np.allclose(total[i, 0, :n].sum(), 3 if n else 0) and np.isnan(total[i, 0, n:]).all()


def test_several_queries_are_single_ones_of_shorter_lengths():
    rng = np.random.default_rng(1)
    lens = np.array([2, 9])
    K, V, table = cache(rng, 2, 2, lens, 4, 8, 8)
    q = rng.standard_normal((2, 4, 4, 8))
    o, _, _ = paged.attend(q, K, V, table, lens)
    for j in range(4):
        one, _, _ = paged.attend(q[:, j:j + 1], K, V, table, lens - (3 - j))
        assert np.array_equal(o[:, j], one[:, 0])
    assert not o[0, :2].any()


def test_append_then_evict_whole_and_part():
    rng = np.random.default_rng(2)
    K, V, table = np.zeros((12, 1, 4, 8)), np.zeros((12, 1, 4, 8)), np.arange(8).reshape(2, 4)
    rows = rng.standard_normal((2, 10, 1, 8))
    lens = paged.append(K, V, table, rows, -rows, np.array([0, 0]), counts=np.array([10, 3]))
    assert lens.tolist() == [10, 3]
    assert paged.append(K, V, table, rows, rows, lens).tolist() == [10, 13]         # (no room for ten more: as it was)
    scores = np.zeros((2, 1, 16))
    scores[0, 0, [1, 4]] = 1, 2
    out = np.array([[8, 9], [10, 11]])
    lens_out, kept, _ = paged.evict(K, V, table, np.array([10, 3]), scores, out, 5, 2)
    assert lens_out.tolist() == [5, 3] and kept[0, 0].tolist() == [0, 1, 4, 8, 9] and kept[1, 0].tolist() == [0, 1, 2, -1, -1]
    flat = K[out][0].reshape(8, 8)
    assert np.array_equal(flat[:5], rows[0, [0, 1, 4, 8, 9], 0])


def test_verification_draws_the_targets_distribution():
    """Accepted or replaced, the first token is distributed as the target's: the point of the method."""
    rng = np.random.default_rng(3)
    b, vocab = 20000, 5
    p, q = np.array([0.5, 0.2, 0.2, 0.1, 0.0]), np.array([0.1, 0.4, 0.1, 0.1, 0.3])
    with np.errstate(divide="ignore"):
        logits = np.broadcast_to(np.log(p), (b, 2, vocab)).astype(np.float32)
        draft_logits = np.broadcast_to(np.log(q), (b, 1, vocab)).astype(np.float32)
    drafts = rng.choice(vocab, size=(b, 1), p=q)
    tokens, accepted = paged.verify(logits, drafts, rng.random((b, 2)), draft_logits)
    got = np.bincount(tokens[:, 0], minlength=vocab) / b
    assert np.abs(got - p).max() < 5 * np.sqrt(0.25 / b)                            # five standard deviations
    assert abs(accepted.mean() - np.minimum(p, q).sum()) < 5 * np.sqrt(0.25 / b)
    greedy, ok = paged.verify(logits[:2], np.array([[0], [3]]), None, temperature=0)
    assert greedy.tolist() == [[0, 0], [0, -1]] and ok.tolist() == [1, 0]
