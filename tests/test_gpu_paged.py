"""Paged caches on the GPU against the float64 oracle (oracle/paged.py)."""
import numpy as np
import pytest

import mqa_inputs as mi

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 2.0 ** -24          # half a step of float32


@pytest.fixture(scope="module")
def m():
    import paper_1911_02150_amd as mod
    mod.load_library()
    return mod


def rounded(x, dtype):
    """x as a cache of this type holds it, in float64."""
    x = np.asarray(x, dtype=np.float32)
    return mi.bf16_bits_to_f64(mi.f32_to_bf16_bits(x)) if dtype == "bf16" else x.astype(np.float64)


def pool(rng, num_pages, h_kv, page_size, width, dtype):
    return rounded(rng.standard_normal((num_pages, h_kv, page_size, width)), dtype)


def on_gpu(x, dtype=None, one_head=False):
    """A numpy array as a device tensor; a pool of one head without the heads' axis."""
    t = torch.from_numpy(np.ascontiguousarray(x))
    if dtype:
        t = t.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    elif t.dtype == torch.float64:
        t = t.float()
    elif t.dtype == torch.int64:
        t = t.to(torch.int32)
    return (t[:, 0] if one_head else t).contiguous().to(DEV)


def tables(rng, b, each, first=0):
    return first + rng.permutation(b * each).reshape(b, each)


def tolerance(q, K, size, scale, length):
    """Half a step for each of: k products and their sum (a logit, at most scale * |q| |K|), the exponential and its argument, as many sums as there are positions, each
    over rounding errors that do not know of one another (eight standard deviations)."""
    k = q.shape[-1]
    logit = abs(scale) * np.abs(q).max() * np.abs(K[np.isfinite(K)]).max() * k ** 0.5 * 4      # (4: a sum of k products of normal numbers)
    return EPS * (2 * (8 + 4) * logit + 16 + 8 * length ** 0.5) * size + 1e-30


# b, n, h, h_kv, k, v, page size, dtype, lengths
ATTEND = [
    (1, 1, 1, 1, 8, 8, 1, "f32", [1]),
    (3, 1, 8, 1, 128, 128, 16, "bf16", [0, 1, 33]),
    (4, 1, 8, 1, 128, 128, 16, "bf16", [511, 512, 513, 700]),
    (2, 1, 32, 1, 128, 128, 64, "bf16", [1500, 31]),
    (2, 1, 64, 1, 128, 128, 16, "bf16", [300, 900]),
    (2, 1, 20, 1, 128, 128, 7, "bf16", [129, 257]),
    (2, 5, 8, 1, 128, 128, 16, "bf16", [5, 400]),
    (2, 3, 8, 8, 128, 128, 16, "bf16", [2, 350]),
    (3, 1, 8, 8, 64, 64, 16, "f32", [1, 128, 600]),
    (2, 4, 8, 2, 64, 64, 5, "f32", [3, 77]),
    (2, 2, 12, 3, 64, 64, 16, "bf16", [290, 33]),
    (2, 1, 8, 1, 128, 128, 16, "f32", [1025, 64]),
    (2, 2, 24, 1, 128, 128, 100, "f32", [99, 301]),
    (2, 2, 6, 2, 40, 24, 3, "bf16", [100, 350]),
    (2, 1, 3, 1, 256, 256, 16, "f32", [513, 17]),
    (1, 1, 9, 1, 16, 256, 16, "bf16", [400]),
    (1, 1, 70, 1, 256, 8, 11, "f32", [290]),
    (1, 128, 8, 1, 128, 128, 16, "bf16", [300]),
    (5, 1, 1, 1, 128, 128, 32, "bf16", [0, 0, 0, 0, 0]),
    (1, 1, 33, 1, 96, 104, 9, "f32", [500]),
    (2, 2, 20, 1, 200, 200, 16, "f32", [600, 50]),
    (2, 1, 40, 1, 200, 248, 16, "bf16", [700, 33]),
    (3, 3, 4, 2, 120, 72, 32, "bf16", [260, 1, 2000]),
]


@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("b,n,h,h_kv,k,v,page,dtype,lens", ATTEND)
def test_attention(m, b, n, h, h_kv, k, v, page, dtype, lens, scored):
    from oracle import paged
    rng = np.random.default_rng(b + 7 * n + 11 * h + k + len(lens))
    each = -(-max(max(lens), 1) // page) + 3
    K, V = (pool(rng, b * each, h_kv, page, w, dtype) for w in (k, v))
    table, lens = tables(rng, b, each), np.array(lens)
    q = rng.standard_normal((b, n, h, k)).astype(np.float32)
    scores = rng.random((b, h_kv, each * page)).astype(np.float32) if scored else None
    scale = 2 / k ** 0.5
    want, total, size = paged.attend(q.astype(np.float64), K, V, table, lens, float(np.float32(scale)), scores)
    one = h_kv == 1
    args = on_gpu(q[:, 0] if n == 1 else q), on_gpu(K, dtype, one), on_gpu(V, dtype, one), on_gpu(table), on_gpu(lens)
    kw = {}
    if scored:
        kw["scores"] = on_gpu(scores, one_head=one)
        kw["scores_out"] = torch.full_like(kw["scores"], 777.0)
    got = m.mqa_paged_decode_step(*args, scale=scale, **kw)
    again = m.mqa_paged_decode_step(*args, scale=scale, **kw)
    assert got.shape == ((b, h, v) if n == 1 else (b, n, h, v)) and torch.equal(got, again)
    off = np.abs(got.cpu().numpy().reshape(want.shape) - want)
    assert (off <= tolerance(q, K, size, scale, max(lens))).all(), off.max()
    if scored:
        out = kw["scores_out"].cpu().numpy().reshape(total.shape)
        left = np.isnan(total)
        assert (out[left] == 777).all()
        bound = tolerance(q, K, 1, scale, max(lens)) * total + EPS * (2 + n * h / h_kv) * total
        assert (np.abs(out - total)[~left] <= bound[~left]).all()
        before = kw["scores"].clone()
        m.mqa_paged_decode_step(*args, scale=scale, scores=before)                # in place
        assert torch.equal(before.view(-1)[torch.from_numpy(~left.reshape(-1)).to(DEV)], kw["scores_out"].view(-1)[torch.from_numpy(~left.reshape(-1)).to(DEV)])
        m.mqa_paged_decode_step(*args, scale=scale, scores_out=before)            # from nothing
        _, zero, _ = paged.attend(q.astype(np.float64), K, V, table, lens, float(np.float32(scale)), np.zeros_like(scores))
        assert (np.abs(before.cpu().numpy().reshape(total.shape) - zero)[~left] <= bound[~left]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,h,h_kv,k", [(1, 8, 1, 128), (4, 8, 1, 128), (3, 4, 4, 64), (2, 40, 1, 128), (2, 4, 2, 24)])
def test_what_is_not_seen_may_hold_anything(m, n, h, h_kv, k, dtype):
    """NaN and infinities behind the length, on missing pages, and at the places of later queries; lengths out of range; pages that hold nothing."""
    from oracle import paged
    rng = np.random.default_rng(n * h + k)
    b, page, each = 5, 16, 6
    K, V = (pool(rng, b * each, h_kv, page, k, dtype) for _ in range(2))
    table, lens = tables(rng, b, each), np.array([40, -3, 1000, 65, 96])
    clean_K, clean_V = K.copy(), V.copy()
    table[0, 1], table[3, 0], table[3, 1], table[4] = -1, b * each, 2 ** 31 - 1, -5
    for i in range(b):
        length = min(max(int(lens[i]), 0), page * each)
        for p in range(length, page * each):
            at = paged.where(table, i, p, b * each, page)
            if at is not None:
                K[at[0], :, at[1]], V[at[0], :, at[1]] = np.nan, np.inf
        for j in range(1, n):                                                 # seen by the later queries alone
            at = paged.where(table, i, length - j, b * each, page) if length - j >= 0 else None
            if at is not None:
                V[at[0], :, at[1], : k // 2] = (np.inf, -np.inf, np.nan)[j % 3]
    q = rng.standard_normal((b, n, h, k)).astype(np.float32)
    one = h_kv == 1
    want, total, size = paged.attend(q.astype(np.float64), K, V, table, lens, 0.25)
    scores = torch.zeros((b, each * page) if one else (b, h_kv, each * page), device=DEV)
    got = m.mqa_paged_decode_step(on_gpu(q), on_gpu(K, dtype, one), on_gpu(V, dtype, one), on_gpu(table), on_gpu(lens), scale=0.25, scores=scores)
    got = got.cpu().numpy().astype(np.float64)
    assert not got[1].any() and not got[4].any() and np.isfinite(got[:, 0]).all()
    finite = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~finite & ~np.isnan(want)], want[~finite & ~np.isnan(want)])
    assert (np.abs(got - want)[finite] <= tolerance(q, clean_K, size, 0.25, 96)[finite]).all()
    there = ~np.isnan(total)
    assert (np.abs(scores.cpu().numpy().reshape(total.shape) - total)[there] <= tolerance(q, clean_K, 1, 0.25, 96) + EPS * (n * h + 2)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [128, 64, 40])
def test_infinite_keys(m, k, dtype):
    """A key of -infinity that is seen has weight 0 where q is positive, and the row stays finite."""
    rng = np.random.default_rng(k)
    from oracle import paged
    K, V, table, lens = pool(rng, 4, 1, 16, k, dtype), pool(rng, 4, 1, 16, k, dtype), np.array([[2, 0, 3, 1]]), np.array([50])
    K[0, 0, 3] = K[3, 0, 15] = -np.inf
    q = np.abs(rng.standard_normal((1, 1, 4, k))).astype(np.float32)
    want, _, size = paged.attend(q.astype(np.float64), K, V, table, lens, 0.25)
    assert np.isfinite(want).all()
    got = m.mqa_paged_decode_step(on_gpu(q), on_gpu(K, dtype, True), on_gpu(V, dtype, True), on_gpu(table), on_gpu(lens), scale=0.25).cpu().numpy()
    assert (np.abs(got - want) <= tolerance(q, K, size, 0.25, 50)).all()


def test_large_logits(m):
    """Logits of hundreds: one position takes all the weight, others none."""
    from oracle import paged
    rng = np.random.default_rng(5)
    K, V, table, lens = pool(rng, 40, 1, 16, 128, "bf16"), pool(rng, 40, 1, 16, 128, "bf16"), tables(rng, 1, 40), np.array([640])
    q = (20 * rng.standard_normal((1, 1, 8, 128))).astype(np.float32)
    want, _, size = paged.attend(q.astype(np.float64), K, V, table, lens)
    got = m.mqa_paged_decode_step(on_gpu(q[:, 0]), on_gpu(K, "bf16", True), on_gpu(V, "bf16", True), on_gpu(table), on_gpu(lens)).cpu().numpy()
    assert (np.abs(got - want[:, 0]) <= tolerance(q, K, size, 1.0, 640)[:, 0]).all()


# b, n, h, k, v, dtype, pages of a sequence: so many sequences that a workgroup has 32 rows, in one launch and in two
MANY = [
    (300, 1, 20, 128, 128, "bf16", 4),
    (300, 2, 20, 128, 128, "bf16", 70),
    (400, 1, 20, 64, 64, "bf16", 70),
    (400, 2, 20, 64, 64, "f32", 5),
    (400, 1, 18, 40, 64, "bf16", 70),
    (400, 1, 18, 64, 24, "f32", 5),
    (300, 1, 20, 120, 96, "bf16", 70),
    (300, 1, 40, 200, 256, "bf16", 4),
    (300, 1, 20, 256, 256, "f32", 70),
]


@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("b,n,h,k,v,dtype,each", MANY)
def test_many_sequences_of_many_rows(m, b, n, h, k, v, dtype, each, scored):
    """Pages shared by all sequences, some of them nothing's."""
    from oracle import paged
    rng = np.random.default_rng(b + h + k + each)
    page, pages = 16, 50
    K, V = (pool(rng, pages, 1, page, w, dtype) for w in (k, v))
    table = rng.integers(0, pages, (b, each))
    table[rng.random(table.shape) < 0.1] = -1
    lens = rng.integers(0, 40, b)
    lens[5], lens[7], lens[-1] = each * page, each * page - 17, 0
    q = rng.standard_normal((b, n, h, k)).astype(np.float32)
    scale = 1 / k ** 0.5
    scores = np.zeros((b, 1, each * page)) if scored else None
    want, total, size = paged.attend(q.astype(np.float64), K, V, table, lens, float(np.float32(scale)), scores)
    kw = dict(scores=torch.zeros((b, each * page), device=DEV)) if scored else {}
    got = m.mqa_paged_decode_step(on_gpu(q[:, 0] if n == 1 else q), on_gpu(K, dtype, True), on_gpu(V, dtype, True), on_gpu(table), on_gpu(lens), scale=scale, **kw)
    off = np.abs(got.cpu().numpy().reshape(want.shape) - want)
    assert (off <= tolerance(q, K, size, scale, lens.max())).all(), off.max()
    if scored:
        out, there = kw["scores"].cpu().numpy()[:, None], ~np.isnan(total)
        bound = tolerance(q, K, 1, scale, lens.max()) * total + EPS * (2 + n * h) * total
        assert (np.abs(out - total)[there] <= bound[there]).all() and not out[~there].any()


@pytest.mark.parametrize("b,k,dtype", [(300, 128, "bf16"), (400, 64, "f32"), (300, 200, "bf16")])
def test_many_rows_and_a_nan_that_half_of_them_see(m, b, k, dtype):
    """The newest token's K and V are NaN in every third sequence: of two queries the first does not see them."""
    from oracle import paged
    rng = np.random.default_rng(b + k)
    page, pages, each, n, h = 16, 40, 4, 2, 20
    K, V = (pool(rng, pages + 1, 1, page, k, dtype) for _ in range(2))
    clean = K[:pages].copy()
    K[pages] = V[pages] = np.nan
    table, lens = rng.integers(0, pages, (b, each)), rng.integers(2, 60, b)
    lens[::3] = 17 + 16 * rng.integers(0, 3, len(lens[::3]))
    for i in range(0, b, 3):
        table[i, lens[i] // page] = pages
    q = rng.standard_normal((b, n, h, k)).astype(np.float32)
    want, _, size = paged.attend(q.astype(np.float64), K, V, table, lens, 0.125)
    got = m.mqa_paged_decode_step(on_gpu(q), on_gpu(K, dtype, True), on_gpu(V, dtype, True), on_gpu(table), on_gpu(lens), scale=0.125).cpu().numpy()
    finite = np.isfinite(want)
    assert np.isnan(got[~finite]).all() and finite[:, 0].all() and not finite[::3, 1].any() and finite[1::3].all()
    assert (np.abs(got - want)[finite] <= tolerance(q, clean, size, 0.125, 60)[finite]).all()


def test_many_short_sequences_and_one_long(m):
    """More sequences than a workgroup has threads, empty ones among them, against the contiguous call."""
    g = torch.Generator(device=DEV).manual_seed(1)
    b, each, page = 700, 40, 16
    lens = torch.randint(0, 60, (b,), generator=g, device=DEV, dtype=torch.int32)
    lens[::7], lens[333] = 0, each * page
    used = torch.randn((b, each * page, 128), generator=g, device=DEV).bfloat16()
    table = torch.randperm(b * each, generator=g, device=DEV).to(torch.int32).view(b, each)
    K = torch.empty((b * each, page, 128), dtype=torch.bfloat16, device=DEV)
    K[table.long()] = used.view(b, each, page, 128)
    q = torch.randn((b, 8, 128), generator=g, device=DEV)
    got = m.mqa_paged_decode_step(q, K, K, table, lens, scale=0.1)
    want = m.mqa_decode_step(q, used, used, lens, scale=0.1)
    assert not got[lens == 0].any()
    # (the contiguous call's q and weights are two bfloat16 terms each: 2^-17 of a logit's products and of a weight)
    assert (got - want).abs().max().item() <= 2 ** -15 * used.abs().max().item()


@pytest.mark.parametrize("b,n,h_kv,k,v,page,dtype", [(3, 1, 1, 128, 128, 16, "bf16"), (4, 9, 3, 24, 40, 5, "f32"), (2, 40, 1, 64, 8, 7, "bf16"), (1, 1, 8, 64, 64, 1, "f32")])
def test_append(m, b, n, h_kv, k, v, page, dtype):
    from oracle import paged
    rng = np.random.default_rng(n)
    each = 12
    K, V = (pool(rng, b * each + 1, h_kv, page, w, dtype) for w in (k, v))
    table = tables(rng, b, each)
    table[0, 1] = -1                                                           # a page that holds nothing: its rows are dropped
    lens = np.array([page, page * each - n + 1, 0, -1])[:b]                    # (the second has no room for n, the fourth no length)
    for counts in (None, np.array([n, max(0, n - 1), -2, n + 5])[:b]):
        k_new, v_new = (rng.standard_normal((b, n, h_kv, w)).astype(np.float32) for w in (k, v))
        wK, wV = K.copy(), V.copy()
        want = paged.append(wK, wV, table, k_new, v_new, lens, counts, lambda x: rounded(x, dtype))
        one = h_kv == 1
        gK, gV, out = on_gpu(K, dtype, one), on_gpu(V, dtype, one), torch.zeros(b, dtype=torch.int32, device=DEV)
        new = [on_gpu(x[:, :, 0] if one else x) for x in (k_new, v_new)]
        assert m.mqa_paged_append_kv_rows(gK, gV, on_gpu(table), *new, on_gpu(lens), out, counts=None if counts is None else on_gpu(counts)) is out
        assert out.tolist() == want.tolist()
        assert np.array_equal(gK.double().cpu().numpy().reshape(K.shape), wK) and np.array_equal(gV.double().cpu().numpy().reshape(V.shape), wV)


def test_append_rounds_as_the_contiguous_call(m):
    """Halfway cases, NaN, infinities, denormals and negative zero."""
    bits = np.array([0x3f808000, 0x3f818000, 0x3f807fff, 0x7fc00001, 0x7f800000, 0xff800000, 0x00000001, 0x80000000, 0x7f7fffff, 0x00008000, 0x807fffff, 0x7f800001],
                    dtype=np.uint32)
    row = torch.from_numpy(np.resize(bits, 64).view(np.float32).copy()).view(1, 1, 64).to(DEV)
    K, lens = torch.zeros((1, 16, 64), dtype=torch.bfloat16, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    pages, table = torch.zeros((2, 16, 64), dtype=torch.bfloat16, device=DEV), torch.ones((1, 1), dtype=torch.int32, device=DEV)
    m.mqa_paged_append_kv_rows(pages, torch.zeros_like(pages), table, row, row, lens, torch.empty_like(lens))
    m.mqa_append_kv(K, torch.zeros_like(K), row[:, 0].contiguous(), row[:, 0].contiguous(), lens)
    a, b = pages[1, 0].view(torch.int16), K[0, 0].view(torch.int16)
    nan = torch.isnan(K[0, 0])
    assert torch.equal(a[~nan], b[~nan]) and torch.isnan(pages[1, 0][nan]).all()


EVICT = [
    (1, 1, 8, 8, 1, "f32", [1], 1, 0),
    (3, 1, 128, 128, 16, "bf16", [0, 40, 700], 64, 16),
    (2, 4, 24, 40, 5, "f32", [33, 60], 20, 20),
    (2, 2, 64, 64, 16, "bf16", [3000, 1025], 1024, 0),
    (2, 1, 64, 8, 16, "f32", [100, 16], 100, 3),
    (1, 1, 16, 16, 16, "f32", [5000], 77, 7),
    (1, 2, 8, 8, 48, "bf16", [16000], 2500, 100),
    (2, 1, 8, 16, 256, "f32", [26000, 24577], 3000, 1),
    (1, 1, 8, 8, 100, "f32", [70001], 5000, 700),
    (2, 1, 8, 8, 64, "f32", [90000, 8193], 90000, 0),
]


@pytest.mark.parametrize("kind", ["random", "ties", "odd"])
@pytest.mark.parametrize("b,h_kv,k,v,page,dtype,lens,budget,recent", EVICT)
def test_evict(m, b, h_kv, k, v, page, dtype, lens, budget, recent, kind):
    from oracle import paged
    rng = np.random.default_rng(budget + len(kind))
    each, out_each = -(-max(lens) // page) + 1, -(-budget // page) + 1
    K, V = (pool(rng, b * (each + out_each), h_kv, page, w, dtype) for w in (k, v))
    table, table_out = tables(rng, b, each), tables(rng, b, out_each, b * each)
    lens = np.array(lens)
    scores = rng.random((b, h_kv, each * page)).astype(np.float32)
    if kind == "ties":
        scores = np.floor(scores * 4).astype(np.float32) * np.where(rng.random(scores.shape) < 0.1, -0.0, 1).astype(np.float32)
    if kind == "odd":                                                          # NaN, infinities, negative and tiny ones; pages that hold nothing
        scores = np.where(rng.random(scores.shape) < 0.3, rng.choice([np.nan, np.inf, -np.inf, -1.5, 1e-42, -1e-42], scores.shape), scores - 0.5).astype(np.float32)
        table[-1, 0], table_out[0, 0] = -1, 2 ** 31 - 1
        lens[0] = 10 ** 9 if b > 1 else lens[0]
    wK, wV = K.copy(), V.copy()
    want_lens, want_kept, want_scores = paged.evict(wK, wV, table, lens, scores, table_out, budget, recent)
    one = h_kv == 1
    gK, gV = on_gpu(K, dtype, one), on_gpu(V, dtype, one)
    lead = (b,) if one else (b, h_kv)
    lens_out, kept = torch.full((b,), 9, dtype=torch.int32, device=DEV), torch.full((*lead, budget), 9, dtype=torch.int32, device=DEV)
    scores_out = torch.full((*lead, out_each * page), 777.0, device=DEV)
    assert m.mqa_paged_evict_kv(gK, gV, on_gpu(table), on_gpu(lens), on_gpu(scores, one_head=one), on_gpu(table_out), lens_out, scores_out, kept, recent) is kept
    assert lens_out.tolist() == want_lens.tolist()
    assert np.array_equal(kept.cpu().numpy().reshape(want_kept.shape), want_kept)
    got = scores_out.cpu().numpy().reshape(want_scores.shape)
    slots = np.arange(want_scores.shape[2]) < want_lens[:, None, None]
    slots = np.broadcast_to(slots, got.shape)
    assert np.array_equal(got[slots], want_scores[slots].astype(np.float32), equal_nan=True) and (got[~slots] == 777).all()
    assert np.array_equal(gK.double().cpu().numpy().reshape(K.shape), wK) and np.array_equal(gV.double().cpu().numpy().reshape(V.shape), wV)


def test_a_cache_on_its_way(m):
    """Prompts appended, steps with scores, an eviction, more steps: as the oracle does them, in one captured graph and without."""
    from oracle import paged
    rng = np.random.default_rng(8)
    b, h, k, page, n = 3, 8, 128, 16, 50
    each, out_each, budget, recent = 5, 4, 40, 8
    prompt, counts = rng.standard_normal((2, b, n, 1, k)).astype(np.float32), np.array([50, 7, 33])
    table, table_out = tables(rng, b, each), tables(rng, b, out_each, b * each)
    new = rng.standard_normal((4, 2, b, 1, 1, k)).astype(np.float32)
    qs = rng.standard_normal((4, b, 1, h, k)).astype(np.float32)
    scale = 0.125
    K, V = (np.zeros((b * (each + out_each), 1, page, k)) for _ in range(2))
    bf = lambda x: rounded(x, "bf16")  # noqa: E731
    lens = paged.append(K, V, table, prompt[0], prompt[1], np.zeros(b, dtype=np.int64), counts, bf)
    scores, outs = np.zeros((b, 1, each * page)), []
    for t in range(2):
        lens = paged.append(K, V, table, new[t, 0], new[t, 1], lens, rounded=bf)
        o, scores, size = paged.attend(qs[t].astype(np.float64), K, V, table, lens, scale, np.nan_to_num(scores))
        outs.append((o, size))
    gpu = [on_gpu(np.zeros_like(K), "bf16", True) for _ in range(2)]
    t_in, t_out, first = on_gpu(table), on_gpu(table_out), on_gpu(counts)
    p, x, queries = [on_gpu(y[:, :, 0]) for y in prompt], [[on_gpu(y[:, :, 0]) for y in z] for z in new], [on_gpu(y[:, 0]) for y in qs]
    ints = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    ls, s_in, s_out, kept, results = [ints(b) for _ in range(6)], torch.zeros((b, each * page), device=DEV), torch.zeros((b, out_each * page), device=DEV), ints(b, budget), {}

    def whole():
        s_in.zero_()
        s_out.zero_()
        ls[0].zero_()
        m.mqa_paged_append_kv_rows(*gpu, t_in, *p, ls[0], ls[1], counts=first)
        for t in range(2):
            m.mqa_paged_append_kv_rows(*gpu, t_in, *x[t], ls[1 + t], ls[2 + t])
            results[t] = m.mqa_paged_decode_step(queries[t], *gpu, t_in, ls[2 + t], scale=scale, scores=s_in)
        m.mqa_paged_evict_kv(*gpu, t_in, ls[3], s_in, t_out, ls[4], s_out, kept, recent)
        for t in range(2, 4):
            m.mqa_paged_append_kv_rows(*gpu, t_out, *x[t], ls[2 + t], ls[3 + t]) if t == 2 else m.mqa_paged_append_kv_rows(*gpu, t_out, *x[t], ls[5], ls[0])
            results[t] = m.mqa_paged_decode_step(queries[t], *gpu, t_out, ls[5] if t == 2 else ls[0], scale=scale, scores=s_out)

    whole()
    torch.cuda.synchronize()
    eager = [results[t].clone() for t in range(4)]
    got_scores = s_in.cpu().numpy().astype(np.float64)[:, None]
    assert ls[3].tolist() == lens.tolist()
    for t in range(2):
        assert (np.abs(eager[t].cpu().numpy()[:, None] - outs[t][0]) <= tolerance(qs, np.concatenate([prompt[0].ravel(), new.ravel()]), outs[t][1], scale, 60)).all()
    # from here on by the scores that the GPU has (a near tie may go either way)
    lens, want_kept, scores = paged.evict(K, V, table, lens, got_scores, table_out, budget, recent)
    assert np.array_equal(kept.cpu().numpy()[:, None], want_kept)
    for t in range(2, 4):
        lens = paged.append(K, V, table_out, new[t, 0], new[t, 1], lens, rounded=bf)
        o, scores, size = paged.attend(qs[t].astype(np.float64), K, V, table_out, lens, scale, np.nan_to_num(scores))
        assert (np.abs(eager[t].cpu().numpy()[:, None] - o) <= tolerance(qs, np.concatenate([prompt[0].ravel(), new.ravel()]), size, scale, 60)).all()
    assert np.array_equal(gpu[0].double().cpu().numpy()[:, None], K)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        whole()
    for _ in range(3):
        for t in range(4):
            results[t].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for t in range(4):
            assert torch.equal(results[t], eager[t])


def test_on_another_stream_and_from_two_threads(m):
    """Calls on streams of their own, at the same time, on workspaces of their own."""
    import threading
    g = torch.Generator(device=DEV).manual_seed(2)
    K = torch.randn((256, 16, 128), generator=g, device=DEV).bfloat16()
    table = torch.randperm(256, generator=g, device=DEV).to(torch.int32).view(2, 128)
    lens = torch.tensor([2000, 1500], dtype=torch.int32, device=DEV)
    qs = [torch.randn((2, 8, 128), generator=g, device=DEV) for _ in range(2)]
    want = [m.mqa_paged_decode_step(q, K, K, table, lens) for q in qs]
    torch.cuda.synchronize()
    bad = []

    def many(x):
        stream = torch.cuda.Stream()
        for r in range(50):
            if r % 2:
                got = m.mqa_paged_decode_step(qs[x], K, K, table, lens, stream=stream)
            else:
                with torch.cuda.stream(stream):
                    got = m.mqa_paged_decode_step(qs[x], K, K, table, lens)
            stream.synchronize()
            if not torch.equal(got, want[x]):
                bad.append((x, r))

    threads = [threading.Thread(target=many, args=(x,)) for x in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_replayed_for_other_lengths_and_pages(m):
    """One captured step, replayed as the lengths grow and pages are exchanged between the replays: what it does is decided on the GPU."""
    g = torch.Generator(device=DEV).manual_seed(4)
    b, each, page, heads = 5, 64, 16, 2
    K, V = (torch.randn((b * each, heads, page, 64), generator=g, device=DEV) for _ in range(2))
    table, lens = torch.randperm(b * each, generator=g, device=DEV).to(torch.int32).view(b, each), torch.zeros(b, dtype=torch.int32, device=DEV)
    q, new = torch.randn((b, 2, 4, 64), generator=g, device=DEV), torch.randn((b, 2, heads, 64), generator=g, device=DEV)
    counts, after = torch.zeros(b, dtype=torch.int32, device=DEV), torch.zeros(b, dtype=torch.int32, device=DEV)
    scores = torch.rand((b, heads, each * page), generator=g, device=DEV)

    def step(K, V, o, out):
        m.mqa_paged_append_kv_rows(K, V, table, new, new, lens, after, counts=counts)
        return m.mqa_paged_decode_step(q, K, V, table, after, o=o, scores=scores, scores_out=out)

    kept = K.clone(), V.clone(), torch.zeros_like(q), torch.zeros_like(scores)
    step(*(t.clone() for t in kept))                       # (before the capture: once outside)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*kept)
    for lengths, rows in (([0, 1, 31, 500, 1022], [2, 1, 0, 2, 2]), ([1024, 1023, 0, -3, 2 ** 31 - 1], [1, 1, 0, 1, 2]), ([900, 900, 900, 900, 900], [2, 2, 2, 2, 9])):
        table.copy_(table[:, torch.randperm(each, generator=g, device=DEV)].roll(1, 0))
        lens.copy_(torch.tensor(lengths, dtype=torch.int32)), counts.copy_(torch.tensor(rows, dtype=torch.int32))
        here = [t.clone() for t in kept]
        step(*here)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(here, kept))


def test_a_page_named_twice(m):
    """Sequences that share pages, and one that has a page twice: to be read as often as it is named."""
    from oracle import paged
    rng = np.random.default_rng(12)
    K, V = (pool(rng, 9, 1, 16, 128, "bf16") for _ in range(2))
    table = np.array([[3, 3, 5, 3], [3, 5, 8, 0], [7, 7, 7, 7]])
    lens, q = np.array([60, 37, 64]), rng.standard_normal((3, 1, 8, 128)).astype(np.float32)
    want, _, size = paged.attend(q.astype(np.float64), K, V, table, lens, 0.125)
    got = m.mqa_paged_decode_step(on_gpu(q[:, 0]), on_gpu(K, "bf16", True), on_gpu(V, "bf16", True), on_gpu(table), on_gpu(lens), scale=0.125)
    assert (np.abs(got.cpu().numpy()[:, None] - want) <= tolerance(q, K, size, 0.125, 64)).all()


@pytest.mark.parametrize("dtype,width", [(torch.float32, 128), (torch.bfloat16, 256)])
def test_pools_of_more_than_4_gib(m, dtype, width):
    """The last pages of a large pool against a small one that holds the same."""
    page, each, heads, b = 64, 20, 3, 2
    row = torch.zeros((), dtype=dtype).element_size() * width
    pages = (5 << 30) // (row * page * heads)
    big = [torch.empty((pages, heads, page, width), dtype=dtype, device=DEV) for _ in range(2)]
    small = [torch.zeros((3 * b * each, heads, page, width), dtype=dtype, device=DEV) for _ in range(2)]
    g = torch.Generator(device=DEV).manual_seed(5)
    for x, y in zip(big, small):
        x[:1].zero_(), x[-len(y):].zero_()
    new = torch.randn((b, 1200, heads, width), generator=g, device=DEV)
    q, lens = torch.randn((b, 2, 6, width), generator=g, device=DEV), torch.tensor([3, 50], dtype=torch.int32, device=DEV)
    order = torch.randperm(2 * b * each, generator=g, device=DEV).to(torch.int32).view(2, b, each)
    results = []
    for K, V, first in ((*big, pages - 3 * b * each), (*small, 0)):
        table, out = order + first
        after, lens_out, kept = torch.zeros_like(lens), torch.zeros_like(lens), torch.zeros((b, heads, 500), dtype=torch.int32, device=DEV)
        scores, left = torch.zeros((b, heads, each * page), device=DEV), torch.zeros((b, heads, each * page), device=DEV)
        m.mqa_paged_append_kv_rows(K, V, table, new, new, lens, after)
        o = m.mqa_paged_decode_step(q, K, V, table, after, scale=0.1, scores=scores)
        m.mqa_paged_evict_kv(K, V, table, after, scores, out, lens_out, left, kept, 10)
        results.append((after, o, scores, lens_out, left, kept, K[first:first + 2 * b * each].clone(), V[first:first + 2 * b * each].clone()))
    assert all(torch.equal(x, y) for x, y in zip(*results))
    assert results[0][1].abs().max() > 0 and results[0][3].tolist() == [500, 500]


@pytest.mark.parametrize("heads", [None, 2])
def test_append_and_evict_on_a_stream(m, heads):
    """On a stream given, and on the current one: one head's pools with and without its axis, too."""
    g = torch.Generator(device=DEV).manual_seed(11)
    b, each, page, k = 3, 6, 16, 64
    lead, per = (2 * b * each, page) if heads is None else (2 * b * each, heads, page), (b,) if heads is None else (b, heads)
    table, out = (torch.randperm(b * each, generator=g, device=DEV).to(torch.int32).view(b, each) + x for x in (0, b * each))
    new, scores = torch.randn((b, 70, *per[1:], k), generator=g, device=DEV), torch.rand((*per, each * page), generator=g, device=DEV)
    results = []
    for stream in (None, torch.cuda.Stream()):
        K, V = (torch.zeros((*lead, k), device=DEV) for _ in range(2))
        lens, after, left = (torch.zeros(b, dtype=torch.int32, device=DEV) for _ in range(3))
        kept, rest = torch.zeros((*per, 40), dtype=torch.int32, device=DEV), torch.zeros_like(scores)
        torch.cuda.synchronize()
        m.mqa_paged_append_kv_rows(K, V, table, new, new, lens, after, stream=stream)
        m.mqa_paged_evict_kv(K, V, table, after, scores, out, left, rest, kept, 7, stream=stream)
        torch.cuda.synchronize()
        results.append((K, V, after, left, kept, rest))
    assert all(torch.equal(x, y) for x, y in zip(*results)) and results[0][3].tolist() == [40] * b
    if heads is None:
        K, V = (torch.zeros((lead[0], 1, page, k), device=DEV) for _ in range(2))
        m.mqa_paged_append_kv_rows(K, V, table, new[:, :, None].contiguous(), new[:, :, None].contiguous(), lens, after)
        m.mqa_paged_evict_kv(K, V, table, after, scores[:, None].contiguous(), out, left, torch.zeros_like(scores)[:, None].contiguous(), kept[:, None].contiguous(), 7)
        assert torch.equal(K[:, 0], results[0][0]) and torch.equal(V[:, 0], results[0][1])


def test_a_given_workspace(m):
    g = torch.Generator(device=DEV).manual_seed(3)
    K = torch.randn((256, 16, 128), generator=g, device=DEV).bfloat16()
    table, lens = torch.arange(256, dtype=torch.int32, device=DEV).view(2, 128), torch.tensor([2000, 1500], dtype=torch.int32, device=DEV)
    q = torch.randn((2, 8, 128), generator=g, device=DEV)
    need = m.mqa_paged_decode_workspace_bytes(2, 1, 8, 1, 16, 128, 128, 128, m.MQA_BF16)
    guard = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
    o = torch.empty((2, 8, 128), device=DEV)
    assert m.mqa_paged_decode_step(q, K, K, table, lens, o=o, workspace=guard[:need]) is o
    assert (guard[need:] == 0x5a).all() and torch.equal(o, m.mqa_paged_decode_step(q, K, K, table, lens))
    with pytest.raises(m.MqaError, match="workspace"):
        m.mqa_paged_decode_step(q, K, K, table, lens, workspace=guard[:need - 16])


def test_wrong_tensors_are_refused(m):
    K, table = torch.zeros((8, 16, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((2, 4), dtype=torch.int32, device=DEV)
    lens, q = torch.ones(2, dtype=torch.int32, device=DEV), torch.zeros((2, 8, 128), device=DEV)
    call = m.mqa_paged_decode_step
    for bad in (dict(q=q[:, :, :64].contiguous()), dict(lens=lens[:1]), dict(table=table[:1]), dict(table=table.view(-1)), dict(o=torch.zeros((2, 8, 64), device=DEV)),
                dict(scores=torch.zeros((2, 63), device=DEV)), dict(V_pages=K[:, :8].contiguous()), dict(q=q.transpose(1, 2)), dict(q=q.view(-1)),
                dict(lens=lens.cpu()), dict(q=q[None, None])):
        with pytest.raises(ValueError):
            call(**{**dict(q=q, K_pages=K, V_pages=K, table=table, lens=lens), **bad})
    for bad in (dict(q=q.double()), dict(V_pages=K.float()), dict(table=table.long()), dict(lens=lens.long()), dict(K_pages=K.half(), V_pages=K.half())):
        with pytest.raises(TypeError):
            call(**{**dict(q=q, K_pages=K, V_pages=K, table=table, lens=lens), **bad})
    new = torch.zeros((2, 1, 128), device=DEV)
    with pytest.raises(ValueError):
        m.mqa_paged_append_kv_rows(K, K, table, new, new[:, :, :64].contiguous(), lens, lens.clone())
    with pytest.raises(m.MqaError):
        m.mqa_paged_append_kv_rows(K, K, table, new, new, lens, lens)
    s, kept = torch.zeros((2, 64), device=DEV), torch.zeros((2, 8), dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        m.mqa_paged_evict_kv(K, K, table, lens, s, table.clone(), lens.clone(), s[:, :32].contiguous(), kept, 0)
    with pytest.raises(m.MqaError):
        m.mqa_paged_evict_kv(K, K, table, lens, s, table.clone(), lens.clone(), s.clone(), kept, 9)


class _Watch:
    """The native calls, with what they returned; or (off) ones that take nothing."""

    def __init__(self, native, on):
        self.native, self.on, self.took = native, on, []

    def __getattr__(self, name):
        def call(*args):
            done = getattr(self.native, name)(*args) if self.on else None
            self.took.append((name, done is not None))
            return done
        return call


@pytest.mark.parametrize("heads", [0, 2])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_native_calls(heads, dtype, monkeypatch):
    """Plain arguments are taken by the native calls, with the general path's results, a captured stream is left to it."""
    import paper_1911_02150_amd.binding as m
    m.load_library()
    g = torch.Generator(device=DEV).manual_seed(9)
    b, n, page, each, k = 3, 2, 16, 40, 64
    lead, per = ((b * each * 2, page) if heads == 0 else (b * each * 2, heads, page)), ((b,) if heads == 0 else (b, heads))
    K, V = (torch.randn((*lead, k), generator=g, device=DEV).to(dtype) for _ in range(2))
    table, out = (torch.randperm(b * each, generator=g, device=DEV).to(torch.int32).view(b, each) + x for x in (0, b * each))
    lens, scores = torch.tensor([600, 7, 0], dtype=torch.int32, device=DEV), torch.rand((*per, each * page), generator=g, device=DEV)
    q, new = torch.randn((b, n, 4, k), generator=g, device=DEV), torch.randn((b, n, *per[1:], k), generator=g, device=DEV)
    logits, drafts, u = torch.randn((b, n + 1, 50), generator=g, device=DEV), torch.ones((b, n), dtype=torch.int32, device=DEV), torch.rand((b, n + 1), generator=g, device=DEV)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)

    def append(counts):
        Kc, Vc, after = K.clone(), V.clone(), torch.zeros_like(lens)
        assert m.mqa_paged_append_kv_rows(Kc, Vc, table, new, new, lens, after, counts=counts) is after
        return Kc, Vc, after

    def scored(**kw):
        s = torch.zeros_like(scores)
        return m.mqa_paged_decode_step(q, K, V, table, lens, scores=scores, scores_out=s, **kw), s

    def evict():
        Kc, Vc, kept, after, s = K.clone(), V.clone(), torch.zeros((*per, 30), dtype=torch.int32, device=DEV), torch.zeros_like(lens), torch.zeros_like(scores)
        assert m.mqa_paged_evict_kv(Kc, Vc, table, lens, scores, out, after, s, kept, 5) is kept
        return Kc, Vc, kept, after, s

    calls = [("paged_append", lambda: append(None)), ("paged_append", lambda: append(torch.tensor([1, 0, 2], dtype=torch.int32, device=DEV))),
             ("paged_decode", lambda: m.mqa_paged_decode_step(q[:, 0].contiguous(), K, V, table, lens)),
             ("paged_decode", lambda: m.mqa_paged_decode_step(q, K, V, table, lens, o=torch.zeros_like(q), scale=0.5, workspace=ws)),
             ("paged_decode", scored), ("paged_decode", lambda: scored(workspace=ws)), ("paged_evict", evict),
             ("verify", lambda: m.mqa_stack_verify_drafts(logits, drafts, u)),
             ("verify", lambda: m.mqa_stack_verify_drafts(logits, drafts, u, draft_logits=logits[:, :n].contiguous(), counts=lens, temperature=0.5, workspace=ws,
                                                          tokens=torch.zeros_like(drafts[:, :1]).repeat(1, n + 1), accepted=torch.zeros_like(lens)))]
    native = m._native
    for name, call in calls:
        got = []
        for on in (True, False):
            watch = _Watch(native, on)
            monkeypatch.setattr(m, "_native", watch)
            got.append(call())
            assert watch.took == [(name, on)], name
        x, y = ((r if isinstance(r, tuple) else (r,)) for r in got)
        assert len(x) == len(y) and all(torch.equal(c, d) and c.dtype == d.dtype and c.shape == d.shape for c, d in zip(x, y)), name
    watch = _Watch(native, True)
    monkeypatch.setattr(m, "_native", watch)
    want, graph = m.mqa_paged_decode_step(q, K, V, table, lens), torch.cuda.CUDAGraph()
    watch.took.clear()
    with torch.cuda.graph(graph):
        got = m.mqa_paged_decode_step(q, K, V, table, lens)
    assert watch.took == [("paged_decode", False)]
    graph.replay()
    assert torch.equal(got, want)
    for bad in (dict(q=q.transpose(1, 2)), dict(lens=lens[:2]), dict(scores=scores[..., 1:].contiguous()), dict(o=q[:, :1].contiguous()), dict(K_pages=K[..., :0], V_pages=V[..., :0, :])):
        with pytest.raises((ValueError, m.MqaError)):
            m.mqa_paged_decode_step(**{**dict(q=q, K_pages=K, V_pages=V, table=table, lens=lens), **bad})


# b, n, h, h_kv, k, dtype, each
NAN_SCORES = [(3, 3, 8, 1, 128, "bf16", 6), (3, 3, 4, 2, 64, "f32", 6), (3, 2, 20, 1, 128, "bf16", 40), (3, 2, 3, 1, 24, "f32", 40)]


@pytest.mark.parametrize("b,n,h,h_kv,k,dtype,each", NAN_SCORES)
def test_scores_of_a_nan_row(m, b, n, h, h_kv, k, dtype, each):
    """A row that is NaN (a NaN in its query; an infinite key) adds NaN to what it sees and nothing to what it does not: positions of later tokens and of pages that hold
    nothing, in one launch and in two."""
    from oracle import paged
    rng = np.random.default_rng(k + each)
    page = 16
    K, V = (pool(rng, b * each, h_kv, page, k, dtype) for _ in range(2))
    table, lens = tables(rng, b, each), np.array([each * page - 20, 40, each * page])
    table[0, 1], table[0, 3], table[2, 0] = -1, 10 ** 6, -7
    q = rng.standard_normal((b, n, h, k)).astype(np.float32)
    q[0, 0, h // 2, 3] = np.nan                                               # the first query of sequence 0: the later tokens' positions are not seen by it
    at = paged.where(table, 1, 5, b * each, page)
    K[at[0], -1, at[1]] = np.inf                                              # a key of sequence 1, in its last K/V head
    one = h_kv == 1
    scores = rng.random((b, h_kv, each * page)).astype(np.float32)
    with np.errstate(all="ignore"):
        want, total, _ = paged.attend(q.astype(np.float64), K, V, table, lens, 0.25, scores)
    written = np.broadcast_to(np.arange(each * page) < lens[:, None, None], total.shape)
    assert np.isnan(total[written]).any() and np.isfinite(total[0, h // 2 * h_kv // h, lens[0] - n + 1:lens[0]]).all()
    out = torch.full((b, each * page) if one else (b, h_kv, each * page), 777.0, device=DEV)
    got = m.mqa_paged_decode_step(on_gpu(q), on_gpu(K, dtype, one), on_gpu(V, dtype, one), on_gpu(table), on_gpu(lens), scale=0.25, scores=on_gpu(scores, one_head=one),
                                  scores_out=out)
    assert np.array_equal(np.isnan(got.cpu().numpy()), np.isnan(want))
    out = out.cpu().numpy().reshape(total.shape)
    assert (out[~written] == 777).all()
    assert np.array_equal(np.isnan(out[written]), np.isnan(total[written]))
    finite = written & ~np.isnan(total)
    bound = tolerance(np.nan_to_num(q), K, 1, 0.25, lens.max()) + EPS * (n * h + 2)      # (of a weight; there are up to n h of them, at most 1 each)
    assert (np.abs(out - total)[finite] <= bound * n * h).all()


@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("b,h_kv,n,h,longest", [(2100, 1, 1, 3, 40), (5000, 2, 2, 4, 300), (40000, 1, 1, 20, 40), (6000, 1, 2, 18, 4500), (3000, 3, 1, 6, 900)])
def test_thousands_of_sequences(m, b, h_kv, n, h, longest, scored):
    """In a table that makes them pieces (more than 1024 positions): against calls for a few hundred sequences each.  Lengths of all kinds, a few far longer than most, or (900)
    none."""
    g = torch.Generator(device=DEV).manual_seed(b)
    page, pages, each, k = 16, 300, 300, 64
    K, V = (torch.randn((pages, h_kv, page, k), generator=g, device=DEV).bfloat16() for _ in range(2))
    table = torch.randint(-1, pages, (b, each), generator=g, device=DEV, dtype=torch.int32)
    lens = torch.randint(0 if longest < 900 else 500, longest, (b,), generator=g, device=DEV, dtype=torch.int32)
    if longest < 900:
        lens[b // 2], lens[-1], lens[7] = each * page, each * page - 5, -1
    q = torch.randn((b, n, h, k), generator=g, device=DEV)
    scores = torch.zeros((b, h_kv, each * page), device=DEV) if scored else None
    got = m.mqa_paged_decode_step(q, K, V, table, lens, scale=0.2, scores=scores)
    again = m.mqa_paged_decode_step(q, K, V, table, lens, scale=0.2)
    assert scored or torch.equal(got, again)
    # (cut into other pieces: float32 sums of up to 4800 weights of another order, half a step each, of values up to 5)
    bound = 2.0 ** -24 * (64 + 8 * 4800 ** 0.5) * 5
    for i in range(0, b, 700):
        part = slice(i, min(b, i + 700))
        s = torch.zeros_like(scores[part]) if scored else None
        want = m.mqa_paged_decode_step(q[part], K, V, table[part], lens[part], scale=0.2, scores=s)
        assert (got[part] - want).abs().max().item() <= bound
        if scored:
            assert (scores[part] - s).abs().max().item() <= 2.0 ** -24 * (64 + 8 * 4800 ** 0.5) * n * h


def test_a_step_grows_with_its_sequences_not_their_square(m):
    """Four times as many short sequences in a table of more than 1024 positions: four times the time, not sixteen (the shortest of several, with room for what else runs)."""
    page, each, k = 16, 66, 8
    K = torch.randn((64, page, k), device=DEV).bfloat16()
    took = []
    for b in (1 << 15, 1 << 17):
        table = torch.zeros((b, each), dtype=torch.int32, device=DEV)
        lens, q = torch.full((b,), 9, dtype=torch.int32, device=DEV), torch.randn((b, 1, k), device=DEV)
        o, times = torch.empty_like(q), []
        for _ in range(6):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            m.mqa_paged_decode_step(q, K, K, table, lens, o=o)
            end.record()
            end.synchronize()
            times.append(start.elapsed_time(end))
        took.append(min(times))
    assert took[1] < 8 * took[0], took


@pytest.mark.parametrize("h_kv", [1, 2])
def test_scores_of_the_tokens_that_stand(m, h_kv):
    """A loop with drafted tokens: attention without scores, verification, then the scores of the tokens that stand, a call for each number of them; as if only those had ever
    been queries.  Twice, so that refused drafts' rows are written over, their places scored from 0 again."""
    from oracle import paged
    rng = np.random.default_rng(h_kv)
    b, n, h, k, page, each, vocab = 6, 3, 4, 64, 16, 5, 50
    one = h_kv == 1
    K, V = (np.zeros((b * each, h_kv, page, k)) for _ in range(2))
    table, lens = tables(rng, b, each), np.array([0, 5, 17, 40, 60, 30])
    first = rng.standard_normal((2, b, 60, h_kv, k)).astype(np.float32)
    bf = lambda x: rounded(x, "bf16")  # noqa: E731
    paged.append(K, V, table, *first, np.zeros(b, dtype=np.int64), lens, bf)
    scores = rng.random((b, h_kv, each * page)).astype(np.float32)
    gK, gV, g_table, g_lens, g_scores = on_gpu(K, "bf16", one), on_gpu(V, "bf16", one), on_gpu(table), on_gpu(lens), on_gpu(scores, one_head=one)
    scores, seen = scores.astype(np.float64), set()
    for _ in range(2):
        new = rng.standard_normal((2, b, n + 1, h_kv, k)).astype(np.float32)
        q = rng.standard_normal((b, n + 1, h, k)).astype(np.float32)
        logits, u = rng.standard_normal((b, n + 1, vocab)).astype(np.float32), rng.random((b, n + 1), dtype=np.float32)
        drafts = np.where(rng.random((b, n)) < 0.8, logits[:, :n].argmax(-1), 7)
        g_q, after = on_gpu(q), torch.zeros_like(g_lens)
        m.mqa_paged_append_kv_rows(gK, gV, g_table, *(on_gpu(x[:, :, 0] if one else x) for x in new), g_lens, after)
        o = m.mqa_paged_decode_step(g_q, gK, gV, g_table, after, scale=0.25)
        tokens, accepted = m.mqa_stack_verify_drafts(on_gpu(logits), on_gpu(drafts), on_gpu(u), temperature=0.0)
        g_lens += accepted + 1
        for j in range(1, n + 2):
            m.mqa_paged_decode_step(g_q[:, :j].contiguous(), gK, gV, g_table, g_lens * (accepted + 1 == j), scale=0.25, scores=g_scores)
        grown = paged.append(K, V, table, *new, lens, rounded=bf)
        want, _, size = paged.attend(q.astype(np.float64), K, V, table, grown, 0.25)
        assert (np.abs(o.cpu().numpy() - want) <= tolerance(q, K, size, 0.25, 80)).all()
        _, stand = paged.verify(logits, drafts, u, temperature=0)
        assert accepted.tolist() == stand.tolist()
        seen.update(stand.tolist())
        lens = lens + stand + 1
        for i in range(b):
            rows = stand[i] + 1
            _, total, _ = paged.attend(q[i:i + 1, :rows].astype(np.float64), K, V, table[i:i + 1], lens[i:i + 1], 0.25, scores[i:i + 1])
            scores[i] = np.where(np.isnan(total[0]), scores[i], total[0])
    assert len(seen) > 2 and g_lens.tolist() == lens.tolist()
    bound = 2 * (tolerance(q, K, 1, 0.25, 80) + EPS * ((n + 1) * h + 2)) * (1 + scores)      # (two steps)
    assert (np.abs(g_scores.cpu().numpy().reshape(scores.shape) - scores) <= bound).all()


@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("b,h_kv,n,h,lengths", [(600, 1, 1, 3, "like"), (300, 2, 2, 4, "like"), (260, 1, 1, 40, "like"), (700, 1, 1, 8, "one long"), (1024, 1, 2, 3, "one long")])
def test_hundreds_of_sequences_in_a_long_table(m, b, h_kv, n, h, lengths, scored):
    """A table of more than 1024 positions, so that work is looked for by length.  Alike: at most 64 tiles each, the longest no more than twice the average, two workgroups or more
    for every compute unit: every cache is left whole, and there is nothing to merge.  Or most of them short or empty, and one that is cut."""
    from oracle import paged
    rng = np.random.default_rng(b)
    page, pages, each, k = 16, 60, 70, 64
    K, V = (pool(rng, pages, h_kv, page, k, "bf16") for _ in range(2))
    table = rng.integers(0, pages, (b, each))
    lens = rng.integers(700, 1100, b) if lengths == "like" else rng.integers(0, 60, b) * (np.arange(b) % 7 != 0)
    if lengths == "one long":
        lens[b // 2] = each * page
    q = rng.standard_normal((b, n, h, k)).astype(np.float32)
    scores = rng.random((b, h_kv, each * page)).astype(np.float32) if scored else None
    want, total, size = paged.attend(q.astype(np.float64), K, V, table, lens, 0.125, scores)
    one = h_kv == 1
    kw = dict(scores=on_gpu(scores, one_head=one), scores_out=torch.full((b, each * page) if one else (b, h_kv, each * page), 777.0, device=DEV)) if scored else {}
    got = m.mqa_paged_decode_step(on_gpu(q), on_gpu(K, "bf16", one), on_gpu(V, "bf16", one), on_gpu(table), on_gpu(lens), scale=0.125, **kw)
    assert (np.abs(got.cpu().numpy() - want) <= tolerance(q, K, size, 0.125, lens.max())).all()
    if scored:
        out, left = kw["scores_out"].cpu().numpy().reshape(total.shape), np.isnan(total)
        bound = (tolerance(q, K, 1, 0.125, lens.max()) + EPS * (2 + n * h / h_kv)) * total
        assert (out[left] == 777).all() and (np.abs(out - total)[~left] <= bound[~left]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k,each", [(128, 3), (64, 40), (40, 40)])
def test_a_row_of_nothing_but_infinite_logits(m, k, each, dtype):
    """Logits of -infinity throughout are as if nothing were seen: a row of 0 and no weight."""
    rng = np.random.default_rng(k)
    page = 16
    lens = np.array([each * page - 3, 20])
    K = np.full((2 * each, 1, page, k), 1.0)
    K[:, :, :, 0] = -np.inf
    V, table = pool(rng, 2 * each, 1, page, k, dtype), tables(rng, 2, each)
    q = np.ones((2, 2, k), dtype=np.float32)
    q[:, 1, 0] = -1                                                            # (the second row's logits: +infinity, which is NaN as a softmax)
    scores = torch.zeros((2, each * page), device=DEV)
    args = [on_gpu(x, d, True) if d else on_gpu(x) for x, d in ((K, dtype), (V, dtype), (table, None), (lens, None))]
    got = m.mqa_paged_decode_step(on_gpu(q[:, :1].copy()), *args, scale=0.25, scores=scores)
    assert not got.any() and not scores.any()
    got = m.mqa_paged_decode_step(on_gpu(q), *args, scale=0.25)
    assert not got[:, 0].any() and torch.isnan(got[:, 1]).all()


def test_the_list_of_a_replayed_step(m):
    """1500 sequences in a long table, captured once: the list of their pieces is written anew at every replay, inside the workspace that the call asks for."""
    g = torch.Generator(device=DEV).manual_seed(14)
    b, each, page, k = 1500, 80, 16, 64
    K, V = (torch.randn((90, page, k), generator=g, device=DEV).bfloat16() for _ in range(2))
    table, q = torch.randint(0, 90, (b, each), generator=g, device=DEV, dtype=torch.int32), torch.randn((b, 4, k), generator=g, device=DEV)
    lens, scores = torch.zeros(b, dtype=torch.int32, device=DEV), torch.zeros((b, each * page), device=DEV)
    need = m.mqa_paged_decode_workspace_bytes(b, 1, 4, 1, page, each, k, k, m.MQA_BF16, True)
    guard = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
    run = lambda o, out, ws=None: m.mqa_paged_decode_step(q, K, V, table, lens, o=o, scale=0.3, scores=scores, scores_out=out, workspace=ws)  # noqa: E731
    o, out = torch.zeros_like(q), torch.zeros_like(scores)
    run(o, out, guard[:need])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(o, out, guard[:need])
    whole = each * page
    for lengths in (torch.randint(0, 30, (b,), generator=g, device=DEV), torch.full((b,), whole, device=DEV), torch.randint(600, 1000, (b,), generator=g, device=DEV),
                    (torch.arange(b, device=DEV) % 97 == 0) * whole):
        lens.copy_(lengths)
        want, want_out = torch.zeros_like(q), torch.zeros_like(scores)
        run(want, want_out)
        guard[:need] = 0x5a
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want) and torch.equal(out, want_out) and (guard[need:] == 0x5a).all()
        some = torch.arange(0, b, 211, device=DEV)                             # (alone: other pieces, sums of another order)
        alone = m.mqa_paged_decode_step(q[some], K, V, table[some], lens[some], scale=0.3)
        assert (alone - want[some]).abs().max().item() <= EPS * (64 + 8 * whole ** 0.5) * 5
