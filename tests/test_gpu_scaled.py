"""Paged caches of 8 bits on the GPU against the float64 oracle (oracle/serving.py)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 2.0 ** -24          # half a step of float32
TYPES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


@pytest.fixture(scope="module")
def m():
    import paper_1911_02150_amd as mod
    mod.load_library()
    return mod


def pool(rng, num_pages, h_kv, page, width, block, kind, powers=True, spread=0.7):
    """Values of 8 bits, and scales of unlike sizes: powers of two, or any."""
    from oracle import serving
    scales = np.exp(spread * rng.standard_normal((num_pages, h_kv, page // block))) * 2.0 ** -5
    scales = 2.0 ** np.round(np.log2(scales)) if powers else scales.astype(np.float32).astype(np.float64)
    return serving.rounded(32 * rng.standard_normal((num_pages, h_kv, page, width)), kind), scales


def bits(values, kind, one=False):
    """Values of 8 bits as a device tensor."""
    t = torch.from_numpy(np.ascontiguousarray(values[:, 0] if one else values)).float()
    return t.to(TYPES[kind]).contiguous().to(DEV)


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.int32).to(DEV)


def f32(x, one=False):
    return torch.from_numpy(np.ascontiguousarray(x[:, 0] if one else x)).float().to(DEV)


def tables(rng, b, each, first=0):
    return first + rng.permutation(b * each).reshape(b, each)


def cache_of(rng, b, each, h_kv, page, block, k, v, kind, powers=True):
    K, Ks = pool(rng, b * each, h_kv, page, k, block, kind, powers)
    V, Vs = pool(rng, b * each, h_kv, page, v, block, kind, powers)
    one = h_kv == 1
    return (K, Ks, V, Vs), (bits(K, kind, one), f32(Ks, one), bits(V, kind, one), f32(Vs, one))


def tolerance(q, K, size, scale, length, kind, top):
    """Half a step for each of: k products and their sum (a logit, at most scale * |q| |K|; q's two terms have 23 bits, two half steps more in every product), its scale and the row's, the
    exponential and its argument, a weight's scale, as many sums as there are positions, each over rounding errors that do not know of one another (eight
    standard deviations).  And for every position half a step of fp16's smallest numbers, 2^-25, in units in which the row's largest weight times scale is 2^10 at least: 2^-35 of
    `top`, which is no less than that largest one, times the type's largest number.  (A position's weight times scale w is 2^10 and more for the largest; its two fp16 terms hold
    w (1 + e) + d, |e| <= 2^-23, |d| <= 2^-25, the second only below 2^-2, that is 2^-12 of the largest; what an earlier maximum was the unit of is scaled down.)"""
    k = q.shape[-1]
    logit = abs(scale) * np.abs(q).max() * np.abs(K[np.isfinite(K)]).max() * k ** 0.5 * 4      # (4: a sum of k products of normal numbers)
    return EPS * ((2 * (8 + 4) + 4 + 3) * logit + 17 + 8 * length ** 0.5) * size + length * 2.0 ** -35 * {"e4m3": 448, "int8": 127}[kind] * top + 1e-30


def attended(q, arrays, table, lens, scale):
    from oracle import paged, serving
    K, Ks, V, Vs = arrays
    with np.errstate(invalid="ignore", over="ignore"):
        K, V = serving.whole(K, Ks), serving.whole(V, Vs)
        sizes = np.abs(np.repeat(Vs, V.shape[2] // Vs.shape[2], axis=2))[..., None]
    o, _, size = paged.attend(q.astype(np.float64), K, V, table, np.array(lens), float(np.float32(scale)))
    top, _, _ = paged.attend(q.astype(np.float64), K, sizes, table, np.array(lens), float(np.float32(scale)))      # (the sum of weight times scale: no less than the largest)
    return o, size, K, np.where(np.isfinite(top), top, 0)


# b, n, h, h_kv, k, v, page size, block, lengths
ATTEND = [
    (1, 1, 1, 1, 16, 16, 1, 1, [1]),
    (3, 1, 8, 1, 128, 128, 16, 16, [0, 1, 33]),
    (4, 1, 8, 1, 128, 128, 16, 16, [511, 512, 513, 700]),
    (2, 1, 32, 1, 128, 128, 64, 64, [1500, 31]),
    (2, 1, 64, 1, 128, 128, 16, 8, [300, 900]),
    (2, 1, 20, 1, 128, 128, 7, 7, [129, 257]),
    (2, 5, 8, 1, 128, 128, 16, 4, [5, 400]),
    (2, 3, 8, 8, 128, 128, 16, 16, [2, 350]),
    (3, 1, 8, 8, 64, 64, 16, 1, [1, 128, 600]),
    (2, 4, 8, 2, 64, 64, 5, 5, [3, 77]),
    (2, 2, 12, 3, 64, 64, 24, 3, [290, 33]),
    (2, 1, 8, 1, 128, 128, 32, 16, [1025, 64]),
    (2, 2, 24, 1, 128, 128, 100, 20, [99, 301]),
    (2, 2, 6, 2, 48, 32, 3, 3, [100, 350]),
    (2, 1, 3, 1, 256, 256, 16, 16, [513, 17]),
    (1, 1, 9, 1, 16, 256, 16, 2, [400]),
    (1, 1, 70, 1, 256, 16, 11, 11, [290]),
    (1, 128, 8, 1, 128, 128, 16, 16, [300]),
    (5, 1, 1, 1, 128, 128, 32, 32, [0, 0, 0, 0, 0]),
    (1, 1, 33, 1, 96, 112, 9, 9, [500]),
    (2, 2, 20, 1, 208, 192, 16, 16, [600, 50]),
    (2, 1, 40, 1, 192, 240, 16, 16, [700, 33]),
    (3, 3, 4, 2, 112, 80, 32, 8, [260, 1, 2000]),
    (2, 1, 16, 1, 128, 64, 512, 256, [1000, 513]),
    (2, 2, 16, 2, 64, 128, 16, 16, [333, 40]),
    (1, 1, 16, 1, 64, 48, 48, 16, [1700]),
]


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("b,n,h,h_kv,k,v,page,block,lens", ATTEND)
def test_attention(m, b, n, h, h_kv, k, v, page, block, lens, kind):
    rng = np.random.default_rng(b + 7 * n + 11 * h + k + len(lens))
    each = -(-max(max(lens), 1) // page) + 3
    arrays, cache = cache_of(rng, b, each, h_kv, page, block, k, v, kind, powers=h % 2 == 0)
    table = tables(rng, b, each)
    q = rng.standard_normal((b, n, h, k)).astype(np.float32)
    scale = 2 / k ** 0.5
    want, size, K, top = attended(q, arrays, table, lens, scale)
    args = (f32(q[:, 0] if n == 1 else q), *cache, i32(table), i32(np.array(lens)))
    got = m.mqa_paged_scaled_decode_step(*args, scale=scale)
    given = torch.full_like(got, 777.0)
    assert got.shape == ((b, h, v) if n == 1 else (b, n, h, v)) and m.mqa_paged_scaled_decode_step(*args, scale=scale, o=given) is given and torch.equal(got, given)
    off = np.abs(got.cpu().numpy().reshape(want.shape) - want)
    assert (off <= tolerance(q, K, size, scale, max(lens), kind, top)).all(), off.max()


# lengths whose pieces fit none of the even shares; as few as a wave looks through and one more; long ones among short ones; more than a thread has one of
UNEVEN = [([830] * 150 + [20] * 100, 1, 1), ([700, 0, 1, 33] * 16, 2, 2), ([40, 1300, 7, 260, 0] * 13, 1, 2), ([9, 2600] + [64] * 61, 4, 4), ([300, 31, 650] * 90, 1, 2), ([64, 0, 1100, 3, 90] * 110, 1, 1),
          ([33] * 1023 + [2100], 1, 1)]


@pytest.mark.parametrize("lens,h_kv,h", UNEVEN)
def test_pieces_of_uneven_lengths(m, lens, h_kv, h):
    """Every piece is somebody's, in a table of a capacity that is cut."""
    b, k, page, block, kind, scale = len(lens), 32, 16, 16, "int8", 0.25
    rng = np.random.default_rng(b + h)
    each = -(-max(lens) // page)
    arrays, cache = cache_of(rng, b, each, h_kv, page, block, k, k, kind)
    table = tables(rng, b, each)
    q = rng.standard_normal((b, 1, h, k)).astype(np.float32)
    want, size, K, top = attended(q, arrays, table, lens, scale)
    wide = np.concatenate([table, np.full((b, 1000 - each), -1)], 1)
    got = m.mqa_paged_scaled_decode_step(f32(q[:, 0]), *cache, i32(wide), i32(np.array(lens)), scale=scale)
    assert (np.abs(got.cpu().numpy().reshape(want.shape) - want) <= tolerance(q, K, size, scale, max(lens), kind, top)).all()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("n,h,h_kv,k", [(1, 8, 1, 128), (4, 8, 1, 128), (3, 4, 4, 64), (2, 40, 1, 128), (2, 4, 2, 32)])
def test_what_is_not_seen_may_hold_anything(m, n, h, h_kv, k, kind):
    """NaN, and scales that are no numbers, behind the length, on missing pages, and at the places of later queries; lengths out of range; pages that hold nothing."""
    from oracle import paged
    rng = np.random.default_rng(n * h + k)
    b, page, each, block = 5, 16, 6, 1
    arrays, cache = cache_of(rng, b, each, h_kv, page, block, k, k, kind)
    K, Ks, V, Vs = arrays
    table, lens = tables(rng, b, each), np.array([40, -3, 1000, 65, 96])
    clean = K * np.repeat(Ks, block, axis=2)[..., None]
    table[0, 1], table[3, 0], table[3, 1], table[4] = -1, b * each, 2 ** 31 - 1, -5
    for i in range(b):
        length = min(max(int(lens[i]), 0), page * each)
        for p in range(length, page * each):
            at = paged.where(table, i, p, b * each, page)
            if at is not None:
                Ks[at[0], :, at[1]], Vs[at[0], :, at[1]] = np.nan, (np.inf, np.nan)[p % 2]
                if kind == "e4m3":
                    K[at[0], :, at[1]], V[at[0], :, at[1]] = np.nan, np.nan
        for j in range(1, n):                                                 # seen by the later queries alone
            at = paged.where(table, i, length - j, b * each, page) if length - j >= 0 else None
            if at is not None:
                Vs[at[0], :, at[1]] = (np.inf, -np.inf, np.nan)[j % 3]
    q = rng.standard_normal((b, n, h, k)).astype(np.float32)
    one = h_kv == 1
    want, size, _, top = attended(q, (K, Ks, V, Vs), table, lens, 0.25)
    got = m.mqa_paged_scaled_decode_step(f32(q), bits(K, kind, one), f32(Ks, one), bits(V, kind, one), f32(Vs, one), i32(table), i32(lens), scale=0.25)
    got = got.cpu().numpy().astype(np.float64)
    assert not got[1].any() and not got[4].any() and np.isfinite(got[:, 0]).all()
    finite = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~finite & ~np.isnan(want)], want[~finite & ~np.isnan(want)])
    assert (np.abs(got - want)[finite] <= tolerance(q, clean, size, 0.25, 96, kind, top)[finite]).all()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("k", [128, 64, 48])
def test_queries_of_any_size(m, k, kind):
    """Rows of zeros, of tiny and of huge numbers, and with an infinity (whose row is NaN: its products with both signs are added)."""
    rng = np.random.default_rng(k)
    arrays, cache = cache_of(rng, 1, 20, 1, 16, 16, k, k, kind)
    table, lens = tables(rng, 1, 20), np.array([300])
    q = rng.standard_normal((1, 1, 8, k)).astype(np.float32)
    q[0, 0, 1] = 0
    q[0, 0, 2] *= 1e-38
    q[0, 0, 3] *= np.float32(1e-42)
    q[0, 0, 4] *= 1e-3
    q[0, 0, 4, 0] = 30
    q[0, 0, 5] *= 50
    want, size, K, top = attended(q, arrays, table, lens, 0.3)
    got = m.mqa_paged_scaled_decode_step(f32(q[:, 0]), *cache, i32(table), i32(lens), scale=0.3).cpu().numpy()
    for r in range(8):
        assert (np.abs(got[:, r] - want[:, 0, r]) <= tolerance(q[:, :, r], K, size[:, 0, r], 0.3, 300, kind, top[:, 0, r])).all(), r
    q[0, 0, 7, 3] = np.inf
    odd = m.mqa_paged_scaled_decode_step(f32(q[:, 0]), *cache, i32(table), i32(lens), scale=0.3).cpu().numpy()
    assert np.isnan(odd[0, 7]).all() and (np.abs(odd[:, :7] - want[:, 0, :7]) <= np.stack([tolerance(q[:, :, r], K, size[:, 0, r], 0.3, 300, kind, top[:, 0, r]) for r in range(7)], 1)).all()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("h", [8, 32])
def test_scales_far_apart(m, h, kind):
    """V's scales from 2^-60 to 2^60 and 0: what a row sees decides about its accuracy, not what others see, or see hardly."""
    rng = np.random.default_rng(h)
    (K, Ks, V, Vs), _ = cache_of(rng, 2, 30, 1, 16, 16, 128, 128, kind)
    table, lens = tables(rng, 2, 30), np.array([470, 100])
    for i, sizes in enumerate(([-60, 0, -30, 3], [60, -20])):
        for x in range(30):
            Vs[table[i, x]] = 2.0 ** sizes[x % len(sizes)]
    Vs[table[1, 1]] = 0
    Ks[table[0, 2]] = 0
    Ks[table[1, 2]] = 2.0 ** -100
    q = (0.3 * rng.standard_normal((2, 1, h, 128))).astype(np.float32)
    want, size, K_all, top = attended(q, (K, Ks, V, Vs), table, lens, 0.1)
    got = m.mqa_paged_scaled_decode_step(f32(q[:, 0]), bits(K, kind, True), f32(Ks, True), bits(V, kind, True), f32(Vs, True), i32(table), i32(lens), scale=0.1).cpu().numpy()
    assert (np.abs(got - want[:, 0]) <= tolerance(q, K_all, size, 0.1, 470, kind, top)[:, 0]).all()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("h,each", [(8, 30), (32, 30), (8, 120)])
def test_scales_apart_and_nothing(m, h, each, kind):
    """V's scales from 2^-45 to 2^45, tile by tile and within tiles, K's of many sizes; blocks of zeros, which have the smallest scale, with most of a row's weight: they count in its sum; scales that are
    no powers of two; one that is smaller than any, whose rows are no zeros and all that a sequence has."""
    rng = np.random.default_rng(h + each)
    (K, Ks, V, Vs), _ = cache_of(rng, 3, each, 1, 16, 16, 128, 128, kind)
    table, lens = tables(rng, 3, each), np.array([16 * each - 5, 16 * each, 20])
    for x in range(each):
        Vs[table[0, x]] = 2.0 ** ((45, -45, 0, 3)[x // 2 % 4] if x < each // 2 else rng.integers(-45, 46))
        Vs[table[1, x]] = np.float32(rng.random() + 0.5)
    Vs[table[1, 3:9]], V[table[1, 3:9]] = 2.0 ** -126, 0
    V[table[1, 4]] = -0.0
    Vs[table[2]] = 2.0 ** -120
    q = (0.3 * rng.standard_normal((3, 1, h, 128))).astype(np.float32)
    K[table[1, 5], 0, 2] = np.sign(q[1, 0, 0]) * 96                          # (a row of zeros takes most of the weight)
    want, size, K_all, top = attended(q, (K, Ks, V, Vs), table, lens, 0.1)
    got = m.mqa_paged_scaled_decode_step(f32(q[:, 0]), bits(K, kind, True), f32(Ks, True), bits(V, kind, True), f32(Vs, True), i32(table), i32(lens), scale=0.1).cpu().numpy()
    bound = tolerance(q, K_all, size, 0.1, 16 * each, kind, top)
    bound[2] = tolerance(q, K_all, size, 0.1, 16 * each, kind, top)[2] - 1e-30 + 2.0 ** -149      # (down to float32's smallest)
    assert (np.abs(got - want[:, 0]) <= bound[:, 0]).all()


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_large_logits(m, kind):
    """Logits of hundreds: one position takes all the weight, others none."""
    rng = np.random.default_rng(5)
    arrays, cache = cache_of(rng, 1, 40, 1, 16, 16, 128, 128, kind)
    table, lens = tables(rng, 1, 40), np.array([640])
    q = (20 * rng.standard_normal((1, 1, 8, 128))).astype(np.float32)
    want, size, K, top = attended(q, arrays, table, lens, 1.0)
    got = m.mqa_paged_scaled_decode_step(f32(q[:, 0]), *cache, i32(table), i32(lens)).cpu().numpy()
    assert (np.abs(got - want[:, 0]) <= tolerance(q, K, size, 1.0, 640, kind, top)[:, 0]).all()


# b, n, h, k, v, pages of a sequence: so many sequences that a workgroup has 32 rows, in one launch and in two, and listed
MANY = [
    (300, 1, 20, 128, 128, 4),
    (300, 2, 20, 128, 128, 70),
    (400, 1, 20, 64, 64, 70),
    (400, 1, 18, 48, 64, 5),
    (300, 1, 20, 112, 96, 70),
    (300, 1, 40, 208, 256, 4),
    (300, 1, 20, 256, 256, 70),
    (1100, 1, 4, 64, 64, 70),
]


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("b,n,h,k,v,each", MANY)
def test_many_sequences_of_many_rows(m, b, n, h, k, v, each, kind):
    """Pages shared by all sequences, some of them nothing's."""
    rng = np.random.default_rng(b + h + k + each)
    page, pages = 16, 50
    arrays, cache = cache_of(rng, 1, pages, 1, page, 8, k, v, kind)
    table = rng.integers(0, pages, (b, each))
    table[rng.random((b, each)) < 0.02] = -1
    lens = rng.integers(0, each * page + 1, b)
    q = rng.standard_normal((b, n, h, k)).astype(np.float32)
    got = m.mqa_paged_scaled_decode_step(f32(q), *cache, i32(table), i32(lens), scale=0.2).cpu().numpy()
    for i in [0, 1, 2, b // 2, b - 1, int(np.argmax(lens)), int(np.argmin(lens))]:
        want, size, K, top = attended(q[i:i + 1], arrays, table[i:i + 1], lens[i:i + 1], 0.2)
        off = np.abs(got[i] - want[0])
        assert (off <= tolerance(q, K, size, 0.2, each * page, kind, top)[0]).all(), (i, off.max())


@pytest.mark.parametrize("k,v,h,kind", [(64, 64, 8, "e4m3"), (64, 64, 33, "int8"), (128, 128, 9, "int8"), (128, 128, 40, "e4m3"), (48, 32, 20, "int8"), (96, 112, 8, "e4m3"), (80, 128, 17, "int8"),
                                        (256, 192, 9, "e4m3"), (16, 256, 20, "int8")])
def test_every_form_over_more_than_4_gib(m, k, v, h, kind):
    """What it is over a small pool of the same pages."""
    page, few, b = 64, 24, 2
    pages = (1 << 32) // (page * max(k, v)) + 40
    rng = np.random.default_rng(k + v + h)
    arrays, small = cache_of(rng, b, few // b, 1, page, 16, k, v, kind)
    table, lens = tables(rng, b, few // b), i32(np.array([few // b * page - 5, 300]))
    q = f32(rng.standard_normal((b, h, k)))
    want = m.mqa_paged_scaled_decode_step(q, *small, i32(table), lens, scale=0.3)
    places = torch.from_numpy(np.concatenate([rng.permutation(few // 2), pages - 1 - rng.permutation(few // 2)])).to(DEV)
    large = []
    for t in small:
        pool = torch.zeros((pages, *t.shape[1:]), dtype=torch.float32 if t.dtype == torch.float32 else torch.uint8, device=DEV)
        pool[places] = t if t.dtype == torch.float32 else t.view(torch.uint8)
        large.append(pool if t.dtype == torch.float32 else pool.view(t.dtype))
    got = m.mqa_paged_scaled_decode_step(q, *large, i32(places.cpu().numpy()[table]), lens, scale=0.3)
    assert torch.equal(got, want)


def test_a_pool_of_more_than_4_gib(m):
    """Rows whose offsets do not fit 32 bits."""
    page, pages, k = 64, (4 << 30) // (64 * 128) + 70, 128
    K, V = (torch.zeros((pages, page, k), dtype=torch.int8, device=DEV) for _ in range(2))
    Ks, Vs = (torch.zeros((pages, 2), device=DEV) for _ in range(2))
    rng = np.random.default_rng(1)
    table = i32(np.array([[pages - 1, 0, pages - 2], [pages - 70, 5, pages // 2]]))
    new = rng.standard_normal((2, 150, k)).astype(np.float32)
    lens, lens_out = i32(np.zeros(2)), i32(np.zeros(2))
    m.mqa_paged_scaled_append_kv_rows(K, Ks, V, Vs, table, f32(new), f32(-new), lens, lens_out)
    assert lens_out.tolist() == [150, 150]
    named = table.long().view(-1)
    small = [t[named].contiguous() for t in (K, Ks, V, Vs)]
    q = torch.from_numpy(rng.standard_normal((2, 8, k)).astype(np.float32)).to(DEV)
    order = torch.arange(6, device=DEV, dtype=torch.int32).view(2, 3)
    assert torch.equal(m.mqa_paged_scaled_decode_step(q, K, Ks, V, Vs, table, lens_out), m.mqa_paged_scaled_decode_step(q, *small, order, lens_out))
    assert int((K != 0).sum()) == int((small[0] != 0).sum()) > 0
    moves = i32(np.array([[pages - 1, 7], [3, pages - 3]]))
    m.mqa_paged_copy_pages([K, Ks], moves)
    assert torch.equal(K[7], K[pages - 1]) and torch.equal(Ks[7], Ks[pages - 1]) and not K[pages - 3].any()


# b, n, h_kv, k, v, page size, block, lengths, counts
APPEND = [
    (1, 1, 1, 16, 16, 1, 1, [0], None),
    (4, 1, 1, 128, 128, 16, 16, [0, 5, 16, 31], None),
    (4, 3, 1, 128, 64, 16, 16, [14, 15, 16, 0], [3, 2, 0, 1]),
    (3, 40, 2, 64, 48, 12, 4, [0, 3, 17], [40, -2, 99]),
    (2, 100, 1, 128, 128, 64, 64, [30, 0], None),
    (2, 33, 8, 32, 256, 8, 1, [1, 8], None),
    (2, 150, 1, 256, 256, 128, 128, [100, 0], [150, 77]),
    (5, 7, 3, 16, 112, 21, 7, [0, 6, 13, 20, 2], None),
    (3, 2, 1, 128, 128, 16, 16, [-1, 1 << 30, 95], None),
    (1, 300, 1, 208, 96, 300, 100, [55], None),
    (2, 400, 1, 256, 112, 300, 300, [299, 10], [400, 1]),
    (3, 40, 2, 128, 80, 32, 32, [31, 0, 32], [40, 33, 1]),
    (2, 100, 1, 144, 64, 64, 64, [1, 64], None),
]


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("b,n,h_kv,k,v,page,block,lens,counts", APPEND)
def test_append(m, b, n, h_kv, k, v, page, block, lens, counts, kind):
    """Bit for bit the oracle's, other blocks as they were; once more onto the same lengths nothing changes."""
    from oracle import serving
    rng = np.random.default_rng(b * n + k)
    each = -(-(max(x for x in lens if x < 1 << 20) + n) // page)
    arrays, cache = cache_of(rng, b, each + 1, h_kv, page, block, k, v, kind)
    table = tables(rng, b, each + 1)[:, :each].copy()
    if b > 2:
        table[1, -1] = -1
    one = h_kv == 1
    k_new, v_new = (rng.standard_normal((b, n, h_kv, w)) * np.exp2(rng.integers(-3, 4, (b, n, h_kv, 1))) for w in (k, v))
    k_new, v_new = k_new.astype(np.float32), v_new.astype(np.float32)
    k_new[0, 0, 0, 0], v_new[-1, -1, -1, -1] = np.nan, np.inf
    if n > 1:
        k_new[0, 1], v_new[-1, 0] = 0, -np.inf
    lens = np.array(lens)
    with np.errstate(invalid="ignore"):
        want_lens = serving.append(*arrays, table, k_new, v_new, lens, counts, kind)
    rows = [torch.from_numpy(x[:, :, 0] if one else x).contiguous().to(DEV) for x in (k_new, v_new)]
    lens_out = i32(np.full(b, 777))
    kw = dict(counts=None if counts is None else i32(np.array(counts)))
    for _ in range(2):
        assert m.mqa_paged_scaled_append_kv_rows(*cache, i32(table), *rows, i32(lens), lens_out, **kw) is lens_out
        assert np.array_equal(lens_out.cpu().numpy(), want_lens)
        for got, want in zip(cache, arrays):
            got = got.float().cpu().double().numpy().reshape(want.shape)
            assert np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_rounding_of_every_size(m, kind):
    """Values around every number of 8 bits and around the middles between them, under scales from 2^-126 to 2^119."""
    from oracle import serving
    every = torch.arange(256, dtype=torch.uint8).view(TYPES["e4m3"]).float().numpy() if kind == "e4m3" else np.arange(-127, 128, dtype=np.float32)
    every = np.unique(every[np.isfinite(every)])
    x = np.concatenate([every, (every[1:] + every[:-1]) / 2]).astype(np.float32)
    x = np.concatenate([x, np.nextafter(x, np.float32(-1e9)), np.nextafter(x, np.float32(1e9))])
    x = np.clip(x, -serving.LARGEST[kind], serving.LARGEST[kind])
    x = np.concatenate([x, np.zeros(-len(x) % 15)]).reshape(-1, 15)
    x = np.concatenate([x, np.full((len(x), 1), serving.LARGEST[kind])], 1).astype(np.float32)       # (every row has the largest number: scale 1)
    for e in (0, -126, -40, 60, 119):
        new = (x.astype(np.float64) * 2.0 ** e).astype(np.float32)[None]
        n = new.shape[1]
        cache = [torch.zeros((n, 1, 16), dtype=TYPES[kind], device=DEV), torch.zeros((n, 1), device=DEV)] * 1
        V = [t.clone() for t in cache]
        table, lens, lens_out = i32(np.arange(n)[None]), i32(np.zeros(1)), i32(np.zeros(1))
        m.mqa_paged_scaled_append_kv_rows(*cache, *V, table, f32(new), f32(new), lens, lens_out)
        assert (cache[1] == 2.0 ** e).all()
        want = serving.rounded(new[0].astype(np.float64) / 2.0 ** e, kind)
        assert np.array_equal(cache[0].float().cpu().numpy()[:, 0], want) and torch.equal(cache[0].view(torch.uint8), V[0].view(torch.uint8))


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_token_by_token_with_refused_drafts(m, kind):
    """Tokens in ones and threes, some taken back; scales only grow while a block has rows, a block begun anew starts anew; scales of the caller's that are no powers of two."""
    from oracle import serving
    rng = np.random.default_rng(9)
    arrays, cache = cache_of(rng, 3, 5, 2, 16, 8, 32, 64, kind, powers=False)
    table, lens = tables(rng, 3, 5), np.array([5, 12, 0])
    for step in range(25):
        n = (1, 3)[step % 2]
        new = [(rng.standard_normal((3, n, 2, w)) * np.exp2(rng.integers(-6, 3))).astype(np.float32) for w in (32, 64)]
        after = serving.append(*arrays, table, *new, lens, kind=kind)
        out = i32(np.zeros(3))
        m.mqa_paged_scaled_append_kv_rows(*cache, i32(table), *[torch.from_numpy(x).to(DEV) for x in new], i32(lens), out)
        assert np.array_equal(out.cpu().numpy(), after)
        lens = np.maximum(after - rng.integers(0, 3, 3), 0)
        for got, want in zip(cache, arrays):
            got = got.float().cpu().double().numpy()
            assert np.abs(got - want).max() <= (0 if got.shape[-1] > 2 else EPS * np.abs(want).max()), step      # (the caller's own scales are float32's)


def test_streams_and_graphs(m):
    """On a stream given, with a workspace given, and captured: replays follow the lengths, rows and pages of their turn, with eager work between them."""
    rng = np.random.default_rng(2)
    b, page, each, k, h = 6, 16, 80, 128, 16
    arrays, cache = cache_of(rng, b, each, 1, page, 16, k, k, "e4m3")
    table, lens, after = i32(tables(rng, b, each)), i32(np.zeros(b)), i32(np.zeros(b))
    q = torch.randn(b, 2, h, k, device=DEV)
    new = [torch.randn(b, 2, k, device=DEV) for _ in range(2)]
    nbytes = m.mqa_paged_scaled_decode_workspace_bytes(b, 2, h, 1, page, each, k, k, m.MQA_E4M3)
    assert nbytes > 0
    ws, o = torch.empty(nbytes, dtype=torch.uint8, device=DEV), torch.empty_like(q)

    def step(c, out, **kw):
        m.mqa_paged_scaled_append_kv_rows(*c, table, *new, lens, after, **{x: y for x, y in kw.items() if x == "stream"})
        return m.mqa_paged_scaled_decode_step(q, *c, table, after, o=out, scale=0.1, **kw)

    eager = [t.clone() for t in cache]
    step(eager, torch.empty_like(q))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    captured = [t.clone() for t in cache]
    with torch.cuda.graph(graph):
        step(captured, o, workspace=ws)
    inner = torch.cuda.CUDAGraph()
    o_inner = torch.empty_like(q)
    with torch.cuda.graph(inner):                                  # a workspace of the call's own
        m.mqa_paged_scaled_decode_step(q, *captured, table, after, o=o_inner, scale=0.1)
    eager = [t.clone() for t in captured]
    side = torch.cuda.Stream()
    for lengths in ([0, 1, 15, 16, 700, 1278], [5] * 6, [1278, 0, 300, 17, 1000, 3], [1279, 1280, -1, 2, 3, 4]):
        lens.copy_(i32(np.array(lengths)))
        q.normal_()
        for t in new:
            t.normal_()
        for x, y in zip(captured, eager):
            y.copy_(x)
        graph.replay()
        inner.replay()
        torch.cuda.synchronize()
        want = step(eager, torch.empty_like(q))
        assert torch.equal(o, want) and torch.equal(o_inner, want)
        for x, y in zip(captured, eager):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        side.wait_stream(torch.cuda.current_stream())
        there = step(eager, torch.empty_like(q), stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(there, want)


def test_what_the_binding_refuses(m):
    K = torch.zeros((4, 16, 32), dtype=torch.int8, device=DEV)
    Ks = torch.ones((4, 2), device=DEV)
    table, lens, new, q = i32(np.zeros((1, 2))), i32(np.zeros(1)), torch.zeros((1, 1, 32), device=DEV), torch.zeros((1, 2, 32), device=DEV)
    out = lens.clone()
    m.mqa_paged_scaled_append_kv_rows(K, Ks, K.clone(), Ks.clone(), table, new, new, lens, out)
    for bad, error in ((dict(K=K.float()), TypeError), (dict(K=K.bfloat16()), TypeError), (dict(Ks=Ks[:, :0]), ValueError), (dict(Ks=torch.ones((4, 3), device=DEV)), ValueError),
                       (dict(Ks=Ks.double()), TypeError), (dict(Vs=torch.ones((4, 1), device=DEV)), ValueError), (dict(V=K.view(torch.float8_e4m3fn)), TypeError),
                       (dict(Ks=Ks.cpu()), ValueError), (dict(K=torch.zeros((4, 32, 16), dtype=torch.int8, device=DEV).transpose(1, 2)), ValueError)):
        c = {**dict(K=K, Ks=Ks, V=K.clone(), Vs=Ks.clone()), **bad}
        if "K" in bad and bad["K"].dtype != torch.int8:
            c["V"] = c["K"].clone()
        with pytest.raises(error):
            m.mqa_paged_scaled_append_kv_rows(*c.values(), table, new, new, lens, out)
        with pytest.raises(error):
            m.mqa_paged_scaled_decode_step(q, *c.values(), table, lens)
    with pytest.raises(m.MqaError) as e:                           # the lengths in place
        m.mqa_paged_scaled_append_kv_rows(K, Ks, K.clone(), Ks.clone(), table, new, new, lens, lens)
    assert e.value.status == 2
    with pytest.raises(ValueError):
        m.mqa_paged_scaled_decode_step(torch.zeros((1, 2, 48), device=DEV), K, Ks, K, Ks, table, lens)
