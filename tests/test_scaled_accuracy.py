"""Attention over pages of 8 bits has the accuracy of two fp16 terms of the queries and of the weights: the root mean square of its errors against float64 is what the form's roundings
make of these inputs, so that a term that were left out or misplaced would show (on the CPU: such a form is told from the right one by the same bound)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_paged_accuracy import DEV, HALF, groups  # noqa: E402

# b, n, h, h_kv, k, v, page, block, kind, V's scales are powers of two, scale * k ** 0.5, lengths: 16 and 32 rows a workgroup, one block of rows and several, one launch and two, each width's
# form; small logits where the weights' terms are to show, larger ones for the queries'
CASES = [
    (2, 1, 8, 1, 128, 128, 16, 16, "e4m3", True, 2.0, [64, 90]),
    (2, 1, 16, 1, 128, 128, 16, 16, "int8", False, 0.1, [40, 64]),
    (4, 2, 20, 1, 128, 128, 16, 8, "int8", False, 2.0, [64, 1700, 100, 33]),
    (3, 1, 40, 1, 128, 128, 7, 7, "e4m3", False, 0.1, [64, 50, 40]),
    (2, 1, 16, 2, 64, 64, 16, 1, "e4m3", True, 2.0, [64, 1000]),
    (2, 1, 8, 1, 64, 64, 16, 16, "int8", True, 0.1, [64, 64]),
    (2, 3, 10, 1, 48, 32, 16, 4, "e4m3", False, 2.0, [64, 80]),
    (2, 3, 10, 1, 48, 64, 16, 4, "int8", False, 0.1, [64, 60]),
    (2, 1, 33, 1, 96, 112, 16, 16, "int8", True, 2.0, [64, 1600]),
    (2, 1, 33, 1, 96, 112, 16, 16, "e4m3", False, 0.1, [64, 60]),
    (2, 1, 12, 1, 208, 256, 16, 16, "e4m3", False, 2.0, [64, 40]),
    (2, 1, 40, 1, 256, 240, 16, 16, "int8", False, 0.1, [64, 40]),
    (300, 1, 20, 1, 128, 128, 16, 16, "e4m3", False, 2.0, [30 + x % 40 for x in range(300)]),
    (300, 1, 20, 1, 128, 128, 16, 16, "int8", False, 0.1, [30 + x % 40 for x in range(300)]),
    (300, 1, 20, 1, 64, 64, 16, 16, "e4m3", False, 0.1, [30 + x % 40 for x in range(300)]),
    (200, 1, 34, 1, 80, 80, 16, 16, "int8", False, 0.1, [30 + x % 40 for x in range(200)]),
    (150, 1, 34, 1, 160, 160, 16, 16, "e4m3", False, 0.1, [30 + x % 40 for x in range(150)]),
]


def inputs(b, n, h, h_kv, k, v, page, block, kind, powers, spread, lens):
    """q, (bits' values, scales) of K and of V, table, lengths, scale.  The scales are within 2^-16 .. 2^16, K's powers of two."""
    from oracle import serving
    rng = np.random.default_rng(b + 3 * n + 5 * h + 7 * k + v + len(kind) + int(10 * spread))
    each = -(-max(lens) // page)
    pages = min(b * each, 200)
    pools = []
    for w, exact in ((k, True), (v, powers)):
        scales = np.exp(0.7 * rng.standard_normal((pages, h_kv, page // block))) * 2.0 ** -5
        scales = 2.0 ** np.round(np.log2(scales)) if exact else scales.astype(np.float32).astype(np.float64)
        pools.append((serving.rounded(32 * rng.standard_normal((pages, h_kv, page, w)), kind), scales))
    table = rng.permutation(b * each).reshape(b, each) % pages
    return rng.standard_normal((b, n, h, k)).astype(np.float32), *pools, table, np.array(lens), float(np.float32(spread / k ** 0.5))


def with_scales(pool, page):
    """A pool's values with their scale as a last column, so that `groups` takes both along."""
    values, scales = pool
    return np.concatenate([values, np.repeat(scales, page // scales.shape[2], axis=2)[..., None]], -1)


def expected(q, K, V, table, lens, scale, n, h, h_kv):
    """Outputs in float64 and the root mean square of the form's errors in them.  Every rounding is off by half a step (at its largest; they do not know of one another).  Of a logit: q * scale,
    q's two terms (two half steps) and 2 k additions to sums of up to the root of the products' squares; scale in the logarithm's base twice, by the logit itself.  Of a weight's exponent: the
    logit with log2 of V's scale (within 16) added, and the difference from the running maximum, which is up to 14 below the largest.  The exponential, a step; the scale's mantissa; the
    weight's two terms, two half steps and 2^-35 of the row's largest weight times scale.  Of an output: 2 L additions of products; the sum of the weights, L additions; its inverse and
    two products."""
    o, off = np.zeros((*q.shape[:3], V[0].shape[-1])), 0.0
    page = K[0].shape[2]
    for qs, Ks, Vs, seen, at, _ in groups(q, with_scales(K, page), with_scales(V, page), table, lens, n, h, h_kv):
        k, L, s = Ks.shape[1] - 1, len(Ks), Vs[:, -1]
        Ks, Vs = Ks[:, :-1] * Ks[:, -1:], Vs[:, :-1] * s[:, None]
        z = np.where(seen, scale * (qs @ Ks.T), -np.inf)
        size = scale ** 2 * ((qs ** 2) @ (Ks.T ** 2))
        w = np.exp(z - z.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        z = np.where(seen, z, 0)
        here = w @ Vs
        ln2, e = np.log(2), np.abs(np.floor(np.log2(s)))
        u = z / ln2 + np.floor(np.log2(s))
        below = np.abs(u - np.where(seen, u, -np.inf).max(-1, keepdims=True)) + 14
        relative = HALF ** 2 * ((2 * k + 1 + 4) * size + 4 * z ** 2 + ln2 ** 2 * ((np.abs(z) / ln2 + e) ** 2 + below ** 2) + 4)      # a weight's
        terms = HALF ** 2 * (4 + 1) * w ** 2 + (2.0 ** -35 * (w * s).max(-1, keepdims=True) / s) ** 2                                 # and what multiplies V of it
        whole = HALF ** 2 * (L + 4)                                                                                                  # a row's
        per = w ** 2 * relative
        spread = per @ (Vs ** 2) - 2 * (per @ Vs) * here + per.sum(-1, keepdims=True) * here ** 2                                    # sum per (V - o)^2
        off += (spread + np.where(seen, terms, 0) @ (Vs ** 2) + HALF ** 2 * (2 * L + 2) * ((w ** 2) @ (Vs ** 2)) + whole * here ** 2).sum()
        o[at] = here
    return o, (off / o.size) ** 0.5


def halves(x, count):
    """x as so many fp16 terms, each in float32."""
    got, x = [], np.asarray(x, dtype=np.float32)
    for _ in range(count):
        got.append(x.astype(np.float16).astype(np.float32))
        x = x - got[-1]
    return got


def model(q, K, V, table, lens, scale, n, h, h_kv, of_q, of_weights):
    """The form with so many terms, its sums in float32."""
    f, page = np.float32, K[0].shape[2]
    o = np.zeros((*q.shape[:3], V[0].shape[-1]))

    def add(products):                                      # [..., terms' values], one after the other
        return np.cumsum(products, axis=-1, dtype=f)[..., -1]
    for qs, Ks, Vs, seen, at, _ in groups(q, with_scales(K, page), with_scales(V, page), table, lens, n, h, h_kv):
        qs = qs.astype(f) * (f(scale) * f(np.log2(np.e)))
        up = int(np.frexp(np.abs(qs).max())[1]) - 14        # the largest: 2^13 .. 2^14
        t = halves(np.ldexp(qs, -up), of_q)
        sc = add(np.concatenate([x[..., None, :] * Ks[:, :-1].astype(f) for x in t], -1))
        mant, e = np.frexp(Vs[:, -1])
        mant, e = f(2 * mant), f(e - 1)
        u = np.where(seen, f(sc.astype(np.float64) * np.ldexp(Ks[:, -1], up) + e), f(-np.inf))
        w = np.exp2(u - (u.max(-1, keepdims=True) - f(10)))
        total = add(w * np.exp2(-e))
        t = halves(w * mant, of_weights)
        o[at] = add(np.concatenate([np.swapaxes(x[..., None] * Vs[:, :-1].astype(f), -1, -2) for x in t], -1)) / total[..., None]
    return o


@pytest.mark.parametrize("case", [c for c in CASES if c[0] < 100 and max(c[-1]) <= 100], ids=str)
def test_the_bound_tells_two_terms_from_one(case):
    b, n, h, h_kv, k, v, page, block, kind, powers, spread, lens = case
    args = (*inputs(*case), n, h, h_kv)
    want, off = expected(*args)
    rms = lambda of_q, of_weights: ((model(*args, of_q, of_weights) - want) ** 2).mean() ** 0.5  # noqa: E731
    assert rms(2, 2) <= off
    if spread >= 1:
        assert rms(1, 2) > 1.5 * off
    assert rms(2, 1) > 1.5 * off


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:11])))
def test_attention_has_two_terms_accuracy(case):
    import paper_1911_02150_amd as m
    b, n, h, h_kv, k, v, page, block, kind, powers, spread, lens = case
    q, K, V, table, lens, scale = inputs(*case)
    want, off = expected(q, K, V, table, lens, scale, n, h, h_kv)
    one = lambda x: np.ascontiguousarray(x[:, 0] if h_kv == 1 else x)  # noqa: E731
    cache = []
    for values, scales in (K, V):
        cache += [torch.from_numpy(one(values)).float().to(torch.float8_e4m3fn if kind == "e4m3" else torch.int8).to(DEV), torch.from_numpy(one(scales)).float().to(DEV)]
    got = m.mqa_paged_scaled_decode_step(torch.from_numpy(q).to(DEV), *cache, *(torch.from_numpy(x.astype(np.int32)).to(DEV) for x in (table, lens)), scale=scale)
    rms = ((got.cpu().numpy() - want) ** 2).mean() ** 0.5
    print(f"rms {rms:.2e}, expected at most {off:.2e}")
    assert rms <= off
