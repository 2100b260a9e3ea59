"""Attention over pages has float32's accuracy: the root mean square of its errors against float64 is what float32's roundings make of these inputs, so that a bfloat16 term of
the queries or of the weights that were left out or misplaced would show (on the CPU: such a form is told from the right one by the same bound)."""
import numpy as np
import pytest

import mqa_inputs as mi

torch = pytest.importorskip("torch")
DEV = "cuda:0"
HALF = 2.0 ** -24          # half a step of float32

# b, n, h, h_kv, k, v, page, dtype, scale * k ** 0.5, lengths: 16 and 32 rows a workgroup, one block of rows and several, one launch and two, each width's form; small logits
# where the weights' terms are to show, larger ones for the queries'
CASES = [
    (2, 1, 8, 1, 128, 128, 16, "bf16", 2.0, [64, 90]),
    (2, 1, 16, 1, 128, 128, 16, "bf16", 0.1, [40, 64]),
    (4, 2, 20, 1, 128, 128, 16, "bf16", 2.0, [64, 700, 100, 33]),
    (3, 1, 40, 1, 128, 128, 7, "bf16", 0.1, [64, 50, 40]),
    (2, 1, 16, 2, 64, 64, 16, "bf16", 2.0, [64, 1000]),
    (2, 1, 8, 1, 64, 64, 16, "bf16", 0.1, [64, 64]),
    (2, 3, 10, 1, 40, 24, 16, "bf16", 2.0, [64, 80]),
    (2, 3, 10, 1, 40, 56, 16, "bf16", 0.1, [64, 60]),
    (2, 1, 33, 1, 96, 104, 16, "bf16", 2.0, [64, 600]),
    (2, 1, 33, 1, 96, 104, 16, "bf16", 0.1, [64, 60]),
    (2, 1, 12, 1, 200, 256, 16, "bf16", 2.0, [64, 40]),
    (2, 1, 40, 1, 256, 248, 16, "bf16", 0.1, [64, 40]),
    (300, 1, 20, 1, 128, 128, 16, "bf16", 2.0, [30 + x % 40 for x in range(300)]),
    (300, 1, 20, 1, 128, 128, 16, "bf16", 0.1, [30 + x % 40 for x in range(300)]),
    (300, 1, 20, 1, 64, 64, 16, "bf16", 0.1, [30 + x % 40 for x in range(300)]),
    (200, 1, 34, 1, 72, 72, 16, "bf16", 0.1, [30 + x % 40 for x in range(200)]),
    (150, 1, 34, 1, 160, 160, 16, "bf16", 0.1, [30 + x % 40 for x in range(150)]),
    (3, 1, 8, 1, 128, 128, 16, "f32", 2.0, [64, 700, 33]),
    (3, 2, 12, 3, 64, 64, 16, "f32", 2.0, [64, 700, 33]),
    (3, 1, 20, 1, 200, 96, 16, "f32", 0.1, [64, 60, 33]),
]


def inputs(b, n, h, h_kv, k, v, page, dtype, spread, lens):
    rng = np.random.default_rng(b + 3 * n + 5 * h + 7 * k + v + len(dtype) + int(10 * spread))
    each = -(-max(lens) // page)
    pages = min(b * each, 200)
    as_held = (lambda x: mi.bf16_bits_to_f64(mi.f32_to_bf16_bits(x))) if dtype == "bf16" else (lambda x: x.astype(np.float64))
    K, V = (as_held(rng.standard_normal((pages, h_kv, page, w)).astype(np.float32)) for w in (k, v))
    table = rng.permutation(b * each).reshape(b, each) % pages
    return rng.standard_normal((b, n, h, k)).astype(np.float32), K, V, table, np.array(lens), float(np.float32(spread / k ** 0.5))


def groups(q, K, V, table, lens, n, h, h_kv):
    """Of every sequence and K/V head: q's rows [n, h / h_kv, k] in float64, K and V rows, [rows, positions] what is seen, and where its outputs are."""
    for i in range(len(lens)):
        for e in range(h_kv):
            rows = [x[table[i], e].reshape(-1, x.shape[-1])[:lens[i]] for x in (K, V)]
            heads = slice(e * (h // h_kv), (e + 1) * (h // h_kv))
            seen = np.arange(lens[i]) < lens[i] - (n - 1 - np.arange(n))[:, None, None]
            yield q[i, :, heads].astype(np.float64), *rows, np.broadcast_to(seen, (n, h // h_kv, lens[i])), (i, slice(None), heads), (i, e)


def expected(q, K, V, table, lens, scale, n, h, h_kv):
    """Outputs and weights' sums in float64 and the mean squares of a float32 form's errors in them.  Every rounding is off by half a step (at its largest; they do not know of
    one another).  Of a logit: q * scale and k additions to sums of up to the root of the products' squares; scale in the logarithm's base twice, and the exponent's
    difference, which go by the logit itself; the exponential, a step.  Of an output: the weights and their products, L additions likewise; the sum of the weights, L additions,
    its inverse and two products."""
    o, o_off = np.zeros((*q.shape[:3], V.shape[-1])), 0.0
    scores, scores_off = np.zeros((len(lens), h_kv, table.shape[1] * K.shape[2])), 0.0
    for qs, Ks, Vs, seen, at, head in groups(q, K, V, table, lens, n, h, h_kv):
        k, L = Ks.shape[1], len(Ks)
        z = np.where(seen, scale * (qs @ Ks.T), -np.inf)
        size = scale ** 2 * ((qs ** 2) @ (Ks.T ** 2))
        w = np.exp(z - z.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        z = np.where(seen, z, 0)
        here = w @ Vs
        relative = HALF ** 2 * ((k + 1) * size + 4 * z ** 2 + (z - z.max(-1, keepdims=True)) ** 2 + 4)      # a weight's
        whole = HALF ** 2 * (L + 4)                                                                          # a row's
        per = w ** 2 * relative
        spread = per @ (Vs ** 2) - 2 * (per @ Vs) * here + per.sum(-1, keepdims=True) * here ** 2             # sum per (V - o)^2
        o_off += (spread + HALF ** 2 * (L + 2) * ((w ** 2) @ (Vs ** 2)) + whole * here ** 2).sum()
        o[at] = here
        scores[head][:L] = w.sum((0, 1))
        scores_off += (w ** 2 * (relative + whole)).sum() + HALF ** 2 * (seen.shape[0] * seen.shape[1] + 2) * (w.sum((0, 1)) ** 2).sum()
    return o, (o_off / o.size) ** 0.5, scores, (scores_off / sum(lens) / h_kv) ** 0.5


def terms(x, count):
    """x as the sum of so many bfloat16 terms, in float64."""
    x, got = np.asarray(x, dtype=np.float32), np.zeros(x.shape)
    for _ in range(count):
        t = mi.bf16_bits_to_f64(mi.f32_to_bf16_bits(x))
        got, x = got + t, (x - t).astype(np.float32)
    return got


def model(q, K, V, table, lens, scale, n, h, h_kv, of_q, of_weights):
    """The form with so many terms, its sums in float32."""
    o = np.zeros((*q.shape[:3], V.shape[-1]))
    f = np.float32
    for qs, Ks, Vs, seen, at, _ in groups(q, K, V, table, lens, n, h, h_kv):
        log2e = f(scale) * f(np.log2(np.e))
        qs = terms(qs.astype(f) * log2e, of_q).astype(f)
        z = np.where(seen, np.cumsum(qs[..., None, :] * Ks.astype(f), axis=-1, dtype=f)[..., -1], f(-np.inf))
        w = np.exp2(z - z.max(-1, keepdims=True))
        total = np.cumsum(w, axis=-1, dtype=f)[..., -1:]
        o[at] = np.cumsum(terms(w, of_weights).astype(f)[..., None] * Vs.astype(f), axis=-2, dtype=f)[..., -1, :] / total
    return o


@pytest.mark.parametrize("case", [c for c in CASES if c[0] < 100 and max(c[-1]) <= 100], ids=str)
def test_the_bound_tells_float32_from_fewer_terms(case):
    b, n, h, h_kv, k, v, page, dtype, spread, lens = case
    args = (*inputs(*case), n, h, h_kv)
    want, off, _, _ = expected(*args)
    rms = lambda of_q, of_weights: ((model(*args, of_q, of_weights) - want) ** 2).mean() ** 0.5  # noqa: E731
    assert rms(3, 3) <= off
    if spread >= 1:
        assert rms(2, 3) > 1.5 * off
    else:
        assert rms(3, 2) > 1.5 * off


@pytest.mark.gpu
@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:9])))
def test_attention_has_float32s_accuracy(case, scored):
    import paper_1911_02150_amd as m
    b, n, h, h_kv, k, v, page, dtype, spread, lens = case
    q, K, V, table, lens, scale = inputs(*case)
    want, off, sums, sums_off = expected(q, K, V, table, lens, scale, n, h, h_kv)
    pools = [torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32) for x in (K, V)]
    pools = [(x[:, 0] if h_kv == 1 else x).contiguous().to(DEV) for x in pools]
    scores = torch.zeros((b, table.shape[1] * page) if h_kv == 1 else (b, h_kv, table.shape[1] * page), device=DEV) if scored else None
    got = m.mqa_paged_decode_step(torch.from_numpy(q).to(DEV), *pools, *(torch.from_numpy(x.astype(np.int32)).to(DEV) for x in (table, lens)), scale=scale, scores=scores)
    rms = ((got.cpu().numpy() - want) ** 2).mean() ** 0.5
    print(f"rms {rms:.2e}, expected at most {off:.2e}")
    assert rms <= off
    if scored:
        rms = (((scores.cpu().numpy().reshape(sums.shape) - sums) ** 2).sum() / lens.sum() / h_kv) ** 0.5
        print(f"scores: rms {rms:.2e}, expected at most {sums_off:.2e}")
        assert rms <= sums_off
