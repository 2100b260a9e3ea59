"""Verification of drafted tokens on the GPU against the float64 oracle: whole numbers, equal."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def m():
    import paper_1911_02150_amd as mod
    mod.load_library()
    return mod


def gpu(x):
    if x is None:
        return None
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t.to(torch.int32) if t.dtype == torch.int64 else t.float()).to(DEV)


def check(m, logits, drafts, u, draft_logits=None, counts=None, temperature=1.0):
    from oracle import paged
    want = paged.verify(logits, drafts, u, draft_logits, counts, temperature)
    args = [gpu(x) for x in (logits, drafts, u)]
    kw = dict(draft_logits=gpu(draft_logits), counts=gpu(counts), temperature=temperature)
    for _ in range(2):
        tokens, accepted = m.mqa_stack_verify_drafts(*args, **kw)
        assert accepted.tolist() == want[1].tolist()
        assert tokens.tolist() == want[0].tolist()
    return want


@pytest.mark.parametrize("temperature", [1.0, 0.7, 0.0])
@pytest.mark.parametrize("draft", ["logits", "none"])
@pytest.mark.parametrize("b,n,vocab", [(1, 1, 1), (2, 3, 2), (7, 4, 100), (3, 5, 4095), (4, 2, 4096), (4, 2, 4097), (8, 4, 32768), (2, 7, 50001), (300, 1, 33), (1, 300, 20),
                                       (3, 40, 60), (130, 2, 1999), (5, 8, 512), (3, 2, 16384), (2, 3, 9001), (1, 2, 16385)])
def test_random(m, b, n, vocab, draft, temperature):
    rng = np.random.default_rng(b + n + vocab)
    logits = (3 * rng.standard_normal((b, n + 1, vocab))).astype(np.float32)
    draft_logits = (logits[:, :n] + 0.5 * rng.standard_normal((b, n, vocab))).astype(np.float32)
    drafts = (draft_logits / (temperature or 0.2) + rng.gumbel(size=draft_logits.shape)).argmax(-1)
    if vocab > 20:
        drafts[rng.random(drafts.shape) < 0.05] = vocab                      # no token
        drafts[rng.random(drafts.shape) < 0.05] = -1
    counts = rng.integers(-1, n + 2, b)
    u = rng.random((b, n + 1), dtype=np.float32)
    for c in (None, counts):
        check(m, logits, drafts, u, draft_logits if draft == "logits" else None, c, temperature)


@pytest.mark.parametrize("vocab", [64, 3000, 5000, 20000])
def test_masked_logits(m, vocab):
    """-infinity for most tokens, whole rows of it, NaN, +infinity; the largest and the smallest random numbers."""
    rng = np.random.default_rng(vocab)
    b, n = 12, 3
    logits = rng.standard_normal((b, n + 1, vocab)).astype(np.float32)
    draft_logits = rng.standard_normal((b, n, vocab)).astype(np.float32)
    logits[:, :, rng.random(vocab) < 0.8] = -np.inf
    logits[0] = -np.inf
    logits[1, 1] = np.nan
    logits[2, 0, 5:] = np.nan
    logits[3, :, 7] = logits[3, :, 11] = np.inf
    logits[4] = np.finfo(np.float32).min                                     # (a mask of the type's lowest value on everything: an even choice)
    logits[5, :, 1:] = np.finfo(np.float32).min
    draft_logits[6] = -np.inf
    draft_logits[7, :, ::2] = np.nan
    draft_logits[8], logits[8, :n] = 0, 0
    drafts = draft_logits[:, :, : min(vocab, 60)].argmax(-1)
    u = rng.random((b, n + 1), dtype=np.float32)
    u[9], u[10] = 0, 1 - 2.0 ** -24
    u[11, n] = 1                                                             # (out of range: the last token that there is)
    for t in (1.0, 0.0, 1e-6, 1e6):
        check(m, logits, drafts, u, draft_logits, None, t)
        check(m, logits, drafts, u, None, None, t)


def test_equal_distributions_stand(m):
    """q = p: every draft stands, whatever u below 1."""
    rng = np.random.default_rng(1)
    logits = rng.standard_normal((4, 6, 1000)).astype(np.float32)
    u = np.full((4, 6), 1 - 2.0 ** -24, dtype=np.float32)
    _, accepted = check(m, logits, rng.integers(0, 1000, (4, 5)), u, logits[:, :5])
    assert (accepted == 5).all()


def test_no_drafts_is_sampling(m):
    """n = 0: a token drawn from each row; over many rows, the distribution."""
    rng = np.random.default_rng(2)
    p = np.array([0.4, 0.0, 0.3, 0.2, 0.1])
    b = 20000
    with np.errstate(divide="ignore"):
        logits = np.broadcast_to(np.log(p), (b, 1, 5)).astype(np.float32)
    u = rng.random((b, 1), dtype=np.float32)
    tokens, accepted = m.mqa_stack_verify_drafts(gpu(logits), None, gpu(u))
    assert not accepted.any() and tokens.shape == (b, 1)
    got = np.bincount(tokens.cpu().numpy().ravel(), minlength=5) / b
    assert np.abs(got - p).max() < 5 * np.sqrt(0.25 / b)                     # five standard deviations
    check(m, logits[:50], np.zeros((50, 0), dtype=np.int64), u[:50])
    check(m, logits[:50], np.zeros((50, 0), dtype=np.int64), u[:50], temperature=0.0)


def test_greedy_is_argmax(m):
    g = torch.Generator(device=DEV).manual_seed(4)
    logits = torch.randn((5, 4, 999), generator=g, device=DEV)
    best = m.mqa_stack_argmax(logits.view(20, 999)).view(5, 4)
    drafts = best[:, :3].clone()
    drafts[1, 2] += 1
    drafts[2, 0] -= 1
    tokens, accepted = m.mqa_stack_verify_drafts(logits, drafts, None, temperature=0.0)
    assert accepted.tolist() == [3, 2, 0, 3, 3]
    for i, a in enumerate(accepted.tolist()):
        assert tokens[i].tolist() == best[i, :a + 1].tolist() + [-1] * (3 - a)


def test_replayed_and_on_a_stream(m):
    g = torch.Generator(device=DEV).manual_seed(5)
    b, n, vocab = 6, 3, 9000
    logits, draft_logits = (3 * torch.randn((b, x, vocab), generator=g, device=DEV) for x in (n + 1, n))
    drafts, u = torch.randint(0, vocab, (b, n), generator=g, device=DEV, dtype=torch.int32), torch.rand((b, n + 1), generator=g, device=DEV)
    drafts[:3] = logits[:3, :n].argmax(-1).int()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    out = torch.zeros((b, n + 1), dtype=torch.int32, device=DEV), torch.zeros(b, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        m.mqa_stack_verify_drafts(logits, drafts, u, draft_logits=draft_logits, tokens=out[0], accepted=out[1])
    for r in range(4):
        u.copy_(torch.rand((b, n + 1), generator=g, device=DEV))
        logits.add_(0.3 * torch.randn((b, n + 1, vocab), generator=g, device=DEV))
        want = m.mqa_stack_verify_drafts(logits, drafts, u, draft_logits=draft_logits)
        torch.cuda.synchronize()
        side = m.mqa_stack_verify_drafts(logits, drafts, u, draft_logits=draft_logits, stream=stream)
        stream.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x in range(2):
            assert torch.equal(out[x], want[x]) and torch.equal(side[x], want[x])


def test_more_than_2_to_31_logits(m):
    """The last rows against a call of their own."""
    b, vocab = 33000, 65536
    g = torch.Generator(device=DEV).manual_seed(6)
    logits, u = torch.empty((b, 1, vocab), device=DEV).normal_(generator=g), torch.rand((b, 1), generator=g, device=DEV)
    tokens, accepted = m.mqa_stack_verify_drafts(logits, None, u)
    some, _ = m.mqa_stack_verify_drafts(logits[-64:].contiguous(), None, u[-64:].contiguous())
    assert torch.equal(tokens[-64:], some) and len(set(tokens[:, 0].tolist())) > 1000 and not accepted.any()


def test_wrong_tensors_are_refused(m):
    logits, drafts, u = torch.zeros((2, 4, 10), device=DEV), torch.zeros((2, 3), dtype=torch.int32, device=DEV), torch.zeros((2, 4), device=DEV)
    for bad in (dict(drafts=drafts[:, :2].contiguous()), dict(u=u[:1]), dict(logits=logits[0]), dict(draft_logits=logits), dict(counts=drafts), dict(tokens=drafts),
                dict(accepted=drafts), dict(u=u.cpu()), dict(logits=logits.transpose(1, 2))):
        with pytest.raises(ValueError):
            m.mqa_stack_verify_drafts(**{**dict(logits=logits, drafts=drafts, u=u), **bad})
    for bad in (dict(drafts=drafts.long()), dict(u=u.double()), dict(logits=logits.bfloat16())):
        with pytest.raises(TypeError):
            m.mqa_stack_verify_drafts(**{**dict(logits=logits, drafts=drafts, u=u), **bad})
    for bad in (dict(temperature=-1.0), dict(temperature=float("nan")), dict(u=None), dict(drafts=None)):
        with pytest.raises(m.MqaError):
            m.mqa_stack_verify_drafts(**{**dict(logits=logits, drafts=drafts, u=u), **bad})


def test_probabilities_are_float64(m):
    """Two borders 4e-15 to 1e-13 of the whole away from the goal, which a 2^x of 43 bits puts on the other side of it: three tokens of weights 1, e^-d and e^-d', where
    1 / u is next to their sum.  (Float64's own errors: u * (1 + w + w'), 3e-16 of the whole.)"""
    rng = np.random.default_rng(0)
    d = rng.uniform(0.34, 0.3465, 2_000_000).astype(np.float32)                # (exponents of nearly -1/2, where a series around 0 is least accurate)
    u = rng.uniform(0.4125, 0.4135, len(d)).astype(np.float32)
    w = np.exp(-d.astype(np.float64))
    other = (-np.log(1 / u.astype(np.float64) - 1 - w)).astype(np.float32)
    left = 1 - u.astype(np.float64) * (1 + w + np.exp(-other.astype(np.float64)))
    near = (np.abs(left) < 1e-13) & (np.abs(left) > 4e-15) & (other < 0.3465)
    d, u, other, first = d[near], u[near], other[near], left[near] > 0
    assert len(d) > 30 and 0 < first.sum() < len(d)
    rows = np.stack([np.zeros_like(d), -d, -other], axis=1)
    for vocab in (3, 5000, 20000):                                             # (one launch, two, three)
        logits = np.full((len(d), 1, vocab), -np.inf, dtype=np.float32)
        logits[:, 0, :3] = rows
        tokens, _ = m.mqa_stack_verify_drafts(gpu(logits), None, gpu(u[:, None]))
        assert ((tokens[:, 0].cpu().numpy() == 0) == first).all()


@pytest.mark.parametrize("vocab", [2, 300, 9000])
def test_greedy_is_argmax_of_odd_rows_too(m, vocab):
    """NaN next to -infinity, the largest number next to +infinity, rows of nothing but NaN or -infinity."""
    top = np.finfo(np.float32).max
    pairs = [(np.nan, -np.inf), (-np.inf, np.nan), (top, np.inf), (np.inf, top), (np.nan, np.nan), (-np.inf, -np.inf), (np.nan, -3.0), (np.inf, np.inf), (np.nan, np.inf),
             (-top, -np.inf)]
    rows = np.full((2 * len(pairs), vocab), np.nan, dtype=np.float32)
    rows[: len(pairs), :2] = pairs                                             # at the row's beginning, the rest of it NaN ...
    rows[len(pairs):, vocab - 2:] = pairs                                      # ... and at its end
    logits = gpu(rows).view(-1, 1, vocab).repeat(1, 3, 1)
    best = m.mqa_stack_argmax(logits[:, 0].contiguous())
    drafts = torch.stack([best, (best + 1) % vocab], dim=1)
    tokens, accepted = m.mqa_stack_verify_drafts(logits, drafts, None, temperature=0.0)
    assert accepted.tolist() == [1] * len(rows)
    assert torch.equal(tokens, torch.stack([best, best, torch.full_like(best, -1)], dim=1))
    check(m, logits.cpu().numpy(), drafts.long().cpu().numpy(), None, temperature=0.0)
