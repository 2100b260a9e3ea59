"""The operators of a serving loop together, as a program uses them: prompts into an 8-bit cache, forks that share their pages, drafted tokens, adjusted logits, verification,
what was refused given back, the pool compacted; every turn against the oracles, whose state is their own."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 2.0 ** -24


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.int32).to(DEV)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
@pytest.mark.parametrize("h_kv", [1, 2])
def test_serving_loop(kind, h_kv):
    import paper_1911_02150_amd as m
    from oracle import paged, serving
    rng = np.random.default_rng(17 + h_kv)
    page, block, each, pages, b, n, k, h, vocab = 16, 8, 12, 60, 6, 3, 64, 4, 200
    lead = (pages,) if h_kv == 1 else (pages, h_kv)
    types = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
    layers = []                                                            # two layers, one table
    for _ in range(2):
        layers.append([torch.zeros((*lead, page, k), dtype=types[kind], device=DEV), torch.ones((*lead, page // block), device=DEV),
                       torch.zeros((*lead, page, k), dtype=types[kind], device=DEV), torch.ones((*lead, page // block), device=DEV)])
    mirror = [[np.zeros((pages, h_kv, page, k)), np.ones((pages, h_kv, page // block)), np.zeros((pages, h_kv, page, k)), np.ones((pages, h_kv, page // block))] for _ in range(2)]
    pools = [t for layer in layers for t in layer]
    refs, table, lens = np.zeros(pages, dtype=np.int64), np.full((b, each), -1), np.zeros(b, dtype=np.int64)
    d_refs, d_table, d_lens, d_after = i32(refs), i32(table), i32(lens), i32(lens)
    history, held = np.zeros((b, each * page + 8), dtype=np.int64), np.zeros(b, dtype=np.int64)

    def append(count_of, rows):
        """Reserved, copied, appended in every layer; the same on the oracle's side."""
        nonlocal lens, d_lens, d_after
        granted, moves = m.mqa_paged_reserve_pages(d_table, d_lens, d_refs, page, rows, counts=i32(count_of))
        m.mqa_paged_copy_pages(pools, moves)
        g, mv = serving.reserve(table, lens, refs, page, rows, count_of)
        assert np.array_equal(granted.cpu().numpy(), g) and np.array_equal(moves.cpu().numpy(), mv)
        for layer, shadow in zip(layers, mirror):
            new = [rng.standard_normal((b, rows, h_kv, k)).astype(np.float32) for _ in range(2)]
            for x in shadow:
                serving.copy(x, mv)
            after = serving.append(*shadow, table, *new, lens, g, kind)
            on = [torch.from_numpy(x[:, :, 0] if h_kv == 1 else x).contiguous().to(DEV) for x in new]
            m.mqa_paged_scaled_append_kv_rows(*layer, d_table, *on, d_lens, d_after, counts=granted)
        d_lens, d_after = d_after, d_lens
        lens = after
        return g

    append(np.array([70, 33, 16, 0, 1, 100]), 100)                        # prompts
    for turn in range(6):
        g = append(np.where(lens > 0, n + 1, 0), n + 1)
        assert np.array_equal(d_lens.cpu().numpy(), lens) and np.array_equal(d_table.cpu().numpy(), table) and np.array_equal(d_refs.cpu().numpy(), refs)
        q = rng.standard_normal((b, n + 1, h, k)).astype(np.float32)
        for layer, shadow in zip(layers, mirror):
            for t, x in zip(layer, shadow):
                assert np.array_equal(t.float().cpu().double().numpy().reshape(x.shape), x)
            o = m.mqa_paged_scaled_decode_step(torch.from_numpy(q).to(DEV), *layer, d_table, d_lens, scale=0.2)
            K, V = serving.whole(*shadow[:2]), serving.whole(*shadow[2:])
            want, _, size = paged.attend(q.astype(np.float64), K, V, table, lens, float(np.float32(0.2)))
            logit = 0.2 * np.abs(q).max() * np.abs(K).max() * k ** 0.5 * 4
            assert (np.abs(o.cpu().numpy() - want) <= EPS * (31 * logit + 17 + 8 * 200 ** 0.5) * size + 1e-30).all()
        logits = rng.standard_normal((b, n + 1, vocab)).astype(np.float32)
        drafts = rng.integers(0, vocab, (b, n))
        for i in range(b):                                                 # (some drafts are likely ones)
            if turn % 2 and i % 2:
                logits[i, np.arange(n), drafts[i]] += 12
        factor = np.full(b, 1.25, dtype=np.float32)
        adjusted = m.mqa_stack_adjust_logits(torch.from_numpy(logits).to(DEV), i32(history), i32(held), drafts=i32(drafts), repetition=torch.from_numpy(factor).to(DEV),
                                             presence=torch.from_numpy(factor).to(DEV))
        want = serving.adjust(logits, history, held, drafts=drafts, repetition=factor, presence=factor)
        assert np.abs(adjusted.cpu().numpy() - want).max() <= EPS * 6 * 1.25 * (np.abs(logits).max() + 1.25)
        tokens, accepted = m.mqa_stack_verify_drafts(adjusted, i32(drafts), None, counts=i32(np.maximum(g - 1, 0)), temperature=0.0)
        w_tokens, w_accepted = paged.verify(adjusted.cpu().numpy().astype(np.float64), drafts, np.zeros((b, n + 1)), counts=np.maximum(g - 1, 0), temperature=0)
        assert np.array_equal(tokens.cpu().numpy(), w_tokens) and np.array_equal(accepted.cpu().numpy(), w_accepted)
        stand = np.where(g > 0, w_accepted + 1, 0)
        for i in range(b):
            history[i, held[i]:held[i] + stand[i]] = w_tokens[i, :stand[i]]
        held += stand
        lens = lens - g + stand
        d_lens.copy_(i32(lens))
        if turn == 2:
            lens[1] = 0                                                    # one ends
            d_lens.copy_(i32(lens))
        m.mqa_paged_free_pages(d_table, d_lens, d_refs, page)
        serving.free(table, lens, refs, page)
        if turn in (1, 4):                                                 # the best ones go on several times, the pool is made compact
            parents = np.array([0, 0, 2, 5, 5, 1])
            d_new, d_new_lens = torch.empty_like(d_table), torch.empty_like(d_lens)
            m.mqa_paged_fork_pages(d_table, d_lens, i32(parents), d_new, d_new_lens, d_refs, page)
            m.mqa_paged_free_pages(d_table, torch.zeros_like(d_lens), d_refs, page)
            new, new_lens = serving.fork(table, lens, parents, refs, page)
            serving.free(table, np.zeros(b, dtype=np.int64), refs, page)
            d_refs_out, moves = torch.empty_like(d_refs), torch.empty((pages // 2, 2), dtype=torch.int32, device=DEV)
            used = torch.empty(1, dtype=torch.int32, device=DEV)
            m.mqa_paged_compact_pages(d_new, d_refs, d_table, d_refs_out, moves, used)
            m.mqa_paged_copy_pages(pools, moves)
            d_refs, d_lens = d_refs_out, d_new_lens
            table, refs, mv, _ = serving.compact(new, refs)
            lens = new_lens
            for shadow in mirror:
                for x in shadow:
                    serving.copy(x, mv)
            history, held = history[parents], held[parents]
        assert np.array_equal(d_table.cpu().numpy(), table) and np.array_equal(d_refs.cpu().numpy(), refs) and np.array_equal(d_lens.cpu().numpy(), lens)
