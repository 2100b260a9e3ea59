"""Who holds which page of a pool, on the GPU against the oracle (oracle/serving.py): whole numbers, equal."""
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


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.int32).to(DEV)


def same(tensor, array):
    return np.array_equal(tensor.cpu().numpy(), array)


def counted(tables, num_pages):
    refs = np.zeros(num_pages, dtype=np.int64)
    for t in tables:
        refs += np.bincount(t[(t >= 0) & (t < num_pages)], minlength=num_pages)
    return refs


def some_tables(rng, b, each, num_pages, page, share=0.3):
    """Tables and lengths of sequences that hold the pages of their positions, some of them shared."""
    lens = rng.integers(0, each * page + 1, b)
    free = list(rng.permutation(num_pages))
    table = np.full((b, each), -1)
    for i in range(b):
        for x in range(-(-int(lens[i]) // page)):
            before = [y for y in range(i) if table[y, x] >= 0]
            if before and rng.random() < share:
                table[i, x] = table[rng.choice(before), x]
            elif free:
                table[i, x] = free.pop()
    return table, lens


# b, pages of a sequence, pool, page size, n
SIZES = [(1, 1, 1, 1, 1), (1, 4, 3, 16, 1), (5, 6, 40, 4, 5), (8, 10, 25, 16, 40), (64, 20, 900, 16, 1), (300, 7, 1500, 3, 9), (1500, 5, 5000, 8, 1), (3000, 3, 4000, 2, 4),
         (8, 40, 200, 2, 30), (1024, 4, 20000, 16, 33), (40, 9, 30000, 5, 16), (40, 200, 30000, 4, 700), (3, 1500, 9000, 1, 1500)]


@pytest.mark.parametrize("b,each,num_pages,page,n", SIZES)
def test_reserve(m, b, each, num_pages, page, n):
    from oracle import serving
    rng = np.random.default_rng(b + num_pages)
    for turn in range(6):
        table, lens = some_tables(rng, b, each, num_pages, page)
        refs = counted([table], num_pages)
        if turn == 1:                                      # somebody else holds some, all the rest is taken
            refs += rng.integers(0, 2, num_pages)
        if turn == 2:                                      # counts that are less than none, lengths and entries out of range
            refs[refs == 0] -= rng.integers(0, 3, int((refs == 0).sum()))
            lens[rng.random(b) < 0.2] = -1
            lens[rng.random(b) < 0.1] = each * page
            lens[rng.random(b) < 0.1] = 2 ** 31 - 1
            table[rng.random(table.shape) < 0.1] = num_pages + 5
        if turn == 3:                                      # many write behind the same page
            lens[:] = max(1, each * page // 2)
            table[:] = table[0]
            refs = counted([table], num_pages)
        counts = None if turn % 2 else rng.integers(-1, n + 2, b)
        t, r = i32(table), i32(refs)
        granted, moves = m.mqa_paged_reserve_pages(t, i32(lens), r, page, min(n, each * page), counts=None if counts is None else i32(counts))
        want, want_moves = serving.reserve(table, lens, refs, page, min(n, each * page), counts)
        assert same(granted, want) and same(moves, want_moves) and same(t, table) and same(r, refs), turn


@pytest.mark.parametrize("b,n,num_pages", [(64, 5, 65536), (1000, 1, 70001), (4, 600, 65536), (1, 4096, 100000), (2000, 3, 40000)])
def test_reserve_from_pools_nearly_full(m, b, n, num_pages):
    """Free pages far apart, and fewer than are needed in some."""
    from oracle import serving
    rng = np.random.default_rng(num_pages + n)
    page, each = 4, -(-n // 4) + 2
    for free in (b * each, b * each // 3, 5, 0):
        table, lens = np.full((b, each), -1), rng.integers(0, 8, b)
        refs = np.ones(num_pages, dtype=np.int64)
        refs[num_pages - 1 - np.sort(rng.choice(num_pages // 2, free, replace=False))] = 0
        t, r = i32(table), i32(refs)
        granted, moves = m.mqa_paged_reserve_pages(t, i32(lens), r, page, n)
        want, want_moves = serving.reserve(table, lens, refs, page, n, None)
        assert same(granted, want) and same(moves, want_moves) and same(t, table) and same(r, refs), free


def test_reserve_where_the_pages_run_out(m):
    """In order of the sequences; one that keeps a shared page may do so only if the others have left it; one that needs nothing is granted all the same."""
    page = 8
    table = np.array([[0, -1], [0, -1], [0, -1], [1, -1], [2, 3]])
    lens, counts = np.array([3, 3, 3, 4, 9]), np.array([1, 1, 1, 1, 9])
    for pool, want in ((6, [1, 1, 1, 1, 0]), (5, [1, 0, 0, 1, 0]), (4, [0, 0, 0, 1, 0])):
        refs = i32(np.array([3, 1, 1, 1, 0, 0][:pool]))
        t = i32(table)
        granted, moves = m.mqa_paged_reserve_pages(t, i32(lens), refs, page, 9, counts=i32(counts))
        assert granted.tolist() == want
        assert moves.tolist() == {6: [[0, 4], [0, 5]] + [[-1, -1]] * 3, 5: [[0, 4]] + [[-1, -1]] * 4, 4: [[-1, -1]] * 5}[pool]
        assert refs.tolist() == {6: [1, 1, 1, 1, 1, 1], 5: [2, 1, 1, 1, 1], 4: [3, 1, 1, 1]}[pool]


@pytest.mark.parametrize("b,each,num_pages,page,n", SIZES)
def test_fork_and_free(m, b, each, num_pages, page, n):
    from oracle import serving
    rng = np.random.default_rng(b + num_pages)
    table, lens = some_tables(rng, b, each, num_pages, page)
    table[rng.random(table.shape) < 0.05] = num_pages      # (no page)
    lens[rng.random(b) < 0.1] = -7
    lens[rng.random(b) < 0.1] = 2 ** 31 - 1
    refs = counted([table], num_pages)
    for b_out in (1, b, 2 * b + 1):
        parents = rng.integers(-1, b + 1, b_out)
        out, lens_out, r = i32(np.full((b_out, each), 777)), i32(np.full(b_out, 777)), i32(refs)
        assert m.mqa_paged_fork_pages(i32(table), i32(lens), i32(parents), out, lens_out, r, page) is out
        want, want_lens = serving.fork(table, lens, parents, refs, page)
        assert same(out, want) and same(lens_out, want_lens) and same(r, refs)
        kept = rng.integers(-2, each * page + 3, b_out)
        assert m.mqa_paged_free_pages(out, i32(kept), r, page) is out
        serving.free(want, kept, refs, page)
        assert same(out, want) and same(r, refs)


@pytest.mark.parametrize("num_pages", [1, 2, 3, 7, 64, 2047, 2048, 2049, 4096, 6000, 16384, 16385, 131072, 131100])
@pytest.mark.parametrize("full", [0.0, 0.1, 0.5, 0.95, 1.0])
def test_compact_and_copy(m, num_pages, full):
    """Pools of several types and page sizes; what is in use is found at its new place."""
    from oracle import serving
    rng = np.random.default_rng(num_pages)
    refs = np.where(rng.random(num_pages) < full, rng.integers(1, 4, num_pages), rng.integers(-1, 1, num_pages))
    table = rng.integers(-2, num_pages + 2, (3, 50))
    want = serving.compact(table, refs)
    table_out, refs_out = torch.full((3, 50), 777, dtype=torch.int32, device=DEV), torch.full((num_pages,), 777, dtype=torch.int32, device=DEV)
    moves, used = torch.full((max(1, num_pages // 2), 2), 777, dtype=torch.int32, device=DEV), torch.full((1,), 777, dtype=torch.int32, device=DEV)
    assert m.mqa_paged_compact_pages(i32(table), i32(refs), table_out, refs_out, moves, used) is moves
    assert same(table_out, want[0]) and same(refs_out, want[1]) and same(moves, want[2]) and used.tolist() == [want[3]]
    pools = [rng.integers(0, 256, (num_pages, *shape)).astype(np.uint8) for shape in ((16, 16), (1, 4), (3, 20), (2, 5, 48))]
    on = [torch.from_numpy(x).to(DEV) for x in pools]
    on[1] = on[1].view(torch.float32)
    m.mqa_paged_copy_pages(on, moves)
    for x, t in zip(pools, on):
        serving.copy(x, want[2])
        assert np.array_equal(t.view(torch.uint8).cpu().numpy(), x)


def test_copy_of_many_pools_and_odd_pairs(m):
    """More pools than a launch takes; pairs with a page outside the pool, and of a page with itself, do nothing; large pages; many pairs."""
    rng = np.random.default_rng(4)
    pools = [torch.from_numpy(rng.integers(-99, 99, (40, 4 * (1 + x % 5)), dtype=np.int32)).to(DEV) for x in range(37)]
    before = [t.clone() for t in pools]
    m.mqa_paged_copy_pages(pools, i32(np.array([[3, 5], [-1, 7], [8, 40], [2 ** 31 - 1, 1], [9, 9], [3, 6], [0, -5]])))
    for x, y in zip(pools, before):
        y[5] = y[3]
        y[6] = y[3]
        assert torch.equal(x, y)
    large = torch.randn((6, 1 << 18), device=DEV)
    want = large.clone()
    m.mqa_paged_copy_pages((large,), i32(np.array([[0, 3], [1, 4]])))
    want[3], want[4] = want[0], want[1]
    assert torch.equal(large, want)
    small = torch.arange(80000, device=DEV, dtype=torch.int32).view(-1, 1).contiguous()
    pairs = np.stack([np.arange(40000), 40000 + rng.permutation(40000)], 1)
    m.mqa_paged_copy_pages([small], i32(pairs))
    assert np.array_equal(small[40000:, 0].cpu().numpy()[pairs[:, 1] - 40000], np.arange(40000))


def test_turns_of_a_pool(m):
    """Forks, reservations, ends and compactions in turn, eager, on a stream given and from a graph: as the oracle's."""
    from oracle import serving
    rng = np.random.default_rng(8)
    page, pages, each, b = 4, 30, 8, 9
    refs, table, lens = np.zeros(pages, dtype=np.int64), np.full((b, each), -1), np.zeros(b, dtype=np.int64)
    t, t_new, r, ls, ls_new = i32(table), i32(table), i32(refs), i32(lens), i32(lens)
    counts, kept, parents, none = (i32(np.zeros(b)) for _ in range(4))
    granted, moves = i32(np.zeros(b)), i32(np.zeros((b, 2)))
    pool = torch.arange(pages * 4, dtype=torch.int32, device=DEV).view(pages, 4).contiguous()
    mirror = pool.cpu().numpy().copy()
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)

    def turn(**kw):
        m.mqa_paged_reserve_pages(t, ls, r, page, 6, counts=counts, granted=granted, moves=moves, workspace=ws, **kw)
        m.mqa_paged_copy_pages([pool], moves, **kw)
        m.mqa_paged_free_pages(t, kept, r, page, **kw)
        m.mqa_paged_fork_pages(t, kept, parents, t_new, ls_new, r, page, **kw)
        m.mqa_paged_free_pages(t, none, r, page, **kw)

    state = [x.clone() for x in (t, r, ls, pool)]
    turn()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turn()
    for x, y in zip((t, r, ls, pool), state):
        x.copy_(y)
    side = torch.cuda.Stream()
    for step in range(60):
        c = rng.integers(0, 7, b)
        g, mv = serving.reserve(table, lens, refs, page, 6, c)
        serving.copy(mirror, mv)
        lens = lens + g
        kp = np.where(rng.random(b) < 0.3, 0, np.maximum(lens - rng.integers(0, 4, b), 0))
        serving.free(table, kp, refs, page)
        pr = rng.integers(-1, b, b)
        new, new_lens = serving.fork(table, kp, pr, refs, page)
        serving.free(table, np.zeros(b, dtype=np.int64), refs, page)
        table, lens = new, new_lens
        counts.copy_(i32(c)), kept.copy_(i32(kp)), parents.copy_(i32(pr))
        if step % 3 == 0:
            turn()
        elif step % 3 == 1:
            graph.replay()
        else:
            side.wait_stream(torch.cuda.current_stream())
            turn(stream=side)
            torch.cuda.current_stream().wait_stream(side)
        assert same(granted, g) and same(moves, mv) and same(t_new, table) and same(r, refs) and same(ls_new, lens), step
        assert np.array_equal(pool.cpu().numpy(), mirror)
        t.copy_(t_new), ls.copy_(ls_new)


def test_what_the_binding_refuses(m):
    t, v, r = i32(np.zeros((2, 3))), i32(np.zeros(2)), i32(np.zeros(8))
    with pytest.raises(TypeError):
        m.mqa_paged_free_pages(t.long(), v, r, 16)
    with pytest.raises(ValueError, match="lens must be"):
        m.mqa_paged_free_pages(t, r, r, 16)
    with pytest.raises(ValueError, match="table_out must be"):
        m.mqa_paged_fork_pages(t, v, v, i32(np.zeros((3, 3))), v.clone(), r, 16)
    with pytest.raises(ValueError, match="moves must be"):
        m.mqa_paged_reserve_pages(t, v, r, 16, 1, moves=i32(np.zeros((2, 3))))
    with pytest.raises(ValueError, match="moves must be"):
        m.mqa_paged_compact_pages(t, r, t.clone(), r.clone(), i32(np.zeros((3, 2))), i32(np.zeros(1)))
    with pytest.raises(ValueError, match=r"pools\[1\] must be"):
        m.mqa_paged_copy_pages([torch.zeros((8, 4), device=DEV), torch.zeros((9, 4), device=DEV)], i32(np.zeros((1, 2))))
    for call in (lambda: m.mqa_paged_reserve_pages(t, v, r, 0, 1), lambda: m.mqa_paged_reserve_pages(t, v, r, 16, 49), lambda: m.mqa_paged_reserve_pages(t, v, r, 16, 2 ** 40),
                 lambda: m.mqa_paged_reserve_pages(t, v, r, 16, 1, granted=v), lambda: m.mqa_paged_compact_pages(t, r, t, r.clone(), i32(np.zeros((4, 2))), i32(np.zeros(1))),
                 lambda: m.mqa_paged_copy_pages([torch.zeros((8, 3), dtype=torch.int8, device=DEV)], i32(np.zeros((1, 2)))), lambda: m.mqa_paged_free_pages(t, v, r, 0)):
        with pytest.raises(m.MqaError) as e:
            call()
        assert e.value.status == 2
