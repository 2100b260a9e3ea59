"""The native calls (csrc/calls.cpp) of 8-bit caches, pages and adjusted logits: taken for plain arguments, with the general path's results; what is not plain is left to
the general path, with its answers and errors."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def m():
    import paper_1911_02150_amd.binding as lib
    lib.load_library()
    return lib


class Watch:
    """The native calls, or none of them, and which were asked and answered."""

    def __init__(self, native, on):
        self.native, self.on, self.took = native, on, []

    def __getattr__(self, name):
        def call(*args):
            done = getattr(self.native, name)(*args) if self.on else None
            self.took.append((name, done is not None))
            return done
        return call


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def cases(m, dtype, heads):
    g = torch.Generator(device=DEV).manual_seed(1)
    b, n, h, k, v, page, block, each, pages = 3, 2, 4, 32, 48, 8, 4, 5, 20
    lead = (pages,) if heads == 1 else (pages, heads)
    K, V = (torch.randn((*lead, page, w), generator=g, device=DEV).mul(20).to(dtype) for w in (k, v))
    Ks, Vs = (torch.rand((*lead, page // block), generator=g, device=DEV) + 0.1 for _ in range(2))
    table = torch.randperm(pages, generator=g, device=DEV)[:b * each].to(torch.int32).view(b, each).contiguous()
    lens = i32(3, 20, 37)
    row = (b, n) if heads == 1 else (b, n, heads)
    k_new, v_new, q = torch.randn((*row, k), generator=g, device=DEV), torch.randn((*row, v), generator=g, device=DEV), torch.randn((b, n, h, k), generator=g, device=DEV)
    new = lambda t: torch.full_like(t, 7)  # noqa: E731

    def append(counts):
        c, out = [t.clone() for t in (K, Ks, V, Vs)], new(lens)
        m.mqa_paged_scaled_append_kv_rows(*c, table, k_new, v_new, lens, out, counts=counts)
        return (*(t.view(torch.uint8) for t in c), out)

    refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
    refs[table.view(-1).long()] = 1

    def fork():
        to, out, r = new(table), new(lens), refs.clone()
        return m.mqa_paged_fork_pages(table, lens, i32(2, 0, 2), to, out, r, page), out, r

    def free():
        t, r = table.clone(), refs.clone()
        return m.mqa_paged_free_pages(t, lens, r, page), r

    def reserve(**kw):
        t, r = table.clone(), refs.clone()
        t[:, 3:] = -1
        return (*m.mqa_paged_reserve_pages(t, i32(20, 24, 10), r, page, 9, **kw), t, r)

    def compact():
        out = new(table), new(refs), torch.zeros((pages // 2, 2), dtype=torch.int32, device=DEV), i32(0)
        m.mqa_paged_compact_pages(table, refs, *out)
        return out

    def copy(as_):
        pools = as_([K.clone(), Ks.clone()])
        m.mqa_paged_copy_pages(pools, i32(1, 2, 3, 4).view(2, 2))
        return pools[0].view(torch.uint8), pools[1]

    logits = torch.randn((b, n + 1, 77), generator=g, device=DEV)
    history, drafts = (torch.randint(0, 77, (b, x), generator=g, device=DEV, dtype=torch.int32) for x in (9, n))
    f = torch.rand(b, generator=g, device=DEV) + 0.5
    allowed = torch.randint(-99, 99, (b, n + 1, 3), generator=g, device=DEV, dtype=torch.int32)
    flat = logits[:, 0].contiguous()
    yield from [
        ("scaled_append", lambda: append(None)), ("scaled_append", lambda: append(i32(1, 2, 0))),
        ("scaled_decode", lambda: (m.mqa_paged_scaled_decode_step(q, K, Ks, V, Vs, table, lens, scale=0.3),)),
        ("scaled_decode", lambda: (m.mqa_paged_scaled_decode_step(q[:, 0].contiguous(), K, Ks, V, Vs, table, lens, o=torch.empty((b, h, v), device=DEV)),)),
        ("fork_pages", fork), ("free_pages", free), ("reserve_pages", reserve),
        ("reserve_pages", lambda: reserve(counts=i32(3, 0, 99), granted=new(lens), moves=torch.zeros((b, 2), dtype=torch.int32, device=DEV))),
        ("compact_pages", compact), ("copy_pages", lambda: copy(list)), ("copy_pages", lambda: copy(tuple)),
        ("adjust_logits", lambda: (m.mqa_stack_adjust_logits(logits, history, lens, drafts=drafts),)),
        ("adjust_logits", lambda: (m.mqa_stack_adjust_logits(logits, history, lens, drafts=drafts, prompts=lens, repetition=f, frequency=f, presence=f, bias_tokens=history,
                                                             biases=torch.rand((b, 9), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV), allowed=allowed,
                                                             out=torch.empty_like(logits)),)),
        ("adjust_logits", lambda: (m.mqa_stack_adjust_logits(flat, history, lens, allowed=allowed[:, 0].contiguous()),)),
    ]


@pytest.mark.parametrize("heads", [1, 2])
@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.int8])
def test_same_as_the_general_path(m, dtype, heads, monkeypatch):
    native = m._native
    for name, call in cases(m, dtype, heads):
        got = []
        for on in (True, False):
            watch = Watch(native, on)
            monkeypatch.setattr(m, "_native", watch)
            got.append(call())
            assert watch.took == [(name, on)], name
        assert len(got[0]) == len(got[1]) and all(torch.equal(x, y) and x.dtype == y.dtype and x.shape == y.shape for x, y in zip(*got)), name


def test_left_to_the_general_path(m, monkeypatch):
    """Subclasses, generators of pools and streams are taken by the general path; wrong tensors are named by it."""
    native = m._native
    watch = Watch(native, True)
    monkeypatch.setattr(m, "_native", watch)

    class Sub(torch.Tensor):
        pass

    table, lens, refs = i32(0, 1, 2, 3).view(2, 2), i32(8, 9), i32(1, 1, 1, 1, 0, 0)
    pool = torch.arange(24, device=DEV, dtype=torch.int32).view(6, 4).contiguous()
    m.mqa_paged_copy_pages((t for t in [pool]), i32(0, 5).view(1, 2))
    assert torch.equal(pool[5], pool[0])
    m.mqa_paged_free_pages(table.as_subclass(Sub), i32(0, 0), refs, 8)
    assert refs.tolist() == [0] * 6 and table.tolist() == [[-1, -1]] * 2
    assert not any(took for _, took in watch.took)
    watch.took.clear()
    m.mqa_paged_reserve_pages(table, i32(0, 0), refs, 8, 9, stream=torch.cuda.current_stream())
    assert not watch.took and table.tolist() == [[0, 1], [2, 3]]
    for error, call in ((TypeError, lambda: m.mqa_paged_free_pages(table.long(), lens, refs, 8)), (ValueError, lambda: m.mqa_paged_free_pages(table, lens[:1], refs, 8)),
                        (ValueError, lambda: m.mqa_paged_reserve_pages(table.t(), lens, refs, 8, 1)), (ValueError, lambda: m.mqa_paged_copy_pages([], i32(0, 5).view(1, 2))),
                        (ValueError, lambda: m.mqa_paged_copy_pages([pool, pool[:5].contiguous()], i32(0, 5).view(1, 2))),
                        (ValueError, lambda: m.mqa_stack_adjust_logits(torch.zeros((2, 5), device=DEV), table, lens[:1]))):
        with pytest.raises(error):
            call()
    assert not any(took for _, took in watch.took)
    for call in (lambda: m.mqa_paged_free_pages(table, lens, refs, 0), lambda: m.mqa_paged_reserve_pages(table, lens, refs, 8, 0),
                 lambda: m.mqa_paged_copy_pages([torch.zeros((6, 3), dtype=torch.int8, device=DEV)], i32(0, 5).view(1, 2))):
        with pytest.raises(m.MqaError) as e:                       # the library's own refusal, from either path
            call()
        assert e.value.status == 2


def test_captured_with_a_workspace_of_its_own(m):
    """While a stream is captured the workspace is the graph's; two graphs have one each, and replays in turn do not meet."""
    table, lens, refs = torch.full((3, 4), -1, dtype=torch.int32, device=DEV), i32(0, 5, 9), torch.zeros(40, dtype=torch.int32, device=DEV)
    granted, moves = i32(0, 0, 0), torch.zeros((3, 2), dtype=torch.int32, device=DEV)
    m.mqa_paged_reserve_pages(table.clone(), lens, refs.clone(), 8, 9, granted=granted, moves=moves)
    graphs, states = [], []
    for _ in range(2):
        state = table.clone(), refs.clone(), granted.clone(), moves.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.mqa_paged_reserve_pages(state[0], lens, state[1], 8, 9, granted=state[2], moves=state[3])
        graphs.append(graph), states.append(state)
    for turn in range(4):
        lens.copy_(i32(turn, 8 * turn % 24, 9))
        for graph, state in zip(graphs, states):
            state[0].fill_(-1), state[1].zero_()
            graph.replay()
        want = table.clone(), refs.clone()
        got = m.mqa_paged_reserve_pages(want[0], lens, want[1], 8, 9)
        torch.cuda.synchronize()
        for state in states:
            assert torch.equal(state[0], want[0]) and torch.equal(state[1], want[1]) and torch.equal(state[2], got[0]) and torch.equal(state[3], got[1])
