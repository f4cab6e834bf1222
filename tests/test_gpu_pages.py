"""Pages of a pool against lists: tables, lengths, counts and copies."""
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import step_ref as ref  # noqa: E402

NONE = -1


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_18703_amd as R
    return R.Context()


def dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


class Both:
    """A pool on the GPU and one of lists, that every call goes to."""

    def __init__(self, ctx, n_pages, page, rows, cols, max_seqs=None):
        self.ctx, self.n_pages, self.page = ctx, n_pages, page
        self.ref = ref.Pool(n_pages, page)
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        self.pool = ctx.pages(self.refs, page, max(rows) if max_seqs is None else max_seqs)
        import paper_2609_18703_amd as R
        self.lists = [([[NONE] * cols for _ in range(n)], [0] * n) for n in rows]
        self.tables = [R.Tables(torch.full((n, cols), NONE, dtype=torch.int32, device="cuda"),
                                torch.zeros(n, dtype=torch.int32, device="cuda")) for n in rows]

    def check(self):
        self.ctx.check("pages")
        self.same()

    def same(self):
        assert self.refs.tolist() == self.ref.refs
        for t, (table, lens) in zip(self.tables, self.lists):
            assert t.len.tolist() == lens
            assert t.table.tolist() == table

    def fork(self, a, parent, b):
        self.pool.fork(self.tables[a], dev(parent), self.tables[b])
        self.ref.fork(*self.lists[a], parent, *self.lists[b])

    def grow(self, a, add):
        n = len(add)
        src, dst, slots = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for _ in range(3))
        free = torch.full((1,), 77, dtype=torch.int64, device="cuda")
        before = sum(r == 0 for r in self.ref.refs)
        self.pool.grow(self.tables[a], dev(add), src, dst, slots, free)
        want = self.ref.grow(*self.lists[a], add)
        if want is None:
            import paper_2609_18703_amd as R
            assert self.ctx.status() == R.ECAP
            want = [NONE] * n, [NONE] * n, [0] * n, before
        assert (src.tolist(), dst.tolist(), slots.tolist(), free.item()) == tuple(want)
        return src, dst, slots

    def release(self, a, keep):
        self.pool.release(self.tables[a], None if keep is None else dev(keep))
        self.ref.release(*self.lists[a], [0] * len(self.lists[a][1]) if keep is None else keep)

    def compact(self):
        half = self.n_pages // 2 + 3
        src, dst = (torch.full((half,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
        moves, free = (torch.full((1,), 77, dtype=torch.int64, device="cuda") for _ in range(2))
        self.pool.compact(self.tables, src, dst, moves, free)
        a, b = self.ref.compact(self.lists)
        n = len(a)
        assert moves.item() == n and free.item() == sum(r == 0 for r in self.ref.refs)
        assert src.tolist() == a + [77] * (half - n) and dst.tolist() == b + [77] * (half - n)
        return src, dst, moves


@pytest.mark.parametrize("n_pages,page,rows,cols,most", [
    (40, 16, (5, 9), 6, 50), (64, 16, (3, 12), 9, 40), (65, 1, (4, 4), 20, 9), (1000, 64, (30, 100), 13, 300),
    (4096, 16, (7, 300), 40, 200), (4097, 32, (40, 257), 30, 500), (13000, 16, (60, 513), 33, 300),
    (9, 65536, (2, 5), 3, 70000)])
def test_pages_through_a_life(ctx, n_pages, page, rows, cols, most):
    """Prompts, children that share them, growth, ends, moves: all tables equal after every call."""
    rng = random.Random(n_pages + page)
    b = Both(ctx, n_pages, page, rows, cols)
    P, N = rows
    room = cols * page
    for life in range(3):
        b.grow(0, [min(rng.randrange(0, most), room - L) for L in b.lists[0][1]])
        b.check()
        b.fork(0, [rng.choice([NONE] + list(range(P))) for _ in range(N)], 1)
        b.check()
        for step in range(4):
            b.grow(1, [min(rng.choice([0, 1, 1, 1, page, rng.randrange(1, most)]), room - L) for L in b.lists[1][1]])
            b.same()
            if step == 1:
                b.release(1, [rng.choice([1 << 30, L, max(0, L - 1), rng.randrange(0, L + 1), 0]) for L in b.lists[1][1]])
                b.check()
            if step == 2:
                b.compact()
                b.check()
        b.release(1, None)
        b.check()
        b.release(0, [rng.choice([0, L, rng.randrange(0, L + 1)]) for L in b.lists[0][1]])
        b.check()
        b.compact()
        b.check()


def test_pages_taken_lowest_first(ctx):
    b = Both(ctx, 20, 16, (3,), 8)
    b.grow(0, [33, 16, 1])
    assert b.tables[0].table[:, :3].tolist() == [[0, 1, 2], [3, NONE, NONE], [4, NONE, NONE]]
    b.release(0, [16, 0, 1])
    b.grow(0, [16, 32, 0])
    assert b.tables[0].table[:, :3].tolist() == [[0, 1, NONE], [2, 3, NONE], [4, NONE, NONE]]
    b.check()


def test_pages_all_or_none(ctx):
    b = Both(ctx, 10, 16, (4,), 12)
    b.grow(0, [40, 1, 0, 16])
    b.check()
    b.grow(0, [0, 16 * 5, 1, 0])                # one more than there are
    b.same()
    b.grow(0, [0, 16 * 4, 1, 0])                # all
    b.check()
    b.grow(0, [0, 0, 1, 0])                     # room in a page
    b.check()
    b.grow(0, [0, 0, 0, 1])
    b.same()


def test_pages_last_sharer_keeps_the_page(ctx):
    """Both children replace a page that their parent has left: it is free from the next call on."""
    b = Both(ctx, 6, 16, (1, 2), 3)
    b.grow(0, [20])
    b.fork(0, [0, 0], 1)
    b.release(0, None)
    src, dst, slots = b.grow(1, [1, 0])
    assert src.tolist() == [1, NONE] and slots.tolist() == [4, 0]
    b.check()
    src, _, _ = b.grow(1, [0, 1])               # the other one has it alone now
    assert src.tolist() == [NONE, NONE]
    b.check()
    b.release(1, None)
    b.grow(0, [20])
    b.fork(0, [0, 0], 1)
    b.release(0, None)
    b.grow(1, [1, 1])
    assert b.refs.tolist() == [2, 0, 1, 1, 0, 0]
    b.check()


def test_pages_nothing(ctx):
    """No sequences, no pages, no positions."""
    b = Both(ctx, 0, 16, (3, 2), 4)
    b.grow(0, [0, 0, 0])
    b.fork(0, [2, NONE], 1)
    b.compact()
    b.release(0, None)
    b.check()
    b.grow(0, [0, 1, 0])
    b.same()
    import paper_2609_18703_amd as R
    refs = dev([0, 1, 0])
    pool = ctx.pages(refs, 16, 0)
    empty = R.Tables(torch.empty(0, 4, dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"))
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    free = torch.zeros(1, dtype=torch.int64, device="cuda")
    pool.grow(empty, none, none, none, none, free)
    ctx.check()
    assert free.item() == 2
    moves = torch.zeros(1, dtype=torch.int64, device="cuda")
    src, dst = dev([9]), dev([9])
    pool.compact([empty], src, dst, moves)
    pool.release(empty)
    pool.fork(empty, none, empty)
    ctx.check()
    assert moves.item() == 1 and (src.item(), dst.item()) == (1, 0) and refs.tolist() == [1, 0, 0]


def test_pages_large_pool(ctx):
    """A pool of many tiles: what is taken and moved lies far apart."""
    n_pages, S = 300001, 700
    g = torch.Generator(device="cuda").manual_seed(1)
    b = Both(ctx, n_pages, 16, (S,), 200, max_seqs=S)
    used = (torch.rand(n_pages, generator=g, device="cuda") < 0.7).int()
    b.refs.copy_(used)
    b.ref.refs = used.tolist()
    b.grow(0, [(37 * s) % 3000 for s in range(S)])
    b.check()
    b.grow(0, [1] * S)
    b.check()
    b.compact()
    b.check()


def test_pages_bad_rows(ctx):
    """What cannot be is refused row by row; the others go on, and counts stay whole."""
    import paper_2609_18703_amd as R
    n = 12
    refs = dev([1, 1, 0, 0, 0, 2, 0, 0, 0, 0, 0, 0])
    pool = ctx.pages(refs, 16, 8)
    table = dev([[0, NONE, NONE], [1, NONE, NONE], [500, NONE, NONE], [5, NONE, NONE], [5, NONE, NONE]])
    t = R.Tables(table, dev([16, 17 + 32, 7, -5, 16]))           # row 1: more than its entries hold
    src, dst, slots = (torch.full((5,), 77, dtype=torch.int32, device="cuda") for _ in range(3))
    free = torch.zeros(1, dtype=torch.int64, device="cuda")
    pool.grow(t, dev([1, 1, 1, 1, 16]), src, dst, slots, free)
    assert ctx.status() == R.ERANGE
    assert t.len.tolist() == [17, 49, 7, -5, 32] and free.item() == 7
    assert table.tolist() == [[0, 2, NONE], [1, NONE, NONE], [500, NONE, NONE], [5, NONE, NONE], [5, 3, NONE]]
    assert src.tolist() == dst.tolist() == [NONE] * 5 and slots.tolist() == [0] * 5
    pool.grow(t, dev([-1, 0, 0, 0, 40]), src, dst, slots, free)   # a negative number; a row too short
    assert ctx.status() in (R.ERANGE, R.ECAP)
    assert t.len.tolist() == [17, 49, 7, -5, 32]
    pool.grow(t, dev([2 ** 31 - 18, 0, 0, 0, 2 ** 31 - 1]), src, dst, slots, free)
    assert ctx.status() in (R.ERANGE, R.ECAP)
    assert t.len.tolist() == [17, 49, 7, -5, 32]

    to = R.Tables(torch.full((6, 1), NONE, dtype=torch.int32, device="cuda"), dev([0, 3, 0, 0, 0, 0]))
    for parent, code in (([NONE, 4, NONE, NONE, NONE, NONE], R.ESTATE),       # the row holds something
                         ([0, NONE, NONE, NONE, NONE, NONE], R.ECAP),         # two pages, one entry
                         ([NONE, NONE, 2, NONE, NONE, NONE], R.ERANGE),       # page 500
                         ([NONE, NONE, NONE, 3, NONE, NONE], R.ERANGE),       # length -5
                         ([NONE, NONE, NONE, NONE, 5, -2], R.ERANGE)):        # no such rows
        pool.fork(t, dev(parent), to)
        assert ctx.status() == code, parent
        assert to.len.tolist() == [0, 3, 0, 0, 0, 0] and (to.table == NONE).all()
    assert refs.tolist() == [1, 1, 1, 1, 0, 2, 0, 0, 0, 0, 0, 0]

    pool.release(t, dev([-1, 0, 7, 0, 32]))
    assert ctx.status() == R.ERANGE
    assert t.len.tolist() == [17, 49, 7, -5, 32]
    pool.release(t, dev([17, 100, 0, 100, 32]))                   # row 2's page is dropped with its error
    assert ctx.status() == R.ERANGE
    assert t.len.tolist() == [17, 49, 0, -5, 32] and table[2].tolist() == [NONE] * 3
    free_page = R.Tables(dev([[9, 9]]), dev([32]))
    pool.release(free_page)
    assert ctx.status() == R.ESTATE
    assert refs.tolist() == [1, 1, 1, 1, 0, 2, 0, 0, 0, 0, 0, 0] and free_page.len.tolist() == [0]

    bad = R.Tables(dev([[9, 4000, 5], [0, 1, 5], [0, 0, 0]]), dev([48, 48, -1]))
    src, dst = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    moves = torch.zeros(1, dtype=torch.int64, device="cuda")
    pool.compact([bad], src, dst, moves)
    assert ctx.status() in (R.ERANGE, R.ESTATE)
    assert moves.item() == 1 and (src[0].item(), dst[0].item()) == (5, 4)
    assert bad.table.tolist() == [[9, 4000, 4], [0, 1, 4], [0, 0, 0]]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("page,heads,dim,layers", [(16, 1, 64, 1), (16, 3, 128, 3), (64, 4, 128, 2), (128, 2, 64, 70)])
@pytest.mark.parametrize("order", ["heads", "slots"])
def test_pages_copy(ctx, page, heads, dim, layers, order, dtype):
    import paper_2609_18703_amd as R
    n_pages = 23
    g = torch.Generator(device="cuda").manual_seed(page + heads)

    def pages():
        if order == "heads":
            return torch.randn(n_pages, heads, page, dim, generator=g, device="cuda").to(dtype)
        return torch.randn(n_pages, page, heads, dim, generator=g, device="cuda").to(dtype).transpose(1, 2)
    kv = [(pages(), pages()) for _ in range(layers)]
    if layers > 1:                              # one of another layout among them
        kv[1] = tuple(torch.randn(n_pages + 2, heads, page, dim + 8, generator=g, device="cuda").to(dtype)[..., :dim]
                      for _ in range(2))
    caches = [R.Cache(k, v) for k, v in kv]
    src, dst = [3, NONE, 5, 5, 0, 22, 9], [1, 2, NONE, 4, 6, 7, 8]
    slots = [page, 1, 1, 1, 0, page - 3, 5]
    pool = ctx.pages(torch.zeros(n_pages, dtype=torch.int32, device="cuda"), page, 1)
    for use, n in ((True, None), (False, None), (False, 3), (True, 0), (False, 100)):
        want = [[t.clone() for t in pair] for pair in kv]
        m = len(src) if n is None else min(n, len(src))
        for i in range(m):
            if src[i] != NONE and dst[i] != NONE:
                upto = slots[i] if use else page
                for pair in want:
                    for t in pair:
                        t[dst[i], :, :upto] = t[src[i], :, :upto]
        pool.copy(caches, dev(src), dev(dst), dev(slots) if use else None, None if n is None else dev([n], torch.int64))
        ctx.check("copy")
        for pair, w in zip(kv, want):
            for a, b in zip(pair, w):
                assert torch.equal(a, b)


def test_pages_copy_bad_entries(ctx):
    import paper_2609_18703_amd as R
    k, v = (torch.randn(6, 2, 16, 64, device="cuda").half() for _ in range(2))
    pool = ctx.pages(torch.zeros(6, dtype=torch.int32, device="cuda"), 16, 1)
    for src, dst, slots in (([6, 1], [0, 2], [4, 4]), ([0, 1], [-2, 2], [4, 4]), ([0, 1], [3, 2], [17, 4]),
                            ([0, 1], [3, 2], [-1, 4])):
        wk = k.clone()
        wk[2, :, :4] = k[1, :, :4]
        pool.copy([R.Cache(k, v)], dev(src), dev(dst), dev(slots))
        assert ctx.status() == R.ERANGE
        assert torch.equal(k, wk)
    before = k.clone()
    pool.copy([R.Cache(k, v)], dev([1]), dev([3]), None, dev([-4], torch.int64))
    ctx.check()
    assert torch.equal(k, before)


@pytest.mark.parametrize("n_pages", [10, 40000])
def test_pages_more_than_any_pool_has(ctx, n_pages):
    """A sequence that wants as many positions, and pages, as there may be."""
    import paper_2609_18703_amd as R
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    pool = ctx.pages(refs, 1, 2)
    t = R.Tables(torch.empty(2, 1 << 30, dtype=torch.int32, device="cuda"), dev([0, 0]))
    out = [torch.full((2,), 77, dtype=torch.int32, device="cuda") for _ in range(3)]
    free = torch.zeros(1, dtype=torch.int64, device="cuda")
    for add in ([1 << 30, 0], [1 << 30, 1 << 30], [(1 << 30) - 1, 3]):
        pool.grow(t, dev(add), *out, free)
        assert ctx.status() == R.ECAP
        assert t.len.tolist() == [0, 0] and free.item() == n_pages and not refs.any()
        assert out[0].tolist() == [NONE] * 2 and out[2].tolist() == [0, 0]


@pytest.mark.parametrize("n_pages,rows", [(12, 8), (40000, 8), (40000, 100)])
@pytest.mark.parametrize("count", [0, -1])
def test_pages_grow_into_a_free_page(ctx, n_pages, rows, count):
    """A sequence goes on in a page that refs call free: an error, and it stays as it is."""
    import paper_2609_18703_amd as R
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[0] = refs[2] = 1
    refs[1] = count
    table = torch.full((rows, 3), NONE, dtype=torch.int32, device="cuda")
    table[:3, 0] = dev([0, 1, 2])
    length = torch.zeros(rows, dtype=torch.int32, device="cuda")
    length[:3] = dev([5, 6, 7])
    t = R.Tables(table, length)
    pool = ctx.pages(refs, 16, rows)
    src, dst, slots = (torch.full((rows,), 77, dtype=torch.int32, device="cuda") for _ in range(3))
    free = torch.zeros(1, dtype=torch.int64, device="cuda")
    pool.grow(t, dev([1, 1, 20] + [0] * (rows - 3)), src, dst, slots, free)
    assert ctx.status() == R.ESTATE
    assert length.tolist() == [6, 6, 27] + [0] * (rows - 3)
    first = 1 if count == 0 else 3                   # (to a count of 0 the page is free: it is the lowest)
    assert table[:3].tolist() == [[0, NONE, NONE], [1, NONE, NONE], [2, first, NONE]]
    assert (src == NONE).all() and (dst == NONE).all() and not slots.any()
    # nothing to add: nothing is looked at
    refs[1] = count
    pool.grow(t, dev([0] * rows), src, dst, slots, free)
    ctx.check()


@pytest.mark.parametrize("n_pages,rows", [(700, 30), (700, 90), (40000, 30)])
def test_pages_in_a_graph(n_pages, rows):
    """A reservation's calls and the moves after it, captured and replayed between eager calls of the same pool and work
    of other kinds."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_18703_amd as R
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        b = Both(R.Context(stream), n_pages, 16, (5, rows), 9)
        k, v = (torch.randn(n_pages, 2, 16, 64, device="cuda").half() for _ in range(2))
        caches = [R.Cache(k, v)]
        b.grow(0, [33, 16, 5, 100, 0])
        rng = random.Random(n_pages + rows)
        parent, add = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(2))
        src, dst, slots = (torch.zeros(rows, dtype=torch.int32, device="cuda") for _ in range(3))
        a, c = (torch.zeros(n_pages // 2, dtype=torch.int32, device="cuda") for _ in range(2))
        free, moves = (torch.zeros(1, dtype=torch.int64, device="cuda") for _ in range(2))
        b.check()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            b.pool.release(b.tables[1])
            b.pool.fork(b.tables[0], parent, b.tables[1])
            b.pool.grow(b.tables[1], add, src, dst, slots, free)
            b.pool.copy(caches, src, dst, slots)
            b.pool.compact(b.tables, a, c, moves, free)
            b.pool.copy(caches, a, c, n=moves)
        for turn in range(6):
            parents = [rng.choice([NONE, 0, 1, 2, 3, 4]) for _ in range(rows)]
            adds = [rng.choice([0, 1, 3, 30]) for _ in range(rows)]
            parent.copy_(dev(parents))
            add.copy_(dev(adds))
            want = [t.clone() for t in (k, v)]
            graph.replay()
            b.ref.release(*b.lists[1], [0] * rows)
            b.ref.fork(*b.lists[0], parents, *b.lists[1])
            s, d, n, _ = b.ref.grow(*b.lists[1], adds)
            assert (src.tolist(), dst.tolist(), slots.tolist()) == (s, d, n)
            for t in want:
                for i in range(rows):
                    if s[i] != NONE:
                        t[d[i], :, :n[i]] = t[s[i], :, :n[i]]
            s, d = b.ref.compact(b.lists)
            for t in want:
                t[dev(d).long()] = t[dev(s).long()]
            b.check()
            assert moves.item() == len(s) and free.item() == sum(r == 0 for r in b.ref.refs)
            assert a[:len(s)].tolist() == s and c[:len(s)].tolist() == d
            live = n_pages - free.item()
            assert all(torch.equal(t[:live], w[:live]) for t, w in zip((k, v), want))
            # eager calls between the replays: some end, some go on
            b.release(1, [rng.choice([0, 1 << 30]) for _ in range(rows)])
            b.grow(1, [rng.choice([0, 1]) if L else 0 for L in b.lists[1][1]])
            b.check()
            _ = (torch.randn(1000, device="cuda") @ torch.randn(1000, 1000, device="cuda")).sum().item()
        stream.synchronize()
