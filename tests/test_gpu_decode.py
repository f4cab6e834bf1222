"""Projections, pages, attention and sampling together, as a batch's children
use them: the same bits as the calls one by one give on pages that nobody
shares, and the tokens that the definition chooses from the logits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import step_ref as ref  # noqa: E402

P, B, HQ, HK, D, PS, HIDDEN, VOCAB, LAYERS = 4, 9, 8, 2, 64, 16, 192, 1003, 2


@pytest.fixture(scope="module")
def R():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_18703_amd as R
    return R


def weights(R, g, n_out, n_in):
    w = torch.randint(-127, 128, (n_out, n_in), generator=g, device="cuda", dtype=torch.int8)
    scale = (torch.rand(n_out, generator=g, device="cuda") + 0.5) / (74 * n_in ** 0.5)
    return R.Weights(w, scale, torch.randn(n_out, generator=g, device="cuda") * 0.1)


def model(R, dtype=torch.bfloat16, n_pages=60):
    g = torch.Generator(device="cuda").manual_seed(7)
    layers = [(weights(R, g, (HQ + 2 * HK) * D, HIDDEN), weights(R, g, HIDDEN, HQ * D)) for _ in range(LAYERS)]
    head = weights(R, g, VOCAB, HIDDEN)
    freq = (1.0e4 ** (-torch.arange(16, device="cuda").float() / 16)).contiguous()
    ctx = R.Context()
    from paper_2609_18703_amd.decode import Decode
    rotary = R.Rotary(freq, [i % 2 for i in range(16)])
    return ctx, g, rotary, layers, head, Decode(ctx, P, B, layers, head, HQ, HK, D, PS, n_pages, 8, rotary, 400, dtype)


def off(new):
    return torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int64, device="cuda")


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Alone:
    """Every sequence with pages of its own, the library's calls one by one."""

    def __init__(self, R, ctx, rotary, layers, dtype, n):
        self.R, self.ctx, self.rotary, self.layers, self.n = R, ctx, rotary, layers, n
        shape = (n * 8, HK, PS, D)
        self.caches = [R.Cache(*(torch.zeros(shape, dtype=dtype, device="cuda") for _ in range(2))) for _ in layers]
        self.table = torch.arange(n * 8, device="cuda").int().flip(0).view(n, 8).contiguous()
        self.len = [0] * n

    def project(self, w, x):
        q = torch.empty(x.shape, dtype=torch.int8, device="cuda")
        scale = torch.empty(x.shape[0], device="cuda")
        out = torch.empty(x.shape[0], w.n_out, dtype=x.dtype, device="cuda")
        self.ctx.quantize(x, q, scale)
        self.ctx.project(q, scale, w, out)
        return out

    def step(self, x, pos, new):
        self.len = [a + b for a, b in zip(self.len, new)]
        T = x.shape[0]
        chunk = self.ctx.chunk(self.n, T, 8)
        chunk.plan(self.caches[0], off(new), i32(self.len), self.table, HQ, n_tokens=T)
        for cache, (a, b) in zip(self.caches, self.layers):
            rows = self.project(a, x).view(T, HQ + 2 * HK, D)
            q = torch.empty(T, HQ, D, dtype=x.dtype, device="cuda")
            chunk.append(cache, rows[:, :HQ], rows[:, HQ:HQ + HK], rows[:, HQ + HK:], q, self.rotary, pos)
            out = torch.empty_like(q)
            chunk.attend(cache, q, out)
            x = x + self.project(b, out.view(T, HQ * D))
        return x

    def fork(self, other, parent):
        for s, p in enumerate(parent):
            self.len[s] = 0 if p < 0 else other.len[p]
            if p >= 0:
                for mine, theirs in zip(self.caches, other.caches):
                    for a, b in ((mine.k, theirs.k), (mine.v, theirs.v)):
                        a[self.table[s].long()] = b[other.table[p].long()]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_decode_as_alone(R, dtype):
    ctx, g, rotary, layers, head, decode = model(R, dtype)
    parents, children = (Alone(R, ctx, rotary, layers, dtype, n) for n in (P, B))

    def tokens(n):
        x = torch.randn(n, HIDDEN, generator=g, device="cuda").to(dtype)
        return x, torch.randint(0, 300, (2, n), generator=g, device="cuda").int()

    lengths = [37, 16, 5, 48]
    x, pos = tokens(sum(lengths))
    got = decode.prompts(x, pos, off(lengths), i32(lengths))
    ctx.check("prompts")
    assert torch.equal(got, parents.step(x, pos, lengths))
    for turn, (parent, news) in enumerate([([0, 0, 2, 1, 3, 3, 0, 2, 1], [[1] * B, [3, 1, 20, 2, 1, 1, 0, 5, 17], [1] * B]),
                                           ([3, 1, 1, 0, 2], [[2, 1, 1, 1, 9, 0, 0, 0, 0]] * 2)]):
        decode.reserve(i32(list(range(len(parent)))), i32(parent))
        children.fork(parents, parent + [-1] * (B - len(parent)))
        for i, new in enumerate(news):
            x, pos = tokens(sum(new))
            got = decode.step(x, pos, off(new), i32(new))
            ctx.check("step")
            assert torch.equal(got, children.step(x, pos, new)), (turn, i)
            assert decode.children.len.tolist() == children.len
            # the last tokens' choice
            last = off(new)[1:][i32(new).long() > 0] - 1
            n = last.numel()
            u = torch.rand(n, generator=g, device="cuda")
            how = dict(temperature=torch.full((n,), 0.8, device="cuda"), top_k=i32([40] * n),
                       top_p=torch.full((n,), 0.95, device="cuda"))
            token, logprob = decode.choose(got[last], u, **how)
            ctx.check("choose")
            logits = children.project(head, got[last]).double().cpu().numpy()
            for r in range(n):
                want = ref.sample(logits[r], float(u[r]), float(how["temperature"][r]), 40, float(how["top_p"][r]))
                assert token[r].item() == want[0]
                assert abs(logprob[r].item() - want[1]) <= 2.0 ** -24 * abs(want[1]) + 1e-11
            # some tokens are taken back, one sequence ends, and the pages move together
            keep = [max(0, L - i) for L in children.len]
            keep[2] = 0 if i == 1 else keep[2]
            decode.keep(i32(keep))
            children.len = keep
            decode.compact()
            ctx.check("compact")
            live = int((decode.refs > 0).sum())
            assert (decode.refs[:live] > 0).all() and decode.n_free.item() == decode.refs.numel() - live
    # nothing is lost: with the children gone and the prompts too, all pages are free
    decode.reserve(i32([]), i32([]))
    decode.pool.release(decode.parents)
    ctx.check()
    assert (decode.refs == 0).all()


def test_decode_on_another_stream(R):
    """Inputs made on the context's stream, called from another current one."""
    outs = []
    for other in (False, True):
        ctx, g, _, _, _, decode = model(R)
        lengths = [30, 20, 10, 1]
        x = torch.randn(61, HIDDEN, generator=g, device="cuda").bfloat16()
        pos = torch.randint(0, 300, (2, 61), generator=g, device="cuda").int()
        q_off, lens, kids = off(lengths), i32(lengths), i32([0, 1, 2, 3, 0, 1, 2, 3, 0])
        one, ones = off([1] * B), i32([1] * B)
        stream = torch.cuda.Stream() if other else torch.cuda.current_stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            decode.prompts(x, pos, q_off, lens)
            decode.reserve(kids, kids)
            h = decode.step(x[:B], pos[:, :B].contiguous(), one, ones)
        ctx.check()
        outs.append(h)
    assert torch.equal(*outs)


def test_decode_in_a_graph(R):
    """A step and its choice, captured and replayed between eager work, against eager steps."""
    outs = {}
    for graphed in (False, True):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            ctx, g, _, _, _, decode = model(R)
            lengths = [30, 20, 10, 1]
            x = torch.randn(61, HIDDEN, generator=g, device="cuda").bfloat16()
            pos = torch.randint(0, 300, (2, 61), generator=g, device="cuda").int()
            decode.prompts(x, pos, off(lengths), i32(lengths))
            kids = i32([0, 1, 2, 3, 0, 1, 2, 3, 0])
            decode.reserve(kids, kids)
            one, ones, u = off([1] * B), i32([1] * B), torch.rand(B, generator=g, device="cuda")
            xs, ps = x[:B].clone(), pos[:, :B].contiguous()

            def step():
                h = decode.step(xs, ps, one, ones)
                return (h, *decode.choose(h, u))
            warm = step()                                # (allocations of the eager kind are made once)
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            if graphed:
                with torch.cuda.graph(graph, stream=stream):
                    captured = step()
            seen = []
            for i in range(20):                          # over the ends of pages
                xs.copy_(x[i:i + B])
                if graphed:
                    graph.replay()
                    seen.append([t.clone() for t in captured])
                else:
                    seen.append(step())
                if i % 3 == 0:
                    torch.cuda.synchronize()
                    _ = (torch.randn(1000, device="cuda") @ torch.randn(1000, 1000, device="cuda")).sum().item()
            ctx.check()
            outs[graphed] = seen
            del warm, graph
    for a, b in zip(outs[False], outs[True]):
        for s, t in zip(a, b):
            assert torch.equal(s, t)


@pytest.mark.parametrize("length", [48, 40])
def test_decode_out_of_pages(R, length):
    """A pool that has too few pages: an error, and the sequences as they were, whole pages shared or partly filled ones."""
    ctx, g, _, _, _, decode = model(R, n_pages=12)
    lengths = [length] * 4
    x = torch.randn(4 * length, HIDDEN, generator=g, device="cuda").bfloat16()
    pos = torch.randint(0, 300, (2, 4 * length), generator=g, device="cuda").int()
    decode.prompts(x, pos, off(lengths), i32(lengths))
    ctx.check()
    assert decode.n_free.item() == 0
    kids = i32([0, 1, 2, 3, 0, 1, 2, 3, 0])
    decode.reserve(kids, kids)
    ctx.check()

    def held():
        pages = decode.parents.table.long()[:, :3]
        return [t[pages].permute(0, 1, 3, 2, 4).reshape(P, 48, HK, D)[:, :length].clone()
                for c in decode.caches for t in (c.k, c.v)]
    before = decode.children.len.tolist(), decode.children.table.tolist(), decode.refs.tolist()
    prompts = held()
    decode.step(x[:B], pos[:, :B].contiguous(), off([1] * B), i32([1] * B))
    assert ctx.status() == R.ECAP
    assert (decode.children.len.tolist(), decode.children.table.tolist(), decode.refs.tolist()) == before
    assert all(torch.equal(a, b) for a, b in zip(held(), prompts))
    decode.keep(i32([0] * B))
    decode.pool.release(decode.parents, i32([length, length, 0, 0]))
    decode.reserve(i32([0, 1]), i32([0, 1]))
    decode.step(x[:2], pos[:, :2].contiguous(), off([1, 1] + [0] * 7), i32([1, 1] + [0] * 7))
    ctx.check()
    assert decode.children.len.tolist() == [length + 1, length + 1] + [0] * 7


@pytest.mark.parametrize("length", [48, 40])
def test_decode_out_of_pages_after_taking_back(R, length):
    """Children that go on before the end of a page which they share, in a pool that has no page for them."""
    ctx, g, _, _, _, decode = model(R, n_pages=12)
    lengths = [length] * 4
    x = torch.randn(4 * length, HIDDEN, generator=g, device="cuda").bfloat16()
    pos = torch.randint(0, 300, (2, 4 * length), generator=g, device="cuda").int()
    decode.prompts(x, pos, off(lengths), i32(lengths))
    kids = i32([0, 1, 2, 3, 0, 1, 2, 3, 0])
    decode.reserve(kids, kids)
    decode.keep(i32([length - 5] * B))
    ctx.check()
    caches = [t.clone() for c in decode.caches for t in (c.k, c.v)]
    state = decode.children.len.tolist(), decode.children.table.tolist(), decode.refs.tolist()
    new = [1, 4, 1, 7, 0, 1, 20, 1, 1]
    decode.step(x[:sum(new)], pos[:, :sum(new)].contiguous(), off(new), i32(new))
    assert ctx.status() == R.ECAP
    assert (decode.children.len.tolist(), decode.children.table.tolist(), decode.refs.tolist()) == state
    assert all(torch.equal(a, b) for a, b in zip(caches, [t for c in decode.caches for t in (c.k, c.v)]))


def state(decode):
    return [t.tolist() for s in (decode.parents, decode.children) for t in (s.len, s.table)] + [decode.refs.tolist()]


def bad_steps(R, x, pos, q_off, new):
    """Arguments of a step that some library call refuses, and how."""
    T = x.shape[0]
    many = x.repeat(401 // T + 1, 1)
    wide = pos.repeat(1, 401 // T + 1)
    return [((many, wide, q_off, new), R.RoError), ((x[:, 1:], pos, q_off, new), ValueError), ((x.half(), pos, q_off, new), TypeError),
            ((x.float(), pos, q_off, new), TypeError), ((x[0], pos, q_off, new), ValueError), ((x.cpu(), pos, q_off, new), ValueError),
            ((x.t().contiguous().t(), pos, q_off, new), ValueError), ((x, pos[:1], q_off, new), ValueError),
            ((x, pos[:, 1:].contiguous(), q_off, new), ValueError), ((x, pos.float(), q_off, new), TypeError),
            ((x, pos, q_off[1:], new), ValueError), ((x, pos, q_off.int(), new), TypeError), ((x, pos, q_off, new.long()), TypeError),
            ((x, pos, q_off, new[1:]), (ValueError, RuntimeError)), ((x, pos, q_off, new.cpu()), (ValueError, RuntimeError)),
            ((x, pos, q_off, torch.cat([new, new])), (ValueError, RuntimeError)),
            ((x.as_strided(x.shape, (3, 1)), pos, q_off, new), R.RoError)]


def test_decode_refused_steps_change_nothing(R):
    """A step or prompts that a library call refuses leave sequences, tables and counts as they were."""
    ctx, g, _, _, _, decode = model(R)
    lengths = [30, 20, 10, 1]
    x = torch.randn(61, HIDDEN, generator=g, device="cuda").bfloat16()
    pos = torch.randint(0, 300, (2, 61), generator=g, device="cuda").int()
    empty = state(decode)
    for args, error in bad_steps(R, x, pos, off(lengths), i32(lengths)):
        with pytest.raises(error):
            decode.prompts(*args)
        assert state(decode) == empty
    decode.prompts(x, pos, off(lengths), i32(lengths))
    kids = i32([0, 1, 2, 3, 0, 1, 2, 3, 0])
    decode.reserve(kids, kids)
    before = state(decode)
    for args, error in bad_steps(R, x[:B], pos[:, :B].contiguous(), off([1] * B), i32([1] * B)):
        with pytest.raises(error):
            decode.step(*args)
        assert state(decode) == before
    decode.step(x[:B], pos[:, :B].contiguous(), off([1] * B), i32([1] * B))
    ctx.check()
    assert decode.children.len.tolist() == [31, 21, 11, 2, 31, 21, 11, 2, 31]


def test_decode_refuses_what_no_step_can_have(R):
    """Weights, pages and rotations that do not go together are refused where they are given."""
    from paper_2609_18703_amd.decode import Decode
    ctx, g, rotary, layers, head, _ = model(R)
    qkv, back = layers[0]

    def make(layers=layers, head=head, q_heads=HQ, page=PS, rotary=rotary):
        return Decode(ctx, P, B, layers, head, q_heads, HK, D, page, 60, 8, rotary, 400)
    make()
    make(head=None)
    wide = R.Rotary(torch.ones(D, device="cuda"))                # twice the head
    for kw in (dict(layers=[(back, back)]), dict(layers=[(qkv, qkv)]), dict(layers=[layers[0], (weights(R, g, (HQ + 2 * HK) * D, 208), back)]),
               dict(head=weights(R, g, VOCAB, 208)), dict(q_heads=HQ + 1), dict(page=8), dict(page=24), dict(rotary=wide)):
        with pytest.raises((ValueError, R.RoError)):
            make(**kw)
    ctx.check()


def test_decode_refused_reservations_change_nothing(R):
    """Tags that do not go together leave the last batch's children in place."""
    ctx, g, _, _, _, decode = model(R)
    lengths = [30, 20, 10, 1]
    x = torch.randn(61, HIDDEN, generator=g, device="cuda").bfloat16()
    pos = torch.randint(0, 300, (2, 61), generator=g, device="cuda").int()
    decode.prompts(x, pos, off(lengths), i32(lengths))
    kids = i32([0, 1, 2, 3, 0, 1, 2, 3, 0])
    decode.reserve(kids, kids)
    before = state(decode)
    for child, parent in ((kids, kids[:5]), (kids, kids[:1]), (kids[:3], kids[:0])):
        with pytest.raises((ValueError, RuntimeError)):
            decode.reserve(child, parent)
        assert state(decode) == before
    decode.reserve(kids[:3], kids)               # tags behind the children are not looked at
    ctx.check()
    assert decode.children.len.tolist() == [30, 20, 10] + [0] * 6
