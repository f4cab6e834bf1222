"""Attention of a model stage over a paged cache: rotary positions, append,
attention, weights and eviction, each against its definition in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import chunk_ref as ref  # noqa: E402

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_18703_amd as R
    c = R.Context()
    yield c
    c.close()


def make(new, kv_len, q_heads, kv_heads, dim, page, dtype, causal=True, window=0, sinks=0, seed=0, spare=3,
         slot_major=False, share=0):
    """Sequences with the given new tokens and lengths; pages in random order;
    table entries beyond a sequence's pages name no page, and every cached
    element that no sequence owns is NaN.  share: leading pages all sequences
    have in common."""
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    need = [-(-L // page) for L in kv_len]
    n_pages = sum(need) + spare
    ids = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = torch.full((len(new), max(need + [1]) + 1), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = ids[at:at + n]
        at += n
        if s and share:
            table[s, :min(share, n, need[0])] = table[0, :min(share, n, need[0])]
    case = dict(new=new, kv_len=kv_len, q_off=[sum(new[:i]) for i in range(len(new) + 1)], page=page, causal=causal,
                window=window, sinks=sinks, table=table, q_heads=q_heads, kv_heads=kv_heads, dim=dim, dtype=dtype)

    def cache():
        x = torch.randn(n_pages, kv_heads, page, dim, generator=g, device="cuda")
        own = torch.zeros(n_pages, page, dtype=torch.bool, device="cuda")
        for s in range(len(new)):
            p, sl = ref.positions(case, s)
            own[p, sl] = True
        x = x.masked_fill(~own[:, None, :, None], math.nan).to(dtype)
        return x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) if slot_major else x
    case["k"], case["v"] = cache(), cache()
    case["q"] = (torch.randn(max(sum(new), 1), q_heads, dim, generator=g, device="cuda") * 1.5).to(dtype)[:sum(new)]
    return case


def plan(ctx, case, **kw):
    import paper_2609_18703_amd as R
    cache = R.Cache(case["k"], case["v"])
    ch = ctx.chunk(len(case["new"]), sum(case["new"]), case["table"].shape[1])
    off = torch.tensor(case["q_off"], dtype=torch.int64, device="cuda")
    kv = torch.tensor(case["kv_len"], dtype=torch.int32, device="cuda")
    ch.plan(cache, off, kv, case["table"], case["q_heads"], sum(case["new"]), max_new=max(case["new"] + [0]),
            causal=case["causal"], window=case["window"], sinks=case["sinks"], **kw)
    ctx.check("plan")
    return cache, ch


CASES = [
    # new tokens, lengths, q heads, kv heads, dim, page, extra
    ([1], [1], 1, 1, 64, 16, {}),
    ([1], [1], 7, 1, 128, 16, {}),
    ([1, 1, 1], [17, 1, 300], 28, 4, 128, 16, {}),
    ([1, 1], [1000, 2049], 8, 8, 64, 64, {}),
    ([1] * 9, [5, 64, 65, 63, 128, 127, 129, 200, 31], 16, 2, 128, 32, {}),
    ([1], [5003], 32, 8, 128, 64, {}),
    ([2, 3], [2, 130], 4, 2, 128, 16, {}),
    ([33], [33], 8, 2, 64, 16, {}),
    ([70, 1, 0, 5], [200, 77, 40, 5], 14, 2, 128, 32, {}),
    ([0, 0], [10, 0], 4, 4, 64, 16, {}),
    ([129], [129], 5, 5, 128, 128, {}),
    ([100, 30], [333, 31], 20, 4, 128, 256, {}),
    ([257], [400], 4, 1, 64, 64, {}),
    ([40, 3], [10, 0], 4, 2, 64, 16, {}),                      # more tokens than positions: rows that see nothing
    ([40, 3], [10, 2], 4, 2, 128, 16, {"causal": False}),
    ([1, 9, 60], [65, 200, 61], 6, 3, 128, 16, {"causal": False}),
    ([1, 1, 50], [300, 20, 130], 8, 2, 128, 16, {"window": 32, "sinks": 4}),
    ([1, 90], [700, 400], 8, 2, 64, 32, {"window": 1, "sinks": 0}),
    ([200], [500], 7, 1, 128, 64, {"window": 100, "sinks": 70}),
    ([130, 1], [260, 1000], 12, 2, 64, 16, {"window": 128, "sinks": 1}),
    ([60, 1], [90, 64], 8, 4, 128, 16, {"window": 1000, "sinks": 3}),
    ([3, 16], [600, 40], 8, 1, 128, 16, {"slot_major": True}),
    ([8, 8, 8], [200, 190, 180], 16, 4, 128, 16, {"share": 8}),
    ([300], [1500], 40, 8, 128, 128, {}),
    # few rows: one, two, three, four and more key / value heads, positions between a window and the sinks
    ([1, 2, 0, 1], [700, 333, 90, 64], 8, 1, 128, 16, {"window": 64, "sinks": 5}),
    ([1, 1], [2000, 450], 14, 2, 64, 32, {"window": 100, "sinks": 130}),
    ([2, 1], [900, 1], 12, 3, 128, 16, {"window": 1, "sinks": 70}),
    ([1] * 5, [64, 1000, 129, 2500, 1], 35, 5, 128, 64, {}),
    ([3, 1], [2, 700], 10, 2, 128, 16, {}),
    ([1, 1], [1300, 70], 40, 20, 64, 256, {"window": 300, "sinks": 1}),
    # weights: shares of several tiles and sequences, and tiles of many shares
    ([700, 1, 0, 300, 1], [4000, 2500, 600, 310, 1700], 4, 2, 64, 64, {}),
    ([1, 650, 40], [3500, 2000, 900], 6, 2, 64, 16, {"window": 200, "sinks": 300}),
]


def close(got, want, tol, what):
    got = got.double()
    bad = ~((got - want).abs() <= tol) & ~((got == want) | (got.isnan() & want.isnan()))
    assert not bad.any(), "%s: %d off, first at %s: %r for %r (tolerance %r)" % (
        what, int(bad.sum()), bad.nonzero()[0].tolist(), float(got[bad][0]), float(want[bad][0]), float(tol[bad][0]))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("at", range(len(CASES)))
def test_attend(ctx, at, dtype):
    new, kv, hq, hk, dim, page, more = CASES[at]
    c = make(new, kv, hq, hk, dim, page, dtype, seed=at, **more)
    cache, ch = plan(ctx, c)
    q = c["q"]
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    print("attend", at, CASES[at], dtype, flush=True)
    ch.attend(cache, q, out, lse)
    ctx.check("attend")
    want, wl, tol, tl = ref.attend(c, c["k"], c["v"], q, dim ** -0.5)
    close(lse, wl, tl, "lse")
    close(out, want, tol, "out")
    again = torch.empty_like(out)
    ch.attend(cache, q, again)                                  # without lse; the same bits
    assert torch.equal(again, out)
    ch.close()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("at", range(len(CASES)))
def test_weigh(ctx, at, dtype):
    new, kv, hq, hk, dim, page, more = CASES[at]
    c = make(new, kv, hq, hk, dim, page, dtype, seed=at + 50, **more)
    cache, ch = plan(ctx, c)
    g = torch.Generator(device="cuda").manual_seed(at)
    _, lse, _, _ = ref.attend(c, c["k"], c["v"], c["q"], dim ** -0.5)
    lse = lse.float()
    w_in = torch.rand(len(new), max(kv) + 5, generator=g, device="cuda")
    w_out = w_in.clone()
    print("weigh", at, CASES[at], dtype, flush=True)
    ch.weigh(cache, c["q"], lse, w_in, w_out)
    ctx.check("weigh")
    want, tol = ref.weigh(c, c["k"], c["q"], lse, w_in, dim ** -0.5)
    close(w_out, want, tol, "weight")
    acc = w_in.clone()
    ch.weigh(cache, c["q"], lse, acc, acc)                      # in place, the same bits
    assert torch.equal(acc, w_out)
    zero = torch.zeros_like(w_in)
    ch.weigh(cache, c["q"], lse, None, zero)
    want, tol = ref.weigh(c, c["k"], c["q"], lse, torch.zeros_like(w_in), dim ** -0.5)
    close(zero, want, tol, "weight from zero")
    ch.close()


@pytest.mark.parametrize("new,kv,heads,dim", [([1, 1], [200, 70], (8, 2), 128), ([60, 90], [160, 90], (8, 2), 128),
                                              ([150], [300], (4, 1), 64)])
def test_hidden_values_do_not_matter(ctx, new, kv, heads, dim):
    """NaN and infinities behind the causal limit and outside the window reach no row that does not see them."""
    for window, sinks in ((0, 0), (40, 3)):
        c = make(new, kv, *heads, dim, 16, BF, window=window, sinks=sinks, seed=5)
        for s in range(len(new)):                               # the last position, and one in the middle
            page, slot = ref.positions(c, s)
            for j, x in ((kv[s] - 1, math.nan), (kv[s] // 2, math.inf), (kv[s] - 2, -math.inf)):
                c["v"][page[j], :, slot[j], ::3] = x
        cache, ch = plan(ctx, c)
        out, lse = torch.empty_like(c["q"]), torch.empty(c["q"].shape[:2], device="cuda")
        print("hidden values", new, kv, window, flush=True)
        ch.attend(cache, c["q"], out, lse)
        ctx.check("attend")
        want, wl, tol, tl = ref.attend(c, c["k"], c["v"], c["q"], dim ** -0.5)
        close(lse, wl, tl, "lse")
        fine = want.isfinite()
        assert torch.equal(fine, out.isfinite())
        assert torch.equal(want.isnan(), out.isnan())
        close(torch.where(fine, out.double(), 0.0), torch.where(fine, want, 0.0), torch.where(fine, tol, 0.0), "out")
        ch.close()


def test_hidden_keys_do_not_matter(ctx):
    c = make([50, 1], [120, 33], 4, 2, 128, 16, HF, seed=9)
    for s in range(2):
        page, slot = ref.positions(c, s)
        c["k"][page[-1], :, slot[-1]] = math.nan                # only the last token sees it
    cache, ch = plan(ctx, c)
    out, lse = torch.empty_like(c["q"]), torch.empty(c["q"].shape[:2], device="cuda")
    print("hidden keys", flush=True)
    ch.attend(cache, c["q"], out, lse)
    ctx.check("attend")
    sees = torch.tensor([49, 50], device="cuda")
    assert out[sees].isnan().all() and lse[sees].isnan().all()
    want, wl, tol, tl = ref.attend(c, c["k"], c["v"], c["q"], 128 ** -0.5)
    close(lse[:49], wl[:49], tl[:49], "lse")
    close(out[:49], want[:49], tol[:49], "out")
    ch.close()


@pytest.mark.parametrize("big", [3.0e4, 1.0])
def test_scores_of_any_size(ctx, big):
    """Scores far above and below zero, whose exponentials alone would overflow, and a rising maximum."""
    c = make([1, 70], [400, 300], 8, 2, 64, 16, HF, seed=3)
    for s in range(2):
        page, slot = ref.positions(c, s)
        up = torch.linspace(-1.0, 1.0, len(page), device="cuda")[:, None, None] * big ** 0.5
        c["k"][page, :, slot] = (c["k"][page, :, slot].float() * 0.01 + up).to(HF)
    c["q"] = (c["q"].float().abs() + big ** 0.25).to(HF)
    cache, ch = plan(ctx, c)
    out, lse = torch.empty_like(c["q"]), torch.empty(c["q"].shape[:2], device="cuda")
    print("scores", big, flush=True)
    ch.attend(cache, c["q"], out, lse, scale=1.0)
    ctx.check("attend")
    want, wl, tol, tl = ref.attend(c, c["k"], c["v"], c["q"], 1.0)
    close(lse, wl, tl, "lse")
    close(out, want, tol, "out")
    ch.close()


@pytest.mark.parametrize("scale", [0.0, -0.125, -1.0e-3])
def test_scale_of_any_sign(ctx, scale):
    c = make([1, 45], [70, 50], 8, 2, 64, 16, BF, window=30, sinks=2, seed=8)
    cache, ch = plan(ctx, c)
    out, lse = torch.empty_like(c["q"]), torch.empty(c["q"].shape[:2], device="cuda")
    print("scale", scale, flush=True)
    ch.attend(cache, c["q"], out, lse, scale=scale)
    w = torch.zeros(2, 70, device="cuda")
    ch.weigh(cache, c["q"], lse, None, w, scale=scale)
    ctx.check("attend")
    want, wl, tol, tl = ref.attend(c, c["k"], c["v"], c["q"], scale)
    close(lse, wl, tl, "lse")
    close(out, want, tol, "out")
    close(w, *ref.weigh(c, c["k"], c["q"], lse, torch.zeros_like(w), scale), "weight")
    ch.close()


def test_hidden_values_where_work_is_cut(ctx):
    """The same as above for rows whose keys several workgroups share."""
    for new, kv in (([1], [9000]), ([20], [9000])):
        c = make(new, kv, 7, 1, 128, 16, BF, window=8000, sinks=5, seed=6)
        page, slot = ref.positions(c, 0)
        for j, x in ((8999, math.nan), (8997, math.inf), (980, -math.inf), (3, math.inf), (8, math.nan)):
            c["v"][page[j], :, slot[j], j % 7::11] = x
        cache, ch = plan(ctx, c)
        out = torch.empty_like(c["q"])
        print("hidden values, cut", new, kv, flush=True)
        ch.attend(cache, c["q"], out)
        ctx.check("attend")
        want, _, tol, _ = ref.attend(c, c["k"], c["v"], c["q"], 128 ** -0.5)
        fine = want.isfinite()
        assert torch.equal(fine, out.isfinite())
        assert torch.equal(want.isnan(), out.isnan())
        close(torch.where(fine, out.double(), 0.0), torch.where(fine, want, 0.0), torch.where(fine, tol, 0.0), "out")
        ch.close()


def test_strided_rows_and_in_place(ctx):
    """Queries inside a fused projection, heads before tokens in the output, and out = q."""
    c = make([37, 1], [90, 200], 8, 2, 128, 32, BF, seed=11)
    cache, ch = plan(ctx, c)
    want, _, tol, _ = ref.attend(c, c["k"], c["v"], c["q"], 128 ** -0.5)
    wide = torch.full((38, 12, 136), 5.0, dtype=BF, device="cuda")
    q = wide[:, 2:10, :128]
    q.copy_(c["q"])
    out = torch.empty(8, 38, 128, dtype=BF, device="cuda").permute(1, 0, 2)
    ch.attend(cache, q, out)
    close(out, want, tol, "out")
    ch.attend(cache, q, q)
    assert torch.equal(q, out)
    assert (wide[:, :2] == 5).all() and (wide[:, 10:] == 5).all() and (wide[..., 128:] == 5).all()
    ctx.check("attend")
    ch.close()


# ---- rotary positions --------------------------------------------------------------

ROPE = [
    # tokens, heads, dim, pairs, axes of the pairs
    (1, 1, 2, 1, 1), (3, 2, 6, 2, 2), (5, 3, 80, 40, 2), (17, 4, 72, 36, 3), (130, 5, 64, 32, 4), (33, 2, 128, 64, 3),
    (9, 3, 128, 32, 3), (4, 2, 130, 64, 1), (1030, 2, 64, 32, 3), (7, 1, 512, 256, 8),
    (9001, 1, 64, 32, 2), (20005, 2, 32, 16, 1),                # several tokens a workgroup
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("at", range(len(ROPE)))
def test_rope(ctx, at, adjacent, dtype):
    import paper_2609_18703_amd as R
    T, H, D, pairs, axes = ROPE[at]
    g = torch.Generator(device="cuda").manual_seed(at)
    x = torch.randn(T, H, D, generator=g, device="cuda").to(dtype)
    axis = [(i * 5 + i // 3) % axes for i in range(pairs)]
    freq = 1.0e4 ** (-torch.arange(pairs, device="cuda").float() / pairs)
    pos = torch.randint(-5, 2_000_000, (axes, T), generator=g, device="cuda").int()
    pos[:, 0] = 0
    rot = R.Rotary(freq, axis, adjacent=adjacent, n_axes=axes)
    print("rope", at, ROPE[at], adjacent, dtype, flush=True)
    for inverse in (False, True):
        y = torch.full_like(x, 9.0)
        ctx.rope(x, y, rot, pos, inverse=inverse)
        ctx.check("rope")
        want, tol = ref.turn(x, pos, freq, axis, adjacent, inverse)
        close(y, want, tol, "y")
        z = x.clone()
        ctx.rope(z, z, rot, pos, inverse=inverse)               # in place
        assert torch.equal(z, y)
        # heads of a wider tensor, shifted off 16 bytes: the same values
        w = torch.full((T, H + 2, D + 3), 5.0, dtype=dtype, device="cuda")
        ctx.rope(x, w[:, 1:H + 1, 1:D + 1], rot, pos, inverse=inverse)
        assert torch.equal(w[:, 1:H + 1, 1:D + 1], y)
        assert (w[:, 0] == 5).all() and (w[..., 0] == 5).all() and (w[..., D + 1:] == 5).all()


def test_rope_gradient(ctx):
    """The inverse rotation of dy is the formula's gradient, and agrees with differences of the forward one."""
    import paper_2609_18703_amd as R
    T, H, D, pairs = 6, 2, 64, 24
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(T, H, D, generator=g, device="cuda").half()
    dy = torch.randn(T, H, D, generator=g, device="cuda").half()
    axis = [i % 3 for i in range(pairs)]
    freq = 100.0 ** (-torch.arange(pairs, device="cuda").float() / pairs)
    pos = torch.randint(0, 1000, (3, T), generator=g, device="cuda").int()
    for adjacent in (False, True):
        rot = R.Rotary(freq, axis, adjacent=adjacent)
        dx = torch.empty_like(dy)
        ctx.rope(dy, dx, rot, pos, inverse=True)
        xd = x.double().requires_grad_(True)
        c, s = (f(pos.double()[torch.tensor(axis, device="cuda")].T * freq.double())[:, None] for f in (torch.cos, torch.sin))
        i = torch.arange(pairs, device="cuda")
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + pairs)
        rest = torch.arange(2 * pairs, D, device="cuda")
        loss = ((xd[..., a] * c - xd[..., b] * s) * dy[..., a].double()).sum() \
            + ((xd[..., b] * c + xd[..., a] * s) * dy[..., b].double()).sum() \
            + (xd[..., rest] * dy[..., rest].double()).sum()
        loss.backward()
        _, tol = ref.turn(dy, pos, freq, axis, adjacent, True)
        close(dx, xd.grad, tol, "gradient")
        # a central difference along a direction v: the rotation is linear, so only rounding is left
        v = torch.randn(T, H, D, generator=g, device="cuda").half()
        y1, y0 = torch.empty_like(x), torch.empty_like(x)
        ctx.rope(x + v, y1, rot, pos)
        ctx.rope(x - v, y0, rot, pos)
        num = ((y1.double() - y0.double()) * dy.double()).sum() / 2
        ana = (dx.double() * ((x + v).double() - (x - v).double())).sum() / 2
        size = (y1.double().abs() + y0.double().abs()).mul(dy.double().abs()).sum()
        assert abs(num - ana) <= 2.0 ** -10 * size + 2.0 ** -10 * (dx.double().abs() * v.double().abs()).sum()
    ctx.check("rope")


APPEND = [
    # new, lengths, q heads, kv heads, dim, page, pairs, axes, adjacent
    ([1], [1], 4, 1, 64, 16, 32, 1, False),
    ([1, 1, 1], [16, 17, 300], 28, 4, 128, 16, 64, 3, False),
    ([40, 0, 7], [40, 9, 100], 8, 2, 128, 32, 64, 3, True),
    ([130, 1030], [150, 1030], 4, 4, 64, 64, 16, 2, False),
    ([9, 5], [30, 5], 6, 2, 128, 16, 20, 2, True),
    ([5000, 4201], [5000, 4300], 1, 1, 64, 64, 32, 2, False),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("at", range(len(APPEND)))
def test_append(ctx, at, dtype):
    import paper_2609_18703_amd as R
    new, kv, hq, hk, dim, page, pairs, axes, adjacent = APPEND[at]
    c = make(new, kv, hq, hk, dim, page, dtype, seed=at)
    g = torch.Generator(device="cuda").manual_seed(at)
    T = sum(new)
    qkv = torch.randn(T, hq + 2 * hk, dim, generator=g, device="cuda").to(dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    axis = [i * axes // pairs for i in range(pairs)]
    freq = 1.0e6 ** (-torch.arange(pairs, device="cuda").float() / pairs)
    pos = torch.randint(0, 100_000, (axes, T), generator=g, device="cuda").int()
    rot = R.Rotary(freq, axis, adjacent=adjacent)
    cache, ch = plan(ctx, c)
    before = c["k"].clone(), c["v"].clone()
    print("append", at, APPEND[at], dtype, flush=True)
    for with_q, with_rot in ((True, True), (False, True), (True, False)):
        c["k"].copy_(before[0])
        c["v"].copy_(before[1])
        qo = torch.full_like(q, 9.0) if with_q else None
        ch.append(cache, q if with_q else None, k, v, qo, rot if with_rot else None, pos if with_rot else None)
        ctx.check("append")
        wk, wv = before[0].double(), before[1].double()
        tk = torch.zeros_like(wk)
        kk, tol = ref.turn(k, pos, freq, axis, adjacent, False) if with_rot else (k.double(), torch.zeros_like(k.double()))
        for s, n in enumerate(new):
            p, sl = (a[kv[s] - n:] for a in ref.positions(c, s))
            t0 = c["q_off"][s]
            wk[p, :, sl], wv[p, :, sl], tk[p, :, sl] = kk[t0:t0 + n], v[t0:t0 + n].double(), tol[t0:t0 + n]
        close(c["k"], wk, tk, "keys")
        close(c["v"], wv, torch.zeros_like(wv), "values")
        if with_q:
            wq, tq = ref.turn(q, pos, freq, axis, adjacent, False) if with_rot else (q.double(), torch.zeros_like(q.double()))
            close(qo, wq, tq, "q")
    ch.append(cache, q, k, v, q, rot, pos)                      # queries in place
    close(q, *ref.turn(qo, pos, freq, axis, adjacent, False), "q in place")
    ctx.check("append")
    ch.close()


# ---- eviction --------------------------------------------------------------------------

EVICT = [
    # lengths, budget, first, last, kv heads, dim, page
    ([1, 0, 3], 2, 0, 1, 1, 64, 16),
    ([40, 17, 16], 17, 4, 5, 2, 128, 16),
    ([300, 2050, 1023, 1024, 1025], 500, 3, 100, 4, 128, 32),
    ([777], 100, 60, 40, 2, 64, 64),                            # nothing competes
    ([5000, 4999], 1, 0, 0, 1, 64, 256),
    ([5000, 100], 4998, 0, 1, 2, 128, 16),
]


@pytest.mark.parametrize("kind", ["random", "ties", "special"])
@pytest.mark.parametrize("at", range(len(EVICT)))
def test_evict(ctx, at, kind):
    import paper_2609_18703_amd as R
    lens, budget, first, last, heads, dim, page = EVICT[at]
    S = len(lens)
    g = torch.Generator(device="cuda").manual_seed(at)
    most = max(1, -(-min(budget, max(lens)) // page))
    c = make([0] * S, lens, heads, heads, dim, page, HF if at % 2 else BF, seed=at, spare=S * most)
    used = set(c["table"][c["table"] >= 0].tolist())
    free = torch.tensor([p for p in range(c["k"].shape[0]) if p not in used], dtype=torch.int32, device="cuda")
    dst = free[torch.randperm(len(free), generator=g, device="cuda")][:S * most].view(S, most).contiguous()
    w = torch.randn(S, max(lens) + 3, generator=g, device="cuda")
    if kind == "ties":
        w = torch.randint(0, 3, w.shape, generator=g, device="cuda").float() * torch.where(w > 0, 1.0, -1.0)   # -0 too
    if kind == "special":
        r = torch.rand(w.shape, generator=g, device="cuda")
        for lo, x in ((0.0, math.nan), (0.2, math.inf), (0.3, -math.inf), (0.4, 0.0), (0.5, -0.0), (0.6, 1e-45)):
            w = torch.where((r > lo) & (r <= lo + 0.1), torch.tensor(x, device="cuda"), w)
    cache, ch = plan(ctx, c)
    k0, v0 = c["k"].clone(), c["v"].clone()
    new_len = torch.full((S,), -7, dtype=torch.int32, device="cuda")
    index = torch.full((S, budget), -7, dtype=torch.int32, device="cuda")
    new_w = torch.full((S, budget), 7.0, device="cuda")
    print("evict", at, EVICT[at], kind, flush=True)
    ch.evict(cache, w, dst, budget, new_len, index, new_w, first=first, last=last)
    ctx.check("evict")
    wk, wv, ww = k0.clone(), v0.clone(), torch.full_like(new_w, 7.0)
    for s, L in enumerate(lens):
        keep = ref.kept(w[s], L, budget, first, last)
        m = len(keep)
        assert int(new_len[s]) == m
        assert index[s].tolist() == keep + [-1] * (budget - m)
        ix = torch.tensor(keep, dtype=torch.long, device="cuda")
        ww[s, :m] = w[s, ix]
        p, sl = (a[ix] for a in ref.positions(c, s))
        r = torch.arange(m, device="cuda")
        wk[dst[s].long()[r // page], :, r % page] = k0[p, :, sl]
        wv[dst[s].long()[r // page], :, r % page] = v0[p, :, sl]
    assert torch.equal(new_w.nan_to_num(nan=123.0), ww.nan_to_num(nan=123.0))
    for got, want in ((c["k"], wk), (c["v"], wv)):
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))
    ch.close()


# ---- errors, streams, graphs ----------------------------------------------------------------

def test_refusals(ctx):
    import paper_2609_18703_amd as R
    c = make([2, 3], [20, 40], 4, 2, 64, 16, BF)
    cache, ch = plan(ctx, c)
    q = c["q"]
    out, lse = torch.empty_like(q), torch.empty(5, 4, device="cuda")

    def refused(code, f):
        with pytest.raises(R.RoError) as e:
            f()
        assert e.value.code == code

    off, kv = (torch.tensor(x, dtype=d, device="cuda") for x, d in (([0, 2, 5], torch.int64), ([20, 40], torch.int32)))
    p = dict(n_tokens=5, max_new=3)
    refused(R.EINVAL, lambda: ch.plan(cache, off, kv, c["table"], 3, **p))          # not a multiple of the heads
    refused(R.EINVAL, lambda: ch.attend(cache, q[:0, :0], out[:0, :0]))              # a refused plan is no plan
    refused(R.EINVAL, lambda: ch.plan(cache, off, kv, c["table"], 4, window=5, causal=False, **p))
    refused(R.EINVAL, lambda: ch.plan(cache, off, kv, c["table"], 4, window=-1, **p))
    refused(R.ECAP, lambda: ch.plan(cache, off, kv, c["table"], 4, n_tokens=6))
    six = make([1] * 3, [3] * 3, 4, 2, 64, 16, BF)
    refused(R.ECAP, lambda: ch.plan(cache, torch.arange(4, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda"),
                                    six["table"], 4, n_tokens=3))
    ch.plan(cache, off, kv, c["table"], 4, **p)
    wide = torch.empty(5, 4, 68, dtype=BF, device="cuda")
    refused(R.EINVAL, lambda: ch.attend(cache, q, wide[..., 1:65]))                  # not on 16 bytes
    refused(R.EINVAL, lambda: ch.attend(cache, q, q[:1].expand(5, 4, 64)))           # a broadcast output
    both = torch.zeros(6, 4, 64, dtype=BF, device="cuda")
    refused(R.EINVAL, lambda: ch.attend(cache, both[:5], both[1:]))                  # overlapping, not the same
    refused(R.EINVAL, lambda: ch.attend(cache, q, out, scale=math.inf))
    refused(R.EINVAL, lambda: ch.attend(cache, q, out, scale=math.nan))
    w = torch.zeros(2, 40, device="cuda")
    refused(R.EINVAL, lambda: ch.weigh(cache, q, None, w, w))
    both_w = torch.zeros(120, device="cuda")
    refused(R.EINVAL, lambda: ch.weigh(cache, q, lse, both_w[:80].view(2, 40), both_w[40:].view(2, 40)))
    other = make([1], [1], 4, 2, 64, 32, BF)
    refused(R.EINVAL, lambda: ch.attend(R.Cache(other["k"], other["v"]), q, out))    # paged differently
    small = R.Cache(c["k"][:2], c["v"][:2])
    refused(R.EINVAL, lambda: ch.attend(small, q, out))                              # fewer pages than planned
    n1, ix = torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty(2, 8, dtype=torch.int32, device="cuda")
    for budget, first, last in ((0, 0, 0), (8, 5, 4), (8, -1, 0), (8, 0, -1)):
        refused(R.EINVAL, lambda: ch.evict(cache, w, c["table"], budget, n1, ix, first=first, last=last))
    for bad in (dict(head_dim=96), dict(page=24), dict(page=8)):
        k = torch.zeros(2, 2, bad.get("page", 16), bad.get("head_dim", 64), dtype=BF, device="cuda")
        refused(R.EINVAL, lambda: ch.plan(R.Cache(k, k), off, kv, c["table"], 4, **p))
    ch.plan(cache, off, kv, c["table"], 4, **p)
    freq = torch.ones(32, device="cuda")
    pos = torch.zeros(2, 5, dtype=torch.int32, device="cuda")
    x = torch.zeros(5, 4, 64, dtype=BF, device="cuda")
    refused(R.EINVAL, lambda: ctx.rope(x, torch.empty_like(x), R.Rotary(torch.ones(33, device="cuda")), pos))
    refused(R.EINVAL, lambda: ctx.rope(x, torch.empty_like(x), R.Rotary(freq, [1] * 32, n_axes=1), pos))
    refused(R.EINVAL, lambda: ctx.rope(both[:5], both[1:], R.Rotary(freq), pos))
    with pytest.raises(TypeError):
        ctx.rope(x.float(), x.float(), R.Rotary(freq), pos)
    with pytest.raises(ValueError):
        ctx.rope(x, torch.empty_like(x)[:4], R.Rotary(freq), pos)
    with pytest.raises(ValueError):
        ch.attend(cache, q[:, :3], out)
    with pytest.raises(ValueError):
        ch.attend(cache, q, out, lse[:4])
    with pytest.raises(ValueError):
        R.Cache(c["k"], c["v"][1:])
    ctx.check("nothing was enqueued")
    ch.close()


@pytest.mark.parametrize("what", ["q_off", "q_off_end", "negative", "long", "page", "max_new", "weight", "dst", "append"])
def test_device_errors(ctx, what):
    """Bad device data is reported, nothing is read or written out of range, and the context goes on."""
    import paper_2609_18703_amd as R
    c = make([2, 3], [20, 40], 4, 2, 64, 16, BF)
    cache = R.Cache(c["k"], c["v"])
    off = torch.tensor([0, 2, 5], device="cuda")
    kv = torch.tensor([20, 40], dtype=torch.int32, device="cuda")
    table, max_new, code = c["table"].clone(), 3, R.ERANGE
    if what == "q_off":
        off[1], code = 9, R.EINVAL
    elif what == "q_off_end":
        off[2], code = 4, R.EINVAL
    elif what == "negative":
        kv[0] = -1
    elif what == "long":
        kv[1] = 16 * table.shape[1] + 1
    elif what == "page":
        table[1, 1] = c["k"].shape[0]
    elif what == "max_new":
        max_new = 2
    elif what == "append":
        kv[0] = 1
    ch = ctx.chunk(2, 5, table.shape[1])
    ch.plan(cache, off, kv, table, 4, n_tokens=5, max_new=max_new)
    q, out, lse = c["q"], torch.empty_like(c["q"]), torch.empty(5, 4, device="cuda")
    w = torch.zeros(2, 39 if what == "weight" else 200, device="cuda")
    dst = torch.full((2, 2), c["k"].shape[0] if what == "dst" else 0, dtype=torch.int32, device="cuda")
    print("device error", what, flush=True)
    if what not in ("weight", "dst", "append"):
        assert ctx.status() == code
    ch.attend(cache, q, out, lse)
    ch.weigh(cache, q, lse, w, w)
    if what == "append":
        ch.append(cache, None, q[:, :2], q[:, :2], None)
    if what == "dst":
        before = c["k"].clone()
        n1, ix = torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty(2, 8, dtype=torch.int32, device="cuda")
        ch.evict(cache, w, dst, 8, n1, ix)
    assert ctx.status() == (code if what in ("weight", "dst", "append") else R.OK)
    if what == "dst":
        assert torch.equal(before.view(torch.int16), c["k"].view(torch.int16))
    ctx.check("cleared")
    ch.close()


def test_own_stream_and_kept_plan():
    """A context on another stream; the plan keeps what it was made from after the caller's arrays change."""
    import paper_2609_18703_amd as R
    stream = torch.cuda.Stream()
    c = make([5, 1], [50, 300], 8, 2, 128, 16, BF, seed=2)
    torch.cuda.synchronize()
    want, _, tol, _ = ref.attend(c, c["k"], c["v"], c["q"], 128 ** -0.5)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        ctx = R.Context()
        cache, ch = plan(ctx, c)
        c["table"].fill_(-1)
        out = torch.empty_like(c["q"])
        for _ in range(3):
            ch.attend(cache, c["q"], out)
    stream.synchronize()
    ctx.check("attend")
    close(out, want, tol, "out")
    ctx.close()


def test_one_plan_after_another(ctx):
    """A plan used for chunks of other shapes in turn: nothing of an earlier one is left."""
    import paper_2609_18703_amd as R
    ch = ctx.chunk(6, 400, 200)
    for i, (new, kv, hq, hk, dim, more) in enumerate([
            ([300, 1], [500, 40], 8, 2, 128, {}), ([1] * 6, [2000, 3, 90, 1, 700, 16], 16, 16, 64, {}),
            ([0], [7], 4, 4, 64, {}), ([40, 40], [41, 900], 28, 4, 128, {"window": 50, "sinks": 2}), ([1], [3001], 8, 1, 128, {})]):
        c = make(new, kv, hq, hk, dim, 16, BF, seed=i, **more)
        cache = R.Cache(c["k"], c["v"])
        off = torch.tensor(c["q_off"], device="cuda")
        ch.plan(cache, off, torch.tensor(kv, dtype=torch.int32, device="cuda"), c["table"], hq, sum(new),
                window=c["window"], sinks=c["sinks"])
        out, lse = torch.empty_like(c["q"]), torch.empty(c["q"].shape[:2], device="cuda")
        print("plan", i, flush=True)
        ch.attend(cache, c["q"], out, lse)
        w = torch.zeros(len(new), max(kv), device="cuda")
        ch.weigh(cache, c["q"], lse, None, w)
        ctx.check("attend")
        want, wl, tol, tl = ref.attend(c, c["k"], c["v"], c["q"], dim ** -0.5)
        close(out, want, tol, "out")
        close(lse, wl, tl, "lse")
        close(w, *ref.weigh(c, c["k"], c["q"], lse, torch.zeros_like(w), dim ** -0.5), "weight")
    ch.close()


def test_captured_step(ctx):
    """Plan, append, attend, weigh and evict in a HIP graph, replayed over changed inputs."""
    import paper_2609_18703_amd as R
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        gctx = R.Context()
        c = make([1, 20, 1], [2000, 60, 9], 8, 2, 128, 16, BF, seed=4, spare=12)
        cache = R.Cache(c["k"].nan_to_num_(), c["v"].nan_to_num_())
        ch = gctx.chunk(3, 22, c["table"].shape[1])
        off = torch.tensor(c["q_off"], device="cuda")
        kv = torch.tensor(c["kv_len"], dtype=torch.int32, device="cuda")
        used = set(c["table"][c["table"] >= 0].tolist())
        dst = torch.tensor([p for p in range(c["k"].shape[0]) if p not in used][:12], dtype=torch.int32,
                           device="cuda").view(3, 4)
        rot = R.Rotary(torch.ones(64, device="cuda") * 0.1)
        pos = torch.arange(22, device="cuda").int()[None]
        qkv = torch.randn(22, 12, 128, device="cuda").to(BF)
        q, out, lse = torch.empty(22, 8, 128, dtype=BF, device="cuda"), torch.empty(22, 8, 128, dtype=BF, device="cuda"), \
            torch.empty(22, 8, device="cuda")
        w = torch.zeros(3, 2000, device="cuda")
        n1, ix = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, 64, dtype=torch.int32, device="cuda")

        def step():
            ch.plan(cache, off, kv, c["table"], 8, n_tokens=22)
            ch.append(cache, qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], q, rot, pos)
            ch.attend(cache, q, out, lse)
            ch.weigh(cache, q, lse, None, w)
            ch.evict(cache, w, dst, 64, n1, ix, first=2, last=8)

        step()
        gctx.check("eager")
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step()
        for i in range(3):
            qkv.copy_(torch.randn(22, 12, 128, device="cuda"))
            kv.copy_(torch.tensor([2000 - 100 * i, 60 - i, 9 - i], dtype=torch.int32))
            got = []
            for f in (graph.replay, step):
                for t in (q, out, lse, w, n1, ix):
                    t.zero_()
                f()
                stream.synchronize()
                got.append([t.clone() for t in (q, out, lse, w, n1, ix, c["k"], c["v"])])
            print("replay", i, flush=True)
            for a, b in zip(*got):
                assert torch.equal(a, b)
            want, _, tol, _ = ref.attend({**c, "kv_len": kv.tolist()}, c["k"], c["v"], q, 128 ** -0.5)
            close(out, want, tol, "out")
        gctx.check("replays")
    torch.cuda.synchronize()
    gctx.close()


def test_offsets_beyond_32_bits(ctx):
    """Pages whose elements lie beyond 2^32 elements into the cache."""
    page, heads, dim = 4096, 2, 128
    per = page * heads * dim
    n_pages = (1 << 32) // per + 3
    k = torch.zeros(n_pages, heads, page, dim, dtype=BF, device="cuda")
    v = torch.zeros(n_pages, heads, page, dim, dtype=BF, device="cuda")
    import paper_2609_18703_amd as R
    kv = [4100]
    table = torch.tensor([[n_pages - 2, n_pages - 1]], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    for p in (n_pages - 2, n_pages - 1):
        k[p] = torch.randn(heads, page, dim, generator=g, device="cuda").to(BF)
        v[p] = torch.randn(heads, page, dim, generator=g, device="cuda").to(BF)
    c = dict(new=[4], kv_len=kv, q_off=[0, 4], page=page, causal=True, window=0, sinks=0, table=table, q_heads=8, k=k, v=v)
    c["q"] = torch.randn(4, 8, dim, generator=g, device="cuda").to(BF)
    cache, ch = plan(ctx, c)
    out, lse = torch.empty_like(c["q"]), torch.empty(4, 8, device="cuda")
    print("far pages", n_pages, flush=True)
    ch.attend(cache, c["q"], out, lse)
    want, wl, tol, tl = ref.attend(c, k, v, c["q"], dim ** -0.5)
    close(out, want, tol, "out")
    close(lse, wl, tl, "lse")
    w = torch.zeros(1, 4100, device="cuda")
    ch.weigh(cache, c["q"], lse, None, w)
    close(w, *ref.weigh(c, k, c["q"], lse, torch.zeros_like(w), dim ** -0.5), "weight")
    dst = torch.tensor([[n_pages - 3]], dtype=torch.int32, device="cuda")
    n1, ix = torch.empty(1, dtype=torch.int32, device="cuda"), torch.empty(1, 50, dtype=torch.int32, device="cuda")
    ch.evict(cache, w, dst, 50, n1, ix, last=3)
    ctx.check("far pages")
    keep = ref.kept(w[0], 4100, 50, 0, 3)
    assert ix[0].tolist() == keep
    src, slot = (a[torch.tensor(keep, device="cuda")] for a in ref.positions(c, 0))
    assert torch.equal(k[n_pages - 3, :, :50], k[src, :, slot].permute(1, 0, 2))
    ch.close()


@pytest.mark.parametrize("what", ["max_new", "page"])
def test_short_sequences_beside_invalid_ones(ctx, what):
    """An invalid sequence counts as empty; one that is shorter than the arguments promise is computed all the same."""
    import paper_2609_18703_amd as R
    new, kv = [60, 1, 39], [80, 50, 70]
    c = make(new, kv, 4, 2, 64, 16, BF, seed=12)
    cache = R.Cache(c["k"], c["v"])
    off = torch.tensor(c["q_off"], device="cuda")
    table, max_new = c["table"].clone(), 60
    if what == "max_new":                        # with 39 at most, no sequence could have fewer than 22 tokens
        max_new = 39
    else:
        table[2, 0] = c["k"].shape[0]
    ch = ctx.chunk(3, 100, table.shape[1])
    ch.plan(cache, off, torch.tensor(kv, dtype=torch.int32, device="cuda"), table, 4, n_tokens=100, max_new=max_new)
    assert ctx.status() == R.ERANGE
    out, lse = torch.zeros_like(c["q"]), torch.zeros(100, 4, device="cuda")
    print("beside invalid ones", what, flush=True)
    ch.attend(cache, c["q"], out, lse)
    w = torch.zeros(3, 80, device="cuda")
    ch.weigh(cache, c["q"], lse, None, w)
    ctx.check("attend")
    want, wl, tol, tl = ref.attend(c, c["k"], c["v"], c["q"], 64 ** -0.5)
    ww, wt = ref.weigh(c, c["k"], c["q"], lse, torch.zeros_like(w), 64 ** -0.5)
    for s in ((1, 2) if what == "max_new" else (0, 1)):
        t = slice(c["q_off"][s], c["q_off"][s + 1])
        close(out[t], want[t], tol[t], "out")
        close(lse[t], wl[t], tl[t], "lse")
        close(w[s], ww[s], wt[s], "weight")
    ch.close()


@pytest.mark.parametrize("new,kv", [([1, 9], [70, 200]), ([150], [300])])
def test_widest_window(ctx, new, kv):
    """A window as wide as its type allows hides nothing."""
    got = []
    for window in (0, 2 ** 31 - 1):
        c = make(new, kv, 4, 2, 64, 16, BF, window=window, sinks=2 ** 31 - 1 if window else 0, seed=13)
        cache, ch = plan(ctx, c)
        out, lse = torch.empty_like(c["q"]), torch.empty(sum(new), 4, device="cuda")
        w = torch.zeros(len(new), max(kv), device="cuda")
        print("widest window", new, window, flush=True)
        ch.attend(cache, c["q"], out, lse)
        ch.weigh(cache, c["q"], lse, None, w)
        ctx.check("attend")
        got.append((out, lse, w))
        ch.close()
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("new,kv", [([1, 1], [200, 70]), ([90], [90])])
def test_infinite_value_of_no_weight(ctx, new, kv):
    """A weight too small for its type does not turn a value's infinity into a NaN, where a row sees it."""
    c = make(new, kv, 4, 2, 64, 16, BF, seed=14)
    for s in range(len(new)):
        page, slot = ref.positions(c, s)
        c["k"][page, :, slot] = 0.0
        c["k"][page[0], :, slot[0]] = -60.0
        c["v"][page[0], :, slot[0], ::5] = math.inf
    c["q"] = c["q"].abs() + 1
    cache, ch = plan(ctx, c)
    out = torch.empty_like(c["q"])
    print("infinite value", new, flush=True)
    ch.attend(cache, c["q"], out)
    ctx.check("attend")
    alone = [t for t, p in ((c["q_off"][s], kv[s] - new[s]) for s in range(len(new))) if p == 0]
    rest = torch.tensor([t for t in range(sum(new)) if t not in alone], device="cuda")
    assert torch.equal(out[rest].isposinf(), torch.arange(64, device="cuda").remainder(5).eq(0).expand_as(out[rest]))
    ch.close()


def test_append_refuses_overlap(ctx):
    import paper_2609_18703_amd as R
    c = make([2, 3], [20, 40], 4, 2, 64, 16, BF)
    cache, ch = plan(ctx, c)
    qkv = torch.zeros(5, 8, 64, dtype=BF, device="cuda")
    q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    for out in (qkv[:, 4:], qkv[:, 2:6], qkv[:, 3:7]):
        with pytest.raises(R.RoError) as e:
            ch.append(cache, q, k, v, out)
        assert e.value.code == R.EINVAL
    ch.append(cache, q, k, v, q)
    n1 = torch.empty(16, dtype=torch.int32, device="cuda")
    with pytest.raises(R.RoError):               # the new lengths inside the new weights
        ch.evict(cache, torch.zeros(2, 40, device="cuda"), c["table"], 8, n1[:2], torch.empty(2, 8, dtype=torch.int32, device="cuda"),
                 n1.view(2, 8))
    ctx.check("append")
    ch.close()


@pytest.mark.parametrize("wide_table", [False, True])
@pytest.mark.parametrize("new,kv,heads,dim,more", [
    ([1, 70, 3, 0, 16, 1], [900, 200, 40, 50, 16, 3000], (8, 2), 128, {}),
    ([17, 1, 1], [700, 1500, 1], (4, 4), 64, {"window": 100, "sinks": 70}),
    ([40, 2], [6000, 9000], (7, 1), 128, {})])
def test_short_sequences_beside_long_ones(ctx, new, kv, heads, dim, more, wide_table):
    """Short sequences in wide tiles, and in narrow ones, which tables of many columns (no pages in most) call for."""
    c = make(new, kv, *heads, dim, 16, BF, seed=15, **more)
    if wide_table:                               # more than 2^30 bytes of keys and values, if all columns had pages
        cols = (1 << 30) // (len(new) * 16 * heads[1] * dim * 4) + 2
        table = torch.full((len(new), cols), -1, dtype=torch.int32, device="cuda")
        table[:, :c["table"].shape[1]] = c["table"]
        c["table"] = table
    cache, ch = plan(ctx, c)
    out, lse = torch.empty_like(c["q"]), torch.empty(c["q"].shape[:2], device="cuda")
    w = torch.zeros(len(new), max(kv), device="cuda")
    print("short beside long", new, kv, wide_table, flush=True)
    for _ in range(2):                           # the second call finds what the first left
        out.fill_(math.nan)
        ch.attend(cache, c["q"], out, lse)
    ch.weigh(cache, c["q"], lse, None, w)
    ctx.check("attend")
    want, wl, tol, tl = ref.attend(c, c["k"], c["v"], c["q"], dim ** -0.5)
    close(out, want, tol, "out")
    close(lse, wl, tl, "lse")
    close(w, *ref.weigh(c, c["k"], c["q"], lse, torch.zeros_like(w), dim ** -0.5), "weight")
    ch.close()
