"""Attention over a paged cache where values are large, infinite or NaN:
scores far beyond what 32 bits tell apart, and what must not reach a row."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import chunk_ref as ref  # noqa: E402
from test_gpu_chunk import BF, HF, close, ctx, make, plan  # noqa: E402,F401

FACTORS = 61


def far_case(new, kv, heads, dim, dtype, score, order, sign=1.0, **more):
    """Scores are whole multiples, up to 61, of a unit; the largest is about `score`.  Every row is won by the
    positions of the largest multiple that it sees (of the smallest where scores are negative): their scores are
    equal to the last bit, and the next ones lie score / 61 below."""
    c = make(new, kv, *heads, dim, 16, dtype, seed=21, **more)
    qk = score / dim ** 0.5
    b = min(10, math.floor(math.log2(qk) / 2) - 5)
    qv = torch.tensor(qk / (FACTORS * 2.0 ** b)).to(dtype)
    assert qv.isfinite()
    c["q"] = torch.full_like(c["q"], float(qv) * sign)
    for s, L in enumerate(kv):
        j = torch.arange(L, device="cuda")
        f = {"rising": 1 + FACTORS * j // L, "falling": FACTORS - FACTORS * j // L, "mixed": 1 + j * 37 % FACTORS}[order]
        page, slot = ref.positions(c, s)
        c["k"][page, :, slot] = (f * 2.0 ** b).to(dtype)[:, None, None]
    return c


def winners(c, dim):
    """(out, lse) in 64 bits: the mean of the values of the positions that win a row, and their score with the
    logarithm of their number.  (The logarithm of a sum of exponentials of such scores loses that number.)"""
    T, Hq, D = c["q"].shape
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device="cuda")
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device="cuda")
    group = Hq // c["k"].shape[1]
    for s, n in enumerate(c["new"]):
        t0, L = c["q_off"][s], c["kv_len"][s]
        page, slot = ref.positions(c, s)
        see = ref.visible(n, L, c["causal"], c["window"], c["sinks"], "cuda")
        for h in range(Hq):
            kk, vv = c["k"][page, h // group, slot].double(), c["v"][page, h // group, slot].double()
            x = (c["q"][t0:t0 + n, h].double()[:, :1] * kk[:, 0] * dim).masked_fill(~see, -math.inf)   # all elements alike
            best = x.amax(1, keepdim=True)
            won = ((x == best) & see).double()
            out[t0:t0 + n, h] = won @ vv / won.sum(1, keepdim=True)
            lse[t0:t0 + n, h] = best[:, 0] * dim ** -0.5 + won.sum(1).log()
    return out, lse


def attend_far(ctx, c, dim, what):
    cache, ch = plan(ctx, c)
    out, lse = torch.full_like(c["q"], 7.0), torch.full(c["q"].shape[:2], 7.0, device="cuda")
    print("far scores", what, flush=True)
    ch.attend(cache, c["q"], out, lse)
    ctx.check("attend")
    want, wl = winners(c, dim)
    # The winners' weights are equal, the others' below e^-60: 2 u as for any weights (both factors of 16 bits).  Sums
    # of D products in 32 bits are off by D 2^-24 of the score.
    big = c["v"].nan_to_num().abs().max().double()
    close(out, want, 2 * ref.U[c["dtype"]] * big.expand_as(want), "out")
    close(lse, wl, 1.0 + dim * 2.0 ** -23 * wl.abs(), "lse")
    ch.close()


@pytest.mark.parametrize("order,sign", [("rising", 1.0), ("falling", 1.0), ("mixed", 1.0), ("mixed", -1.0)])
@pytest.mark.parametrize("dtype,score", [(HF, 2.0 ** e) for e in (12, 14, 20, 28, 30, 34)] + [(BF, 2.0 ** e) for e in (28, 31, 36, 90)])
@pytest.mark.parametrize("new,kv,heads,dim", [([70], [300], (8, 2), 64), ([20], [2500], (7, 1), 128)])
def test_far_scores_of_many_rows(ctx, new, kv, heads, dim, dtype, score, order, sign):
    c = far_case(new, kv, heads, dim, dtype, score, order, sign)
    attend_far(ctx, c, dim, (new, kv, dim, dtype, score, order, sign))


def test_far_scores_in_a_window(ctx):
    c = far_case([90, 17], [400, 60], (8, 2), 128, HF, 2.0 ** 30, "mixed", window=40, sinks=3)
    attend_far(ctx, c, 128, "window")


@pytest.mark.parametrize("order,sign", [("rising", 1.0), ("falling", 1.0), ("mixed", 1.0), ("mixed", -1.0)])
@pytest.mark.parametrize("dtype,score", [(HF, 2.0 ** e) for e in (12, 14, 20, 28, 30, 34)] + [(BF, 2.0 ** e) for e in (28, 31, 36, 90)])
@pytest.mark.parametrize("new,kv,heads,dim", [([1, 2, 1], [300, 64, 1], (8, 2), 64), ([1], [2500], (7, 1), 128)])
def test_far_scores_of_few_rows(ctx, new, kv, heads, dim, dtype, score, order, sign):
    c = far_case(new, kv, heads, dim, dtype, score, order, sign)
    attend_far(ctx, c, dim, (new, kv, dim, dtype, score, order, sign))


def test_far_scores_of_few_rows_in_a_window(ctx):
    c = far_case([1, 2], [400, 60], (8, 2), 128, HF, 2.0 ** 30, "mixed", window=40, sinks=3)
    attend_far(ctx, c, 128, "window")


@pytest.mark.parametrize("new,kv,heads,dim,light", [
    ([1], [200], (4, 2), 64, 64), ([1, 2], [200, 300], (4, 2), 128, 32), ([1], [200], (4, 2), 64, 32),
    ([1], [9000], (7, 1), 128, 4500), ([2], [9000], (7, 1), 64, 100),
    ([60], [200], (4, 2), 64, 64), ([20], [9000], (7, 1), 128, 4500), ([20], [9000], (7, 1), 64, 100)])
def test_infinite_values_far_below_the_rest(ctx, new, kv, heads, dim, light):
    """Infinities at positions whose weights are far too small for 32 bits: in a half tile of their own, in a tile,
    in a part of rows that several workgroups share."""
    c = make(new, kv, *heads, dim, 16, BF, seed=31)
    c["q"] = c["q"].abs() + 1
    plain = c["v"].clone()
    for s in range(len(new)):
        page, slot = ref.positions(c, s)
        c["k"][page, :, slot] = 0.0
        c["k"][page[:light], :, slot[:light]] = -60.0
        for j, at, x in ((3, 0, math.inf), (5, 1, -math.inf), (light - 1, 0, math.inf), (7, 2, math.inf), (9, 2, -math.inf)):
            c["v"][page[j], :, slot[j], at::7] = x
            plain[page[j], :, slot[j], at::7] = 0.0
    cache, ch = plan(ctx, c)
    out, lse = torch.empty_like(c["q"]), torch.empty(c["q"].shape[:2], device="cuda")
    print("far below", new, kv, light, flush=True)
    ch.attend(cache, c["q"], out, lse)
    ctx.check("attend")
    want, wl, tol, tl = ref.attend(c, c["k"], plain, c["q"], dim ** -0.5)      # (their weights are nothing to a finite sum)
    d = torch.arange(dim, device="cuda") % 7
    for at, x in ((0, math.inf), (1, -math.inf), (2, math.nan)):
        want[..., d == at] = x
    close(lse, wl, tl, "lse")
    close(out, want, tol, "out")
    ch.close()


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
@pytest.mark.parametrize("new,kv,heads,dim,bad", [
    ([100, 30], [300, 31], (8, 2), 128, [50, 110]), ([150], [300], (4, 1), 64, [70]),
    ([4, 1], [200, 70], (4, 2), 128, [1]), ([3], [900], (8, 2), 64, [0])])
def test_weights_of_a_row_that_is_not_finite(ctx, new, kv, heads, dim, bad, window, sinks):
    """A token with NaN in its query, whose lse is NaN: positions that it does not see keep their weights."""
    c = make(new, kv, *heads, dim, 16, BF, window=window, sinks=sinks, seed=33)
    c["q"][bad, :, 3] = math.nan
    cache, ch = plan(ctx, c)
    lse = ref.attend(c, c["k"], c["v"], c["q"], dim ** -0.5)[1].float()
    assert lse[bad].isnan().all()
    w = torch.zeros(len(new), max(kv), device="cuda")
    print("weights beside NaN", new, kv, window, flush=True)
    ch.weigh(cache, c["q"], lse, None, w)
    ctx.check("weigh")
    seen = torch.zeros_like(w, dtype=torch.bool)
    for t in bad:
        s = max(i for i in range(len(new)) if c["q_off"][i] <= t)
        see = ref.visible(new[s], kv[s], True, window, sinks, "cuda")[t - c["q_off"][s]]
        seen[s, :kv[s]] |= see
    assert torch.equal(w.isnan(), seen)
    lse[bad] = -math.inf                         # (adds nothing to the others)
    c["q"][bad] = 0.0
    want, tol = ref.weigh(c, c["k"], c["q"], lse, torch.zeros_like(w), dim ** -0.5)
    close(w[~seen], want[~seen], tol[~seen], "weight")
    ch.close()


@pytest.mark.parametrize("window", [0, 40])
def test_weights_of_repeated_rows(ctx, window):
    """Seven heads a key / value head: tiles of rows have one that repeats the last.  Whatever token that is the row
    of, positions behind it keep their weights."""
    new, kv = [30, 11], [140, 60]
    for t in (8, 17, 26, 29, 38, 40):
        c = make(new, kv, 7, 1, 128, 16, BF, window=window, seed=34)
        lse = ref.attend(c, c["k"], c["v"], c["q"], 128 ** -0.5)[1].float()
        c["q"][t, :, 5] = math.nan
        lse[t] = math.nan
        cache, ch = plan(ctx, c)
        w = torch.zeros(2, 140, device="cuda")
        print("repeated rows", t, window, flush=True)
        ch.weigh(cache, c["q"], lse, None, w)
        ctx.check("weigh")
        s = int(t >= 30)
        seen = torch.zeros_like(w, dtype=torch.bool)
        seen[s, :kv[s]] = ref.visible(new[s], kv[s], True, window, 0, "cuda")[t - c["q_off"][s]]
        assert torch.equal(w.isnan(), seen)
        ch.close()


@pytest.mark.parametrize("new,kv,heads,dim,idle", [
    ([100, 30], [600, 31], (8, 2), 128, [0, 50, 110]), ([150], [1200], (7, 1), 64, [70, 149]),
    ([4, 1], [200, 70], (4, 2), 128, [1, 4]), ([3], [900], (8, 2), 64, [0]), ([2, 2], [90, 700], (6, 3), 64, [0, 3])])
def test_rows_without_weight_may_hold_anything(ctx, new, kv, heads, dim, idle):
    """A row whose lse is -inf adds nothing, whatever its query holds."""
    c = make(new, kv, *heads, dim, 16, BF, seed=35)
    lse = ref.attend(c, c["k"], c["v"], c["q"], dim ** -0.5)[1].float()
    lse[idle] = -math.inf
    got = []
    for fill in (0.0, math.nan, math.inf, -math.inf):
        c["q"][idle] = fill
        cache, ch = plan(ctx, c)
        w = torch.zeros(len(new), max(kv), device="cuda")
        print("rows without weight", new, kv, fill, flush=True)
        ch.weigh(cache, c["q"], lse, None, w)
        ctx.check("weigh")
        got.append(w)
        ch.close()
    c["q"][idle] = 0.0
    close(got[0], *ref.weigh(c, c["k"], c["q"], lse, torch.zeros_like(got[0]), dim ** -0.5), "weight")
    for w in got[1:]:
        assert torch.equal(w, got[0])


@pytest.mark.parametrize("dtype,score", [(HF, 2.0 ** e) for e in (14, 20, 28, 33)] + [(BF, 2.0 ** e) for e in (28, 31, 36, 90)])
@pytest.mark.parametrize("new,kv,heads,dim", [([90], [250], (8, 2), 64), ([40, 3], [250, 90], (7, 1), 128),
                                              ([1, 2], [250, 90], (8, 4), 128), ([2, 1], [60, 250], (6, 3), 64)])
def test_weights_of_far_scores(ctx, new, kv, heads, dim, dtype, score):
    """Scores that are exact in 32 bits, one position of each row far above the others: it gets a weight of one."""
    c = make(new, kv, *heads, dim, 16, dtype, seed=37)
    b = min(8, math.floor(math.log2(score / dim) / 2) - 4)
    a = math.log2(score * 8 / (256 * dim)) - b
    c["q"] = torch.full_like(c["q"], 2.0 ** math.floor(a))
    want = torch.zeros(len(new), max(kv), dtype=torch.float64, device="cuda")
    for s, (n, L) in enumerate(zip(new, kv)):
        page, slot = ref.positions(c, s)
        f = 1 + torch.arange(L, device="cuda") * 37 % 251           # all different, exact in 8 bits
        c["k"][page, :, slot] = (f * 2.0 ** b).to(dtype)[:, None, None]
        won = f.double().expand(n, L).masked_fill(~ref.visible(n, L, True, 0, 0, "cuda"), 0.0).argmax(1)
        want[s].index_add_(0, won, torch.full((n,), float(heads[0]), dtype=torch.float64, device="cuda"))
    assert c["q"].isfinite().all()
    cache, ch = plan(ctx, c)
    out, lse = torch.empty_like(c["q"]), torch.empty(c["q"].shape[:2], device="cuda")
    w = torch.zeros(len(new), max(kv), device="cuda")
    print("weights of far scores", new, kv, dim, dtype, score, flush=True)
    ch.attend(cache, c["q"], out, lse, scale=0.125)
    ch.weigh(cache, c["q"], lse, None, w, scale=0.125)
    ctx.check("weigh")
    won = want > 0
    close(w[won], want[won], 2.0 ** -20 * want[won], "weight")      # (a weight of one in the exponent's last place)
    other, tol = ref.weigh(c, c["k"], c["q"], lse, torch.zeros_like(w), 0.125)
    other = other.float().double()                                  # what 32 bits hold of weights down to 10^-10000
    close(w[~won], other[~won], tol[~won], "weight of nothing")     # (e^-64 where scores are smallest)
    ch.close()


@pytest.mark.parametrize("window", [0, 5000])
@pytest.mark.parametrize("heads", [(2, 1), (4, 2), (6, 3), (16, 4), (20, 5), (40, 20)])
def test_weights_before_of_single_tokens(ctx, heads, window):
    """The weights before, of many tiles in a row, for every way that waves share heads and tiles."""
    new, kv = [1] * 40, [20000 - 491 * s for s in range(40)]
    c = make(new, kv, *heads, 64, 256, HF, window=window, sinks=100 if window else 0, seed=41)
    cache, ch = plan(ctx, c)
    before = (torch.arange(40 * 20000, device="cuda") % 16384).float().view(40, 20000)
    lse = torch.full((40, heads[0]), math.inf, device="cuda")       # no token adds anything
    w = torch.full_like(before, -1.0)
    print("weights before", heads, window, flush=True)
    ch.weigh(cache, c["q"], lse, before, w)
    ctx.check("weigh")
    for s, L in enumerate(kv):
        assert torch.equal(w[s, :L], before[s, :L]) and (w[s, L:] == -1.0).all()
    ch.close()


@pytest.mark.parametrize("new,kv,off", [([5, 5, 5], [20, 30, 40], [0, 5, 0, 5]), ([40, 40], [50, 60], None)])
def test_overlapping_sequences(ctx, new, kv, off):
    """Offsets that fall, so that two sequences have the same tokens: an error, and nothing is computed or written."""
    import paper_2609_18703_amd as R
    c = make(new, kv, 4, 2, 64, 16, BF, seed=43)
    S, T = len(new), sum(new)
    off = off or [0, T, 0] + [T]                 # (the second of three sequences falls)
    if len(off) - 1 > S:
        c["table"] = c["table"][[0, 1, 1]].contiguous()
        kv = [*kv, kv[-1]]
    S, T = len(off) - 1, off[-1]
    cache = R.Cache(c["k"], c["v"])
    ch = ctx.chunk(S, T, c["table"].shape[1])
    ch.plan(cache, torch.tensor(off, device="cuda"), torch.tensor([max(x, T) for x in kv], dtype=torch.int32, device="cuda"),
            torch.where(c["table"] < 0, 0, c["table"]), 4, n_tokens=T)
    print("overlapping", off, flush=True)
    assert ctx.status() == R.EINVAL
    q = c["q"][:T].contiguous()
    out, lse = torch.full_like(q, 7.0), torch.full((T, 4), 7.0, device="cuda")
    w, k0 = torch.full((S, 200), 7.0, device="cuda"), c["k"].clone()
    n1, ix = torch.full((S,), 7, dtype=torch.int32, device="cuda"), torch.full((S, 8), 7, dtype=torch.int32, device="cuda")
    ch.append(cache, None, q[:, :2], q[:, :2], None)
    ch.attend(cache, q, out, lse)
    ch.weigh(cache, q, lse, None, w)
    ch.evict(cache, w, torch.zeros(S, 1, dtype=torch.int32, device="cuda"), 8, n1, ix)
    ctx.check("nothing to do")
    assert (out == 7.0).all() and (lse == 7.0).all() and (w == 7.0).all()
    assert torch.equal(k0.view(torch.int16), c["k"].view(torch.int16))
    assert (n1 == 0).all() and (ix == -1).all()
    ch.close()


def test_after_a_refused_allocation(ctx):
    """A plan too large for the GPU is refused, and the next call, of whatever library, knows nothing of it."""
    import paper_2609_18703_amd as R
    with pytest.raises(R.RoError) as e:
        ctx.chunk(1 << 20, 8, 1 << 20)           # 2^42 bytes of page numbers
    assert e.value.code == R.EHIP
    c = make([1, 9], [40, 30], 4, 2, 64, 16, BF, seed=45)
    cache, ch = plan(ctx, c)
    with pytest.raises(R.RoError):
        ctx.chunk(1 << 20, 8, 1 << 20)
    out = torch.empty_like(c["q"])
    ch.attend(cache, c["q"], out)
    ctx.check("attend")
    want, _, tol, _ = ref.attend(c, c["k"], c["v"], c["q"], 64 ** -0.5)
    close(out, want, tol, "out")
    ch.close()
