"""The choice of tokens against its definition: equal tokens."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import step_ref as ref  # noqa: E402

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_18703_amd as R
    return R.Context()


def check(ctx, logits, u, mask=None, **how):
    """how: lists, one entry a row.  mask: booleans [rows, vocab]."""
    n, V = logits.shape
    dev = {k: torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in how.items()}
    if mask is not None:
        words = (V + 31) // 32
        bits = np.zeros((n, words * 32), np.uint8)
        bits[:, :V] = mask
        bits[:, V:] = 1                          # what lies behind the vocabulary says nothing
        dev["mask"] = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).cuda()
    uu = torch.tensor(u, dtype=torch.float32, device="cuda")
    token = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    logprob = torch.full((n,), 9.0, device="cuda")
    ctx.sample(logits, uu, token, logprob, **dev)
    bad = any(not 0 <= t < math.inf for t in how.get("temperature", [])) or \
        any(x != x for k in ("top_p", "min_p") for x in how.get(k, []))
    import paper_2609_18703_amd as R
    assert ctx.status() == (R.EINVAL if bad else R.OK)
    got, lp = token.tolist(), logprob.cpu().double().tolist()
    rows = logits.double().cpu().numpy()
    uu = uu.double().tolist()
    host = {k: dev[k].double().tolist() for k in how}
    for r in range(n):
        want = ref.sample(rows[r], uu[r], allowed=None if mask is None else mask[r], **{k: host[k][r] for k in how})
        assert got[r] == want[0], (r, got[r], want, {k: host[k][r] for k in how})
        # the logarithm in 64 bits (sums of up to 2^20 numbers), rounded to 32
        if math.isinf(want[1]):
            assert lp[r] == want[1]
        else:
            assert abs(lp[r] - want[1]) <= 2.0 ** -24 * abs(want[1]) + 1e-12 * (1 + abs(want[1]))
    ctx.sample(logits, torch.tensor(u, dtype=torch.float32, device="cuda"), token2 := torch.empty_like(token), None, **dev)
    ctx.status()
    assert token2.tolist() == got
    return got


HOW = dict(temperature=[1.0, 0.7, 0.0, 1.3, 0.3, 5.0, 0.05], top_k=[0, 50, 0, 20, 1, 1000, 3, -1],
           top_p=[1.0, 0.9, 0.95, 0.5, 0.999, 0.0, 1e-7, 2.0, 0.99999], min_p=[0.0, 0.05, 0.0, 1.0, 1e-6, 0.3])


def turn(n, at=0):
    return {k: [v[(r + at) % len(v)] for r in range(n)] for k, v in HOW.items()}


def normal(n, V, dtype, seed, spread=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(n, V, generator=g, device="cuda") * spread).to(dtype), \
        torch.rand(n, generator=g, device="cuda").tolist()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 63, 64, 65, 511, 513, 1000, 8191, 8193, 32003, 70001, 150001])
def test_sample(ctx, V, dtype):
    n = 64 if V < 10000 else 24
    x, u = normal(n, V, dtype, V)
    check(ctx, x, u, **turn(n, V))
    check(ctx, x, u)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("spread", [0.01, 0.3, 30.0, 2000.0])
def test_sample_spreads(ctx, spread, dtype):
    x, u = normal(63, 3001, dtype, 5, spread)
    check(ctx, x, u, **turn(63, 3))


@pytest.mark.parametrize("name", list(HOW))
def test_sample_one_filter(ctx, name):
    x, u = normal(40, 5003, BF, 11)
    check(ctx, x, u, **{name: turn(40)[name]})


def test_sample_all_random_numbers(ctx):
    """Over evenly spaced u every token comes as often as its weight says."""
    n, V = 4096, 11
    x = torch.tensor([[3.0, 1.0, 2.0, 2.0, -1.0, 0.5, 2.0, -3.0, 1.0, 0.0, 3.0]]).repeat(n, 1).to(HF).cuda()
    u = [(i + 0.5) / n for i in range(n)]
    got = check(ctx, x, u)
    p = torch.softmax(x[0].double(), 0).cpu()
    count = torch.bincount(torch.tensor(got), minlength=V)
    assert ((count.double() - n * p).abs() <= 1.0).all()


def test_sample_random_numbers_at_the_ends(ctx):
    x, _ = normal(9, 777, BF, 2)
    edge = [0.0, 1 - 2.0 ** -24, 1.0, 2.0, -1.0, math.nan, math.inf, -math.inf, 1e-38]
    for at in range(3):
        check(ctx, x, edge, **turn(9, at))
    check(ctx, x, edge)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("V", [5, 32, 33, 1000, 66000])
def test_sample_masks(ctx, V, dtype):
    n = 24
    x, u = normal(n, V, dtype, V + 1)
    r = np.random.default_rng(V)
    mask = r.random((n, V)) < np.array([0.02, 0.5, 1.0, 0.0])[np.arange(n) % 4][:, None]
    mask[5] = False
    mask[5, V - 1] = True
    mask[6] = False
    mask[6, 0] = True
    check(ctx, x, u, mask=mask, **turn(n))
    check(ctx, x[:, 1:], u, mask=mask[:, 1:])                     # rows at odd places


def test_sample_mask_stride(ctx):
    x, u = normal(3, 100, BF, 8)
    words = torch.full((3, 9), -1, dtype=torch.int32, device="cuda")
    words[:, 2:6] = torch.tensor([[1, 0, 0, 0], [0, 2, 0, 0], [0, 0, 0, 8]], dtype=torch.int32, device="cuda")
    token = torch.empty(3, dtype=torch.int32, device="cuda")
    ctx.sample(x, torch.tensor(u, device="cuda"), token, mask=words[:, 2:6])
    ctx.check()
    assert token.tolist() == [0, 33, 99]


@pytest.mark.parametrize("dtype", [BF, HF])
def test_sample_values(ctx, dtype):
    """Infinities, NaN, the lowest numbers, zeros of both signs, equal rows."""
    V = 1234
    x, u = normal(16, V, dtype, 77)
    low = torch.finfo(dtype).min
    x[0] = -math.inf
    x[1] = math.nan
    x[2, ::2] = math.nan
    x[3, 5:] = -math.inf
    x[4, 100:] = low
    x[5] = low
    x[6, [7, 70, 700]] = math.inf
    x[7] = math.inf
    x[8] = 0.0
    x[8, ::3] = -0.0
    x[9] = 2.5
    x[10] = torch.finfo(dtype).max
    x[11] = x[11].abs() * 1e-4
    x[11, ::2] *= -1
    x[12, 0], x[12, 1:] = 100.0, -100.0
    x[13, :] = low
    x[13, 9] = -math.inf
    x[14, 3] = torch.finfo(dtype).max
    x[15] = torch.finfo(dtype).smallest_normal / 8 * torch.arange(V, device="cuda").remainder(5).to(dtype)
    for at in range(7):
        check(ctx, x, u, **turn(16, at))
    check(ctx, x, u)
    for t in (1e-45, 1e-30, 1e-3, 1e4, 1e30, 3e38):
        check(ctx, x, u, temperature=[t] * 16)
        check(ctx, x, u, temperature=[t] * 16, top_p=[0.7] * 16, min_p=[0.01] * 16)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_sample_many_equal(ctx, dtype):
    """More tokens of one value than 16 bits count, and as many as they do."""
    V = 200003
    x = torch.zeros(12, V, dtype=dtype, device="cuda")
    x[1] = 1.5
    x[2, :65535] = 1.0
    x[2, 65535:] = -40.0
    x[3, :65536] = 1.0
    x[4, 1:65538] = 1.0
    x[5, ::2] = 1.0
    x[6, ::2] = -1.0
    x[7, 5] = 3.0
    x[8] = torch.finfo(dtype).min
    x[8, 40:45] = 2.0
    x[9, :131072] = 1.0
    x[9, 131072:] = 0.5
    x[10, :131071] = -1.0
    x[11, :65536], x[11, 65536:131072], x[11, 131072:] = 1.0, 1.0078125, 0.9921875
    u = [0.0, 0.1, 0.3, 0.5, 0.7, 0.9, 0.99, 0.999, 0.2, 0.6, 0.8, 0.45]
    for at in range(4):
        check(ctx, x, u, **turn(12, at))
    check(ctx, x, u)


def test_sample_largest(ctx):
    V = 1 << 20
    x, u = normal(3, V, HF, 9)
    check(ctx, x, u, **turn(3))
    check(ctx, x, u)


@pytest.mark.parametrize("off", range(8))
def test_sample_any_place(ctx, off):
    """Rows that begin at any element, and end at any."""
    room, u = normal(6, 1031, BF, off)
    for V in (1, 5, 8, 1000 + off):
        check(ctx, room[:, off:off + V], u, **turn(6, off))


def test_sample_bad_parameters(ctx):
    x, u = normal(8, 100, BF, 1)
    check(ctx, x, u, temperature=[1.0, -1.0, math.nan, math.inf, 0.5, 1.0, -0.0, 1.0])
    check(ctx, x, u, top_p=[1.0, math.nan] * 4)
    check(ctx, x, u, min_p=[math.nan, 0.1] * 4)


def test_sample_rows_and_more(ctx):
    """Two thousand rows; outputs behind the rows stay."""
    x, u = normal(2000, 257, HF, 4)
    check(ctx, x, u, **turn(2000))
    token = torch.full((5,), -7, dtype=torch.int32, device="cuda")
    lp = torch.full((5,), 9.0, device="cuda")
    ctx.sample(x[:3], torch.tensor(u, device="cuda"), token, lp)
    ctx.check()
    assert token[3:].tolist() == [-7, -7] and lp[3:].tolist() == [9.0, 9.0]


def whole_rows(ctx, x, u, mask, **how):
    """As check does, with so many rows that none of them is cut; the rows' tokens and logprobs."""
    n, V = x.shape
    many = 1000
    turns = torch.arange(many, device="cuda") % n
    rows = torch.empty(many, V, dtype=x.dtype, device="cuda")
    torch.index_select(x, 0, turns, out=rows)
    dev = {k: v[turns].contiguous() for k, v in how.items()}
    if mask is not None:
        dev["mask"] = mask[turns].contiguous()
    token, lp = torch.empty(many, dtype=torch.int32, device="cuda"), torch.empty(many, device="cuda")
    ctx.sample(rows, u[turns].contiguous(), token, lp, **dev)
    ctx.check()
    return token[:n], lp[:n]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("V,off", [(131072, 0), (131073, 0), (131073, 5), (150001, 3), (262144, 7), (500009, 1)])
def test_sample_slices(ctx, V, off, dtype):
    """Rows that are cut into slices: by the definition, and as whole rows to the bit."""
    n = 9
    room, u = normal(n, V + off, dtype, V + off)
    x = room[:, off:]
    x[1] = float("-inf")
    x[1, 131071 - off] = 0.5                     # one candidate, in one slice
    x[2, V - 1] = 90.0                           # the others out of its reach
    x[3, ::3] = math.nan
    x[3, 40000:110000] = math.nan                # slices of nothing else
    x[4, V // 2:] = float("inf")
    x[5] = float("-inf")
    x[6] = 0.25
    mask = np.ones((n, V), bool)
    mask[7, :100000] = False
    mask[0, 70000:] = False
    mask[6, 1::2] = False
    for at, m in ((0, None), (1, mask), (2, mask)):
        how = turn(n, at)
        got = check(ctx, x, u, m, **how)
        dev = {k: torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in how.items()}
        words = None
        if m is not None:
            bits = np.zeros((n, (V + 31) // 32 * 32), np.uint8)
            bits[:, :V] = m
            words = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).cuda()
        uu = torch.tensor(u, device="cuda")
        token, lp = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
        ctx.sample(x, uu, token, lp, mask=words, **dev)
        ctx.check()
        if V <= 150001:
            t2, lp2 = whole_rows(ctx, x, uu, words, **dev)
            assert torch.equal(token, t2) and torch.equal(lp.view(torch.int32), lp2.view(torch.int32))
        assert token.tolist() == got


def test_sample_slices_bad_parameters(ctx):
    x, u = normal(5, 140000, BF, 1)
    check(ctx, x, u, temperature=[1.0, -1.0, math.nan, math.inf, 0.0])
    check(ctx, x, u, top_p=[1.0, math.nan, 0.5, 0.0, 0.9], min_p=[0.1, 0.0, math.nan, 1.0, 0.0])


def test_sample_slices_in_graphs():
    """Captured before the context has room for slices and after, replayed between eager calls."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_18703_amd as R
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = R.Context(stream)
        x, u = normal(6, 160000, BF, 5)
        other, _ = normal(6, 160000, BF, 6)
        at = x.clone()
        u = torch.tensor(u, device="cuda")
        dev = {k: torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda")
               for k, v in turn(6).items()}
        token, lp = torch.empty(6, dtype=torch.int32, device="cuda"), torch.empty(6, device="cuda")
        stream.synchronize()
        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                ctx.sample(at, u, token, lp, **dev)
            graphs.append(g)
            want = []
            for rows in (x, other):              # (the first of them makes the room)
                ctx.sample(rows, u, token, lp, **dev)
                ctx.check()
                want.append((token.clone(), lp.clone()))
        assert not torch.equal(want[0][0], want[1][0])
        for turn_of in range(6):
            at.copy_((x, other)[turn_of % 2])
            token.fill_(-5)
            graphs[turn_of // 2 % 2].replay()
            ctx.check()
            assert torch.equal(token, want[turn_of % 2][0]) and torch.equal(lp, want[turn_of % 2][1])
            ctx.sample(other, u, token, lp, **dev)
        stream.synchronize()


BEYOND = [1.0, 2.0, math.inf, math.nan]          # numbers that take the last kept token


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("V", [2, 777, 140000])
def test_sample_last_kept_far_below(ctx, V, dtype, monkeypatch):
    """The last kept token, however little of the sum it has: whole rows and, of the longest, cut ones."""
    plain = ref.sample

    def in_32_bits(*a, **k):
        # beyond the largest 32-bit number, 2^128 - 2^104, and half a step more, a logarithm is rounded to infinity
        at, lp, n = plain(*a, **k)
        return at, -math.inf if lp <= -(2.0 ** 128 - 2.0 ** 103) else lp, n
    monkeypatch.setattr(ref, "sample", in_32_bits)
    x, _ = normal(8, V, dtype, V + 3, 30.0)
    x[0] = -100.0
    x[0, 0] = 0.0                                # {0, -100, ...}
    x[1, V // 2] = math.inf                      # the others have no weight at all
    x[2, 1:] = torch.finfo(dtype).min
    x[3, ::2] = -math.inf
    x[4, 1] = x[4].min()                         # two of the least: the later one
    x[5, V - 1] = math.nan
    x[6, 0] = 300.0
    mask = np.random.default_rng(V).random((8, V)) < 0.5
    mask[:, :2] = True
    for shift in range(4):
        u = [BEYOND[(r + shift) % 4] for r in range(8)]
        check(ctx, x, u)
        check(ctx, x, u, mask=mask)
        for t in (0.05, 1.0, 4.0):
            check(ctx, x, u, temperature=[t] * 8)
        check(ctx, x, u, top_k=[V, V - 1, 5, 0, V // 2 + 1, 2, 300, V + 1], temperature=[0.05] * 8)
        check(ctx, x, u, top_p=[1.0, 0.5, 0.999, 2.0, 1 - 2.0 ** -24, 0.0, 1.0, 0.9])
        check(ctx, x, u, min_p=[0.0, -1.0, 1e-30, 1e-40, 1e-20, 0.0, 1e-36, 2.0])
        check(ctx, x, u, **turn(8, shift))


# The largest logit, another one, a temperature, and a 32-bit number that the other one's
# weight exceeds by 4e-16 to 9e-15 of itself: by more than the weight's rounding (2^-52), and
# by less than a logarithm of 2 in 53 bits loses, 2.3e-17 for every power of 2 in the weight.
CLOSE = [(5.125, -54.25, 1.110068917274475, 5.896577888776472e-24), (29.125, -56.25, 1.4169886112213135, 6.812669029478745e-27),
         (25.0, -27.125, 0.8485968708992004, 2.1061707945346375e-27), (1.25, -58.25, 1.1741161346435547, 9.806438460062956e-23),
         (17.375, -58.25, 1.4801291227340698, 6.462019107256508e-23), (13.0, -42.25, 0.9567762613296509, 8.34126175370901e-26)]


def test_sample_weights_in_64_bits(ctx):
    """min_p next to a far token's weight: kept, as the weight's first 70 digits say."""
    from decimal import Decimal, localcontext
    with localcontext() as of:
        of.prec = 70
        for most, other, t, p in CLOSE:
            t32, p32 = (Decimal(float(np.float32(v))) for v in (t, p))
            assert 4e-16 < ((Decimal(other) - Decimal(most)) / t32).exp() / p32 - 1 < 9e-15
    x = torch.tensor([[a, b] for a, b, _, _ in CLOSE]).to(BF).cuda()
    n = len(CLOSE)
    token = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    ctx.sample(x, torch.full((n,), math.nan, device="cuda"), token,
               temperature=torch.tensor([c[2] for c in CLOSE], device="cuda"),
               min_p=torch.tensor([c[3] for c in CLOSE], device="cuda"))
    ctx.check()
    assert token.tolist() == [1] * n


def test_sample_without_memory_for_slices():
    """The room for slices is not to be had: whole rows, and the same tokens; slices once it is."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_18703_amd as R
    ctx = R.Context()
    x, u = normal(6, 150001, BF, 12)
    u = torch.tensor(u, device="cuda")
    dev = {k: torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in turn(6).items()}
    outs = []
    for refuse in (2, 0, 0):
        token, lp = torch.full((6,), -7, dtype=torch.int32, device="cuda"), torch.full((6,), 9.0, device="cuda")
        ctx.debug_refuse(refuse)
        try:
            ctx.sample(x, u, token, lp, **dev)
        finally:
            ctx.debug_refuse(0)
        ctx.check()
        outs.append((token.tolist(), lp.view(torch.int32).tolist()))
    assert outs[0] == outs[1] == outs[2]
    assert -7 not in outs[0][0]
    torch.zeros(1, device="cuda").add_(1).item()     # (no error is left behind)


def filled(n, V, off, dtype):
    """Rows with infinities, NaN, repeated values and lone candidates among ordinary ones, and a mask."""
    room, u = normal(n, V + off, dtype, V + off)
    x = room[:, off:]
    x[1] = float("-inf")
    x[1, V // 2] = 0.5
    x[2, V - 1] = 90.0
    x[3, ::3] = math.nan
    x[3, V // 4:V // 2] = math.nan
    x[4, V // 2:] = float("inf")
    x[5] = float("-inf")
    x[6] = 0.25
    x[7, ::2], x[7, 1::2] = -1.5, 1.5
    mask = np.ones((n, V), bool)
    mask[0, V // 2:] = False
    mask[6, 1::2] = False
    mask[8] = np.random.default_rng(V).random(V) < 0.03
    return x, u, mask


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("V,off", [(32770, 0), (40000, 3), (49152, 0), (65529, 7), (65530, 2), (98290, 0), (98299, 1), (100000, 0),
                                   (128000, 0), (131000, 5)])
def test_sample_lengths(ctx, V, off, dtype):
    """Rows that registers hold, in each of the sizes that they come in."""
    x, u, mask = filled(10, V, off, dtype)
    for at, m in ((0, None), (1, mask), (2, None), (3, mask)):
        check(ctx, x, u, m, **turn(10, at))
    check(ctx, x, u)


def uncut(ctx, x, u, mask=None, **how):
    """As check does, in cut rows, and whole rows of the same: equal to the bit."""
    n, V = x.shape
    got = check(ctx, x, u, mask, **how)
    dev = {k: torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in how.items()}
    words = None
    if mask is not None:
        bits = np.zeros((n, (V + 31) // 32 * 32), np.uint8)
        bits[:, :V] = mask
        words = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).cuda()
    uu = torch.tensor(u, dtype=torch.float32, device="cuda")
    token, lp = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda")
    ctx.sample(x, uu, token, lp, mask=words, **dev)
    ctx.check()
    t2, lp2 = whole_rows(ctx, x, uu, words, **dev)
    assert torch.equal(token, t2) and torch.equal(lp.view(torch.int32), lp2.view(torch.int32))
    assert token.tolist() == got


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("V,off", [(163826, 0), (163827, 0), (200003, 3), (262144, 0), (500009, 1)])
def test_sample_whole_rows_of_any_length(ctx, V, off, dtype):
    """More rows than can be cut, longer than registers hold."""
    x, u, mask = filled(9, V, off, dtype)
    for at, m in ((0, None), (1, mask)):
        uncut(ctx, x, u, m, **turn(9, at))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("V", [140001, 200003])
def test_sample_whole_rows_many_equal(ctx, V, dtype):
    """Counters of 16 bits that run over, some of both signs, in rows that are not cut: held in registers, and read again."""
    x = torch.zeros(11, V, dtype=dtype, device="cuda")
    x[1, :65535], x[1, 65535:] = 1.0, -40.0
    x[2, :65536] = 1.0
    x[3, 1:65538] = 1.0
    x[4, ::2] = 1.0
    x[5, ::2] = -1.0
    x[6] = torch.finfo(dtype).min
    x[6, 40:45] = 2.0
    x[7, :131072], x[7, 131072:] = 1.0, 0.5
    x[8, :131071] = -1.0
    x[9, :65536], x[9, 65536:131072], x[9, 131072:] = 1.0, -1.0, 0.9921875
    x[10, :66000], x[10, 66000:] = 0.0078125, -0.0078125
    u = [0.0, 0.1, 0.3, 0.5, 0.7, 0.9, 0.99, 0.999, 0.2, 0.6, 0.45]
    for at in range(3):
        uncut(ctx, x, u, **turn(11, at))
    uncut(ctx, x, [math.nan] * 11)
