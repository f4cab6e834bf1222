"""Projections in 8-bit integers against their definition: every integer of
the rounding, and products within the rounding of the result."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import step_ref as ref  # noqa: E402

BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_18703_amd as R
    return R.Context()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def check_quantize(ctx, x, q=None):
    n, dim = x.shape
    q = torch.full((n, dim), 99, dtype=torch.int8, device="cuda") if q is None else q
    scale = torch.full((n,), 7.0, device="cuda")
    ctx.quantize(x, q, scale)
    ctx.check("quantize")
    want, want_scale = ref.quantize(x)
    assert torch.equal(q.cpu(), want)
    got = scale.cpu().double()
    same = got.isnan() & want_scale.isnan()
    # one division, rounded to 32 bits
    assert (same | ((got - want_scale).abs() <= 2.0 ** -24 * want_scale + 2.0 ** -150)).all()
    return q, scale


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("n,dim", [(1, 1), (1, 16), (3, 7), (5, 3584), (2, 8192), (64, 129), (1000, 48), (2, 20000),
                                   (1, 131056), (3, 4097)])
def test_quantize(ctx, n, dim, dtype):
    g = gen(n * 1000 + dim)
    check_quantize(ctx, (torch.randn(n, dim, generator=g, device="cuda") * 5).to(dtype))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("n,dim", [(1, 8), (7, 504), (9, 512), (5, 520), (6, 2048), (3, 2056), (70, 1000), (4, 4096),
                                   (3, 4104), (2, 8200), (3, 16384), (2, 16392), (5, 11111)])
def test_quantize_lengths(ctx, n, dim, dtype):
    """Rows around those that a wave, or a workgroup's registers, hold."""
    check_quantize(ctx, (torch.randn(n, dim, generator=gen(n + dim), device="cuda") * 0.7).to(dtype))


@pytest.mark.parametrize("dtype", [BF, HF])
def test_quantize_halves(ctx, dtype):
    """Quotients that end in a half go to the even integer."""
    steps = torch.arange(-254, 255, device="cuda").float() / 2
    x = torch.cat([steps, torch.tensor([127.0], device="cuda")])[None].to(dtype)
    q, _ = check_quantize(ctx, x)
    assert q[0, 255].item() == 0 and q[0, 254 + 3].item() == 2 and q[0, 254 + 5].item() == 2


@pytest.mark.parametrize("dtype", [BF, HF])
def test_quantize_every_number_below_one(ctx, dtype):
    """Every number of the type as an element, under several largest ones."""
    bits = torch.arange(1 << 16, device="cuda").to(torch.int32)
    every = torch.where(bits >= 1 << 15, bits - (1 << 16), bits).to(torch.int16).view(dtype)
    every = torch.where(every.isfinite(), every, 0.0)
    rows = []
    for top in (1.0, 1.5703125, 3.1, 127.0, 60000.0, torch.finfo(dtype).tiny, torch.finfo(dtype).max):
        t = torch.tensor(top, device="cuda").to(dtype)
        rows.append(torch.cat([torch.where(every.abs() <= t, every, 0.0), t[None], -t[None]]))
    check_quantize(ctx, torch.stack(rows))


@pytest.mark.parametrize("dtype", [BF, HF])
def test_quantize_values(ctx, dtype):
    """Zeros, the largest and the least numbers, infinities, NaN: a row's own affair."""
    big, tiny = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    x = torch.zeros(9, 33, device="cuda").to(dtype)
    x[1, 4], x[1, 5] = big, -big / 2
    x[2, 7], x[2, 8] = tiny, tiny / 4
    x[3, 9] = tiny / 64
    x[4, 1], x[4, 2] = math.inf, 1.0
    x[5, 1], x[5, 2] = -math.inf, 1.0
    x[6, 32] = math.nan
    x[7] = -0.0
    x[8] = -1.0
    check_quantize(ctx, x)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_quantize_strides(ctx, dtype):
    g = gen(3)
    wide = torch.randn(9, 2, 70, generator=g, device="cuda").to(dtype)
    for cols in (slice(0, 64), slice(1, 65), slice(3, 70)):
        x = wide[:, 1, cols]
        room = torch.full((9, 83), 55, dtype=torch.int8, device="cuda")
        check_quantize(ctx, x, room[:, 5:5 + x.shape[1]])
        assert (room[:, :5] == 55).all() and (room[:, 5 + x.shape[1]:] == 55).all()
    one = wide[:1, 0].expand(5, 70)
    check_quantize(ctx, one)


def make(m, k, n, seed, bias=True, full=False):
    g = gen(seed)
    lo = -128 if full else -127
    q = torch.randint(lo, 128, (m, k), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(lo, 128, (n, k), generator=g, device="cuda", dtype=torch.int8)
    scale = torch.rand(m, generator=g, device="cuda") * 0.05 + 0.001
    w_scale = (torch.rand(n, generator=g, device="cuda") + 0.1) / (74 * k ** 0.5)
    b = torch.randn(n, generator=g, device="cuda") if bias else None
    return q, scale, w, w_scale, b


def check_project(ctx, q, scale, w, w_scale, b, out):
    import paper_2609_18703_amd as R
    ctx.project(q, scale, R.Weights(w, w_scale, b), out)
    ctx.check("project")
    want, tol = ref.project(q, scale, w, w_scale, b, out.dtype)
    off = (out.cpu().double() - want).abs()
    assert (off <= tol).all(), (off - tol).max()


SIZES = [(1, 16, 1), (1, 16, 17), (2, 32, 5), (5, 3584, 4608), (1, 4096, 33), (16, 48, 64), (17, 80, 65), (31, 1040, 129),
         (33, 128, 1000), (64, 512, 2049), (65, 112, 257), (100, 272, 100), (127, 64, 127), (129, 144, 257), (200, 1024, 513),
         (257, 176, 130), (300, 2064, 640), (513, 256, 1030), (1000, 16, 1), (1100, 96, 1027), (3, 131056, 7), (260, 20000, 270)]


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_project(ctx, m, k, n, dtype):
    q, scale, w, w_scale, b = make(m, k, n, m + k + n, bias=(m + n) % 2 == 0)
    room = torch.full((m, n + 3), 77.0, dtype=dtype, device="cuda")
    check_project(ctx, q, scale, w, w_scale, b, room[:, :n])
    assert (room[:, n:] == 77).all()


@pytest.mark.parametrize("dtype", [BF, FL])
@pytest.mark.parametrize("m,k,n", [(17, 1536, 16), (33, 1552, 100), (64, 2064, 2047), (100, 4096, 64), (1000, 1600, 17),
                                   (31, 131056, 33), (490, 2048, 250), (32, 1520, 4096), (17, 4096, 4096), (33, 4096, 2049),
                                   (64, 640, 8300), (40, 112, 8193), (64, 1040, 8192), (30, 1040, 5000), (20, 96, 4100), (32, 1408, 8192),
                                   (17, 2064, 8193), (25, 128, 31)])
def test_project_few_tokens(ctx, m, k, n, dtype):
    """Sizes on both sides of where rows are shared among a workgroup's waves, and weights read once."""
    q, scale, w, w_scale, b = make(m, k, n, m + k + n, bias=(m + n) % 2 == 0, full=True)
    room = torch.full((m, n + 3), 77.0, dtype=dtype, device="cuda")
    check_project(ctx, q, scale, w, w_scale, b, room[:, :n])
    assert (room[:, n:] == 77).all()


@pytest.mark.parametrize("m", [1, 8, 40, 300])
def test_project_strides(ctx, m):
    """Parts of wider tensors, out at any element."""
    k, n = 160, 75
    q, scale, w, w_scale, b = make(m, 3 * k, 2 * n, m)
    room = torch.full((m, n + 9), 77.0, dtype=BF, device="cuda")
    for at in (0, 1, 2, 5):
        room.fill_(77.0)
        check_project(ctx, q[:, 16:16 + k], scale, w[1::2, 2 * k - 32:3 * k - 32], w_scale[:n].contiguous(), b[n:].contiguous(),
                      room[:, at:at + n])
        assert (room[:, :at] == 77).all() and (room[:, at + n:] == 77).all()


@pytest.mark.parametrize("m", [1, 64, 257])
def test_project_largest_sums(ctx, m):
    """-128 * -128, as often as sums allow."""
    import paper_2609_18703_amd as R
    q = torch.full((m, 131056), -128, dtype=torch.int8, device="cuda")
    w = torch.full((3, 131056), -128, dtype=torch.int8, device="cuda")
    w[1] = 127
    out = torch.empty(m, 3, device="cuda")
    one = torch.ones(max(m, 3), device="cuda")
    ctx.project(q, one, R.Weights(w, one), out)
    ctx.check()
    want = torch.tensor([128.0 * 128 * 131056, -128.0 * 127 * 131056, 128.0 * 128 * 131056], dtype=torch.float64)
    assert ((out.cpu().double() - want).abs() <= 2.0 ** -24 * want.abs()).all()


def test_project_rows_are_their_own(ctx):
    """A row that is not finite, and a channel whose scale is not, stay where they are."""
    import paper_2609_18703_amd as R
    for m in (5, 300):
        x = torch.randn(m, 256, generator=gen(1), device="cuda").to(BF)
        x[1, 3] = math.inf
        x[3, 5] = math.nan
        q, scale = check_quantize(ctx, x)
        _, _, w, w_scale, b = make(m, 256, 100, 4)
        w_scale[7] = math.inf
        out = torch.empty(m, 100, dtype=BF, device="cuda")
        ctx.project(q, scale, R.Weights(w, w_scale, b), out)
        ctx.check()
        bad = torch.zeros(m, 100, dtype=torch.bool, device="cuda")
        bad[[1, 3]] = True
        bad[:, 7] = True
        assert (out.isfinite() == ~bad).all()
        assert out[[1, 3]].isnan().all()


def test_project_same_bits(ctx):
    import paper_2609_18703_amd as R
    for m, k, n in ((5, 2048, 500), (300, 2048, 500)):
        q, scale, w, w_scale, b = make(m, k, n, 9)
        outs = [torch.empty(m, n, device="cuda") for _ in range(3)]
        for o in outs:
            ctx.project(q, scale, R.Weights(w, w_scale, b), o)
        ctx.check()
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("m,n", [(1, 4096), (16, 8001), (200, 300), (32, 8192), (20, 20001), (64, 20001), (300, 2500), (513, 1030), (1100, 1027),
                                 (388, 4717), (1679, 2323), (901, 8309), (1167, 6427)])
def test_project_roundings(ctx, m, n, dtype):
    """A result is rounded to a 32-bit number, and that to its type, wherever in a tile of whichever size it lies: to the bit."""
    import paper_2609_18703_amd as R
    k = 1600
    q, scale, w, w_scale, _ = make(m, k, n, m + n)
    out = torch.empty(m, n, dtype=dtype, device="cuda")
    ctx.project(q, scale, R.Weights(w, w_scale), out)
    ctx.check("project")
    total = q.double() @ w.double().T                            # (whole numbers below 2^53)
    row = (total.float() * scale[:, None]).double()
    want = (row * w_scale.double()).float().to(dtype)            # (a product of two 32-bit numbers is exact in 64 bits)
    assert torch.equal(out, want), (out != want).sum()


# (tokens, channels) for which tiles of 128 x 128 by eight waves, 256 x 128, 256 x 256, and 128 x 128 by four are taken
# on 256 CUs, with tokens and channels left over in the last ones.
LARGE = [(217, 8309), (388, 4717), (521, 7283), (1679, 2323), (901, 8309), (1281, 5915), (1167, 6427), (1585, 4889)]


@pytest.mark.parametrize("k", [16, 112, 144, 656, 1168])
@pytest.mark.parametrize("m,n", LARGE)
def test_project_large_tiles(ctx, m, n, k):
    """Rows shorter than a stage, of one and of several, with a part of one left over; rows of the result that begin on 16
    bytes and that do not; each type; and a row's bits are those that it has alone."""
    import paper_2609_18703_amd as R
    q, scale, w, w_scale, b = make(m, k, n, m + k + n, bias=k % 32 == 0, full=True)
    weights = R.Weights(w, w_scale, b)
    rows = [0, m // 3, m - 2, m - 1]
    for dtype in (BF, HF, FL):
        want, tol = ref.project(q, scale, w, w_scale, b, dtype)
        for stride in (n + 3, (n + 7) // 8 * 8 + 8):
            room = torch.full((m, stride), 77.0, dtype=dtype, device="cuda")
            ctx.project(q, scale, weights, room[:, :n])
            ctx.check("project")
            off = (room[:, :n].cpu().double() - want).abs()
            assert (off <= tol).all(), (dtype, stride, (off - tol).max())
            assert (room[:, n:] == 77).all()
            alone = torch.empty(len(rows), n, dtype=dtype, device="cuda")
            ctx.project(q[rows], scale[rows], weights, alone)
            assert torch.equal(alone, room[rows, :n])
