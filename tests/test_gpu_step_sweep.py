"""Projections, sampling and pages at random sizes, strides, values and filters, against their definitions.  A case
is a number; RO_STEP_CASES (30) says how many of each kind are run, RO_STEP_FIRST (0) from which on."""
import math
import os
import random

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import step_ref as ref  # noqa: E402
import test_gpu_pages as pages  # noqa: E402
import test_gpu_project as project  # noqa: E402
import test_gpu_sample as sample  # noqa: E402

BF, HF, FL = torch.bfloat16, torch.float16, torch.float32
FIRST = int(os.environ.get("RO_STEP_FIRST", "0"))
CASES = range(FIRST, FIRST + int(os.environ.get("RO_STEP_CASES", "30")))


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_18703_amd as R
    return R.Context()


def log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


@pytest.mark.parametrize("case", CASES)
def test_quantize(ctx, case):
    rng = random.Random(case)
    dim = log(rng, 1, 40000)
    n = log(rng, 1, max(1, min(3000, 2000000 // dim)))
    at, more, q_at = rng.choice([0, 0, 8, 1, 3]), rng.choice([0, 0, 8, 5]), rng.choice([0, 0, 8, 3])
    dtype = rng.choice([BF, HF])
    g = project.gen(case)
    x = (torch.randn(n, at + dim + more, generator=g, device="cuda") * rng.choice([1e-6, 0.1, 1.0, 300.0])).to(dtype)
    for _ in range(rng.randrange(4)):
        x[rng.randrange(n), rng.randrange(x.shape[1])] = rng.choice([math.inf, math.nan, 0.0, -0.0, torch.finfo(dtype).max, torch.finfo(dtype).tiny / 4])
    if rng.random() < 0.1:
        x[rng.randrange(n)] = 0.0
    room = torch.full((n, q_at + dim + 7), 55, dtype=torch.int8, device="cuda")
    project.check_quantize(ctx, x[:, at:at + dim], room[:, q_at:q_at + dim])
    assert (room[:, :q_at] == 55).all() and (room[:, q_at + dim:] == 55).all()


@pytest.mark.parametrize("case", CASES)
def test_project(ctx, case):
    """To the bit without a bias, within its roundings with one."""
    import paper_2609_18703_amd as R
    rng = random.Random(case)
    while True:
        m, k, n = log(rng, 1, 6000), 16 * log(rng, 1, 1000), log(rng, 1, 20000)
        if m * n <= 12000000 and m * n * k <= 3 << 33 and n * k <= 1 << 28:
            break
    dtype, bias = rng.choice([BF, HF, FL]), rng.random() < 0.3
    q, scale, w, w_scale, b = project.make(m, k + rng.choice([0, 16, 112, 128]), n, case, bias=bias, full=True)
    q, w = q[:, :k], w[:, :k]
    at, more = rng.choice([0, 0, 1, 8]), rng.choice([0, 0, 3, 8])
    room = torch.full((m, at + n + more), 77.0, dtype=dtype, device="cuda")
    out = room[:, at:at + n]
    ctx.project(q, scale, R.Weights(w, w_scale, b), out)
    ctx.check("project")
    row = ((q.double() @ w.double().T).float() * scale[:, None]).double()
    if bias:
        want = row * w_scale.double() + b.double()               # (off by 2^-53 of itself)
        tol = 2.0 ** -24 * (1 + 2.0 ** -20) * want.abs() + ref.TINY[FL]
        if dtype is not FL:
            tol = tol + ref.U[dtype] * (want.abs() + tol) + ref.TINY[dtype]
        assert ((out.double() - want).abs() <= tol).all()
    else:
        assert torch.equal(out, (row * w_scale.double()).float().to(dtype))
    assert (room[:, :at] == 77).all() and (room[:, at + n:] == 77).all()


@pytest.mark.parametrize("case", CASES)
def test_sample(ctx, case, monkeypatch):
    rng = random.Random(case)
    V = log(rng, 1, 400000)
    n = log(rng, 1, max(1, min(300, 3000000 // V)))
    dtype, off = rng.choice([BF, HF]), rng.choice([0, 0, 1, 3, 6])
    room, u = sample.normal(n, V + off, dtype, case, rng.choice([0.01, 0.5, 2.0, 8.0, 200.0]))
    x = room[:, off:]
    for _ in range(rng.randrange(4)):
        r, c = rng.randrange(n), rng.randrange(V)
        x[r, c:c + rng.choice([1, 1, V])] = rng.choice([math.inf, -math.inf, math.nan, 0.0, -0.0, torch.finfo(dtype).min, 1.0])
    for _ in range(rng.randrange(3)):
        u[rng.randrange(n)] = rng.choice([0.0, 1 - 2.0 ** -24, 1.0, 2.0, -1.0, math.nan, math.inf, 1e-38])
    how = {name: [rng.choice(values) for _ in range(n)] for name, values in sample.HOW.items() if rng.random() < 0.5}
    if "temperature" in how and rng.random() < 0.2:
        how["temperature"][rng.randrange(n)] = rng.choice([1e-30, 1e-3, 1e4, 1e30])
    mask = None
    if rng.random() < 0.4:
        mask = np.random.default_rng(case).random((n, V)) < rng.choice([0.001, 0.1, 0.9])
    plain = ref.sample

    def in_32_bits(*a, **k):
        # beyond the largest 32-bit number, 2^128 - 2^104, and half a step more, a logarithm is rounded to infinity
        at, lp, kept = plain(*a, **k)
        return at, -math.inf if lp <= -(2.0 ** 128 - 2.0 ** 103) else lp, kept
    monkeypatch.setattr(ref, "sample", in_32_bits)
    sample.check(ctx, x, u, mask, **how)


@pytest.mark.parametrize("case", CASES)
def test_pages(ctx, case):
    rng = random.Random(case)
    page = rng.choice([1, 2, 16, 16, 64, 128, 4096])
    rows, cols = (log(rng, 1, 80), log(rng, 1, 400)), log(rng, 1, 60)
    n_pages = log(rng, 1, rng.choice([60, 3000, 20000, 60000]))
    b = pages.Both(ctx, n_pages, page, rows, cols)
    room = cols * page
    most = log(rng, 1, room)
    for _ in range(rng.randrange(3, 12)):
        a = rng.randrange(2)
        lens = b.lists[a][1]
        what = rng.choice(["grow", "grow", "grow", "fork", "release", "compact"])
        if what == "grow":
            b.grow(a, [min(rng.choice([0, 1, rng.randrange(0, most + 1)]), room - L) for L in lens])
        elif what == "fork":
            parent = [rng.choice([pages.NONE] + list(range(rows[0]))) for _ in range(rows[1])]
            b.release(1, [0 if p >= 0 else L for p, L in zip(parent, b.lists[1][1])])
            b.fork(0, parent, 1)
        elif what == "release":
            b.release(a, rng.choice([None, [rng.choice([1 << 30, 0, L, rng.randrange(0, L + 1)]) for L in lens]]))
        else:
            b.compact()
        b.same()
    b.release(0, None)
    b.release(1, None)
    b.check()
    assert not b.refs.any()
