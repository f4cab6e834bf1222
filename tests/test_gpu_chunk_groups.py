"""Attention, weights and a step's order with many query heads a key / value
head, up to the 64 that are accepted, against definitions in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import chunk_ref as ref  # noqa: E402
from test_gpu_chunk import BF, HF, close, ctx, make, plan  # noqa: E402,F401

CASES = [
    # new tokens, lengths, q heads, kv heads, dim, extra
    ([1, 1, 1], [300, 70, 1], 64, 1, 128, {}),                  # single tokens that fill half a wide tile
    ([1, 2], [2100, 40], 64, 1, 64, {}),
    ([1, 1], [500, 17], 16, 1, 128, {}),                        # exactly as many as a narrow tile has rows
    ([1, 1], [500, 17], 17, 1, 128, {}),                        # and one more
    ([70], [150], 48, 1, 64, {}),                               # one token a tile of weights
    ([33, 4], [200, 9], 66, 2, 128, {}),                        # 33 heads: one token and a row to spare
    ([30, 1], [90, 400], 40, 2, 64, {"window": 37, "sinks": 5}),
    ([5, 1], [5, 1000], 96, 3, 128, {"window": 100, "sinks": 1}),
    ([9], [300], 64, 1, 128, {"causal": False}),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("at", range(len(CASES)))
def test_many_heads_a_group(ctx, at, dtype):
    new, kv, hq, hk, dim, more = CASES[at]
    c = make(new, kv, hq, hk, dim, 16, dtype, seed=60 + at, **more)
    cache, ch = plan(ctx, c)
    out, lse = torch.full_like(c["q"], 7.0), torch.full(c["q"].shape[:2], 7.0, device="cuda")
    w = torch.zeros(len(new), max(kv), device="cuda")
    print("groups", at, CASES[at], dtype, flush=True)
    ch.attend(cache, c["q"], out, lse)
    ch.weigh(cache, c["q"], lse, None, w)
    ctx.check("attend and weigh")
    want, wl, tol, tl = ref.attend(c, c["k"], c["v"], c["q"], dim ** -0.5)
    close(lse, wl, tl, "lse")
    close(out, want, tol, "out")
    close(w, *ref.weigh(c, c["k"], c["q"], lse, torch.zeros_like(w), dim ** -0.5), "weight")
    ch.close()
