"""A model stage between a batch and its gather: prompts shared by siblings,
a chunk of new tokens, single tokens, eviction, and the children's results
gathered by parent in ordinal order, against dense attention in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import chunk_ref as ref  # noqa: E402
import oracle as O  # noqa: E402


def test_stage_from_batch_to_gather():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_18703_amd as R
    from paper_2609_18703_amd.stage import Stage

    counts = np.array([3, 0, 5, 1, 4], np.int32)
    P, N, B, Hq, Hk, D, ps = 5, 13, 13, 8, 2, 64, 16
    pairs, axes = 24, 3
    g = torch.Generator(device="cuda").manual_seed(4)
    freq = 1.0e4 ** (-torch.arange(pairs, device="cuda").float() / pairs)
    axis = [i % axes for i in range(pairs)]
    ctx = R.Context()
    rot = R.Rotary(freq, axis)
    st = Stage(ctx, P, N, B, Hq, Hk, D, ps, prompt_pages=3, child_pages=2, rotary=rot, max_new=20)

    # expand, and one reservation of all children in a shuffled ready order
    offsets = torch.empty(P + 1, dtype=torch.int64, device="cuda")
    ctx.expand(torch.from_numpy(counts).cuda(), offsets)
    queue = torch.randperm(N, generator=g, device="cuda").int()
    child, parent, ordinal = (torch.empty(N, dtype=torch.int32, device="cuda") for _ in range(3))
    ctx.batch(queue, None, offsets, B, child, parent, ordinal)

    def tokens(n):
        qkv = torch.randn(n, Hq + 2 * Hk, D, generator=g, device="cuda").bfloat16()
        return qkv, torch.randint(0, 500, (axes, n), generator=g, device="cuda").int()

    def off(new):
        return torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int64, device="cuda")

    lengths = [48, 16, 32, 16, 48]
    prompt_qkv, prompt_pos = tokens(sum(lengths))
    kv = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    st.prompts(prompt_qkv, prompt_pos, off(lengths), kv)
    st.reserve(child, parent)
    news = [[1 + (7 * s) % 20 for s in range(B)], [1] * B, [1] * B, [2] * B]
    inputs, outs, shrunk = [], [], {}
    budgets = {1: (30, 2, 5), 2: (25, 1, 3)}
    for i, new in enumerate(news):
        qkv, pos = tokens(sum(new))
        inputs.append((qkv, pos))
        print("step", i, flush=True)
        outs.append(st.step(qkv, pos, off(new), torch.tensor(new, dtype=torch.int32, device="cuda")))
        if i in budgets:
            weight = st.weight.clone()
            shrunk[i] = weight, st.shrink(budgets[i][0], first=budgets[i][1], last=budgets[i][2])
    ctx.check("stage")

    # each child's result is its last token's row; they come back in batch order
    rows = outs[-1][1::2].reshape(B, -1).contiguous().view(torch.uint8)
    size = rows.shape[1]
    state = torch.zeros(B, dtype=torch.uint8, device="cuda")
    rep_off = torch.arange(B + 1, device="cuda") * size
    out_off = torch.empty(P + 1, dtype=torch.int64, device="cuda")
    out = torch.empty(N * size, dtype=torch.uint8, device="cuda")
    ctx.gather(parent, ordinal, state, rep_off, rows.view(-1), offsets, out_off, out)
    ctx.check("gather")

    # ---- the same, dense, in 64 bits
    c, p, o = (t.cpu().numpy() for t in (child, parent, ordinal))
    offs = O.expand(counts, tags=False)
    assert np.array_equal(np.sort(c), np.arange(N)) and np.array_equal(offs[p] + o, c)

    def keys_values(qkv, pos):
        k = ref.turn(qkv[:, Hq:Hq + Hk], pos, freq, axis, False, False)[0].bfloat16()
        q = ref.turn(qkv[:, :Hq], pos, freq, axis, False, False)[0].bfloat16()
        return q, k, qkv[:, Hq + Hk:]
    _, pk, pv = keys_values(prompt_qkv, prompt_pos)
    starts = np.cumsum([0] + lengths)
    K = [pk[starts[x]:starts[x + 1]] for x in p]
    V = [pv[starts[x]:starts[x + 1]] for x in p]
    W = [torch.zeros(len(k), dtype=torch.float64, device="cuda") for k in K]
    last = torch.zeros(N, Hq, D, dtype=torch.float64, device="cuda")
    for i, new in enumerate(news):
        q, k, v = keys_values(*inputs[i])
        t0 = 0
        for s, n in enumerate(new):
            K[s], V[s] = torch.cat([K[s], k[t0:t0 + n]]), torch.cat([V[s], v[t0:t0 + n]])
            W[s] = torch.cat([W[s], torch.zeros(n, dtype=torch.float64, device="cuda")])
            L = len(K[s])
            see = ref.visible(n, L, True, 0, 0, "cuda")
            kk, vv = K[s].double().repeat_interleave(Hq // Hk, 1), V[s].double().repeat_interleave(Hq // Hk, 1)
            x = torch.einsum("ihd,jhd->ihj", q[t0:t0 + n].double(), kk) * D ** -0.5
            x = x.masked_fill(~see[:, None], -math.inf)
            z = torch.logsumexp(x, -1, keepdim=True)
            pr = (x - z).exp()
            want = torch.einsum("ihj,jhd->ihd", pr, vv)
            # the rotated queries and keys, and the outputs, are rounded to 8 bits: u of each factor of the score
            score = (q[t0:t0 + n].double().abs()[:, None] * kk.abs()[None]).sum(-1).amax() * D ** -0.5
            tol = (4 * ref.U[torch.bfloat16] * (1 + score)) * torch.einsum("ihj,jhd->ihd", pr, vv.abs()) + 1e-3
            assert ((outs[i][t0:t0 + n].double() - want).abs() <= tol).all(), (i, s)
            W[s] += pr.sum((0, 1))
            if i == 3:
                last[c[s]] = want[-1]
            t0 += n
        if i in budgets:
            weight, index = shrunk[i]
            budget, first, end = budgets[i]
            for s in range(B):
                keep = ref.kept(weight[s], len(K[s]), budget, first, end)
                assert index[s].tolist() == keep + [-1] * (budget - len(keep))
                got = weight[s, :len(K[s])].double()
                assert ((got - W[s]).abs() <= 0.05 * W[s] + 1e-2).all()
                ix = torch.tensor(keep, device="cuda")
                K[s], V[s], W[s] = K[s][ix], V[s][ix], W[s][ix]
    # parents' slots hold their children's rows in ordinal order, bit for bit those of the last step
    got = out.view(torch.bfloat16).view(N, Hq, D)
    for s in range(B):
        assert torch.equal(got[c[s]], outs[-1][2 * s + 1])
    assert out_off.tolist() == (offs * size).tolist()
    assert (got.double() - last).abs().max() < 0.2
    ctx.close()
