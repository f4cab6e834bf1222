"""Operators of a model stage's attention over a paged cache, as cases to time.

A stage takes batches of ready children of many parents.  Each child is a
sequence with its own number of new tokens and its own cached length; cached
keys and values lie in pages that a block table names.  Five kinds of work:

  rope    rotary positions of several axes (time, height, width) on the heads
          of every token, and the inverse rotation, which is its gradient.
  append  the rotation of a step's queries and keys; keys and values go to the
          cache positions of their tokens.
  attend  attention of every sequence's new tokens over its cache, causal,
          optionally with a sliding window and first tokens that stay visible;
          single tokens and chunks of a prompt.
  weigh   the attention that every cached position received, added up over new
          tokens and heads.
  evict   the heaviest positions of every sequence, the first and the last
          ones among them, copied in order to pages of their own.

`own` says which side `run` takes: the plain form in 32 bits, or the library.
New-token counts and lengths are evenly spaced over their range and dealt to
the sequences in an order drawn from the seed, so that the size of a case does
not depend on the seed.  All values are drawn from the seed on the GPU.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # one page image in an encoder: height and width on small heads, neighbouring elements paired
        {"name": "rope-image", "kind": "rope", "tokens": 1179, "heads": 16, "dim": 64, "rot": 64, "axes": 2,
         "pairs": True, "inverse": False, "dtype": "f16"},
        # the gradient of the rotation for a long video's tokens: time, height, width
        {"name": "rope-video-gradient", "kind": "rope", "tokens": 32771, "heads": 36, "dim": 128, "rot": 128,
         "axes": 3, "pairs": False, "inverse": True, "dtype": "bf16"},
        # one more token of every sequence of a batch: latency
        {"name": "append-tokens", "kind": "append", "seqs": 64, "new_lo": 1, "new_hi": 1, "len_lo": 1,
         "len_hi": 300, "q_heads": 28, "kv_heads": 4, "dim": 128, "rot": 128, "axes": 3, "pairs": False, "page": 16,
         "dtype": "bf16"},
        # prompts of odd lengths enter the cache, half of each head rotated
        {"name": "append-prompts", "kind": "append", "seqs": 7, "new_lo": 333, "new_hi": 4700, "len_lo": 400,
         "len_hi": 5001, "q_heads": 32, "kv_heads": 8, "dim": 128, "rot": 64, "axes": 1, "pairs": True, "page": 64,
         "dtype": "f16"},
        # the next token of a few short sequences: latency counts
        {"name": "attend-tokens-few", "kind": "attend", "seqs": 5, "new_lo": 1, "new_hi": 1, "len_lo": 1,
         "len_hi": 901, "q_heads": 28, "kv_heads": 4, "dim": 128, "page": 16, "window": 0, "sinks": 0,
         "dtype": "bf16"},
        # the next token of a full batch over long caches: the cache is read once
        {"name": "attend-tokens-long", "kind": "attend", "seqs": 64, "new_lo": 1, "new_hi": 1, "len_lo": 700,
         "len_hi": 32768, "q_heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "window": 0, "sinks": 0,
         "dtype": "bf16"},
        # a long prompt's chunk over what is cached of it already
        {"name": "attend-prompt", "kind": "attend", "seqs": 1, "new_lo": 8000, "new_hi": 8000, "len_lo": 12001,
         "len_hi": 12001, "q_heads": 28, "kv_heads": 4, "dim": 128, "page": 128, "window": 0, "sinks": 0,
         "dtype": "bf16"},
        # chunks and single tokens in one batch, a sliding window and first tokens that stay, small heads
        {"name": "attend-mixed-window", "kind": "attend", "seqs": 13, "new_lo": 1, "new_hi": 1500, "len_lo": 1,
         "len_hi": 6007, "q_heads": 16, "kv_heads": 2, "dim": 64, "page": 32, "window": 1024, "sinks": 4,
         "dtype": "f16"},
        # what the cached positions received from a batch's single tokens
        {"name": "weigh-tokens", "kind": "weigh", "seqs": 48, "new_lo": 1, "new_hi": 1, "len_lo": 33,
         "len_hi": 8191, "q_heads": 28, "kv_heads": 4, "dim": 128, "page": 16, "window": 0, "sinks": 0,
         "dtype": "bf16"},
        # the same for chunks of prompts
        {"name": "weigh-chunks", "kind": "weigh", "seqs": 4, "new_lo": 257, "new_hi": 2050, "len_lo": 1000,
         "len_hi": 9001, "q_heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "window": 0, "sinks": 0,
         "dtype": "f16"},
        # short sequences, some within the budget already: latency
        {"name": "evict-short", "kind": "evict", "seqs": 9, "len_lo": 200, "len_hi": 1203, "budget": 513, "first": 4,
         "last": 64, "kv_heads": 4, "dim": 128, "page": 16, "dtype": "bf16"},
        # half of a batch's long caches goes
        {"name": "evict-long", "kind": "evict", "seqs": 16, "len_lo": 9000, "len_hi": 32768, "budget": 16384,
         "first": 4, "last": 1024, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16"},
    ]


MOST_PAIRS = 28 * 8000 * 12001          # padded scores of the largest listed chunk
MOST_CACHE = 64 * 32768 * 8 * 128       # padded keys of the largest listed cache


def draw(rng):
    def log(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return n + 1 if n == 3072 else n

    kind = rng.choice(["rope", "append", "attend", "attend", "attend", "weigh", "weigh", "evict"])
    dim = rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "f16"])
    q_heads, kv_heads = rng.choice([(32, 8), (28, 4), (16, 2), (16, 16), (20, 20), (8, 1), (40, 8)])
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "rope":
        return {"kind": "rope", "tokens": log(1, 32771), "heads": rng.choice([1, 5, 16, 28, 36]), "dim": dim,
                "rot": rng.choice([dim, dim, dim // 2]), "axes": rng.choice([1, 2, 3, 4]),
                "pairs": rng.random() < 0.5, "inverse": rng.random() < 0.5, "dtype": dtype}
    if kind == "evict":
        while True:
            seqs, hi = log(1, 64), log(16, 32768)
            lo = max(1, hi // rng.randrange(1, 9))
            if seqs * hi * kv_heads * dim <= 16 * 32768 * 8 * 128 and lo != 3072:
                break
        budget = log(max(2, hi // 8), hi)
        last = rng.randrange(0, budget // 2 + 1)
        return {"kind": "evict", "seqs": seqs, "len_lo": lo, "len_hi": hi,
                "budget": budget, "first": min(rng.choice([0, 4]), budget - last), "last": last,
                "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype}
    window, sinks = (0, 0) if rng.random() < 0.6 else (log(1, 4096), rng.choice([0, 1, 4, 64]))
    while True:
        seqs = log(1, 128)
        new_hi = 1 if rng.random() < 0.4 else log(2, 8000)
        new_lo = rng.choice([1, max(1, new_hi // 2), new_hi])
        len_hi = new_hi + (log(1, 32768) if rng.random() < 0.7 else 0)
        len_lo = max(1, len_hi // rng.randrange(1, 16))
        cache = seqs * len_hi * kv_heads * dim
        if kind == "append":
            len_hi = min(len_hi, new_hi + 600)
            len_lo = min(len_lo, len_hi)
            fits = seqs * new_hi <= 20000
        else:
            fits = cache <= MOST_CACHE and seqs * new_hi * len_hi * q_heads <= MOST_PAIRS
        if fits and 3072 not in (len_hi, len_lo, new_hi, new_lo):
            break
    case = {"kind": kind, "seqs": seqs, "new_lo": new_lo, "new_hi": new_hi, "len_lo": len_lo, "len_hi": len_hi,
            "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype}
    if kind == "append":
        return {**case, "rot": rng.choice([dim, dim, dim // 2]), "axes": rng.choice([1, 2, 3, 4]),
                "pairs": rng.random() < 0.5}
    return {**case, "window": window, "sinks": sinks}


# ------------------------------------------------------------------ sizes that follow from a case

def _spread(lo, hi, n):
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [hi]


def _sizes(case):
    """(new tokens, cached length with them) of every sequence, in an order of no seed."""
    S = case["seqs"]
    new = _spread(case.get("new_lo", 0), case.get("new_hi", 0), S)
    step = next(k for k in range(max(1, S * 5 // 8), 2 * S + 2) if math.gcd(k, S) == 1)
    total = _spread(case["len_lo"], case["len_hi"], S)
    return [(n, max(n, total[i * step % S])) for i, n in enumerate(new)]


def _seen(n, L, window, sinks):
    """Visible (new token, cached position) pairs of one sequence, and the positions seen by any token."""
    p0 = L - n
    if window <= 0:
        return n * p0 + n * (n + 1) // 2, L
    pairs, lo = 0, max(0, p0 - window + 1)
    for i in range(n):
        first = max(0, p0 + i - window + 1)
        pairs += p0 + i + 1 - first + min(sinks, first)
    return pairs, L - lo + min(sinks, lo)


def work(case):
    kind, D = case["kind"], case["dim"]
    if kind == "rope":
        T, H = case["tokens"], case["heads"]
        return {"bytes": 4.0 * T * H * D + 4.0 * T * case["axes"] + 2.0 * case["rot"],
                "flops": 3.0 * T * H * case["rot"]}
    sizes = _sizes(case)
    T = sum(n for n, _ in sizes)
    Hk = case["kv_heads"]
    if kind == "evict":
        kept = sum(min(L, case["budget"]) for _, L in sizes)
        return {"bytes": 4.0 * sum(L for _, L in sizes) + kept * (2 * 4.0 * Hk * D + 8.0), "flops": 0.0}
    Hq = case["q_heads"]
    if kind == "append":
        return {"bytes": 4.0 * T * (Hq + 2 * Hk) * D + 4.0 * T * case["axes"],
                "flops": 3.0 * T * (Hq + Hk) * case["rot"]}
    seen = [_seen(n, L, case["window"], case["sinks"]) for n, L in sizes]
    pairs, rows = Hq * sum(p for p, _ in seen), sum(r for _, r in seen)
    if kind == "attend":
        return {"bytes": 4.0 * rows * Hk * D + T * Hq * (4.0 * D + 4.0), "flops": 4.0 * D * pairs}
    return {"bytes": 2.0 * rows * Hk * D + T * Hq * (2.0 * D + 4.0) + 8.0 * sum(L for _, L in sizes),
            "flops": 2.0 * D * pairs}


# ------------------------------------------------------------------ what a program has in hand

def _sections(pairs, axes):
    """The axis of every rotated pair: runs of pairs per axis, time the shortest of three."""
    runs = {1: [pairs], 2: [pairs // 2] * 2, 3: [pairs // 4, pairs * 3 // 8, pairs * 3 // 8], 4: [pairs // 4] * 4}[axes]
    return [a for a, r in enumerate(runs) for _ in range(r)]


def _positions(axes, T, gen):
    """Positions of T tokens: the first axis counts on, the others run over a picture's rows and columns."""
    at = torch.arange(T, device=DEV)
    base = torch.randint(0, 40000, (1,), generator=gen, device=DEV)
    wide = torch.randint(20, 120, (1,), generator=gen, device=DEV)
    rows = [at + base, at // wide % 96, at % wide, at // (wide * 96)]
    return torch.stack(rows[:axes]).to(torch.int32).contiguous()


def _inputs(case, seed):
    """All tensors of a case, on the GPU."""
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    dtype, D = DTYPES[case["dtype"]], case["dim"]

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32) * scale).to(dtype)

    s = {"case": case}
    if "rot" in case:
        R = case["rot"]
        s["inv_freq"] = (1.0e6 ** (-torch.arange(R // 2, device=DEV, dtype=torch.float64) * 2 / R)).float()
        s["axis"] = _sections(R // 2, case["axes"])
        s["axis_dev"] = torch.tensor(s["axis"], device=DEV)
    if case["kind"] == "rope":
        T = case["tokens"]
        s["pos"] = _positions(case["axes"], T, gen)
        s["x"] = normal(T, case["heads"], D)
        s["y"] = torch.empty_like(s["x"])
        return s

    S, Hk, ps = case["seqs"], case["kv_heads"], case["page"]
    order = torch.randperm(S, generator=gen, device=DEV).tolist()
    sizes = [_sizes(case)[i] for i in order]
    new, total = [n for n, _ in sizes], [L for _, L in sizes]
    T, longest = sum(new), max(total)
    s["new"], s["total"], s["T"] = new, total, T
    s["kv_len"] = torch.tensor(total, dtype=torch.int32, device=DEV)
    s["q_off"] = torch.tensor([0] + new, device=DEV).cumsum(0)
    # pages in the order of an allocator that has been running for a while
    need = [-(-L // ps) for L in total]
    kept = [-(-min(L, case["budget"]) // ps) for L in total] if case["kind"] == "evict" else [0] * S
    n_pages = sum(need) + sum(kept)
    pages = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)

    def table(counts, first):
        most = max(1, max(counts))
        off = torch.tensor([0] + counts[:-1], device=DEV).cumsum(0)
        col = torch.arange(most, device=DEV)
        at = torch.where(col < torch.tensor(counts, device=DEV)[:, None], off[:, None] + col, 0)
        return pages[first + at].contiguous()

    s["table"] = table(need, 0)
    s["k"] = normal(n_pages, Hk, ps, D)
    s["v"] = normal(n_pages, Hk, ps, D)
    if case["kind"] == "evict":
        s["dst"] = table(kept, sum(need))
        # attention that positions received: many light ones, a few heavy ones, some never seen
        w = torch.randn(S, longest, generator=gen, device=DEV).mul_(2.0).exp_()
        s["weight"] = torch.where(torch.rand(S, longest, generator=gen, device=DEV) < 0.02, torch.zeros_like(w), w)
        keep = [min(L, case["budget"]) for L in total]
        s["rows"] = (torch.repeat_interleave(torch.arange(S, device=DEV), torch.tensor(keep, device=DEV)),
                     torch.cat([torch.arange(n, device=DEV) for n in keep]))
        s["index"] = torch.empty(S, case["budget"], dtype=torch.int32, device=DEV)
        s["new_len"] = torch.empty(S, dtype=torch.int32, device=DEV)
        s["new_weight"] = torch.zeros(S, case["budget"], device=DEV)
        return s

    Hq = case["q_heads"]
    s["seq"] = torch.repeat_interleave(torch.arange(S, device=DEV), torch.tensor(new, device=DEV))
    s["nth"] = torch.arange(T, device=DEV) - s["q_off"][s["seq"]]
    if case["kind"] == "append":
        s["pos"] = _positions(case["axes"], T, gen)
        qkv = normal(T, Hq + 2 * Hk, D)                 # one projection's output, read in place
        s["q"], s["kn"], s["vn"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
        s["q_out"] = torch.empty(T, Hq, D, dtype=dtype, device=DEV)
        return s
    s["scale"] = D ** -0.5
    s["q"] = normal(T, Hq, D, scale=1.5)
    if case["kind"] == "attend":
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(T, Hq, device=DEV)
        return s
    # what the attention of normal keys gives: the logarithm of the mean of exp over the visible ones, and their number
    p = s["kv_len"].long()[s["seq"]] - s["q_off"].diff()[s["seq"]] + s["nth"]
    seen = p + 1
    if case["window"] > 0:
        first = (p - case["window"] + 1).clamp(min=0)
        seen = p + 1 - first + first.clamp(max=case["sinks"])
    s["lse"] = seen.float().log()[:, None] + s["q"].float().square().sum(-1) * (s["scale"] ** 2 / 2)
    s["weight"] = torch.rand(S, longest, generator=gen, device=DEV)
    s["new_weight"] = torch.zeros(S, longest, device=DEV)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    import paper_2609_18703_amd as R
    ctx = s["ctx"] = R.Context()
    if "rot" in case:
        s["rotary"] = R.Rotary(s["inv_freq"], s["axis"], adjacent=case["pairs"])
    if case["kind"] == "rope":
        return s
    # a step's plan: one for all layers of a model
    s["cache"] = R.Cache(s["k"], s["v"])
    s["chunk"] = ctx.chunk(case["seqs"], s["T"], s["table"].shape[1])
    s["chunk"].plan(s["cache"], s["q_off"], s["kv_len"], s["table"], case.get("q_heads", case["kv_heads"]),
                    n_tokens=s["T"], max_new=max(s["new"]), window=case.get("window", 0), sinks=case.get("sinks", 0))
    ctx.check("plan")
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    kind = s["case"]["kind"]
    return (_library if own else _plain)[kind](s)


def _own_rope(s):
    s["ctx"].rope(s["x"], s["y"], s["rotary"], s["pos"], inverse=s["case"]["inverse"])
    return {"y": s["y"]}


def _own_append(s):
    s["chunk"].append(s["cache"], s["q"], s["kn"], s["vn"], s["q_out"], s["rotary"], s["pos"])
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _own_attend(s):
    s["chunk"].attend(s["cache"], s["q"], s["out"], s["lse"], scale=s["scale"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_weigh(s):
    s["chunk"].weigh(s["cache"], s["q"], s["lse"], s["weight"], s["new_weight"], scale=s["scale"])
    return {"weight": s["new_weight"]}


def _own_evict(s):
    c = s["case"]
    s["chunk"].evict(s["cache"], s["weight"], s["dst"], c["budget"], s["new_len"], s["index"], s["new_weight"],
                     first=c["first"], last=c["last"])
    return {"len": s["new_len"], "index": s["index"], "weight": s["new_weight"], "k": s["k"], "v": s["v"]}


_library = {"rope": _own_rope, "append": _own_append, "attend": _own_attend, "weigh": _own_weigh, "evict": _own_evict}


def _rotate(x, s, sign=1.0):
    c = s["case"]
    R = c["rot"]
    angle = s["pos"].float()[s["axis_dev"]].T * s["inv_freq"]              # [T, R/2]
    cos, sin = angle.cos()[:, None], angle.sin()[:, None] * sign
    f = x.float()
    if c["pairs"]:
        a, b = f[..., 0:R:2], f[..., 1:R:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = f[..., :R // 2], f[..., R // 2:R]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, f[..., R:]], -1).to(x.dtype)


def _plain_rope(s):
    return {"y": _rotate(s["x"], s, -1.0 if s["case"]["inverse"] else 1.0)}


def _plain_append(s):
    ps = s["case"]["page"]
    at = s["kv_len"].long()[s["seq"]] - s["q_off"].diff()[s["seq"]] + s["nth"]
    page = s["table"].long()[s["seq"], at // ps]
    s["k"][page, :, at % ps] = _rotate(s["kn"], s)
    s["v"][page, :, at % ps] = s["vn"]
    return {"q": _rotate(s["q"], s), "k": s["k"], "v": s["v"]}


def _padded(s):
    """Queries [S, kv heads, new x group, D], scores' mask [S, new, length] and the page and slot of every position."""
    c = s["case"]
    S, Hk, ps, D = c["seqs"], c["kv_heads"], c["page"], c["dim"]
    n, L = max(s["new"]), max(s["total"])
    group = c["q_heads"] // Hk
    new, total = s["q_off"].diff(), s["kv_len"].long()
    i, j = torch.arange(n, device=DEV), torch.arange(L, device=DEV)
    at = (s["q_off"][:-1, None] + i).clamp(max=s["T"] - 1)
    q = s["q"][at].float().view(S, n, Hk, group, D).permute(0, 2, 1, 3, 4).reshape(S, Hk, n * group, D)
    p = (total - new)[:, None] + i
    see = (j <= p[..., None]) & (i < new[:, None])[..., None]
    if c["window"] > 0:
        see &= (j > p[..., None] - c["window"]) | (j < c["sinks"])
    page = s["table"].long()[:, j // ps]
    return q, see, page, j % ps, group


def _scores(s):
    c = s["case"]
    q, see, page, slot, group = _padded(s)
    k = s["k"][page, :, slot].float().transpose(1, 2)                        # [S, kv heads, length, D]
    x = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"])
    x = x.view(c["seqs"], c["kv_heads"], -1, group, x.shape[-1])
    return x.masked_fill_(~see[:, None, :, None], -math.inf), page, slot


def _plain_attend(s):
    c = s["case"]
    x, page, slot = _scores(s)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top.masked_fill(top == -math.inf, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    v = s["v"][page, :, slot].float().transpose(1, 2)
    o = torch.matmul(p.flatten(2, 3), v).view(*p.shape[:-1], c["dim"]) / total.clamp(min=1e-30)
    lse = torch.where(total > 0, top + total.log(), -math.inf)[..., 0]
    o, lse = o.permute(0, 2, 1, 3, 4), lse.permute(0, 2, 1, 3)               # [S, new, kv heads, group, ...]
    return {"out": o[s["seq"], s["nth"]].reshape(s["q"].shape).to(s["q"].dtype),
            "lse": lse[s["seq"], s["nth"]].reshape(s["T"], -1)}


def _plain_weigh(s):
    c = s["case"]
    n, L, S, Hq = max(s["new"]), max(s["total"]), c["seqs"], c["q_heads"]
    lse = torch.zeros(S, n, Hq, device=DEV)
    lse[s["seq"], s["nth"]] = s["lse"]
    x, _, _ = _scores(s)
    lse = lse.view(S, n, c["kv_heads"], -1).transpose(1, 2)
    got = x.sub_(lse[..., None]).exp_().sum((1, 2, 3))
    j = torch.arange(L, device=DEV)
    return {"weight": torch.where(j < s["kv_len"][:, None], s["weight"] + got, s["new_weight"])}


def _plain_evict(s):
    c = s["case"]
    ps, budget = c["page"], c["budget"]
    total = s["kv_len"].long()[:, None]
    j = torch.arange(max(s["total"]), device=DEV)
    stays = (j < c["first"]) | (j >= total - c["last"])
    key = torch.where(j < total, torch.where(stays, math.inf, s["weight"]), -math.inf)
    ranked = key.sort(dim=-1, descending=True, stable=True).indices[:, :budget]
    m = ranked.shape[1]
    keep = total.clamp(max=budget)
    rank = torch.arange(m, device=DEV)
    index = torch.where(rank < keep, ranked, total.max()).sort(-1).values
    seq, nth = s["rows"]
    src = index[seq, nth]
    page, to = s["table"].long()[seq, src // ps], s["dst"].long()[seq, nth // ps]
    s["k"][to, :, nth % ps] = s["k"][page, :, src % ps]
    s["v"][to, :, nth % ps] = s["v"][page, :, src % ps]
    s["index"].fill_(-1)
    s["index"][seq, nth] = src.int()
    s["new_weight"][seq, nth] = s["weight"][seq, src]
    return {"len": keep[:, 0].int(), "index": s["index"], "weight": s["new_weight"], "k": s["k"], "v": s["v"]}


_plain = {"rope": _plain_rope, "append": _plain_append, "attend": _plain_attend, "weigh": _plain_weigh,
          "evict": _plain_evict}


# ------------------------------------------------------------------ the definitions, in 64 bits

def _turn(x, s, back=False):
    """The rotation as complex numbers."""
    c, R = s["case"], s["case"]["rot"]
    out = x.double()
    a = torch.empty(x.shape[0], R // 2, dtype=torch.float64, device=DEV)
    for i, axis in enumerate(s["axis"]):
        a[:, i] = s["pos"][axis].double() * s["inv_freq"][i].double()
    turn = torch.polar(torch.ones_like(a), -a if back else a)[:, None]
    first = slice(0, R, 2) if c["pairs"] else slice(0, R // 2)
    second = slice(1, R, 2) if c["pairs"] else slice(R // 2, R)
    z = torch.complex(out[..., first].clone(), out[..., second].clone()) * turn
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _sequence(s, n):
    """Tokens, cached pages' positions of sequence n: (first token, new, length, flat row of every position)."""
    t0, new, L = int(s["q_off"][n]), s["new"][n], s["total"][n]
    ps = s["case"]["page"]
    page = s["table"][n].long().repeat_interleave(ps)[:L]
    return t0, new, L, page, torch.arange(L, device=DEV) % ps


def exact(case, seed):
    s = _inputs(dict(case), seed)
    kind = case["kind"]
    if kind == "rope":
        return {"y": _turn(s["x"], s, case["inverse"])}
    if kind == "append":
        k, v = s["k"].double(), s["v"].double()
        kn = _turn(s["kn"], s)
        for n in range(case["seqs"]):
            t0, new, L, page, slot = _sequence(s, n)
            k[page[L - new:], :, slot[L - new:]] = kn[t0:t0 + new]
            v[page[L - new:], :, slot[L - new:]] = s["vn"][t0:t0 + new].double()
        return {"q": _turn(s["q"], s), "k": k, "v": v}
    if kind == "evict":
        return _exact_evict(s)
    Hk, group, D = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["dim"]
    out = torch.zeros(s["T"], case["q_heads"], D, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["T"], case["q_heads"], dtype=torch.float64, device=DEV)
    weight = s["new_weight"].double() if kind == "weigh" else None
    for n in range(case["seqs"]):
        t0, new, L, page, slot = _sequence(s, n)
        if kind == "weigh":
            weight[n, :L] = s["weight"][n, :L].double()
        p, j = torch.arange(L - new, L, device=DEV)[:, None], torch.arange(L, device=DEV)
        hidden = j > p
        if case["window"] > 0:
            hidden = hidden | ((p - j >= case["window"]) & (j >= case["sinks"]))
        hidden = hidden.repeat_interleave(group, 0)
        keys, values = s["k"][page, :, slot], s["v"][page, :, slot]
        step = max(1, (1 << 27) // (L * group))
        for h in range(Hk):
            for a in range(0, new, step):
                b = min(new, a + step)
                heads = slice(h * group, (h + 1) * group)
                q = s["q"][t0 + a:t0 + b, heads].double().reshape(-1, D)
                x = (q @ keys[:, h].double().T.contiguous()) * s["scale"]
                x[hidden[a * group:b * group]] = -math.inf
                if kind == "weigh":
                    weight[n, :L] += (x - s["lse"][t0 + a:t0 + b, heads].double().reshape(-1, 1)).exp().sum(0)
                    continue
                z = torch.logsumexp(x, -1, keepdim=True)
                out[t0 + a:t0 + b, heads] = ((x - z).exp() @ values[:, h].double()).view(b - a, group, D)
                lse[t0 + a:t0 + b, heads] = z.view(b - a, group)
    return {"weight": weight} if kind == "weigh" else {"out": out, "lse": lse}


def _exact_evict(s):
    c = s["case"]
    ps, budget = c["page"], c["budget"]
    k, v, weight = s["k"].double(), s["v"].double(), s["new_weight"].double()
    index = torch.full((c["seqs"], budget), -1, dtype=torch.int32, device=DEV)
    length = torch.empty(c["seqs"], dtype=torch.int32, device=DEV)
    for n in range(c["seqs"]):
        _, _, L, page, slot = _sequence(s, n)
        kept = list(range(L))
        if L > budget:
            w = s["weight"][n, :L].tolist()
            middle = sorted(range(c["first"], L - c["last"]), key=lambda i: (-w[i], i))
            kept = sorted(list(range(c["first"])) + middle[:budget - c["first"] - c["last"]]
                          + list(range(L - c["last"], L)))
        at = torch.tensor(kept, device=DEV)
        m = len(kept)
        to, into = s["dst"][n].long().repeat_interleave(ps)[:m], torch.arange(m, device=DEV) % ps
        k[to, :, into] = s["k"][page[at], :, slot[at]].double()
        v[to, :, into] = s["v"][page[at], :, slot[at]].double()
        weight[n, :m] = s["weight"][n, at].double()
        index[n, :m] = at.int()
        length[n] = m
    return {"len": length, "index": index, "weight": weight, "k": k, "v": v}
