"""Operators of a model stage's step around its attention, as cases to time.

One more token of every child in a batch takes, besides attention over its
paged cache: projections, a choice, and pages to put it in.  Four kinds of
work:

  project  rows to 8-bit integers with a scale each, then the product with
           8-bit weights that have a scale for each channel.
  sample   the next token from logits: temperature, top-k, top-p, min-p, a
           mask of allowed tokens; the random numbers are inputs.
  fork     the children of the last batch give their pages back; those of the
           next one share their parents' prompts and get room for new tokens,
           a shared last page is copied in every layer.
  compact  a pool with holes: live pages move to the lowest numbers, tables
           and every layer's keys and values follow.

`own` says which side `run` takes: the plain form in 32 bits (64 for sums and
near borders), or the library.  All values are drawn from the seed on the GPU.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
NONE = -1                               # no page


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # queries, keys and values of a few children's next tokens: latency, the weights are read once
        {"name": "project-tokens", "kind": "project", "m": 5, "k": 3584, "n": 4608, "bias": True, "x": "bf16",
         "out": "bf16"},
        # a full batch's logits over a large vocabulary of odd size
        {"name": "project-logits", "kind": "project", "m": 64, "k": 4096, "n": 150001, "bias": False, "x": "bf16",
         "out": "bf16"},
        # prompts of a few hundred tokens beside single ones
        {"name": "project-mixed", "kind": "project", "m": 777, "k": 5120, "n": 7168, "bias": True, "x": "f16",
         "out": "f16"},
        # a long prompt's chunk through a wide layer
        {"name": "project-prompt", "kind": "project", "m": 12001, "k": 4096, "n": 16384, "bias": False, "x": "bf16",
         "out": "bf16"},
        # a few sequences, every kind of filter among them: latency
        {"name": "sample-few", "kind": "sample", "rows": 5, "vocab": 32003, "filters": "mixed", "mask": 0.0,
         "spread": 3.0, "dtype": "bf16"},
        # a full batch over a large vocabulary
        {"name": "sample-batch", "kind": "sample", "rows": 64, "vocab": 150001, "filters": "mixed", "mask": 0.0,
         "spread": 2.5, "dtype": "bf16"},
        # a grammar allows few tokens
        {"name": "sample-masked", "kind": "sample", "rows": 48, "vocab": 65537, "filters": "mixed", "mask": 0.97,
         "spread": 2.0, "dtype": "f16"},
        # many short generations at once, temperature alone
        {"name": "sample-many", "kind": "sample", "rows": 1024, "vocab": 128000, "filters": "temperature",
         "mask": 0.0, "spread": 3.0, "dtype": "f16"},
        # a few children of short prompts: latency
        {"name": "fork-few", "kind": "fork", "parents": 3, "children": 13, "len_lo": 9, "len_hi": 901, "add_lo": 1,
         "add_hi": 1, "page": 16, "layers": 2, "kv_heads": 4, "dim": 128, "spare": 40, "dtype": "bf16"},
        # a batch of siblings of long prompts, some with chunks of their own
        {"name": "fork-batch", "kind": "fork", "parents": 61, "children": 500, "len_lo": 100, "len_hi": 4001,
         "add_lo": 1, "add_hi": 130, "page": 64, "layers": 4, "kv_heads": 4, "dim": 128, "spare": 500,
         "dtype": "bf16"},
        # some of a few sequences have ended: latency
        {"name": "compact-few", "kind": "compact", "seqs": 17, "len_lo": 1, "len_hi": 700, "gone": 5, "page": 16,
         "layers": 2, "kv_heads": 4, "dim": 128, "spare": 31, "dtype": "f16"},
        # a pool after a day: half of the sequences have ended
        {"name": "compact-many", "kind": "compact", "seqs": 700, "len_lo": 1, "len_hi": 6007, "gone": 350, "page": 16,
         "layers": 2, "kv_heads": 4, "dim": 128, "spare": 9000, "dtype": "bf16"},
    ]


MOST_PRODUCT = 12001 * 4096 * 16384
MOST_LOGITS = 1024 * 128000
MOST_SLOTS = 8 * 320000 * 4 * 128       # elements of all layers' keys


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["project", "project", "sample", "sample", "fork", "compact"])
    if kind == "project":
        while True:
            m, k, n = log(1, 12001), 16 * log(2, 1024), log(1, 160000)
            if m * k * n <= MOST_PRODUCT and m * n <= 12001 * 16384 and k * n <= 1 << 30:
                break
        x = rng.choice(["bf16", "f16"])
        return {"kind": "project", "m": m, "k": k, "n": n, "bias": rng.random() < 0.5, "x": x,
                "out": rng.choice([x, x, "f32"])}
    if kind == "sample":
        while True:
            rows, vocab = log(1, 1024), log(1, 262144)
            if rows * vocab <= MOST_LOGITS:
                break
        return {"kind": "sample", "rows": rows, "vocab": vocab,
                "filters": rng.choice(["mixed", "mixed", "temperature", "greedy"]),
                "mask": rng.choice([0.0, 0.0, 0.3, 0.97]), "spread": rng.choice([0.5, 2.0, 3.0, 8.0]),
                "dtype": rng.choice(["bf16", "f16"])}
    while True:
        case = {"kind": kind, "page": rng.choice([16, 32, 64, 128]), "layers": rng.randrange(1, 9),
                "kv_heads": rng.choice([1, 2, 4, 8]), "dim": rng.choice([64, 128]), "spare": log(1, 9000),
                "len_hi": log(2, 8000), "dtype": rng.choice(["bf16", "f16"])}
        case["len_lo"] = max(1, case["len_hi"] // rng.randrange(1, 50))
        if kind == "fork":
            case.update(parents=log(1, 100), children=log(1, 1000), add_lo=rng.choice([0, 1]), add_hi=log(1, 300))
            slots = case["parents"] * case["len_hi"] + case["children"] * (case["add_hi"] + case["page"])
        else:
            case["seqs"] = log(1, 1000)
            case["gone"] = rng.randrange(0, case["seqs"] + 1)
            slots = case["seqs"] * case["len_hi"]
        slots += case["spare"] * case["page"]
        if slots * case["layers"] * case["kv_heads"] * case["dim"] <= MOST_SLOTS:
            return case


# ------------------------------------------------------------------ sizes that follow from a case

def _spread(lo, hi, n):
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [hi]


def _pages(positions, page):
    return -(-positions // page)


def _fork_sizes(case):
    """(parents' lengths, child's parent, child's new tokens): as many children a parent as its turn gives."""
    P, C = case["parents"], case["children"]
    lens = _spread(case["len_lo"], case["len_hi"], P)
    return lens, [(i * 7 + i // P) % P for i in range(C)], _spread(case["add_lo"], case["add_hi"], C)


def _fork_need(case):
    """(pages that the children take, positions of shared last pages that are copied)."""
    lens, parent, add = _fork_sizes(case)
    ps = case["page"]
    need = slots = 0
    for p, a in zip(parent, add):
        need += _pages(lens[p] + a, ps) - _pages(lens[p], ps)
        if a > 0 and lens[p] % ps:
            need += 1
            slots += lens[p] % ps
    return need, slots


def work(case):
    if case["kind"] == "project":
        m, k, n = case["m"], case["k"], case["n"]
        size = 4.0 if case["out"] == "f32" else 2.0
        return {"bytes": 2.0 * m * k + n * k + 4.0 * (n + (n if case["bias"] else 0)) + size * m * n,
                "flops": 2.0 * m * n * k}
    if case["kind"] == "sample":
        n, V = case["rows"], case["vocab"]
        return {"bytes": 2.0 * n * V + (n * V / 8.0 if case["mask"] > 0 else 0.0) + 28.0 * n, "flops": 0.0}
    ps = case["page"]
    row = 4.0 * case["layers"] * case["kv_heads"] * case["dim"]          # keys and values of one position
    if case["kind"] == "fork":
        lens, parent, _ = _fork_sizes(case)
        need, slots = _fork_need(case)
        held = sum(_pages(lens[p], ps) for p in parent)
        pool = sum(_pages(x, ps) for x in lens) + need + case["spare"]
        return {"bytes": 2 * row * slots + 4.0 * pool + 8.0 * held + 4.0 * need, "flops": 0.0}
    lens = _spread(case["len_lo"], case["len_hi"], case["seqs"])
    stay = _stays(case)
    live = sum(_pages(x, ps) for x, s in zip(lens, stay) if s)
    pool = sum(_pages(x, ps) for x in lens) + case["spare"]
    moved = live * (pool - live) / pool                  # pages lie anywhere: the live ones beyond the live count
    return {"bytes": 2 * row * ps * moved + 4.0 * pool + 8.0 * live, "flops": 0.0}


def _stays(case):
    """Which sequences have not ended: those that have are spread over all lengths."""
    S, gone = case["seqs"], case["gone"]
    return [(i + 1) * gone // S == i * gone // S for i in range(S)]


# ------------------------------------------------------------------ what a program has in hand

def _inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    s = {"case": case}

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)

    if case["kind"] == "project":
        m, k, n = case["m"], case["k"], case["n"]
        # some channels of a hidden state are far larger than the rest
        loud = 1.0 + 20.0 * (torch.rand(k, generator=gen, device=DEV) < 0.003)
        s["x"] = (normal(m, k) * loud).to(DTYPES[case["x"]])
        s["w"] = torch.randint(-127, 128, (n, k), generator=gen, device=DEV, dtype=torch.int8)
        s["w_scale"] = (torch.rand(n, generator=gen, device=DEV) + 0.5) / (74.0 * k ** 0.5)
        s["bias"] = normal(n) if case["bias"] else None
        s["out"] = torch.empty(m, n, dtype=DTYPES[case["out"]], device=DEV)
        return s
    if case["kind"] == "sample":
        n, V = case["rows"], case["vocab"]
        x = normal(n, V) * case["spread"]
        # a few tokens stand out, by as much as the row is sure
        few = min(V, 24)
        at = torch.randint(0, V, (n, few), generator=gen, device=DEV)
        x.scatter_add_(1, at, torch.rand(n, few, generator=gen, device=DEV) * 12.0
                       * torch.rand(n, 1, generator=gen, device=DEV))
        s["logits"] = x.to(DTYPES[case["dtype"]])
        s["u"] = torch.rand(n, generator=gen, device=DEV)
        nth = torch.arange(n, device=DEV) + int(torch.randint(0, 64, (1,), generator=gen, device=DEV))

        def turn(values, dtype):
            return torch.tensor(values, dtype=dtype, device=DEV)[nth % len(values)].contiguous()
        if case["filters"] == "greedy":
            s["temperature"] = torch.zeros(n, device=DEV)
        else:
            s["temperature"] = turn([1.0, 0.7, 0.0, 1.3, 0.3] if case["filters"] == "mixed" else [0.8, 1.0, 1.1],
                                    torch.float32)
        if case["filters"] == "mixed":
            s["top_k"] = turn([0, 50, 0, 20, 1000, 0, 1], torch.int32)
            s["top_p"] = turn([1.0, 0.9, 0.95, 1.0, 0.5, 0.99], torch.float32)
            s["min_p"] = turn([0.0, 0.0, 0.05, 0.0, 0.1, 0.0, 0.0, 0.02], torch.float32)
        if case["mask"] > 0:
            words = _pages(V, 32)
            bit = torch.rand(n, words * 32, generator=gen, device=DEV) >= case["mask"]
            weight = 1 << torch.arange(32, device=DEV)
            s["mask"] = (bit.view(n, words, 32) * weight).sum(-1)
            s["mask"] = torch.where(s["mask"] >= 1 << 31, s["mask"] - (1 << 32), s["mask"]).int()
        s["token"] = torch.empty(n, dtype=torch.int32, device=DEV)
        s["logprob"] = torch.empty(n, device=DEV)
        return s

    ps, spare = case["page"], case["spare"]
    if case["kind"] == "fork":
        lens, parent, add = _fork_sizes(case)
        order = torch.randperm(len(lens), generator=gen, device=DEV).tolist()
        lens = [lens[i] for i in order]
        parent = [order.index(p) for p in parent]
        turn = torch.randperm(len(parent), generator=gen, device=DEV).tolist()
        parent, add = [parent[i] for i in turn], [add[i] for i in turn]
        n_pages = sum(_pages(x, ps) for x in lens) + _fork_need(case)[0] + spare
        cols = max(_pages(lens[p] + a, ps) for p, a in zip(parent, add))
        cols = max(cols, _pages(max(lens), ps))
    else:
        lens = _spread(case["len_lo"], case["len_hi"], case["seqs"])
        n_pages = sum(_pages(x, ps) for x in lens) + spare
        cols = _pages(max(lens), ps)
    # an allocator that has been running for a while: pages in any order, sequences in any place
    pages = torch.randperm(n_pages, generator=gen, device=DEV).int()
    held = [_pages(x, ps) for x in lens]
    if case["kind"] == "compact":
        # those that have ended have given theirs back
        stay = _stays(case)
        lens = [x if t else 0 for x, t in zip(lens, stay)]
    off = torch.tensor([0] + held, device=DEV).cumsum(0)[:-1]
    col = torch.arange(cols, device=DEV)
    have = torch.tensor([_pages(x, ps) for x in lens], device=DEV)
    at = torch.where(col < have[:, None], off[:, None] + col, 0)
    table = torch.where(col < have[:, None], pages[at], NONE)
    length = torch.tensor(lens, dtype=torch.int32, device=DEV)
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[table[table != NONE].long()] = 1
    # the pool's words lie in one block, as they would be saved: references, tables, lengths
    S = len(lens)
    block = torch.cat([refs, table.flatten().int(), length])
    s["block"], s["saved"] = block, block.clone()
    s["refs"], s["table"], s["len"] = block[:n_pages], block[n_pages:n_pages + S * cols].view(S, cols), block[-S:]
    shape = (n_pages, case["kv_heads"], ps, case["dim"])
    kv = [normal(*shape).to(DTYPES[case["dtype"]]) for _ in range(2 * case["layers"])]
    s["k"], s["v"] = kv[::2], kv[1::2]
    if case["kind"] == "fork":
        C = case["children"]
        s["parent"] = torch.tensor(parent, dtype=torch.int32, device=DEV)
        s["add"] = torch.tensor(add, dtype=torch.int32, device=DEV)
        s["to"] = torch.full((C, cols), NONE, dtype=torch.int32, device=DEV)
        s["to_len"] = torch.zeros(C, dtype=torch.int32, device=DEV)
        s["src"], s["dst"], s["slots"] = (torch.empty(C, dtype=torch.int32, device=DEV) for _ in range(3))
    else:
        # (entries behind the moves stay as they are)
        s["src"], s["dst"] = (torch.full((n_pages,), NONE, dtype=torch.int32, device=DEV) for _ in range(2))
        s["moves"] = torch.zeros(1, dtype=torch.int64, device=DEV)
    s["free"] = torch.zeros(1, dtype=torch.int64, device=DEV)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    import paper_2609_18703_amd as R
    ctx = s["ctx"] = R.Context()
    if case["kind"] == "project":
        s["weights"] = R.Weights(s["w"], s["w_scale"], s["bias"])
        s["q"] = torch.empty(case["m"], case["k"], dtype=torch.int8, device=DEV)
        s["scale"] = torch.empty(case["m"], device=DEV)
    elif case["kind"] in ("fork", "compact"):
        s["pool"] = ctx.pages(s["refs"], case["page"], max(s["table"].shape[0], case.get("children", 0)))
        s["tables"] = R.Tables(s["table"], s["len"])
        s["caches"] = [R.Cache(k, v) for k, v in zip(s["k"], s["v"])]
        if case["kind"] == "fork":
            s["children"] = R.Tables(s["to"], s["to_len"])
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return (_library if own else _plain)[s["case"]["kind"]](s)


def _own_project(s):
    s["ctx"].quantize(s["x"], s["q"], s["scale"])
    s["ctx"].project(s["q"], s["scale"], s["weights"], s["out"])
    return {"out": s["out"], "scale": s["scale"]}


def _own_sample(s):
    s["ctx"].sample(s["logits"], s["u"], s["token"], s["logprob"], temperature=s["temperature"],
                    top_k=s.get("top_k"), top_p=s.get("top_p"), min_p=s.get("min_p"), mask=s.get("mask"))
    return {"token": s["token"], "logprob": s["logprob"]}


def _own_fork(s):
    pool = s["pool"]
    pool.release(s["children"])
    pool.fork(s["tables"], s["parent"], s["children"])
    pool.grow(s["children"], s["add"], s["src"], s["dst"], s["slots"], s["free"])
    pool.copy(s["caches"], s["src"], s["dst"], s["slots"])
    return {x: s[x] for x in ("to", "to_len", "refs", "src", "dst", "slots", "free", "k", "v")}


def _own_compact(s):
    s["block"].copy_(s["saved"])
    s["pool"].compact([s["tables"]], s["src"], s["dst"], s["moves"], s["free"])
    s["pool"].copy(s["caches"], s["src"], s["dst"], n=s["moves"])
    return {x: s[x] for x in ("table", "len", "refs", "src", "dst", "moves", "free", "k", "v")}


_library = {"project": _own_project, "sample": _own_sample, "fork": _own_fork, "compact": _own_compact}


def _plain_project(s):
    f = s["x"].float()
    top = f.abs().amax(-1, keepdim=True)
    q = torch.where(top > 0, f * 127.0 / top, 0.0).round()
    w = s["w"].float()
    acc = torch.zeros(q.shape[0], w.shape[0], dtype=torch.float64, device=DEV)
    for a in range(0, q.shape[1], 1024):                 # sums of 1,024 such products are exact in 32 bits
        acc += q[:, a:a + 1024] @ w[:, a:a + 1024].T
    scale = top / 127.0
    out = acc.float() * scale * s["w_scale"]
    if s["bias"] is not None:
        out = out + s["bias"]
    return {"out": out.to(s["out"].dtype), "scale": scale[:, 0]}


def _allowed(s):
    V = s["case"]["vocab"]
    ok = s["logits"] > -math.inf                         # NaN is not
    if "mask" in s:
        bit = (s["mask"][..., None] >> torch.arange(32, device=DEV)) & 1
        ok &= bit.flatten(1)[:, :V] != 0
    return ok


def _plain_sample(s):
    V = s["case"]["vocab"]
    x = torch.where(_allowed(s), s["logits"].float(), -math.inf)
    T = s["temperature"].double()[:, None]
    x, order = x.sort(dim=-1, descending=True, stable=True)
    z = x.double() / torch.where(T > 0, T, 1.0)
    # the largest is the first; an infinite one leaves the rest nothing
    diff = torch.where(z == z[:, :1], 0.0, z - z[:, :1]).masked_fill(x == -math.inf, -math.inf)
    w = diff.exp()
    total = w.sum(-1, keepdim=True)
    rank = torch.arange(V, device=DEV)
    keep = x > -math.inf
    if "top_k" in s:
        k = s["top_k"].long()[:, None]
        keep &= (rank < k) | (k <= 0)
    if "top_p" in s:
        p = s["top_p"].double()[:, None]
        left = w * keep
        before = left.cumsum(-1).roll(1, -1)
        before[:, 0] = 0.0
        keep &= (before < p * left.sum(-1, keepdim=True)) | (p >= 1)
    if "min_p" in s:
        keep &= w >= s["min_p"].double()[:, None]
    keep &= (T > 0) | (rank == 0)
    keep[:, 0] |= x[:, 0] > -math.inf
    sums = (w * keep).cumsum(-1)
    pick = (sums <= s["u"].double()[:, None] * sums[:, -1:]).sum(-1, keepdim=True)
    pick = pick.minimum(keep.sum(-1, keepdim=True) - 1)
    none = pick < 0
    pick = pick.clamp(min=0)
    token = order.gather(1, pick).masked_fill(none, -1)
    logprob = (diff.gather(1, pick) - total.log()).masked_fill(none, -math.inf)
    return {"token": token[:, 0].int(), "logprob": logprob[:, 0].float()}


def _held(table, length, page):
    """Which entries of a table are held."""
    return torch.arange(table.shape[1], device=DEV) < ((length.long() + page - 1) // page)[:, None]


def _copy(s, src, dst, slots=None):
    """Pages src to pages dst, the first `slots` positions of them, in every layer."""
    src, dst = src.long(), dst.long()
    for t in s["k"] + s["v"]:
        if slots is None:
            t[dst] = t[src]
        else:
            inside = (torch.arange(t.shape[2], device=DEV) < slots[:, None])[:, None, :, None]
            t[dst] = torch.where(inside, t[src], t[dst])


def _plain_fork(s):
    ps, refs, to, length = s["case"]["page"], s["refs"], s["to"], s["to_len"]

    def count(pages, by):
        refs.index_add_(0, pages.long(), torch.full_like(pages, by))
    # the last children leave
    count(to[_held(to, length, ps)], -1)
    to.fill_(NONE)
    # the next ones share their parents' pages
    parent = s["parent"].long()
    length.copy_(s["len"][parent])
    held = _held(to, length, ps)
    to.copy_(torch.where(held, s["table"][parent], NONE))
    count(to[held], 1)
    # ... and grow: a shared last page that is partly filled, then new ones
    have = (length.long() + ps - 1) // ps
    want = (length.long() + s["add"] + ps - 1) // ps
    last = to.gather(1, (have - 1).clamp(min=0)[:, None])[:, 0]
    own_copy = (s["add"] > 0) & (length % ps != 0) & (refs[last.clamp(min=0).long()] > 1)
    first = have - own_copy.long()
    need = want - first
    free = (refs == 0).nonzero()[:, 0]
    take = need.cumsum(0) - need
    col = torch.arange(to.shape[1], device=DEV)
    new = (col >= first[:, None]) & (col < want[:, None])
    at = torch.where(new, take[:, None] + col - first[:, None], 0)
    src = torch.where(own_copy, last, NONE)
    fresh = torch.cat([free, free.new_zeros(1)])[at].int()
    to.copy_(torch.where(new, fresh, to))
    count(to[new], 1)
    count(last[own_copy], -1)
    dst = torch.where(own_copy, to.gather(1, first.clamp(max=to.shape[1] - 1)[:, None])[:, 0], NONE)
    slots = torch.where(own_copy, length % ps, 0)
    length += s["add"]
    _copy(s, src[own_copy], dst[own_copy], slots[own_copy])
    return {"to": to, "to_len": length, "refs": refs, "src": src, "dst": dst, "slots": slots,
            "free": (refs == 0).sum().view(1), "k": s["k"], "v": s["v"]}


def _plain_compact(s):
    s["block"].copy_(s["saved"])
    refs, table = s["refs"], s["table"]
    live = (refs > 0).sum()
    at = torch.arange(refs.numel(), device=DEV)
    src = ((refs > 0) & (at >= live)).nonzero()[:, 0]
    dst = ((refs == 0) & (at < live)).nonzero()[:, 0]
    new = at.clone()
    new[src] = dst
    held = _held(table, s["len"], s["case"]["page"])
    table.copy_(torch.where(held, new[table.clamp(min=0).long()].int(), table))
    refs[dst] = refs[src]
    refs[src] = 0
    _copy(s, src, dst)
    n = src.numel()
    s["src"][:n], s["dst"][:n] = src.int(), dst.int()
    return {"table": table, "len": s["len"], "refs": refs, "src": s["src"], "dst": s["dst"],
            "moves": torch.full((1,), n, device=DEV), "free": (refs == 0).sum().view(1), "k": s["k"], "v": s["v"]}


_plain = {"project": _plain_project, "sample": _plain_sample, "fork": _plain_fork, "compact": _plain_compact}


# ------------------------------------------------------------------ the definitions, in 64 bits

def exact(case, seed):
    s = _inputs(dict(case), seed)
    return {"project": _exact_project, "sample": _exact_sample, "fork": _exact_fork,
            "compact": _exact_compact}[case["kind"]](s)


def _exact_project(s):
    x = s["x"].double()
    m, n = s["out"].shape
    top = torch.stack([row.abs().max() for row in x]) if m <= 64 else x.abs().max(1).values
    q = (x * 127 / torch.where(top == 0, 1.0, top)[:, None]).round()
    out = torch.empty(m, n, dtype=torch.float64, device=DEV)
    step = max(1, (1 << 28) // max(1, x.shape[1]))
    for a in range(0, n, step):
        b = min(n, a + step)
        # whole numbers below 2^53: exact
        out[:, a:b] = torch.mm(q, s["w"][a:b].double().T.contiguous())
        out[:, a:b] *= (top / 127)[:, None] * s["w_scale"][a:b].double()
        if s["bias"] is not None:
            out[:, a:b] += s["bias"][a:b].double()
    return {"out": out, "scale": top / 127}


def _exact_sample(s):
    n, V = s["logits"].shape
    ok = _allowed(s)
    tokens, logprobs = [], []
    for r in range(n):
        index = ok[r].nonzero()[:, 0]
        if index.numel() == 0:
            tokens.append(torch.tensor(-1, device=DEV))
            logprobs.append(torch.tensor(-math.inf, dtype=torch.float64, device=DEV))
            continue
        T = float(s["temperature"][r])
        z = s["logits"][r, index].double() / (T if T > 0 else 1.0)
        by = torch.sort(-z, stable=True).indices
        z, index = z[by], index[by]
        p = torch.exp(z - torch.logsumexp(z, 0))          # probabilities, in the order of the choice
        m = index.numel()
        if T == 0:
            m = 1
        if "top_k" in s and int(s["top_k"][r]) > 0:
            m = min(m, int(s["top_k"][r]))
        if "top_p" in s and float(s["top_p"][r]) < 1:
            c = torch.cumsum(p[:m], 0)
            m = min(m, int(torch.searchsorted(c, float(s["top_p"][r]) * c[-1])) + 1)
        if "min_p" in s:
            m = min(m, max(1, int((p >= float(s["min_p"][r]) * p[0]).sum())))
        c = torch.cumsum(p[:m], 0)
        at = min(m - 1, int(torch.searchsorted(c, float(s["u"][r]) * c[-1], right=True)))
        tokens.append(index[at])
        logprobs.append(z[at] - torch.logsumexp(z, 0))
    return {"token": torch.stack(tokens).int(), "logprob": torch.stack(logprobs)}


def _exact_fork(s):
    ps = s["case"]["page"]
    refs, table, lens = s["refs"].tolist(), s["table"].tolist(), s["len"].tolist()
    to, to_len = s["to"].tolist(), []
    k, v = [t.double() for t in s["k"]], [t.double() for t in s["v"]]
    parent, add = s["parent"].tolist(), s["add"].tolist()
    for i, p in enumerate(parent):
        to_len.append(lens[p])
        for c in range(_pages(lens[p], ps)):
            to[i][c] = table[p][c]
            refs[to[i][c]] += 1
    shared = list(refs)
    free = iter([p for p, r in enumerate(refs) if r == 0])
    src, dst, slots = [], [], []
    for i, a in enumerate(add):
        L = to_len[i]
        have, part = _pages(L, ps), L % ps
        if a > 0 and part and shared[to[i][have - 1]] > 1:
            old, new = to[i][have - 1], next(free)
            to[i][have - 1] = new
            refs[old] -= 1
            refs[new] = 1
            src.append(old), dst.append(new), slots.append(part)
            for t in k + v:
                t[new, :, :part] = t[old, :, :part]
        else:
            src.append(NONE), dst.append(NONE), slots.append(0)
        for c in range(have, _pages(L + a, ps)):
            to[i][c] = next(free)
            refs[to[i][c]] = 1
        to_len[i] = L + a

    def whole(values, dtype=torch.int32):
        return torch.tensor(values, dtype=dtype, device=DEV)
    return {"to": whole(to), "to_len": whole(to_len), "refs": whole(refs), "src": whole(src), "dst": whole(dst),
            "slots": whole(slots), "free": whole([sum(r == 0 for r in refs)], torch.int64), "k": k, "v": v}


def _exact_compact(s):
    ps = s["case"]["page"]
    refs, table, lens = s["refs"].tolist(), s["table"].tolist(), s["len"].tolist()
    k, v = [t.double() for t in s["k"]], [t.double() for t in s["v"]]
    live = sum(r > 0 for r in refs)
    holes = [p for p in range(live) if refs[p] == 0]
    late = [p for p in range(live, len(refs)) if refs[p] > 0]
    new = dict(zip(late, holes))
    for row, L in zip(table, lens):
        for c in range(_pages(L, ps)):
            row[c] = new.get(row[c], row[c])
    for a, b in new.items():
        refs[b], refs[a] = refs[a], 0
    a, b = torch.tensor(late, device=DEV).long(), torch.tensor(holes, device=DEV).long()
    for t in k + v:
        t.index_copy_(0, b, t.index_select(0, a))

    def padded(values):
        return torch.tensor(values + [NONE] * (len(refs) - len(values)), dtype=torch.int32, device=DEV)
    return {"table": torch.tensor(table, dtype=torch.int32, device=DEV), "len": s["len"], "refs": padded(refs),
            "src": padded(late), "dst": padded(holes), "moves": torch.tensor([len(late)], device=DEV),
            "free": torch.tensor([len(refs) - live], device=DEV), "k": k, "v": v}
