"""Plain definitions of the operators around a stage's attention: projections
in 8-bit integers, the choice of tokens, pages of a pool.  Python and 64-bit
numbers on the CPU."""
import math

import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}   # half of the least number
NONE = -1


def quantize(x):
    """(q, scale) of rows x, in 64 bits: quotients of such numbers are never so
    near to a half that 64 bits do not tell."""
    f = x.double().cpu()
    top = f.abs().amax(-1, keepdim=True)
    bad = ~torch.isfinite(top)
    q = torch.where((top > 0) & ~bad, f * 127 / torch.where(top > 0, top, 1.0), 0.0).round()
    scale = torch.where(bad, math.nan, top / 127)[:, 0]
    return q.nan_to_num(0).to(torch.int8), scale


def project(q, scale, w, w_scale, bias, dtype):
    """(out, how far a result may be from it).  Whole numbers are exact; their
    sum becomes a 32-bit float, is multiplied twice and added to once, and the
    result is rounded to its type."""
    total = (q.cpu().double() @ w.cpu().double().T)
    prod = total * scale.cpu().double()[:, None] * w_scale.cpu().double()
    out = prod + (bias.cpu().double() if bias is not None else 0.0)
    near = 3 * 2.0 ** -24 * prod.abs() * (1 + 2.0 ** -20) + 2.0 ** -24 * out.abs()
    return out, near + U[dtype] * (out.abs() + near) + TINY[dtype]


def candidates(row, allowed=None):
    """Tokens of a row (float64 numpy) in the order of the choice."""
    ok = row > -math.inf
    if allowed is not None:
        ok &= allowed
    index = np.nonzero(ok)[0]
    return index[np.argsort(-row[index], kind="stable")]


def sample(row, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, allowed=None):
    """(token, logprob) of one row, and how many candidates are kept."""
    row = np.asarray(row, np.float64)
    order = candidates(row, allowed)
    if len(order) == 0 or not 0 <= temperature < math.inf or top_p != top_p or min_p != min_p:
        return -1, -math.inf, 0
    z = row[order] / (temperature if temperature > 0 else 1.0)
    if z[0] == math.inf:
        diff = np.where(z == math.inf, 0.0, -math.inf)
    else:
        diff = z - z[0]
    w = np.exp(diff)
    n = len(order)
    if top_k > 0:
        n = min(n, int(top_k))
    if top_p < 1:
        left = math.fsum(w[:n])
        sums = np.concatenate([[0.0], np.cumsum(w[:n])[:-1]])
        n = max(1, int((sums < top_p * left).sum()))
    n = max(1, min(n, int((w >= min_p).sum())))
    if temperature == 0:
        n = 1
    sums = np.cumsum(w[:n])
    if u < 1:
        at = min(n - 1, int((sums <= u * sums[-1]).sum()))
    else:                                       # NaN among them
        at = n - 1
    return int(order[at]), float(diff[at] - math.log(math.fsum(w))), n


class Pool:
    """The pool and its tables, as lists."""

    def __init__(self, n_pages, page):
        self.refs, self.page = [0] * n_pages, page

    def need(self, positions):
        return -(-positions // self.page)

    def fork(self, tables, lens, parent, to, to_len):
        for i, p in enumerate(parent):
            if p < 0:
                continue
            to_len[i] = lens[p]
            for c in range(self.need(lens[p])):
                to[i][c] = tables[p][c]
                self.refs[to[i][c]] += 1

    def grow(self, tables, lens, add):
        """(src, dst, slots, free), or None where the pool has too few."""
        n = len(lens)
        first, want, replace = [0] * n, [0] * n, [False] * n
        for s in range(n):
            first[s], want[s] = self.need(lens[s]), self.need(lens[s] + add[s])
            if add[s] > 0 and lens[s] % self.page and self.refs[tables[s][first[s] - 1]] > 1:
                replace[s] = True
                first[s] -= 1
        free = [p for p, r in enumerate(self.refs) if r == 0]
        if sum(want) - sum(first) > len(free):
            return None
        src, dst, slots = [NONE] * n, [NONE] * n, [0] * n
        free = iter(free)
        for s in range(n):
            old = tables[s][first[s]] if replace[s] else None
            for c in range(first[s], want[s]):
                tables[s][c] = next(free)
                self.refs[tables[s][c]] = 1
            if replace[s]:
                src[s], dst[s], slots[s] = old, tables[s][first[s]], lens[s] % self.page
                self.refs[old] -= 1
            lens[s] += add[s]
        return src, dst, slots, sum(r == 0 for r in self.refs)

    def release(self, tables, lens, keep):
        for s in range(len(lens)):
            if keep[s] >= lens[s]:
                continue
            for c in range(self.need(keep[s]), self.need(lens[s])):
                self.refs[tables[s][c]] -= 1
                tables[s][c] = NONE
            lens[s] = keep[s]

    def compact(self, list_of_tables):
        """(src, dst): pages that move, and where to."""
        live = sum(r > 0 for r in self.refs)
        src = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        dst = [p for p in range(live) if self.refs[p] == 0]
        new = dict(zip(src, dst))
        for tables, lens in list_of_tables:
            for s, L in enumerate(lens):
                for c in range(self.need(L)):
                    tables[s][c] = new.get(tables[s][c], tables[s][c])
        for a, b in new.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        return src, dst
