"""Plain definitions in 64 bits of the operators over a paged cache, and how
far a 16-bit result may be from them.

Bounds are worked out from the formulas.  u is the unit roundoff of the 16-bit
type.  Attention multiplies each weight, rounded to that type, with a value
and rounds the result: 2 u sum(p |v|) / sum(p) covers both (|o| is at most
that sum).  Weights under the smallest normal number of float16 are off by up
to 2^-25 each, with the largest weight at least 1.  Scores are 32-bit sums of
D exact products: off by at most D 2^-24 sum |q k|, and a score's error is the
relative error of its weight."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def positions(case, s):
    """Page and slot of every cached position of sequence s."""
    L, ps = case["kv_len"][s], case["page"]
    page = case["table"][s].long()[: -(-L // ps)].repeat_interleave(ps)[:L]
    return page, torch.arange(L, device=page.device) % ps


def visible(n, L, causal, window, sinks, device):
    p = torch.arange(L - n, L, device=device)[:, None]
    j = torch.arange(L, device=device)[None]
    if not causal:
        return torch.ones(n, L, dtype=torch.bool, device=device)
    see = j <= p
    if window > 0:
        see = see & ((j > p - window) | (j < sinks))
    return see


def attend(case, k, v, q, scale):
    """(out, lse, tolerance of out, tolerance of lse), in 64 bits."""
    T, Hq, D = q.shape
    Hk = k.shape[1]
    group, u = Hq // Hk, U[q.dtype]
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device=q.device)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64, device=q.device)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for s, n in enumerate(case["new"]):
        t0, L = case["q_off"][s], case["kv_len"][s]
        if n == 0 or L == 0:
            continue
        page, slot = positions(case, s)
        see = visible(n, L, case["causal"], case["window"], case["sinks"], q.device)
        for h in range(Hq):
            kk, vv = k[page, h // group, slot].double(), v[page, h // group, slot].double()
            qq = q[t0:t0 + n, h].double()
            for i in range(n):                   # row by row: only what is visible enters
                m = see[i].nonzero()[:, 0]
                if m.numel() == 0:
                    continue
                x = (kk[m] * qq[i]).sum(-1) * scale
                z = torch.logsumexp(x, 0)
                p = (x - z).exp()[:, None]
                off = D * 2.0 ** -24 * (kk[m].abs() * qq[i].abs()).sum(-1).max() * abs(scale)
                out[t0 + i, h] = (p * vv[m]).sum(0)
                lse[t0 + i, h] = z
                big = vv[m].abs()
                tol[t0 + i, h] = ((2 * u + 2 * off + 1e-5) * (p * big).sum(0)
                                  + m.numel() * 2.0 ** -25 * big.amax(0) + 2.0 ** -25)
                tol_lse[t0 + i, h] = off + m.numel() * 2.0 ** -24 + 1e-6 * (1 + z.abs())
    return out, lse, tol, tol_lse


def weigh(case, k, q, lse, w_in, scale):
    """(weights, tolerance) in 64 bits; entries at or beyond a sequence's length are None's: zero tolerance, w_in."""
    Hq, D = q.shape[1:]
    group = Hq // k.shape[1]
    out, tol = w_in.double().clone(), torch.zeros(w_in.shape, dtype=torch.float64, device=q.device)
    for s, n in enumerate(case["new"]):
        t0, L = case["q_off"][s], case["kv_len"][s]
        if n == 0 or L == 0:
            continue
        page, slot = positions(case, s)
        see = visible(n, L, case["causal"], case["window"], case["sinks"], q.device)
        add, err = torch.zeros(L, dtype=torch.float64, device=q.device), torch.zeros(L, dtype=torch.float64, device=q.device)
        for h in range(Hq):
            kk, qq = k[page, h // group, slot].double(), q[t0:t0 + n, h].double()
            x = (kk[None] * qq[:, None]).sum(-1) * scale
            off = D * 2.0 ** -24 * (kk.abs()[None] * qq.abs()[:, None]).sum(-1) * abs(scale)
            z = lse[t0:t0 + n, h].double()[:, None]
            p = torch.where(see, (x - z).exp(), 0.0)
            add += p.sum(0)
            err += torch.where(see, p * (off + 2.0 ** -21 + 2.0 ** -22 * (x.abs() + z.abs())), 0.0).sum(0)
        out[s, :L] += add
        tol[s, :L] = err + (n * Hq + 4) * 2.0 ** -24 * (add + w_in[s, :L].double().abs())
    return out, tol


def turn(x, pos, freq, axis, adjacent, inverse):
    """(y, tolerance) in 64 bits."""
    R, u = 2 * freq.numel(), U[x.dtype]
    a = pos.double()[torch.tensor(axis, device=x.device)].T * freq.double()
    if inverse:
        a = -a
    c, s = a.cos()[:, None], a.sin()[:, None]
    y = x.double().clone()
    i = torch.arange(R // 2, device=x.device)
    f, g = (2 * i, 2 * i + 1) if adjacent else (i, i + R // 2)
    p, q = x[..., f].double(), x[..., g].double()
    y[..., f], y[..., g] = p * c - q * s, q * c + p * s
    tol = torch.zeros_like(y)
    both = 1e-6 * (p.abs() + q.abs()) + 2.0 ** -25
    tol[..., f] = u * y[..., f].abs() + both
    tol[..., g] = u * y[..., g].abs() + both
    return y, tol


def kept(weight, L, budget, first, last):
    """The positions that eviction keeps, in order."""
    if L <= budget:
        return list(range(L))
    w = [(-math.inf, 0) if x != x else (x, 1) for x in weight[:L].tolist()]     # a NaN is lighter than any number
    middle = sorted(range(first, L - last), key=lambda j: (-w[j][0], -w[j][1], j))
    return sorted(list(range(first)) + middle[:budget - first - last] + list(range(L - last, L)))
