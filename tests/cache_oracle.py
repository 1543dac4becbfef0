"""Plain fp64 CPU implementations of the paged-cache operators, with the bounds that
their fp32 sums and roundings to the stored type allow."""
from __future__ import annotations

import math

import torch


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


U = 2.0 ** -24      # half a step of fp32


def rotary(x, positions, freqs, scale=1.0, interleaved=False, transpose=False):
    """(y, sizes) in fp64: y and |x0| + |x1| of every turned pair (0 where copied)."""
    n = freqs.numel()
    t = positions.double()[:, None] * freqs.double()[None, :]
    c, s = scale * t.cos()[:, None], scale * t.sin()[:, None] * (-1 if transpose else 1)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n),
                                                                         slice(n, 2 * n))
    x = x.double()
    y, size = x.clone(), torch.zeros_like(x)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, size


def rotary_bound(y, size, dtype, scale=1.0):
    """Factors are off by 4 half steps of fp32 (2 of the sine, 1 of its argument, 1 of
    the scale), a product and a sum by one each: 8 in all on |x0| + |x1|; then the
    rounding to dtype (or half its smallest value)."""
    return half_step(dtype) * y.abs() + 8 * U * abs(scale) * size * 1.001 + \
        torch.finfo(dtype).tiny * torch.finfo(dtype).eps


def rows_of(cache_k, table, s, h, length, page):
    """The keys 0 .. length - 1 of a sequence and whether each is there (no hole)."""
    j = torch.arange(length)
    p = table[s, j // page].long()
    there = (p >= 0) & (p < cache_k.shape[0])
    return cache_k[p.clamp(0, cache_k.shape[0] - 1), h, j % page], there, p, j % page


def attention(q, k, v, table, lengths, offsets, scale, causal, weight=None):
    """out, its bound, gains and theirs. q, k, v as stored (CPU tensors of the type
    under test); gains: pages x heads x page or None."""
    dtype, (tokens, hq, d), (pages, hkv, page, _) = q.dtype, q.shape, k.shape
    group, most = hq // hkv, table.shape[1] * page
    out = torch.zeros(q.shape, dtype=torch.float64)
    bound = torch.full(q.shape, -1.0, dtype=torch.float64)     # -1: no row of a sequence
    gain = torch.zeros(pages, hkv, page, dtype=torch.float64)
    slack = torch.zeros_like(gain)
    off = offsets.clamp(0, tokens).tolist()
    for s in range(table.shape[0]):
        L, (a, b) = min(max(int(lengths[s]), 0), most), off[s:s + 2]
        n = b - a
        for h in range(hq):
            if n <= 0:
                break
            K, there, p, slot = rows_of(k, table, s, h // group, L, page)
            V = rows_of(v, table, s, h // group, L, page)[0]
            Q = q[a:b, h].double()
            seen = there[None, :].expand(n, L).clone()
            if causal:
                seen &= torch.arange(L)[None, :] <= (L - n + torch.arange(n))[:, None]
            z = torch.where(seen, scale * Q @ torch.where(there[:, None], K.double(), 0.0).T,
                            -math.inf)
            top = z.amax(1, keepdim=True) if L else torch.full((n, 1), -math.inf).double()
            e = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
            total = e.sum(1, keepdim=True)
            w = torch.where(total > 0, e / total, 0.0)
            Vd = torch.where(there[:, None], V.double(), 0.0)
            y = w @ torch.where(Vd.isfinite(), Vd, 0.0)
            # Values that are not finite reach the rows that see them, and no others.
            wild = ~Vd.isfinite()
            for j in torch.nonzero(wild.any(1))[:, 0].tolist():
                y[seen[:, j]] += torch.where(wild[j], Vd[j], 0.0)
            # A score of d products is off by d + 2 half steps of their sizes (which
            # errs p by as much, twice through the maximum), exp2 and the sum over L
            # keys by L + 8 more, rescalings by one per 16 keys. The rounding of p to
            # the stored type is half a step of it.
            reach = (abs(scale) * Q.abs() @ torch.where(there[:, None], K.double(), 0.0).abs().T)
            reach = torch.where(seen, reach, 0.0).amax(1, keepdim=True) if L else 0.0
            rel = U * (2 * (d + 4) * reach + 2 * L + 16)
            size = w @ torch.where(Vd.isfinite(), Vd, 0.0).abs()
            out[a:b, h] = y
            bound[a:b, h] = half_step(dtype) * y.abs() + \
                (2 * rel + (half_step(dtype) if dtype != torch.float32 else 0.0)) * size * 1.01 + \
                torch.finfo(dtype).tiny
            if L:
                gain[p[there], h // group, slot[there]] += w.sum(0)[there]
                slack[p[there], h // group, slot[there]] += \
                    ((2 * rel + U * n * group) * w).sum(0)[there] + 1e-37
    if weight is None:
        return out, bound, None, None
    return out, bound, weight.double() + gain, slack + U * (weight.double() + gain).abs()


def evict(weight, table, lengths, budget, recent, page):
    """kept indices (sequences x heads x budget, -1 behind) by plain sorting."""
    seqs, heads = table.shape[0], weight.shape[1]
    kept = torch.full((seqs, heads, budget), -1, dtype=torch.int32)
    for s in range(seqs):
        L = min(max(int(lengths[s]), 0), table.shape[1] * page)
        n = min(L, budget)
        r = min(recent, n)
        for h in range(heads):
            w, there, _, _ = rows_of(weight[..., None], table, s, h, L, page)
            w = torch.where(there, w[:, 0].double(), math.nan)
            key = [(-math.inf, -j) if math.isnan(x) else (x, -j)
                   for j, x in enumerate(w[:L - r].tolist())]
            # a NaN is lighter than minus infinity
            nan = [math.isnan(x) for x in w[:L - r].tolist()]
            order = sorted(range(L - r), key=lambda j: (not nan[j], *key[j]), reverse=True)
            index = sorted(order[:n - r]) + list(range(L - r, L))
            kept[s, h, :n] = torch.tensor(index, dtype=torch.int32)
    return kept
