"""GPU: the operators over a paged cache against plain fp64 implementations."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

TYPES = ["bf16", "f16", "f32"]


def _t(torch, name):
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[name]


def torch_equal(a, b):
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def _check(got, want, bound, what=""):
    """got within bound of want; equal infinities and NaNs where want has them."""
    got = got.double().cpu()
    fine = want.isfinite()
    assert torch_equal(got[~fine], want[~fine]), what
    worst = float(((got - want).abs() - bound)[fine].max()) if bool(fine.any()) else 0.0
    assert worst <= 0.0, what


# --------------------------------------------------------------- rotary -----

ROTARY = [(1, 1, 8, 4), (5, 3, 64, 32), (3, 2, 80, 33), (2, 5, 12, 6), (7, 1, 7, 3), (4, 4, 96, 7),
          (300, 32, 128, 64), (2, 2, 256, 1), (3, 3, 40, 0), (1000, 40, 72, 20)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,dim,pairs", ROTARY)
def test_rotary(torch_dev, dtype, interleaved, tokens, heads, dim, pairs):
    torch, dev = torch_dev
    import cache_oracle as O
    import paper_2202_12674_amd as P
    g = torch.Generator().manual_seed(tokens * 1000 + dim)
    x = torch.randn(tokens, heads, dim, generator=g).to(_t(torch, dtype))
    pos = torch.randint(-50, 2_000_000, (tokens,), generator=g)
    f = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / max(pairs, 1))
    for transpose, wide in ((False, True), (True, False)):
        p = pos if wide else pos.to(torch.int32)
        y = P.rotary(x.to(dev), p.to(dev), f.to(dev), 1.25, interleaved, transpose)
        want, size = O.rotary(x, pos, f, 1.25, interleaved, transpose)
        _check(y, want, O.rotary_bound(want, size, x.dtype, 1.25))


@pytest.mark.parametrize("dtype", TYPES)
def test_rotary_strides_in_place_and_its_gradient(torch_dev, dtype):
    torch, dev = torch_dev
    import cache_oracle as O
    import paper_2202_12674_amd as P
    g = torch.Generator().manual_seed(4)
    wide = torch.randn(11, 9, 53, generator=g).to(_t(torch, dtype)).to(dev)
    x = wide[:, 2:7, 3:47]                       # rows that begin on odd places
    pos, f, _ = torch.arange(11, device=dev) * 37, *P.rotary_frequencies(30, device=dev)
    want, size = O.rotary(x.cpu(), pos.cpu(), f.cpu())
    y = P.rotary(x, pos, f)
    _check(y, want, O.rotary_bound(want, size, x.dtype))
    buf = torch.full((5, 11, 50), 7.0, dtype=x.dtype, device=dev)
    out = buf.transpose(0, 1)[..., :44]          # heads before tokens
    P.rotary(x, pos, f, out=out)
    assert torch.equal(out, y) and bool((buf[..., 44:] == 7.0).all())
    keep = wide.clone()
    P.rotary(x, pos, f, out=x)
    assert torch.equal(x, y)
    keep[:, 2:7, 3:47] = y
    assert torch.equal(wide, keep)
    if dtype == "f32":
        # the transposed map is the gradient: by differences of <dy, rotary(x)>, which
        # is linear in x, so that a difference over one unit is exact but for rounding
        dy = torch.randn(11, 5, 44, generator=g).to(dev)
        dx = P.rotary(dy, pos, f, transpose=True)
        x0 = torch.randn(11, 5, 44, generator=g).to(dev)
        for at in ((0, 0, 0), (3, 2, 17), (10, 4, 29), (5, 1, 40)):
            x1 = x0.clone()
            x1[at] += 1.0
            diff = ((P.rotary(x1, pos, f).double() - P.rotary(x0, pos, f).double())
                    * dy.double()).sum()
            assert abs(float(diff - dx[at])) < 64 * 2.0 ** -24 * 10


def test_rotary_of_nothing(torch_dev):
    torch, dev = torch_dev
    import paper_2202_12674_amd as P
    f = torch.ones(4, dtype=torch.float64, device=dev)
    y = P.rotary(torch.zeros(0, 3, 8, device=dev), torch.zeros(0, dtype=torch.int64, device=dev), f)
    assert y.shape == (0, 3, 8)


# ---------------------------------------------------------------- cache -----

def make(torch, dev, dtype, lengths, hkv, d, page, seed=0, layout="heads", spare=3, holes=0,
         columns=0):
    """A cache of random pages whose unused places hold NaN: (cache, CPU copies)."""
    import paper_2202_12674_amd as P
    g = torch.Generator().manual_seed(seed)
    need = [-(-max(L, 0) // page) for L in lengths]
    pool = sum(need) + spare
    order = torch.randperm(pool, generator=g).int()
    columns = max(columns, max(need), 1)
    table = torch.full((len(lengths), columns), -1, dtype=torch.int32)
    k = torch.full((pool, hkv, page, d), math.nan)
    v, w, at = k.clone(), torch.full((pool, hkv, page), math.nan), 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        for i in range(n):
            fill = min(page, lengths[s] - i * page)
            p = int(order[at + i])
            k[p, :, :fill] = torch.randn(hkv, fill, d, generator=g)
            v[p, :, :fill] = torch.randn(hkv, fill, d, generator=g)
            w[p, :, :fill] = torch.rand(hkv, fill, generator=g)
        at += n
    for i in range(holes):
        s = i % len(lengths)
        if need[s] > 1:
            table[s, (5 * i + 1) % need[s]] = (-1, pool, 2 ** 31 - 1, -2 ** 31)[i % 4]
    dt = _t(torch, dtype)
    k, v = k.to(dt), v.to(dt)
    if layout == "slots":              # slots before heads
        kd = k.to(dev).transpose(1, 2).contiguous().transpose(1, 2)
        vd = v.to(dev).transpose(1, 2).contiguous().transpose(1, 2)
    elif layout == "both":             # keys and values of a page behind each other
        kv = torch.stack([k, v], 1).to(dev)
        kd, vd = kv[:, 0], kv[:, 1]
    elif layout == "gaps":             # rows with room between them
        kd = torch.full((pool, hkv, page + 1, d + 16), math.nan, dtype=dt, device=dev)
        vd = kd.clone()
        kd, vd = kd[:, :, :page, 8:d + 8], vd[:, :, :page, 8:d + 8]
        kd.copy_(k), vd.copy_(v)
    else:
        kd, vd = k.to(dev), v.to(dev)
    wd = w.to(dev)
    if layout == "gaps":
        wd = torch.full((hkv, pool, page + 3), math.nan, device=dev).transpose(0, 1)[..., :page]
        wd.copy_(w)
    tab = torch.full((len(lengths), columns + (5 if layout == "gaps" else 0)), 2 ** 30,
                     dtype=torch.int32)
    tab[:, :columns] = table
    cache = P.PagedCache(kd, vd, tab.to(dev)[:, :columns],
                         torch.tensor(lengths, dtype=torch.int32, device=dev), wd)
    return cache, (k, v, table, torch.tensor(lengths, dtype=torch.int32), w)


def offsets_of(torch, new):
    return torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32)


def run_attention(torch_dev, dtype, lengths, new, hq, hkv, d, page, causal=True, accumulate=False,
                  layout="heads", holes=0, behind=0, scale=None, seed=1, split_q=False, big=1.0,
                  wild=()):
    torch, dev = torch_dev
    import cache_oracle as O
    import paper_2202_12674_amd as P
    cache, (k, v, table, lens, w) = make(torch, dev, dtype, lengths, hkv, d, page, seed, layout,
                                         holes=holes)
    g = torch.Generator().manual_seed(seed + 1)
    for s, j, h, x, value in wild:     # values (x of head h of key j) that are not finite
        v[int(table[s, j // page]), h, j % page, x] = value
    cache.v.copy_(v)
    tokens = sum(new) + behind
    q = (big * torch.randn(tokens, hq, d, generator=g)).to(k.dtype)
    off = offsets_of(torch, new)
    qd = q.to(dev)
    if split_q:                        # queries within wider rows, on odd places
        wide = torch.full((tokens, hq + 2, d + 7), math.nan, dtype=k.dtype, device=dev)
        wide[:, 1:-1, 3:3 + d] = qd
        qd = wide[:, 1:-1, 3:3 + d]
    out = torch.full((hq, tokens, d + 5), 3.0, dtype=k.dtype, device=dev)
    out = out.transpose(0, 1)[..., :d]
    wout = torch.full(w.shape, -5.0, device=dev) if accumulate else None
    y = P.attention(qd, cache, off.to(dev), scale=scale, causal=causal, accumulate=accumulate,
                    weight_out=wout, out=out)
    want, bound, ww, slack = O.attention(q, k, v, table, lens, off,
                                         d ** -0.5 if scale is None else scale, causal,
                                         w if accumulate else None)
    there = bound != -1
    _check(y[there.to(dev)], want[there], bound[there], "out")
    assert bool((y.cpu()[~there] == 3.0).all())
    if accumulate:
        there = torch.zeros(w.shape, dtype=torch.bool)
        for s, L in enumerate(lengths):
            _, ok, p, slot = O.rows_of(k, table, s, 0, L, page)
            there[p[ok], :, slot[ok]] = True
        _check(wout.cpu()[there], ww[there], slack[there], "weight")
        assert bool((wout.cpu()[~there] == -5.0).all())
        before = cache.weight.clone()
        P.attention(qd, cache, off.to(dev), scale=scale, causal=causal, accumulate=True, out=out)
        new_w = cache.weight.cpu()
        assert torch.equal(new_w[there], wout.cpu()[there])       # the same sums, in place
        assert torch.equal(new_w[~there].nan_to_num(-1.0), before.cpu()[~there].nan_to_num(-1.0))
    return y


SHAPES = [  # lengths, new, hq, hkv, d, page
    ([1], [1], 1, 1, 8, 1),
    ([5, 0, 17], [1, 1, 1], 4, 2, 64, 16),
    ([33, 64, 1], [1, 1, 1], 8, 1, 128, 16),
    ([700, 31, 32], [1, 1, 1], 12, 4, 96, 7),
    ([100, 40, 0, 9], [3, 0, 2, 9], 6, 2, 72, 24),
    ([3, 200], [5, 2], 5, 5, 80, 128),                 # more rows than keys
    ([257, 130], [257, 70], 4, 4, 64, 64),
    ([300, 90], [129, 90], 7, 1, 256, 16),
    ([515], [200], 14, 2, 40, 48),
    ([1030, 65, 64], [40, 65, 1], 16, 2, 128, 33),
    ([2100], [1], 40, 2, 16, 5),
    ([190, 333], [33, 20], 9, 3, 248, 32),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,new,hq,hkv,d,page", SHAPES)
@pytest.mark.parametrize("causal", [True, False])
def test_attention(torch_dev, dtype, lengths, new, hq, hkv, d, page, causal):
    run_attention(torch_dev, dtype, lengths, new, hq, hkv, d, page, causal)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,new,hq,hkv,d,page", SHAPES)
def test_attention_that_accumulates_weights(torch_dev, dtype, lengths, new, hq, hkv, d, page):
    run_attention(torch_dev, dtype, lengths, new, hq, hkv, d, page, True, True)
    run_attention(torch_dev, dtype, lengths, new, hq, hkv, d, page, False, True, seed=8)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["slots", "both", "gaps"])
@pytest.mark.parametrize("new", [[1, 1, 1], [70, 3, 40]])
def test_attention_layouts(torch_dev, dtype, layout, new):
    run_attention(torch_dev, dtype, [150, 61, 77], new, 6, 3, 104, 19, True, True, layout=layout,
                  split_q=True)
    run_attention(torch_dev, dtype, [150, 61, 77], new, 6, 3, 64, 32, True, True, layout=layout,
                  split_q=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [[1, 1, 1], [50, 45, 66]])
def test_attention_holes_and_rows_behind_the_last_sequence(torch_dev, dtype, new):
    run_attention(torch_dev, dtype, [210, 45, 166], new, 8, 2, 64, 16, True, True, holes=9,
                  behind=5)
    run_attention(torch_dev, dtype, [210, 45, 166], new, 8, 2, 128, 21, True, True, holes=6,
                  behind=33, split_q=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [0.0, -0.7, 3.0])
def test_attention_scales(torch_dev, dtype, scale):
    run_attention(torch_dev, dtype, [99, 260], [1, 1], 4, 2, 64, 16, True, True, scale=scale)
    run_attention(torch_dev, dtype, [99, 260], [80, 100], 4, 2, 64, 16, True, True, scale=scale)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [5, 60, 200])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 21), (256, 32)])
def test_values_that_are_not_finite_reach_only_rows_that_see_them(torch_dev, dtype, new, d, page):
    """Infinities and NaNs in the values of new tokens, one the first, one the last of a
    chunk: rows before them must not change, rows from them on take them over."""
    wild = [(0, 299, 0, 3, math.inf), (0, 299, 0, 4, math.nan), (0, 298, 0, 3, -math.inf),
            (0, 300 - new, 1, d - 1, math.inf), (0, 300 - new // 2, 0, 0, -math.inf),
            (1, 130 - new // 2 if new < 130 else 70, 1, 5, math.inf)]
    run_attention(torch_dev, dtype, [300, 130], [new, min(new, 130)], 4, 2, d, page, True, True,
                  wild=wild)


def test_attention_of_large_scores(torch_dev):
    """Scores in the thousands: one key holds all the weight, nothing overflows."""
    run_attention(torch_dev, "f32", [400, 90], [1, 1], 4, 2, 64, 16, True, True, big=300.0)
    run_attention(torch_dev, "f32", [400, 90], [200, 90], 4, 2, 64, 16, True, True, big=300.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_of_long_sequences_and_many(torch_dev, dtype):
    run_attention(torch_dev, dtype, [20011, 3, 9000], [1, 1, 1], 8, 2, 64, 64, True, True)
    run_attention(torch_dev, dtype, [5000], [20], 2, 1, 128, 16, True, True)
    run_attention(torch_dev, dtype, [37 + i for i in range(70)], [1 + i % 3 for i in range(70)], 4,
                  1, 64, 16, True, True)


@pytest.mark.parametrize("d,page", [(64, 24), (96, 16), (128, 64)])
def test_attention_of_chunks_over_long_caches(torch_dev, d, page):
    """Hundreds of rows over keys that outgrow an L2, where single precision too goes by
    tiles of 128 rows; values that are not finite among the last."""
    lengths, new = [9000, 8301], [300, 277]
    wild = [(0, 8999, 0, 3, math.inf), (0, 8800, 0, d - 1, math.nan), (1, 8150, 0, 7, -math.inf)]
    for dtype in TYPES:
        run_attention(torch_dev, dtype, lengths, new, 2, 1, d, page, True, True, wild=wild)
        run_attention(torch_dev, dtype, lengths, new, 2, 1, d, page, False, split_q=True, holes=5)


def test_attention_of_nothing(torch_dev):
    torch, dev = torch_dev
    import paper_2202_12674_amd as P
    cache, (_, _, _, _, w) = make(torch, dev, "bf16", [20, 5], 2, 64, 16)
    off = torch.zeros(3, dtype=torch.int32, device=dev)
    q = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device=dev)
    assert P.attention(q, cache, off).shape == (0, 4, 64)
    out = torch.full(w.shape, -5.0, device=dev)
    P.attention(q, cache, off, accumulate=True, weight_out=out)
    seen = ~w.isnan()
    assert torch.equal(out.cpu()[seen], w[seen]) and bool((out.cpu()[~seen] == -5.0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [4, 90])
def test_lengths_and_offsets_out_of_range_are_cut(torch_dev, dtype, new):
    torch, dev = torch_dev
    import cache_oracle as O
    import paper_2202_12674_amd as P
    cache, (k, v, table, lens, w) = make(torch, dev, dtype, [96, 96], 2, 64, 16, spare=0)
    cache.lengths.copy_(torch.tensor([2 ** 31 - 1, -7]))
    g = torch.Generator().manual_seed(3)
    q = torch.randn(new, 4, 64, generator=g).to(k.dtype)
    off = torch.tensor([-3, new - 1, 2 ** 31 - 1], dtype=torch.int32)
    y = P.attention(q.to(dev), cache, off.to(dev))
    want, bound, _, _ = O.attention(q, k, v, table, cache.lengths.cpu(), off, 0.125, True)
    _check(y, want, bound)


# --------------------------------------------------------------- append -----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("layout", ["heads", "slots", "gaps"])
@pytest.mark.parametrize("d,pairs,page", [(64, 32, 16), (8, 3, 1), (136, 20, 7), (256, 0, 64)])
def test_append(torch_dev, dtype, interleaved, layout, d, pairs, page):
    torch, dev = torch_dev
    import cache_oracle as O
    import paper_2202_12674_amd as P
    lengths, new, hkv = [40, 3, 17, 0, 66], [1, 5, 17, 0, 30], 3   # 3 keys cannot hold 5 tokens
    cache, (k, v, table, lens, w) = make(torch, dev, dtype, lengths, hkv, d, page, 2, layout,
                                         holes=2)
    g = torch.Generator().manual_seed(9)
    tokens = sum(new) + 4
    nk = torch.randn(tokens, hkv, d, generator=g).to(k.dtype)
    nv = torch.randn(tokens, hkv, d, generator=g).to(k.dtype)
    pos = torch.randint(0, 100000, (tokens,), generator=g)
    f = 100.0 ** (-torch.arange(pairs, dtype=torch.float64) / max(pairs, 1))
    both = torch.cat([nk, nv], 1).to(dev)                          # strided inputs
    turned = dict(positions=pos.to(dev), freqs=f.to(dev), scale=0.9, interleaved=interleaved) \
        if pairs else {}
    P.cache_append(cache, both[:, :hkv], both[:, hkv:], offsets_of(torch, new).to(dev), **turned)
    want_k, size = O.rotary(nk, pos, f, 0.9 if pairs else 1.0, interleaved)
    bound = O.rotary_bound(want_k, size, k.dtype) * (size > 0)      # copied values are equal
    ek, ev, ew, slack = k.double(), v.double(), w.double(), torch.zeros(k.shape).double()
    t = 0
    for s, n in enumerate(new):
        for i in range(n):
            j = lengths[s] - n + i
            p = int(table[s, j // page]) if j >= 0 else -1
            if 0 <= p < k.shape[0]:
                ek[p, :, j % page], ev[p, :, j % page] = want_k[t + i], nv[t + i].double()
                slack[p, :, j % page] = bound[t + i]
                ew[p, :, j % page] = 0.0
        t += n
    _check(cache.k, ek, slack)
    _check(cache.v, ev, torch.zeros_like(slack))
    _check(cache.weight, ew, torch.zeros_like(ew))


# ---------------------------------------------------------------- evict -----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["heads", "slots", "gaps"])
@pytest.mark.parametrize("lengths,budget,recent,d,page", [
    ([1], 1, 0, 8, 1), ([50, 7, 0, 20], 20, 5, 64, 16), ([300, 64, 65], 64, 64, 128, 7),
    ([300, 64, 65], 64, 100, 40, 32), ([1500, 900], 700, 0, 72, 24), ([90], 90, 3, 256, 64),
    ([33, 4000], 1, 1, 16, 48)])
@pytest.mark.parametrize("kind", ["rand", "ties", "odd"])
def test_evict(torch_dev, dtype, layout, lengths, budget, recent, d, page, kind):
    torch, dev = torch_dev
    import cache_oracle as O
    import paper_2202_12674_amd as P
    hkv = 2
    cache, (k, v, table, lens, w) = make(torch, dev, dtype, lengths, hkv, d, page, 5, layout,
                                         holes=1 if kind == "odd" else 0)
    g = torch.Generator().manual_seed(12)
    there = ~w.isnan()
    if kind == "ties":
        w[there] = torch.randint(0, 3, w.shape, generator=g).float()[there]
        w[there & (torch.rand(w.shape, generator=g) < 0.1)] = -0.0
    if kind == "odd":
        w[there] = torch.randn(w.shape, generator=g)[there]
        for x in (math.inf, -math.inf, math.nan, 1e-40):
            w[there & (torch.rand(w.shape, generator=g) < 0.1)] = x
    cache.weight.copy_(w)
    kept_n = [min(L, budget) for L in lengths]
    target, (tk, tv, ttable, _, tw) = make(torch, dev, dtype, kept_n, hkv, d, page, 6, layout,
                                           columns=-(-budget // page))
    kept = P.cache_evict(cache, target, budget, recent)
    want = O.evict(w, table, lens, budget, recent, page)
    assert torch.equal(kept.cpu(), want)
    assert target.lengths.tolist() == kept_n
    for s, n in enumerate(kept_n):
        for h in range(hkv):
            src, ok, p, slot = O.rows_of(k, table, s, h, lengths[s], page)
            index = want[s, h, :n].long()
            _, _, tp, tslot = O.rows_of(tk, ttable, s, h, n, page)
            for x, y in ((k, tk), (v, tv), (w, tw)):
                row = x[p.clamp(0, k.shape[0] - 1), h, slot]
                row = torch.where(ok.view(-1, *[1] * (row.dim() - 1)), row, 0.0)   # holes give 0
                y[tp, h, tslot] = row[index]
    for x, y in ((target.k, tk), (target.v, tv), (target.weight, tw)):
        assert torch.equal(x.cpu().nan_to_num(7.0), y.nan_to_num(7.0))


def test_evict_of_sequences_that_lds_does_not_hold(torch_dev):
    torch, dev = torch_dev
    import cache_oracle as O
    import paper_2202_12674_amd as P
    lengths = [60001, 24000]
    cache, (_, _, table, lens, w) = make(torch, dev, "bf16", lengths, 1, 8, 64, 3)
    target, _ = make(torch, dev, "bf16", [30000, 24000], 1, 8, 64, 4)
    kept = P.cache_evict(cache, target, 30000, 100)
    assert torch.equal(kept.cpu(), O.evict(w, table, lens, 30000, 100, 64))


# ------------------------------------------------------------- together -----

@pytest.mark.parametrize("dtype", TYPES)
def test_a_prompt_tokens_and_an_eviction(torch_dev, dtype):
    """Rotate, append, attend and evict as a serving loop does: a prompt in two chunks,
    then single tokens, then half of the cache goes and tokens follow. Every step is
    checked against the oracle on what the cache holds at that moment."""
    torch, dev = torch_dev
    import cache_oracle as O
    import paper_2202_12674_amd as P
    g = torch.Generator().manual_seed(2)
    seqs, hq, hkv, d, page, columns = 2, 4, 2, 64, 16, 12
    dt = _t(torch, dtype)
    f, scale = P.rotary_frequencies(d, scaling="yarn", factor=4.0, original=64.0, device=dev)
    pool = torch.zeros(2, 2 * seqs * columns, hkv, page, d, dtype=dt, device=dev)
    weight = torch.zeros(2 * seqs * columns, hkv, page, device=dev)
    order = torch.randperm(2 * seqs * columns, generator=g).int().view(2 * seqs, columns).to(dev)
    caches = [P.PagedCache(pool[0], pool[1], order[i * seqs:(i + 1) * seqs],
                           torch.zeros(seqs, dtype=torch.int32, device=dev), weight)
              for i in (0, 1)]
    cache, position = caches[0], [0, 0]

    def step(new):
        tokens = sum(new)
        q, k, v = (torch.randn(tokens, h, d, generator=g).to(dt) for h in (hq, hkv, hkv))
        at = torch.cat([torch.arange(p, p + n) for p, n in zip(position, new)]).to(dev)
        for s, n in enumerate(new):
            position[s] += n
        off = offsets_of(torch, new).to(dev)
        cache.lengths.add_(torch.tensor(new, dtype=torch.int32, device=dev))
        P.cache_append(cache, k.to(dev), v.to(dev), off, at, f, scale)
        qr = P.rotary(q.to(dev), at, f, scale)
        wb = weight.clone()
        y = P.attention(qr, cache, off, accumulate=True)
        want, bound, w, slack = O.attention(qr.cpu(), pool[0].cpu(), pool[1].cpu(),
                                            cache.table.cpu(), cache.lengths.cpu(), off.cpu(),
                                            d ** -0.5, True, wb.cpu())
        _check(y, want, bound)
        _check(weight, w, slack)

    step([60, 37])
    step([30, 64])
    for _ in range(3):
        step([1, 1])
    want = O.evict(weight.cpu(), cache.table.cpu(), cache.lengths.cpu(), 48, 16, page)
    assert torch.equal(P.cache_evict(cache, caches[1], 48, 16).cpu(), want)
    cache = caches[1]
    assert cache.lengths.tolist() == [48, 48]
    for _ in range(2):
        step([1, 1])
    step([20, 1])


@pytest.mark.parametrize("new,longest", [(1, 333), (70, 333), (1, 20000)])
def test_a_captured_step_replays(torch_dev, new, longest):
    """Append, attention with weights and eviction in one graph, replayed with eager
    work between: every replay as the eager calls."""
    torch, dev = torch_dev
    import paper_2202_12674_amd as P
    cache, _ = make(torch, dev, "bf16", [200, longest], 2, 64, 16, 3)
    target, _ = make(torch, dev, "bf16", [128, 128], 2, 64, 16, 4)
    off = offsets_of(torch, [new, new]).to(dev)
    f, _ = P.rotary_frequencies(64, device=dev)
    at = torch.arange(2 * new, device=dev)
    q = torch.randn(2 * new, 8, 64, device=dev).bfloat16()
    k, v = (torch.randn(2 * new, 2, 64, device=dev).bfloat16() for _ in range(2))
    wout = torch.zeros(cache.weight.shape, device=dev)
    ws = P.alloc_workspace(P.attention_workspace_bytes(cache, 2 * new, 8, True), dev)

    def step():
        P.cache_append(cache, k, v, off, at, f)
        y = P.attention(P.rotary(q, at, f), cache, off, accumulate=True, weight_out=wout,
                        workspace=ws)
        return y, P.cache_evict(cache, target, 128, 10)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, kept = step()
    for i in range(4):
        q.copy_(torch.randn(2 * new, 8, 64, device=dev))
        k.copy_(torch.randn(2 * new, 2, 64, device=dev))
        y, want = step()
        y, want, w = y.clone(), want.clone(), wout.clone()
        wout.zero_(), got.zero_(), ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, y) and torch.equal(kept, want), i
        assert torch.equal(wout.nan_to_num(-1), w.nan_to_num(-1)), i


def test_two_captured_graphs_share_a_workspace(torch_dev):
    """Two captured calls of other sizes that use one workspace, replayed in turn: a call
    reads nothing there that it has not written."""
    torch, dev = torch_dev
    import paper_2202_12674_amd as P
    parts = []
    for new, lengths in ((1, [900, 40]), (60, [300, 77])):
        cache, _ = make(torch, dev, "f16", lengths, 2, 64, 16, new)
        parts.append((cache, offsets_of(torch, [new, new]).to(dev),
                      torch.randn(2 * new, 8, 64, device=dev).half(),
                      torch.zeros(cache.weight.shape, device=dev)))
    ws = P.alloc_workspace(max(P.attention_workspace_bytes(c, q.shape[0], 8, True)
                               for c, _, q, _ in parts), dev)

    def step(c, off, q, w):
        return P.attention(q, c, off, accumulate=True, weight_out=w, workspace=ws)

    want = []
    for p in parts:
        want.append((step(*p).clone(), p[3].clone()))
    graphs, got = [], []
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for p in parts:
            step(*p)
    side.synchronize()
    for p in parts:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(step(*p))
        graphs.append(g)
    for i in (0, 1, 1, 0, 1, 0):
        got[i].zero_(), parts[i][3].zero_(), ws.fill_(255)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(got[i], want[i][0])
        assert torch.equal(parts[i][3].nan_to_num(-1), want[i][1].nan_to_num(-1))


def test_results_do_not_depend_on_the_run(torch_dev):
    torch, dev = torch_dev
    import paper_2202_12674_amd as P
    for new in (1, 90):
        cache, _ = make(torch, dev, "bf16", [900, 1333, 90], 2, 128, 32, 3)
        q = torch.randn(3 * new, 8, 128, device=dev).bfloat16()
        off = offsets_of(torch, [new] * 3).to(dev)
        out = [(P.attention(q, cache, off, accumulate=True, weight_out=w), w)
               for w in (torch.zeros(cache.weight.shape, device=dev) for _ in range(5))]
        for y, w in out[1:]:
            assert torch.equal(y, out[0][0]) and torch.equal(w, out[0][1])


def test_calls_on_streams_of_their_own(torch_dev):
    torch, dev = torch_dev
    import paper_2202_12674_amd as P
    cache, _ = make(torch, dev, "f16", [700, 20], 2, 64, 16, 3)
    off = offsets_of(torch, [1, 1]).to(dev)
    q = [torch.randn(2, 8, 64, device=dev).half() for _ in range(6)]
    want = [P.attention(x, cache, off) for x in q]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(3)], []
    for i, x in enumerate(q):
        with torch.cuda.stream(streams[i % 3]):
            got.append(P.attention(x, cache, off))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("new", [1, 90])
def test_sequences_may_share_pages_and_weights_may_go_in_place(torch_dev, new):
    """A shared prefix: the first pages of three sequences are the same; and weight_out
    given as the cache's own weights."""
    torch, dev = torch_dev
    import cache_oracle as O
    import paper_2202_12674_amd as P
    cache, (k, v, table, lens, w) = make(torch, dev, "bf16", [300, 280, 333], 2, 64, 16, 7)
    q = torch.randn(3 * new, 4, 64, generator=torch.Generator().manual_seed(1)).bfloat16()
    off = offsets_of(torch, [new] * 3)
    weight = cache.weight.clone()
    P.attention(q.to(dev), cache, off.to(dev), accumulate=True)
    first = cache.weight.clone()
    cache.weight.copy_(weight)
    P.attention(q.to(dev), cache, off.to(dev), accumulate=True, weight_out=cache.weight)
    assert torch.equal(first.nan_to_num(-1), cache.weight.nan_to_num(-1))
    table[1, :9] = table[2, :9] = table[0, :9]
    cache.table.copy_(table)
    y = P.attention(q.to(dev), cache, off.to(dev))
    want, bound, _, _ = O.attention(q, k, v, table, lens, off, 0.125, True)
    _check(y, want, bound)


@pytest.mark.parametrize("page", [64, 21])
@pytest.mark.parametrize("new", [1, 90])
def test_pages_beyond_32_bit_offsets(torch_dev, new, page):
    """The same cache in a small pool and at the end of one of 5 GiB: equal in every bit."""
    torch, dev = torch_dev
    import paper_2202_12674_amd as P
    heads, d = 2, 128
    small, _ = make(torch, dev, "bf16", [500, 300], heads, d, page, 7)
    pages = 5 * 2 ** 30 // (heads * page * d * 2)
    base = pages - small.pages
    k, v = (torch.empty(pages, heads, page, d, dtype=torch.bfloat16, device=dev) for _ in "kv")
    w = torch.empty(pages, heads, page, device=dev)
    k[base:], v[base:], w[base:] = small.k, small.v, small.weight
    table = torch.where(small.table >= 0, small.table + base, small.table)
    large = P.PagedCache(k, v, table, small.lengths, w)
    q = torch.randn(2 * new, 8, d, device=dev).bfloat16()
    nk, nv = (torch.randn(2 * new, heads, d, device=dev).bfloat16() for _ in "kv")
    off, at = offsets_of(torch, [new, new]).to(dev), torch.arange(2 * new, device=dev)
    f, _ = P.rotary_frequencies(d, device=dev)
    out = []
    for c in (small, large):
        P.cache_append(c, nk, nv, off, at, f)
        out.append(P.attention(q, c, off, accumulate=True))
    assert torch.equal(out[0], out[1])
    for a, b in ((k, small.k), (v, small.v), (w, small.weight)):
        assert torch.equal(a[base:].nan_to_num(9.0), b.nan_to_num(9.0))
    del k, v, w, large
    torch.cuda.empty_cache()


def test_calls_of_two_threads(torch_dev):
    torch, dev = torch_dev
    import threading
    import paper_2202_12674_amd as P
    cache, _ = make(torch, dev, "f16", [700, 320], 2, 64, 16, 3)
    off = {n: offsets_of(torch, [n, n]).to(dev) for n in (1, 50)}
    q = {n: torch.randn(2 * n, 8, 64, device=dev).half() for n in off}
    want = {n: P.attention(q[n], cache, off[n]) for n in off}
    torch.cuda.synchronize()
    got, errors = {n: [] for n in off}, []

    def work(n):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got[n].append(P.attention(q[n], cache, off[n]))
                    try:
                        P.attention(q[n][:, :3], cache, off[n])
                        errors.append("not refused")
                    except P.LssvmError:
                        pass
                torch.cuda.current_stream().synchronize()
        except Exception as e:      # noqa: BLE001 - reported below
            errors.append(e)

    threads = [threading.Thread(target=work, args=(n,)) for n in off]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for n in off:
        for y in got[n]:
            assert torch.equal(y, want[n])


def test_tensor_refusals(torch_dev):
    torch, dev = torch_dev
    import paper_2202_12674_amd as P
    cache, _ = make(torch, dev, "bf16", [20, 5], 2, 64, 16)
    off = offsets_of(torch, [1, 1]).to(dev)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device=dev)
    pos, f = torch.zeros(2, dtype=torch.int64, device=dev), P.rotary_frequencies(64, device=dev)[0]
    kv = q[:, :2]
    bad = [lambda: P.attention(q.half(), cache, off), lambda: P.attention(q[:, :3], cache, off),
           lambda: P.attention(q[..., :32], cache, off), lambda: P.attention(q, cache, off[:2]),
           lambda: P.attention(q, cache, off.long()), lambda: P.attention(q, cache, off.cpu()),
           lambda: P.attention(q, cache, off, out=q), lambda: P.attention(q, cache, off, out=q[:1]),
           lambda: P.attention(q, cache, off, scale=math.nan),
           lambda: P.attention(q, cache, off, weight_out=cache.weight),
           lambda: P.attention(q, cache, off, accumulate=True, weight_out=cache.weight[:1]),
           lambda: P.attention(q, cache, off, workspace=torch.empty(0, device=dev)),
           lambda: P.attention(q.transpose(1, 2), cache, off),
           lambda: P.cache_append(cache, kv, kv[:1], off), lambda: P.cache_append(cache, q, q, off),
           lambda: P.cache_append(cache, kv, kv, off, pos), lambda: P.rotary(q, pos, f.float()),
           lambda: P.rotary(q, pos[:1], f), lambda: P.rotary(q, pos.float(), f),
           lambda: P.rotary(q, pos, torch.cat([f, f])), lambda: P.rotary(q, pos, f, out=q[:, :2]),
           lambda: P.cache_evict(cache, cache, 4), lambda: P.cache_evict(cache, cache, 0),
           lambda: P.PagedCache(cache.k, cache.v[:1], cache.table, cache.lengths),
           lambda: P.PagedCache(cache.k, cache.v, cache.table.long(), cache.lengths),
           lambda: P.PagedCache(cache.k, cache.v, cache.table, cache.lengths[:1]),
           lambda: P.PagedCache(cache.k, cache.v, cache.table, cache.lengths, cache.weight[:1])]
    for i, call in enumerate(bad):
        with pytest.raises((TypeError, ValueError, P.LssvmError)):
            call()
            print("not refused:", i)
    plain = P.PagedCache(cache.k, cache.v, cache.table, cache.lengths)
    with pytest.raises(P.LssvmError):
        P.attention(q, plain, off, accumulate=True)
