"""GPU: the operators over a paged cache where their numbers run out of range: weights,
values, angles and scores far from 1, and calls as large as the limits allow."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24      # half a step of fp32


def one_sequence(torch, dev, k, v, page=16):
    """A cache of one sequence and one head, keys and values (L x d) in order."""
    import paper_2202_12674_amd as P
    L, d = k.shape
    pages = -(-L // page)
    pool = torch.zeros(2, pages * page, d, dtype=k.dtype)
    pool[0, :L], pool[1, :L] = k, v
    pool = pool.view(2, pages, 1, page, d).to(dev)
    return P.PagedCache(pool[0], pool[1], torch.arange(pages, dtype=torch.int32, device=dev)[None],
                        torch.tensor([L], dtype=torch.int32, device=dev),
                        torch.zeros(pages, 1, page, device=dev))


def attend(torch, dev, q, k, v, page=16, causal=False, accumulate=False):
    """(out, weights) of rows q over one sequence, scale 1."""
    import paper_2202_12674_amd as P
    cache = one_sequence(torch, dev, k, v, page)
    off = torch.tensor([0, q.shape[0]], dtype=torch.int32, device=dev)
    y = P.attention(q.to(dev), cache, off, scale=1.0, causal=causal, accumulate=accumulate)
    return y.cpu(), cache.weight.view(-1)[:k.shape[0]].double().cpu()


# ------------------------------------------ weights far below the largest ---

def _faint(torch, dev, gaps, v, new, page):
    """Keys `gaps` nats below a score of 0 with values v >= 0, all in half precision."""
    L, d, heads = len(gaps), v.shape[1], 2
    k = torch.zeros(L, d)
    k[:, 0] = -torch.tensor(gaps)
    k, v = k.half(), v.half()
    q = torch.zeros(new, heads, d)
    q[..., 0] = 1.0
    y, w = attend(torch, dev, q.half(), k, v, page, accumulate=True)
    p = torch.softmax(k[:, 0].double(), 0)
    want = p @ v.double()
    # Nothing cancels. Half a step of fp16 for the weights and one for the result; the
    # sums over L keys of 2 terms each, and scores of up to 32 nats with three roundings,
    # in fp32.
    rel = U * (4 * L + 8 * 32 + 16)
    bound = want * (2 * 2.0 ** -11 + rel) + 2.0 ** -24
    worst = float(((y.double() - want).abs() / bound).max())
    assert worst <= 1.0, worst
    gain = new * heads * p
    assert bool(((w - gain).abs() <= gain * (rel + U * new * heads) + 1e-37).all())


@pytest.mark.parametrize("new", [1, 5, 200])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 21), (256, 32)])
@pytest.mark.parametrize("gap,every", [(8.0, 32), (15.0, 32), (17.5, 32), (22.0, 32), (15.0, 4096),
                                       (25.0, 4096), (28.0, 4096)])
def test_many_small_weights_in_half_precision(torch_dev, new, d, page, gap, every):
    """Single keys of value zero take nearly all the weight, thousands of others share
    the rest: what they add up to is a normal number."""
    torch, dev = torch_dev
    g = torch.Generator().manual_seed(1)
    v = 2e4 + 4e4 * torch.rand(4096, d, generator=g)
    v[::every] = 0.0
    _faint(torch, dev, [0.0 if j % every == 0 else gap for j in range(4096)], v, new, page)


@pytest.mark.parametrize("new", [1, 200])
@pytest.mark.parametrize("least", [0.0, 7.0, 14.0, 21.0])
def test_weights_of_all_sizes_in_half_precision(torch_dev, new, least):
    """Weights over forty powers of two; those above the bound meet values of zero."""
    torch, dev = torch_dev
    g = torch.Generator().manual_seed(2)
    gaps = (28.0 * torch.rand(3000, generator=g)).half().float()
    gaps[0] = 0.0
    v = (2e4 + 4e4 * torch.rand(3000, 64, generator=g)) * (gaps >= least)[:, None]
    _faint(torch, dev, gaps.tolist(), v, new, 16)


@pytest.mark.parametrize("new", [1, 9, 150])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 21), (256, 32)])
def test_small_weights_beside_values_that_are_not_finite(torch_dev, new, d, page):
    """Half precision, causal rows: faint weights in steps that are masked, and gone over
    again for the infinities and NaNs of the last tokens."""
    torch, dev = torch_dev
    import cache_oracle as O
    g = torch.Generator().manual_seed(12)
    L, pages = 700, -(-700 // page)
    k, v = torch.zeros(L, d), 2e4 + 4e4 * torch.rand(L, d, generator=g)
    k[:, 0], v[0] = -14.0 - 14.0 * torch.rand(L, generator=g), 0.0
    k[0, 0] = 0.0
    v[L - 1, 3], v[L - 1 - new // 2, 4], v[L - new, 5] = math.inf, math.nan, -math.inf
    k, v = k.half(), v.half()
    q = torch.zeros(new, 2, d).half()
    q[..., 0] = 1.0
    pool = torch.zeros(2, pages * page, d).half()
    pool[0, :L], pool[1, :L] = k, v
    pool = pool.view(2, pages, 1, page, d)
    want, bound, w, slack = O.attention(
        q, pool[0], pool[1], torch.arange(pages, dtype=torch.int32)[None], torch.tensor([L]),
        torch.tensor([0, new], dtype=torch.int32), 1.0, True, torch.zeros(pages, 1, page))
    y, weight = attend(torch, dev, q, k, v, page, causal=True, accumulate=True)
    fine = want.isfinite()
    # (the plain bound's absolute part, the least normal number, down to half a step there)
    bound = bound - torch.finfo(torch.float16).tiny + 2.0 ** -24
    assert torch.equal(y.double()[~fine].nan_to_num(7.0), want[~fine].nan_to_num(7.0))
    assert bool(((y.double() - want).abs() <= bound)[fine].all())
    assert bool(((weight - w.view(-1)[:L]).abs() <= slack.view(-1)[:L]).all())


# ----------------------------------------------------------- wide angles ----

@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_rotary_of_positions_as_large_as_their_type(torch_dev, dtype, interleaved):
    """The angle is position x frequency in fp64, however large; an infinite one is NaN."""
    torch, dev = torch_dev
    import cache_oracle as O
    import paper_2202_12674_amd as P
    g = torch.Generator().manual_seed(3)
    near = [s * 2 ** e + o for e in (30, 40, 44, 45, 46, 49, 52, 53, 55, 58, 62) for s in (1, -1)
            for o in (-1, 0, 1)]
    pos = torch.tensor(near + [2 ** 63 - 1, -2 ** 63, 0], dtype=torch.int64)
    f = torch.tensor([1.0, 0.7390851332151607, 1e-3, 1e-9, 3.0, 1e5, 1e30, 1e300],
                     dtype=torch.float64)
    x = torch.randn(len(pos), 2, 21, generator=g)
    x = x.half() if dtype == "f16" else x
    y = P.rotary(x.to(dev), pos.to(dev), f.to(dev), interleaved=interleaved).double().cpu()
    for t in range(len(pos)):
        angles = [float(pos[t]) * a for a in f.tolist()]
        for i, a in enumerate(angles):
            m, n = (2 * i, 2 * i + 1) if interleaved else (i, i + len(angles))
            x0, x1 = x[t, :, m].double(), x[t, :, n].double()
            if math.isinf(a):
                assert bool(y[t, :, [m, n]].isnan().all())
                continue
            c, s = math.cos(a), math.sin(a)
            for at, want in ((m, x0 * c - x1 * s), (n, x1 * c + x0 * s)):
                bound = O.rotary_bound(want, x0.abs() + x1.abs(), x.dtype)
                assert bool(((y[t, :, at] - want).abs() <= bound).all()), (int(pos[t]), a)
    assert torch.equal(y[..., 16:], x[..., 16:].double())


# ------------------------------------------------------------ wide values ---

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,L,d,page", [(n, *c) for n in (1, 200) for c in (
    (300, 64, 16), (5000, 128, 21), (2000, 256, 32))] + [(300, 5000, 128, 16)])
def test_values_near_the_largest(torch_dev, dtype, new, L, d, page):
    """A mean of finite values is finite, though their sum is not; an infinity among them
    reaches the rows that see it."""
    torch, dev = torch_dev
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(4)
    k, q = torch.randn(L, d, generator=g).to(dt), torch.randn(new, 1, d, generator=g)
    q = (q / math.sqrt(d)).to(dt)
    v = (3e38 * (0.5 + 0.5 * torch.rand(L, d, generator=g))).to(dt)
    v[:, 1] = torch.randn(L, generator=g).abs().to(dt)      # an ordinary column among them
    v[L - 1 - new // 2, 5] = math.inf
    y = attend(torch, dev, q, k, v, page, causal=True)[0][:, 0].double()
    z = q[:, 0].double() @ k.double().T
    z[torch.arange(L)[None, :] > L - new + torch.arange(new)[:, None]] = -math.inf
    p = torch.softmax(z, 1)
    want = p @ torch.where(v.isinf(), 0.0, v.double())
    want[p[:, L - 1 - new // 2] > 0, 5] = math.inf
    reach = float((q.double().abs()[:, 0] @ k.double().abs().T).max())
    rel = 2 * U * (2 * (d + 4) * reach + 2 * L + 16) + \
        (2 * 2.0 ** -9 * 2 if dtype == "bf16" else 2 * U)
    fine = want.isfinite()
    assert torch.equal(fine, y.isfinite()) and torch.equal(y[~fine], want[~fine])
    assert bool(((y - want).abs() <= rel * want)[fine].all())


# -------------------------------------------------- scores that are infinite ---

@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new,L,page", [(1, 400, 16), (1, 1500, 21), (150, 400, 16), (150, 1500, 21),
                                        (300, 9000, 32)])
def test_scores_of_minus_infinity(torch_dev, dtype, new, L, page):
    """Such a key weighs exactly nothing: finite values under it are left out, one that is
    not finite gives NaN; and a row of no other keys has no softmax."""
    torch, dev = torch_dev
    dt = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype]
    g = torch.Generator().manual_seed(5)
    d = 64
    k, v = torch.randn(L, d, generator=g).to(dt), torch.randn(L, d, generator=g).to(dt)
    q = torch.zeros(new, 1, d, dtype=dt)
    q[..., 0] = 1.0
    lost = [3, 77, L - new // 2 - 1, L - 1]
    k[lost, 0] = -math.inf
    v[3, 5], v[77, 6], v[L - new // 2 - 1, 7] = math.inf, math.nan, -math.inf
    v[8, 9], v[9, 10] = math.inf, math.nan                   # under finite scores
    y = attend(torch, dev, q, k, v, page, causal=True)[0][:, 0].double()
    z = (q[:, 0].double() @ torch.where(k.isinf(), 0.0, k.double()).T)
    z[:, lost] = -math.inf
    seen = torch.arange(L)[None, :] <= L - new + torch.arange(new)[:, None]
    p = torch.softmax(torch.where(seen, z, -math.inf), 1)
    want, size = (p @ torch.where(v.isfinite(), x, 0.0) for x in (v.double(), v.double().abs()))
    want[:, [5, 6, 10]], want[:, 9] = math.nan, math.inf
    want[seen[:, L - new // 2 - 1], 7] = math.nan
    half = torch.finfo(dt).eps / 2
    bound = half * want.abs() + (half * (dtype != "f32") + U * (4 * L + 4 * d * 8)) * size + 1e-7
    fine = want.isfinite()
    assert torch.equal(want.isnan(), y.isnan()) and torch.equal(want.isinf(), y.isinf())
    assert bool(((y - want).abs() <= bound)[fine].all())

    k[:, 0] = -math.inf
    y, w = attend(torch, dev, q, k, v, page, causal=True, accumulate=True)
    assert bool(y.isnan().all()) and bool(w.isnan().all())
    k[L - new, 0] = 2.0                                      # one key that is seen by all
    y = attend(torch, dev, q, k, v, page, causal=True)[0][:, 0]
    others = [x for x in range(d) if x not in (5, 6, 7, 9, 10)]
    only = v[L - new, others].double()
    assert bool(((y[:, others].double() - only).abs() <= 8 * U * only.abs()).all())


# ---------------------------------------------------------- largest sizes ---

def test_evict_to_the_largest_budget(torch_dev):
    """A budget of 2^29 keys of 512 bytes: 2^32 pieces of 16 bytes, of which a grid's side
    cannot have a thread each. The sequence itself is short."""
    torch, dev = torch_dev
    import paper_2202_12674_amd as P
    page, d, L = 1 << 12, 128, 9
    columns = (1 << 29) // page
    pool = torch.zeros(2, 2, 1, page, d, device=dev)
    pool[:, 0, 0, :L] = torch.randn(2, L, d, device=dev)
    weight = torch.zeros(2, 1, page, device=dev)
    weight[0, 0, :L] = torch.arange(L, device=dev)
    cache, target = (P.PagedCache(pool[0], pool[1],
                                  torch.full((1, columns), i, dtype=torch.int32, device=dev),
                                  torch.tensor([L * (1 - i)], dtype=torch.int32, device=dev), weight)
                     for i in (0, 1))
    kept = P.cache_evict(cache, target, 1 << 29, 0)
    assert kept[0, 0, :L].tolist() == list(range(L)) and int(target.lengths) == L
    assert bool((kept[0, 0, L:] == -1).all())
    assert torch.equal(pool[:, 1, 0, :L], pool[:, 0, 0, :L]) and not pool[:, 1, 0, L:].any()
    assert torch.equal(weight[1], weight[0])
    del kept
    torch.cuda.empty_cache()


def test_evict_of_the_longest_sequence(torch_dev):
    """2^29 keys, all recent: what stands first and last of them arrives there. Every page
    is the same one, and all but two of the target's are holes."""
    torch, dev = torch_dev
    import paper_2202_12674_amd as P
    page, d = 1 << 12, 128
    columns = (1 << 29) // page
    pool = torch.zeros(2, 3, 1, page, d, device=dev)
    pool[:, 0] = torch.randn(2, 1, page, d, device=dev)
    weight = torch.zeros(3, 1, page, device=dev)
    weight[0, 0] = torch.rand(page, device=dev)
    to = torch.full((1, columns), -1, dtype=torch.int32, device=dev)
    to[0, 0], to[0, -1] = 1, 2
    cache = P.PagedCache(pool[0], pool[1], torch.zeros_like(to),
                         torch.full((1,), 1 << 29, dtype=torch.int32, device=dev), weight)
    target = P.PagedCache(pool[0], pool[1], to, torch.zeros(1, dtype=torch.int32, device=dev),
                          weight)
    kept = P.cache_evict(cache, target, 1 << 29, 1 << 29)
    assert int(target.lengths) == 1 << 29
    assert int(kept[0, 0, 0]) == 0 and bool((kept[0, 0].diff() == 1).all())
    for p in (1, 2):
        assert torch.equal(pool[:, p], pool[:, 0]) and torch.equal(weight[p], weight[0])
    del kept
    torch.cuda.empty_cache()


def test_attention_of_as_many_rows_as_a_call_may_have(torch_dev):
    """1024 sequences of 64 rows and 4096 heads, which in tiles of 16 rows would be more
    workgroups than a grid holds. Every sequence has the same two keys."""
    torch, dev = torch_dev
    import paper_2202_12674_amd as P
    seqs, new, heads, d = 1024, 64, 4096, 8
    g = torch.Generator().manual_seed(6)
    k, v = (torch.randn(1, heads, 16, d, generator=g).bfloat16().to(dev) for _ in "kv")
    cache = P.PagedCache(k, v, torch.zeros(seqs, 1, dtype=torch.int32, device=dev),
                         torch.full((seqs,), 2, dtype=torch.int32, device=dev))
    off = (new * torch.arange(seqs + 1, device=dev)).int()
    q = torch.randn(1, heads, d, generator=g).bfloat16().to(dev)
    out = torch.full((seqs * new, heads, d), 7.0, dtype=torch.bfloat16, device=dev)
    P.attention(q.expand(seqs * new, heads, d), cache, off, causal=False, out=out)
    one = P.PagedCache(k, v, cache.table[:1], cache.lengths[:1])
    want = P.attention(q.expand(new, heads, d), one, off[:2], causal=False)
    p = torch.softmax(d ** -0.5 * (q[0, :, None].double() * k[0, :, :2].double()).sum(-1), -1)
    exact = (p[..., None] * v[0, :, :2].double()).sum(1)
    size = (p[..., None] * v[0, :, :2].double().abs()).sum(1)
    # half a step of bf16 for the result and one for the weights
    bound = 2.0 ** -8 * (exact.abs() + size) * 1.01 + 1e-6
    assert bool(((want.double() - exact).abs() <= bound).all())
    assert bool(((out[0].double() - exact).abs() <= bound).all())
    for rows in out.split(1 << 12):
        assert torch.equal(rows, out[:1].expand_as(rows))
    del out, rows
    torch.cuda.empty_cache()


@pytest.mark.parametrize("pairs,interleaved", [(0, False), (3, True)])
def test_append_of_as_many_tokens_as_a_call_may_have(torch_dev, pairs, interleaved):
    """2^30 tokens of four and five pieces of 16 bytes each, 2^32 and more; all but the
    last three lie outside the offsets."""
    torch, dev = torch_dev
    import paper_2202_12674_amd as P
    tokens, d = 1 << 30, 8
    k, v = (torch.arange(1.0, d + 1, device=dev).mul(s).view(1, 1, d) for s in (1, -2))
    pool = torch.zeros(2, 1, 1, 16, d, device=dev)
    weight = torch.ones(1, 1, 16, device=dev)
    cache = P.PagedCache(pool[0], pool[1], torch.zeros(1, 1, dtype=torch.int32, device=dev),
                         torch.tensor([5], dtype=torch.int32, device=dev), weight)
    off = torch.tensor([tokens - 3, tokens], dtype=torch.int32, device=dev)
    turned = {}
    if pairs:       # every angle is 0
        turned = dict(positions=torch.zeros(1, dtype=torch.int32, device=dev).expand(tokens),
                      freqs=torch.ones(pairs, dtype=torch.float64, device=dev),
                      interleaved=interleaved)
        turned["positions"] = turned["positions"].contiguous()
    P.cache_append(cache, k.expand(tokens, 1, d), v.expand(tokens, 1, d), off, **turned)
    assert torch.equal(pool[0, 0, 0, 2:5], k[0].expand(3, d))
    assert torch.equal(pool[1, 0, 0, 2:5], v[0].expand(3, d))
    assert not pool[:, 0, 0, :2].any() and not pool[:, 0, 0, 5:].any()
    assert weight.flatten().tolist() == [1.0] * 2 + [0.0] * 3 + [1.0] * 11
    del turned
    torch.cuda.empty_cache()


# --------------------------------------------------------------- gradients ---

def test_calls_that_would_lose_a_gradient_are_refused(torch_dev):
    torch, dev = torch_dev
    import paper_2202_12674_amd as P
    cache = one_sequence(torch, dev, *torch.randn(2, 20, 64).bfloat16())
    target = one_sequence(torch, dev, *torch.randn(2, 20, 64).bfloat16())
    leaf = P.PagedCache(cache.k.clone().requires_grad_(), cache.v, cache.table, cache.lengths,
                        cache.weight)
    off = torch.tensor([0, 2], dtype=torch.int32, device=dev)
    x = torch.randn(2, 1, 64, device=dev).bfloat16()
    g = x.clone().requires_grad_()
    pos, f = torch.arange(2, device=dev), P.rotary_frequencies(64, device=dev)[0]
    calls = [lambda x, c: P.rotary(x, pos, f), lambda x, c: P.attention(x, c, off),
             lambda x, c: P.cache_append(c, x, x, off, pos, f)]
    for call in calls:
        for a, c in [(g, cache)] + ([(x, leaf)] if call is not calls[0] else []):
            with pytest.raises(ValueError, match="gradient"):
                call(a, c)
            with torch.no_grad():
                call(a, c)
        call(g.detach(), cache), call(x, cache)
    with pytest.raises(ValueError, match="gradient"):
        P.rotary(x, pos, f, out=g * 1)
    with pytest.raises(ValueError, match="gradient"):
        P.cache_evict(leaf, target, 4)
    with torch.no_grad():
        assert torch.equal(P.rotary(g, pos, f), P.rotary(x, pos, f))
        P.cache_evict(leaf, target, 4)


# ------------------------------------------------------- views of one array ---

def test_results_beside_their_inputs_in_one_array(torch_dev):
    """Inputs and results that are parts of every row of one array do not overlap, those
    that share a value do."""
    torch, dev = torch_dev
    import paper_2202_12674_amd as P
    g = torch.Generator().manual_seed(8)
    heads, d, tokens = 3, 64, 7
    wide = torch.randn(tokens, 2 * heads + 1, d, generator=g).bfloat16().to(dev)
    x, y = wide[:, :heads], wide[:, heads + 1:]
    keep = wide.clone()
    pos, f = torch.arange(tokens, device=dev), P.rotary_frequencies(d, device=dev)[0]
    k, v = torch.randn(2, 50, d, generator=g).bfloat16()
    cache = one_sequence(torch, dev, k, v)
    off = torch.tensor([0, tokens], dtype=torch.int32, device=dev)
    for a, b in ((x, y), (y, x)):
        wide.copy_(keep)
        want = P.rotary(a, pos, f), P.attention(a, cache, off)
        for i, call in enumerate((lambda: P.rotary(a, pos, f, out=b),
                                  lambda: P.attention(a, cache, off, out=b))):
            call()
            assert torch.equal(b, want[i])
        rest = slice(0, heads + 1) if b is y else slice(heads, None)
        assert torch.equal(wide[:, rest], keep[:, rest])
    with pytest.raises(P.LssvmError, match="overlap"):
        P.rotary(x, pos, f, out=wide[:, 1:heads + 1])
    with pytest.raises(P.LssvmError, match="overlap"):
        P.attention(x, cache, off, out=wide[:, 2:heads + 2])
    # the next token's row, some heads on
    with pytest.raises(P.LssvmError, match="overlap"):
        P.rotary(wide.view(-1, d)[:24].view(4, 6, d)[:3, :4], pos[:3], f,
                 out=wide.view(-1, d)[3:21].view(3, 6, d)[:, :4])


# ------------------------------------- keys and queries that are not finite ---

@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new,page", [(1, 16), (9, 21), (200, 16)])
def test_keys_and_queries_that_are_not_finite(torch_dev, dtype, new, page):
    """A NaN in a key, an infinite score or a NaN in a query makes a NaN of every row that
    it enters, and changes no other."""
    torch, dev = torch_dev
    import cache_oracle as O
    import paper_2202_12674_amd as P
    dt = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype]
    g = torch.Generator().manual_seed(9)
    L, d, heads = 333, 64, 2
    k, v = (torch.randn(L, d, generator=g).to(dt) for _ in "kv")
    q = torch.randn(new, heads, d, generator=g).to(dt)
    q[:, 0, 7] = 1.0
    q[:, 1, 7] = -1.0
    last, pages = L - new // 3 - 1, -(-L // page)      # seen by the last third of the rows
    table = torch.arange(pages, dtype=torch.int32)[None]
    off = torch.tensor([0, new], dtype=torch.int32)

    def plain(k, v):
        pool = torch.zeros(2, pages * page, d, dtype=dt)
        pool[0, :len(k)], pool[1, :len(k)] = k, v
        pool = pool.view(2, pages, 1, page, d)
        return O.attention(q, pool[0], pool[1], table, torch.tensor([len(k)]), off, 1.0, True)[:2]

    want, bound = plain(k, v)
    for what in ("nan key", "inf key", "nan query"):
        kk, qq, out = k.clone(), q.clone(), want.clone()
        rows = torch.arange(new) >= last - (L - new)
        if what == "nan key":
            kk[last, 7], out[rows] = math.nan, math.nan
        elif what == "inf key":       # head 0: a score of infinity, head 1: of minus infinity
            kk[last, 7], out[rows, 0] = math.inf, math.nan
        else:
            qq[new // 2, 1, 3], out[new // 2, 1] = math.nan, math.nan
        y, w = attend(torch, dev, qq, kk, v, page, causal=True, accumulate=True)
        y, slack = y.double(), bound.clone()
        assert bool(w.isnan()[:L - new + 1].all()), what     # seen by every row
        if what == "inf key":         # as without that key, for the rows that see it
            less = [torch.cat([x[:last], x[last + 1:]]) for x in (k, v)]
            out[rows, 1], slack[rows, 1] = (x[rows, 1] for x in plain(*less))
        fine = out.isfinite()
        assert torch.equal(y.isnan(), out.isnan()), what
        assert bool(((y - out).abs() <= slack)[fine].all()), what


# ------------------------------------------------------------ wide tables ---

@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new", [[1, 1, 1], [1, 60, 3], [100, 40, 120]])
@pytest.mark.parametrize("columns", [40, 900])
def test_tables_much_wider_than_their_sequences(torch_dev, dtype, new, columns):
    """Room for many times the keys that are there, in steps of one plan and another: as
    in a table of just the sequences' pages, and prompts and single tokens in one call."""
    torch, dev = torch_dev
    import cache_oracle as O
    import paper_2202_12674_amd as P
    from test_gpu_cache import make, offsets_of, _check
    lengths, page, d = [130, 61, 250], 16, 64
    cache, (k, v, table, lens, w) = make(torch, dev, dtype, lengths, 2, d, page, 3, columns=columns)
    q = torch.randn(sum(new), 6, d, generator=torch.Generator().manual_seed(3)).to(k.dtype)
    off = offsets_of(torch, new)
    wout = torch.full(w.shape, -5.0, device=dev)
    y = P.attention(q.to(dev), cache, off.to(dev), accumulate=True, weight_out=wout)
    want, bound, ww, slack = O.attention(q, k, v, table, lens, off, d ** -0.5, True, w)
    _check(y, want, bound, "out")
    there = ~w.isnan()
    _check(wout.cpu()[there], ww[there], slack[there], "weight")
    assert bool((wout.cpu()[~there] == -5.0).all())
    target, _ = make(torch, dev, dtype, [40] * 3, 2, d, page, 4, columns=columns)
    kept = P.cache_evict(cache, target, 40, 7)
    assert torch.equal(kept.cpu(), O.evict(w, table, lens, 40, 7, page))
