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
