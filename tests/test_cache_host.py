"""Checks of the paged-cache operators that need no GPU: the library exports what
include/lssvm_cache.h declares, refuses bad arguments on the host before any GPU
work, and computes the rotary frequencies of the formulas."""
from __future__ import annotations

import ctypes
import math
import os
import re

import pytest

import paper_2202_12674_amd as P
from paper_2202_12674_amd import _binding as B
from paper_2202_12674_amd import cache as C

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20                  # never dereferenced: validation fails first


def two(*v):
    return (ctypes.c_int64 * 2)(*v)


def cache(**change):
    c = C._Cache(FAKE, FAKE, FAKE, FAKE, FAKE, 10, 2, 16, 64, 3, 4, (2048, 1024, 64),
                 (2048, 1024, 64), (32, 16), 4, C.BF16)
    for k, v in change.items():
        setattr(c, k, (ctypes.c_int64 * len(v))(*v) if isinstance(v, tuple) else v)
    return c


def test_library_exports_every_declared_function():
    txt = open(os.path.join(ROOT, "include", "lssvm_cache.h")).read()
    txt = re.sub(r"/\*.*?\*/", "", txt, flags=re.S)
    names = sorted(set(re.findall(r"\b(lssvm_[a-z_]+)\s*\(", txt)))
    assert set(names) == set(C._SIGS)
    for nm in names:
        assert hasattr(P.lib(), nm), nm


BAD_CACHES = [dict(k=None), dict(v=None), dict(table=None), dict(lengths=None), dict(dtype=0),
              dict(dtype=9), dict(dim=0), dict(dim=12), dict(dim=264), dict(pages=0),
              dict(pages=1 << 31), dict(heads=0), dict(heads=65536), dict(page=0),
              dict(sequences=0), dict(sequences=65536), dict(columns=0), dict(columns=1 << 28), dict(sequences=65535, heads=65, k_stride=(66560, 1024, 64),
                                                   v_stride=(66560, 1024, 64),
                                                   weight_stride=(1040, 16)),
              dict(table_stride=3), dict(k=FAKE + 8), dict(v=FAKE + 2),
              dict(k_stride=(2048, 1024, 60)), dict(v_stride=(2044, 1024, 64)),
              dict(k_stride=(0, 1024, 64)), dict(k_stride=(2048, 1024, 32)),
              dict(v_stride=(2048, 64, 64)), dict(k_stride=(-2048, 1024, 64)),
              dict(k_stride=(1 << 41, 1024, 64)), dict(weight_stride=(16, 16)),
              dict(weight_stride=(32, 8))]


@pytest.mark.parametrize("change", BAD_CACHES, ids=lambda c: "-".join(c))
def test_every_call_refuses_a_bad_cache(change):
    L, good, c = C._lib(), cache(), cache(**change)
    s = two(128, 64)
    assert L.lssvm_attention_workspace_bytes(ctypes.byref(c), 4, 4, 0) == 0
    assert L.lssvm_attention(ctypes.byref(c), FAKE, s, 4, 4, FAKE, 1.0, 1, 0, None, None,
                             2 * FAKE, s, FAKE, 1 << 40, None) == B.EINVAL
    assert P.last_error().startswith("cache")
    assert L.lssvm_cache_append(ctypes.byref(c), FAKE, s, FAKE, s, 4, FAKE, None, 0, None, 0, 1.0,
                                0, None) == B.EINVAL
    assert L.lssvm_cache_evict(ctypes.byref(c), ctypes.byref(good), 4, 0, FAKE, None) == B.EINVAL
    assert L.lssvm_cache_evict(ctypes.byref(good), ctypes.byref(c), 4, 0, FAKE, None) == B.EINVAL


def test_a_missing_cache_is_refused():
    L, s = C._lib(), two(128, 64)
    assert L.lssvm_attention_workspace_bytes(None, 4, 4, 0) == 0
    assert L.lssvm_attention(None, FAKE, s, 4, 4, FAKE, 1.0, 1, 0, None, None, 2 * FAKE, s, FAKE,
                             1 << 40, None) == B.EINVAL


def test_a_dimension_of_one_may_have_any_stride():
    c = cache(pages=1, k_stride=(7, 1024, 64))
    assert C._lib().lssvm_attention_workspace_bytes(ctypes.byref(c), 4, 4, 0) > 0


def test_attention_refusals():
    L, c = C._lib(), cache()
    s = two(256, 64)
    need = L.lssvm_attention_workspace_bytes(ctypes.byref(c), 4, 4, 1)
    assert need > 0
    good = dict(q=FAKE, qs=s, tokens=4, heads=4, offsets=FAKE, scale=1.0, accumulate=1, wo=FAKE,
                ws=two(32, 16), out=2 * FAKE, os=s, work=FAKE, size=need)

    def call(cc=c, **change):
        a = {**good, **change}
        return L.lssvm_attention(ctypes.byref(cc), a["q"], a["qs"], a["tokens"], a["heads"],
                                 a["offsets"], a["scale"], 1, a["accumulate"], a["wo"], a["ws"],
                                 a["out"], a["os"], a["work"], a["size"], None)

    for change in (dict(q=None), dict(qs=None), dict(out=None), dict(os=None), dict(offsets=None),
                   dict(tokens=-1), dict(tokens=1 << 31), dict(heads=0), dict(heads=3),
                   dict(heads=65536), dict(tokens=1 << 29), dict(scale=math.inf), dict(scale=math.nan), dict(ws=None),
                   dict(ws=two(16, 16)), dict(os=two(64, 64)), dict(os=two(256, 32)),
                   dict(os=two(-256, 64)), dict(q=FAKE + 1), dict(out=2 * FAKE + 1),
                   dict(out=FAKE), dict(out=FAKE + 1024), dict(work=None), dict(work=FAKE + 8),
                   dict(size=need - 1)):
        assert call(**change) == B.EINVAL, change
    assert call(cache(weight=None), wo=None) == B.EINVAL
    assert L.lssvm_attention_workspace_bytes(ctypes.byref(c), 4, 3, 0) == 0
    assert L.lssvm_attention_workspace_bytes(ctypes.byref(c), -1, 4, 0) == 0
    # nothing to do: no rows, no weights
    assert call(tokens=0, accumulate=0, q=None, out=None) == B.OK


def test_rotary_refusals():
    L, s = C._lib(), two(256, 64)
    good = dict(x=FAKE, xs=s, out=2 * FAKE, os=s, tokens=4, heads=4, dim=64, pos=FAKE, bytes=8,
                freqs=FAKE, pairs=32, scale=1.0, dtype=C.BF16)

    def call(**change):
        a = {**good, **change}
        return L.lssvm_rotary(a["x"], a["xs"], a["out"], a["os"], a["tokens"], a["heads"],
                              a["dim"], a["pos"], a["bytes"], a["freqs"], a["pairs"], a["scale"],
                              0, 0, a["dtype"], None)

    for change in (dict(x=None), dict(xs=None), dict(out=None), dict(os=None), dict(tokens=-1),
                   dict(heads=0), dict(dim=0), dict(pairs=-1), dict(pairs=33), dict(pos=None),
                   dict(bytes=2), dict(pos=FAKE + 4), dict(freqs=None), dict(freqs=FAKE + 4),
                   dict(scale=math.inf), dict(dtype=0), dict(dtype=7), dict(os=two(64, 64)),
                   dict(x=FAKE + 1), dict(out=FAKE + 64), dict(out=FAKE, os=two(512, 64)),
                   dict(tokens=1 << 30, heads=1 << 15), dict(tokens=1 << 20, heads=1 << 10, dim=64)):
        assert call(**change) == B.EINVAL, change
    assert call(tokens=0, x=None, out=None, pos=None) == B.OK


def test_append_refusals():
    L, s, c = C._lib(), two(128, 64), cache()
    good = dict(k=FAKE, ks=s, v=FAKE, vs=s, tokens=4, offsets=FAKE, pos=FAKE, bytes=4, freqs=FAKE,
                pairs=32, scale=1.0)

    def call(**change):
        a = {**good, **change}
        return L.lssvm_cache_append(ctypes.byref(c), a["k"], a["ks"], a["v"], a["vs"], a["tokens"],
                                    a["offsets"], a["pos"], a["bytes"], a["freqs"], a["pairs"],
                                    a["scale"], 0, None)

    for change in (dict(k=None), dict(ks=None), dict(v=None), dict(vs=None), dict(tokens=-1),
                   dict(offsets=None), dict(pos=None), dict(bytes=3), dict(pos=FAKE + 2),
                   dict(freqs=None), dict(pairs=33), dict(pairs=-1), dict(scale=math.nan),
                   dict(k=FAKE + 1), dict(v=FAKE + 1), dict(vs=two(-1, 64))):
        assert call(**change) == B.EINVAL, change
    assert call(tokens=0, k=None, v=None) == B.OK


def test_evict_refusals():
    L = C._lib()
    a = cache()
    other = dict(table=2 * FAKE, lengths=2 * FAKE)

    def call(b=None, budget=8, recent=2, kept=FAKE, source=a):
        b = cache(**other) if b is None else b
        return L.lssvm_cache_evict(ctypes.byref(source), ctypes.byref(b), budget, recent, kept,
                                   None)

    for b in (cache(**other, weight=None), cache(**other, heads=1), cache(**other, page=8),
              cache(**other, dim=56), cache(**other, sequences=2), cache(**other, dtype=C.F16),
              cache(table=2 * FAKE), cache(lengths=2 * FAKE)):
        assert call(b) == B.EINVAL
    for change in (dict(budget=0), dict(budget=65), dict(recent=-1), dict(kept=None),
                   dict(source=cache(weight=None))):
        assert call(**change) == B.EINVAL, change


@pytest.mark.parametrize("dim", [2, 4, 64, 130])
def test_rotary_frequencies_are_those_of_the_formulas(dim):
    n, factor, original = dim // 2, 4.0, 2048.0
    plain, one = P.rotary_frequencies(dim)
    assert one == 1.0
    want = [10000.0 ** (-2.0 * i / dim) for i in range(n)]
    assert plain.tolist() == pytest.approx(want, rel=1e-14)
    linear, _ = P.rotary_frequencies(dim, scaling="linear", factor=factor)
    assert linear.tolist() == pytest.approx([f / factor for f in want], rel=1e-14)
    ntk, _ = P.rotary_frequencies(dim, scaling="ntk", factor=factor)
    assert ntk[0] == 1.0
    if n > 1:     # the slowest pair is stretched by factor
        assert float(ntk[-1]) == pytest.approx(want[-1] / factor, rel=1e-12)
    yarn, scale = P.rotary_frequencies(dim, scaling="yarn", factor=factor, original=original)
    assert scale == pytest.approx(0.1 * math.log(factor) + 1.0, rel=1e-15)
    for f, y in zip(want, yarn.tolist()):
        turns = original * f / (2 * math.pi)
        keep = min(1.0, max(0.0, (turns - 1.0) / 31.0))
        assert y == pytest.approx(f * keep + f / factor * (1 - keep), rel=1e-13)


def test_rotary_frequencies_refusals():
    for a in (dict(dim=0), dict(dim=3), dict(dim=-2), dict(dim=8, scaling="more")):
        with pytest.raises(ValueError):
            P.rotary_frequencies(**a)
    for a in (dict(base=0.0), dict(base=math.inf), dict(factor=0.5), dict(factor=math.nan),
              dict(scaling="yarn", original=0.0)):
        with pytest.raises(P.LssvmError):
            P.rotary_frequencies(8, **a)


def test_tensors_that_are_not_on_a_gpu_are_refused():
    torch = pytest.importorskip("torch")
    k = torch.zeros(4, 2, 16, 64)
    with pytest.raises(TypeError):
        P.PagedCache(k, k, torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(TypeError):
        P.rotary(torch.zeros(2, 2, 8), torch.zeros(2, dtype=torch.int64),
                 torch.zeros(4, dtype=torch.float64))
    for call in (lambda: P.attention(k[0], None, None), lambda: P.cache_append(None, k, k, None),
                 lambda: P.cache_evict(None, None, 3)):
        with pytest.raises(TypeError):
            call()
