"""Refusals of the paged-cache operators that need no GPU."""
from __future__ import annotations

import ctypes

import pytest

from paper_2202_12674_amd import _binding as B
from paper_2202_12674_amd import cache as C

FAKE = 1 << 20                  # never dereferenced: validation fails first


def test_calls_that_require_a_gradient_are_refused_while_gradients_are_on():
    torch = pytest.importorskip("torch")
    C._no_gradient(False)
    with pytest.raises(ValueError, match="gradient"):
        C._no_gradient(True)
    with torch.no_grad():
        C._no_gradient(True)


@pytest.mark.parametrize("scale", [1e39, -1e300, 3.4e38])
def test_scales_beyond_single_precision_are_refused(scale):
    """Finite in double precision; 3.4e38 only where it is multiplied by log2(e)."""
    L, s = C._lib(), (ctypes.c_int64 * 2)(256, 64)
    cache = C._Cache(FAKE, FAKE, FAKE, FAKE, FAKE, 10, 2, 16, 64, 3, 4, (2048, 1024, 64),
                     (2048, 1024, 64), (32, 16), 4, C.BF16)
    assert L.lssvm_attention(ctypes.byref(cache), FAKE, s, 4, 4, FAKE, scale, 1, 0, None, None,
                             2 * FAKE, s, FAKE, 1 << 40, None) == B.EINVAL
    assert b"scale" in L.lssvm_last_error()
    if abs(scale) > 3.41e38:
        assert L.lssvm_rotary(FAKE, s, 2 * FAKE, s, 4, 4, 64, FAKE, 8, FAKE, 32, scale, 0, 0,
                              C.BF16, None) == B.EINVAL
        assert L.lssvm_cache_append(ctypes.byref(cache), FAKE, s, FAKE, s, 4, FAKE, FAKE, 8, FAKE,
                                    32, scale, 0, None) == B.EINVAL
