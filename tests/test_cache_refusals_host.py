"""Refusals of the paged-cache operators that need no GPU."""
from __future__ import annotations

import pytest

from paper_2202_12674_amd import cache as C


def test_tensors_that_require_a_gradient_are_refused_while_gradients_are_on():
    torch = pytest.importorskip("torch")
    x, leaf = torch.zeros(2), torch.zeros(2, requires_grad=True)
    C._no_gradient(x, x)
    for t in (leaf, leaf * 2):
        with pytest.raises(ValueError, match="gradient"):
            C._no_gradient(x, t)
        with torch.no_grad():
            C._no_gradient(x, t)
