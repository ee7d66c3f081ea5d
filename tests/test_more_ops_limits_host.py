"""What position bias, routing, balance loss and activations in 8 bits accept at the ends of
their arguments, and what the functions on tensors need of torch (no GPU call is made)."""

import numpy as np
import pytest

arplan = pytest.importorskip(
    "paper_2409_04202_amd.arplan",
    reason="HIP library not built (run python -m paper_2409_04202_amd.build)")

P = 1 << 40     # an address that is never used
BIG = 1 << 30   # apart from the next


def at(i):
    return P + i * BIG


@pytest.mark.parametrize("coefficient", (float(np.finfo(np.float32).max), -3.4e38, 1e-45, 0.0))
def test_every_finite_coefficient_is_accepted(coefficient):
    """The refusal that such a call meets is one that is checked later: the loss in the mass."""
    with pytest.raises(arplan.ArError, match="overlaps"):
        arplan.ar_balance("bf16", 4, 16, 2, at(0), 16, at(1), at(2), at(3), coefficient, 1, at(4),
                          at(3), at(6), 16)
