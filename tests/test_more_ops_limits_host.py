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


@pytest.mark.parametrize("E,rows", [(8, 1024), (61, 128), (128, 64), (512, 16), (1024, 8)])
def test_routings_that_one_block_takes(E, rows):
    """A routing without a workspace is one block's for both types: two passes over its
    wavefronts' rows at most, and of many choices or all experts one, for another would take
    longer in fp32 than the blocks' join."""
    for k in (1, 8, 9, 32):
        if k <= E:
            passes = 2 if k <= 8 and k < E else 1
            assert arplan.ar_route_workspace(passes * rows, E, k) == 0
            assert arplan.ar_route_workspace(passes * rows + 1, E, k) > 0
