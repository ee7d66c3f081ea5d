"""What position bias, routing, balance loss and activations in 8 bits accept at the ends of
their arguments, and what the functions on tensors need of torch (no GPU call is made)."""

import os
import subprocess
import sys

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


def test_tensors_are_refused_by_a_torch_without_gpu_functions():
    """The module imports, and refuses what is not on a GPU, where torch has no functions for
    the current device and stream."""
    pytest.importorskip("torch")
    code = ("import torch\n"
            "for n in ('_cuda_getDevice', '_cuda_getCurrentRawStream'):\n"
            "    if hasattr(torch._C, n):\n"
            "        delattr(torch._C, n)\n"
            "from paper_2409_04202_amd import ops\n"
            "try:\n"
            "    ops.checkpoint_store(torch.zeros(2, 2))\n"
            "except ValueError as e:\n"
            "    print('refused:', e)\n")
    r = subprocess.run([sys.executable, "-c", code], stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                       text=True, timeout=300, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0 and "refused: x: a GPU tensor expected" in r.stdout, r.stdout


@pytest.mark.parametrize("k", (2.0, "2", None, -1, (1 << 64) + 2))
def test_a_number_of_choices_that_is_none(k):
    torch = pytest.importorskip("torch")
    from paper_2409_04202_amd import ops
    with pytest.raises(ValueError, match="k: a whole number"):
        ops.route(torch.zeros(4, 8), k)


def test_workspaces_of_several_blocks_are_asked_for():
    """A byte less than asked for, none, one off 16 bytes, and those that are an operand's, at the
    smallest sizes that need any."""
    def refused(f, *args):
        with pytest.raises(arplan.ArError) as e:
            f(*args)
        assert e.value.status == arplan.AR_ERR_INVALID_ARG

    for dtype, B, Q, K in (("bf16", 5, 32, 32), ("f32", 9, 32, 32), ("f32", 2, 130, 1100)):
        need = arplan.ar_position_bias_grad_workspace(dtype, 32, B, 4, Q, K)
        assert need > 0
        for space, n in ((at(2), need - 1), (None, need), (at(2) + 8, need), (at(0), need), (at(1), need)):
            refused(arplan.ar_position_bias_grad, dtype, 32, 128, 0, B, 4, Q, K, 0, at(0), 4 * Q * K,
                    Q * K, K, 0, at(1), 4, space, n)
    need = arplan.ar_route_workspace(385, 40, 2)
    assert need > 0
    for dtype in ("bf16", "f32"):
        for space, n in ((at(6), need - 1), (None, need), (at(6) + 8, need), (at(0), need), (at(2), need)):
            refused(arplan.ar_route, dtype, 385, 40, 2, at(0), 40, None, 1, at(2), at(3), at(4), at(5),
                    space, n)
