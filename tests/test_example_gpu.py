"""The data-parallel example: the replicas' gradients through an AllReduce plan
against automatic differentiation of the whole batch in 64 bits, and training."""

import importlib.util
import math
import os

import pytest
import torch

pytest.importorskip(
    "paper_2409_04202_amd.arplan",
    reason="HIP library not built (run python -m paper_2409_04202_amd.build)")
from paper_2409_04202_amd import arplan  # noqa: E402

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location(
        "data_parallel_distill", os.path.join(ROOT, "examples", "data_parallel_distill.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_allreduced_gradient_is_the_whole_batchs():
    ex, n = _example(), 3
    model = ex.Model(7, torch.float32)
    rows = [torch.zeros(ex.Model.SIZE, device="cuda") for _ in range(n)]
    data = [ex.batch(0, r, n) for r in range(n)]
    losses = torch.cat([ex.gradients(model, *d, row) for d, row in zip(data, rows)])
    with arplan.Plan(n, ex.Model.SIZE, "f32", "rhd") as p:
        p.execute(rows, torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert all(torch.equal(rows[0], r) for r in rows)

    w = {k: v.double().cpu().requires_grad_() for k, v in model.views(model.vector).items()}
    tokens, teacher, ids, weights = (torch.cat(x).cpu() for x in zip(*data))
    x = torch.where((tokens >= 0)[:, None], w["table"][tokens.clamp(min=0)], 0.0) * math.sqrt(ex.D)
    g = x @ w["wg"].t()
    logits = (g * torch.sigmoid(g) * (x @ w["wu"].t())) @ w["head"].t()
    tau = ex.TEMPERATURE
    lq = torch.log_softmax(logits / tau, 1).gather(1, ids)
    lp = torch.log_softmax(teacher.double() / tau, 1)
    loss = weights.double() * tau * tau * (lp.exp() * (lp - lq)).sum(1)
    loss.sum().backward()
    assert torch.allclose(losses.double().cpu(), loss.detach(), rtol=1e-4, atol=1e-9)
    got = ex.Model.views(rows[0].double().cpu())
    for name in w:
        off = (got[name] - w[name].grad).norm() / w[name].grad.norm()
        # sums of at most 4096 fp32 terms each, four products deep
        assert off < 4 * 4096 * 2.0 ** -24, (name, float(off))


@pytest.mark.parametrize("dtype,plan", [("f32", "rhd"), ("bf16", "ring")])
def test_training_lowers_the_loss(dtype, plan):
    ex = _example()
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    means = ex.train(n=2, steps=6, dtype=dt, plan=plan, say=lambda s: None)
    assert all(math.isfinite(m) for m in means) and means[-1] < 0.9 * means[0]
