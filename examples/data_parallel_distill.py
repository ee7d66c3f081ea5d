"""Data-parallel distillation steps of a small model on one GPU: n replicas make
their gradients with the replica operators, an AllReduce plan sums them, and
every replica applies the same update.

A replica's model is an embedding, a gated feed-forward block and a linear
head.  Its gradients are written straight into its row of one (n, P) matrix,
the buffers of the plan:

    tokens -> embed_lookup -> glu_forward -> head -> distill (loss, dlogits)
           <- embed_grad   <- glu_backward <- head <-

    python examples/data_parallel_distill.py [--replicas 4] [--steps 8]
        [--dtype f32|bf16] [--plan ring|rhd|cps|rb]
"""

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2409_04202_amd import arplan, ops  # noqa: E402

V, D, F, T, K = 4096, 256, 512, 512, 16     # vocabulary, widths, tokens a replica, teacher entries
TEMPERATURE = 2.0


class Model:
    """Weights as views of one vector, in the order of their gradients."""

    SHAPES = {"table": (V, D), "wg": (F, D), "wu": (F, D), "head": (V, F)}
    SIZE = sum(math.prod(s) for s in SHAPES.values())

    @classmethod
    def views(cls, vector):
        out, at = {}, 0
        for name, shape in cls.SHAPES.items():
            n = math.prod(shape)
            out[name] = vector[at:at + n].view(shape)
            at += n
        return out

    def __init__(self, seed, dtype, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.vector = torch.empty(self.SIZE, dtype=dtype, device=device)
        for name, w in self.views(self.vector).items():
            w.copy_(torch.randn(w.shape, generator=g, device=device) / math.sqrt(w.shape[1]))
        self.__dict__.update(self.views(self.vector))


def gradients(model, tokens, teacher, ids, weights, vector):
    """One replica's step up to its gradients, which go into ``vector``; the
    losses of its tokens."""
    grad = Model.views(vector)
    x = ops.embed_lookup(model.table, tokens, scale=math.sqrt(D))
    h, saved = ops.glu_forward(x, model.wg, model.wu, save=True)
    logits = torch.mm(h, model.head.t())
    # in place: the logits' memory takes their gradient
    loss, dlogits = ops.distill(logits, teacher, ids, temperature=TEMPERATURE, weights=weights,
                                grad=logits)
    torch.mm(dlogits.t(), h, out=grad["head"])
    dh = torch.mm(dlogits, model.head)
    dx, _, _ = ops.glu_backward(dh, x, model.wg, model.wu, saved, dwg=grad["wg"], dwu=grad["wu"])
    ops.embed_grad(dx, tokens, grad["table"], scale=math.sqrt(D))
    return loss


def batch(step, replica, n, device="cuda"):
    """A replica's tokens (the last eighth padding) and its teacher's entries."""
    g = torch.Generator(device=device)
    g.manual_seed(1000 * step + replica)
    tokens = torch.randint(0, V, (T,), generator=g, device=device)
    tokens[T - T // 8:] = -1
    weights = torch.full((T,), 1.0 / (n * (T - T // 8)), device=device)
    weights[T - T // 8:] = 0
    # the teacher's answer depends on the token alone, so that there is something to learn
    ids = (tokens[:, None].clamp(min=0) * 31 + torch.arange(K, device=device) * 257) % V
    teacher = torch.linspace(8, 2, K, device=device).expand(T, K).contiguous()
    return tokens, teacher, ids, weights


def train(n=4, steps=8, dtype=torch.float32, plan="rhd", rate=0.1, say=print):
    """The mean loss of each step."""
    model = Model(7, dtype)
    buffers = torch.zeros(n, Model.SIZE, dtype=dtype, device="cuda")
    name = {torch.float32: "f32", torch.bfloat16: "bf16"}[dtype]
    rows = list(buffers.unbind(0))
    means = []
    with arplan.Plan(n, Model.SIZE, name, plan) as allreduce:
        for step in range(steps):
            losses = [gradients(model, *batch(step, r, n), rows[r]) for r in range(n)]
            allreduce.execute(rows, torch.cuda.current_stream())
            # every row now holds the sum; the replicas' weights are one copy here
            # (a step of a fixed share of the weights' length)
            g = rows[0].float()
            model.vector.sub_((g * (rate * model.vector.float().norm() / g.norm())).to(dtype))
            means.append(float(torch.stack(losses).sum()))
            say("step %d: mean loss %.4f" % (step, means[-1]))
    return means


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--replicas", type=int, default=4)
    p.add_argument("--steps", type=int, default=8)
    p.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    p.add_argument("--plan", choices=("ring", "rhd", "cps", "rb"), default="rhd")
    a = p.parse_args(argv)
    train(a.replicas, a.steps, {"f32": torch.float32, "bf16": torch.bfloat16}[a.dtype], a.plan,
          say=lambda s: print(s, flush=True))


if __name__ == "__main__":
    main()
