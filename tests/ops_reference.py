"""Plain definitions of the replica operators in 64 bits, on the CPU, with
the error each of them allows a 32-bit kernel.

``U`` is the unit roundoff of fp32, ``UB`` that of bf16.  A sum of n fp32
terms is off by at most n U times the sum of their magnitudes whatever its
order; a result stored as bf16 by UB of its magnitude more.
"""

import math

import numpy as np
import torch

U = 2.0 ** -24
UB = 2.0 ** -8     # a significand of 8 bits, as U is 2^-24 for one of 24
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def stored(x, dtype):
    """The error of storing x (half a unit in the last place, and of a
    denormal result)."""
    return x.abs() * (UB if dtype == "bf16" else U) * 1.01 + 1e-38


# ------------------------------------------------------------- embedding

def embed_lookup(table, ids, scale):
    """Bit for bit: the fp32 product, rounded once to the table's type."""
    V = table.shape[0]
    ok = (ids >= 0) & (ids < V)
    rows = table[ids.clamp(0, max(V - 1, 0))] if V else torch.zeros(len(ids), table.shape[1])
    out = rows.float() * np.float32(scale)
    out[~ok] = 0
    return out.to(table.dtype)


def embed_grad(dout, ids, V, scale, run, old=None):
    """Bit for bit: tokens in increasing order, in runs whose sums are then
    added in order, all in fp32."""
    d = dout.float().numpy()
    out = np.zeros((V, d.shape[1]), np.float32) if old is None else old.float().numpy().copy()
    ids = ids.numpy()
    for v in np.unique(ids):
        if v < 0 or v >= V:
            continue
        t = np.flatnonzero(ids == v)
        sums = []
        for i in range(0, len(t), run):
            s = np.zeros(d.shape[1], np.float32)
            for j in t[i:i + run]:
                s = s + d[j]
            sums.append(s)
        s = sums[0]
        if len(sums) > 1:
            s = np.zeros(d.shape[1], np.float32)
            for x in sums:
                s = s + x
        s = s * np.float32(scale)
        out[v] = s if old is None else s + out[v]
    return torch.from_numpy(out).to(dout.dtype)


def embed_grad64(dout, ids, V, scale):
    """The value in 64 bits and the error allowed before storing."""
    d = dout.double()
    out, mag = torch.zeros(V, d.shape[1]).double(), torch.zeros(V, d.shape[1]).double()
    ok = (ids >= 0) & (ids < V)
    out.index_add_(0, ids[ok], d[ok])
    mag.index_add_(0, ids[ok], d[ok].abs())
    n = torch.bincount(ids[ok], minlength=V).double()[:, None]
    return out * scale, mag * abs(scale) * (n + 2) * U


# ------------------------------------------------------ gated feed-forward

def activate(act, g):
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    cdf = 0.5 * torch.special.erfc(-g / math.sqrt(2.0))
    return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def glu(x, wg, wu, act, dh, dtype):
    """[(value, error allowed)] for h, dx, dwg, dwu."""
    x, wg, wu, dh = (t.double() for t in (x, wg, wu, dh))
    M, D = x.shape
    F = wg.shape[0]
    ub = UB if dtype == "bf16" else U
    g, u = x @ wg.t(), x @ wu.t()
    eg = (D + 1) * U * (x.abs() @ wg.abs().t())
    eu = (D + 1) * U * (x.abs() @ wu.abs().t())
    a, da = activate(act, g)
    # the activation in fp32: its own error (its few operations and library
    # calls, of some units each, on values up to 1 + |g|) and its slopes (both
    # activations' first derivatives stay below 1.2, the second below 1)
    ea, eda = 1.2 * eg + 16 * U * (1 + g.abs()), eg + 16 * U * (1 + g.abs())
    h = a * u
    eh = ea * u.abs() + a.abs() * eu + ea * eu
    dg, du = dh * u * da, dh * a
    # the saved factors and their products with dh are stored once each
    edg = dh.abs() * (eda * u.abs() + da.abs() * eu + eda * eu) + 2.1 * ub * dg.abs() + 2 * U * dg.abs()
    edu = dh.abs() * ea + 2.1 * ub * du.abs()
    dx = dg @ wg + du @ wu
    mag = (dg.abs() + edg) @ wg.abs() + (du.abs() + edu) @ wu.abs()
    edx = edg @ wg.abs() + edu @ wu.abs() + (2 * F + 1) * U * mag
    out = [(h, eh + stored(h, dtype)), (dx, edx + stored(dx, dtype))]
    for d, e in ((dg, edg), (du, edu)):
        v = d.t() @ x
        ev = e.t() @ x.abs() + (M + 1) * U * ((d.abs() + e).t() @ x.abs())
        out.append((v, ev + stored(v, dtype)))
    return out


# ----------------------------------------------------------- distillation

def distill(logits, teacher, ids, tau, weights, dtype):
    """(loss, error allowed), (gradient, error allowed)."""
    T, V = logits.shape
    K = teacher.shape[1]
    loss, eloss = torch.zeros(T).double(), torch.zeros(T).double()
    grad, egrad = torch.zeros(T, V).double(), torch.zeros(T, V).double()
    for t in range(T):
        w = 1.0 if weights is None else float(weights[t])
        z = logits[t].double()
        here = [k for k in range(K) if 0 <= int(ids[t, k]) < V
                and float(teacher[t, k]) != -math.inf]
        if w == 0 or not here or bool((z == -math.inf).all()):
            continue
        s = torch.tensor([float(teacher[t, k]) for k in here]).double() / tau
        at = torch.tensor([int(ids[t, k]) for k in here])
        # a largest value of +inf, less itself, is NaN
        lp, lq = s - s.max(), (z - z.max()) / tau
        lp, lq = lp - torch.logsumexp(lp, 0), lq - torch.logsumexp(lq, 0)
        p, q = lp.exp(), lq.exp()
        term = torch.where(p == 0, torch.zeros(()).double(), p * (lp - lq[at]))
        loss[t] = w * tau * tau * term.sum()
        grad[t] = q
        grad[t].index_add_(0, at, -p)
        grad[t] *= w * tau
        # In fp32 a logarithm of a probability is off by a few roundings of
        # its own size and by its sum's relative error: a thread's share of
        # the V terms, the joins and the exponentials' own errors.
        d = U * (math.ceil(V / 1024) + K / 32 + 64)
        big = lambda l: torch.where(l.abs() < 1e30, l.abs(), torch.zeros(()).double())  # noqa: E731
        elp, elq = d + 6 * U * big(lp), d + 6 * U * big(lq)
        eloss[t] = w * tau * tau * (p * (elp * (1 + big(lp) + big(lq[at])) + elq[at])).sum() \
            + (K + 8) * U * w * tau * tau * (p * (big(lp) + big(lq[at]))).sum()
        mag = q.clone().index_add_(0, at, p)
        egrad[t] = w * tau * (q * (elq + 4 * U)).index_add(0, at, p * (elp + (K + 4) * U)) \
            + 4 * U * w * tau * mag + 1e-37
    return (loss, eloss + loss.abs() * 4 * U + 1e-37), (grad, egrad + stored(grad, dtype))


def compare(name, got, want, allowed):
    got = got.double().cpu()
    same = (got == want) | (got.isnan() & want.isnan())
    off = (got - want).abs()
    bad = ~(same | (off <= allowed))
    assert not bool(bad.any()), "%s: %d of %d off, the worst by %.3g where %.3g is allowed" % (
        name, int(bad.sum()), bad.numel(), float(off[bad].max()), float(allowed[bad][off[bad].argmax()]))
