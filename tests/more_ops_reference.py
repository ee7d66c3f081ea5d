"""Plain definitions, on the CPU in 64 bits or whole numbers, of the position
bias, the routing with its balance loss, and activations kept in 8 bits."""

import math

import numpy as np
import torch

U = 2.0 ** -24
UB = 2.0 ** -8
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


# --------------------------------------------------------- position bias

def bucket(n, side, most):
    """The bucket of distance n >= 0 of a side, by whole numbers."""
    ones = side // 2
    if n < ones:
        return n
    q, b = side - ones, ones
    while b + 1 < side and n ** q >= ones ** (q - (b + 1 - ones)) * most ** (b + 1 - ones):
        b += 1
    return b


def buckets(Q, K, offset, count, most, causal):
    """(Q, K) buckets, -1 at later keys of a causal bias."""
    side = count if causal else count // 2
    near = {}

    def one(n):
        if n < 0 and causal:
            return -1
        d = min(abs(n), most)
        if d not in near:
            near[d] = bucket(d, side, most)
        return near[d] + (side if n < 0 else 0)
    line = [one(offset + Q - 1 - g) for g in range(Q + K - 1)]
    at = torch.arange(K)[None, :] + (Q - 1) - torch.arange(Q)[:, None]
    return torch.tensor(line)[at]


def position_bias(table, Q, K, offset, most, causal):
    b = buckets(Q, K, offset, table.shape[0], most, causal)
    out = table[b.clamp(min=0)].permute(2, 0, 1).clone()
    out[:, b < 0] = -math.inf
    return out


def position_bias_grad(d, count, offset, most, causal):
    """(gradient, sum of magnitudes) in 64 bits, for d (B, H, Q, K)."""
    B, H, Q, K = d.shape
    b = buckets(Q, K, offset, count, most, causal).flatten()
    seen = b >= 0
    flat = d.double().permute(2, 3, 0, 1).reshape(Q * K, B, H)[seen]
    out, size = torch.zeros(count, H).double(), torch.zeros(count, H).double()
    out.index_add_(0, b[seen], flat.sum(1))
    size.index_add_(0, b[seen], flat.abs().sum(1))
    return out, size


# --------------------------------------------------------------- routing

def route(logits, k, live=None, normalize=False):
    """(ids, gates, counts, mass) of rows without NaN and +inf, in 64 bits."""
    T, E = logits.shape
    z = logits.double().numpy()
    ids, gates = np.full((T, k), -1, np.int64), np.zeros((T, k))
    counts, mass = np.zeros(E + 1, np.int64), np.zeros(E)
    order = np.argsort(-z, axis=1, kind="stable")[:, :k]    # (of equal ones the lower first)
    for t in range(T):
        if (live is not None and not live[t]) or np.all(np.isneginf(z[t])):
            continue
        p = np.exp(z[t] - z[t].max())
        p /= p.sum()
        at = order[t][z[t, order[t]] > -np.inf]
        ids[t, :len(at)] = at
        gates[t, :len(at)] = p[at] / (p[at].sum() if normalize else 1)
        counts[at] += 1
        counts[E] += 1
        mass += p
    return tuple(torch.from_numpy(x) for x in (ids, gates, counts, mass))


def balance(logits, ids, counts, mass, coefficient, normalize=False, dgates=None):
    """(loss, gradient, the magnitude that the gradient's error is relative to)."""
    T, E = logits.shape
    k = ids.shape[1]
    N = float(counts[E])
    c = coefficient * E * counts[:E].double() / (k * N * N) if N > 0 else torch.zeros(E).double()
    loss = float((c * mass.double()).sum())
    grad, size = torch.zeros(T, E).double(), torch.zeros(T, E).double()
    for t in range(T):
        if ids[t, 0] < 0:
            continue
        p = torch.softmax(logits[t].double(), 0)
        a = c.clone()
        there = [j for j in range(k) if 0 <= ids[t, j] < E]
        if dgates is not None and not normalize:
            for j in there:
                a[ids[t, j]] += dgates[t, j].double()
        grad[t] = p * (a - (p * a).sum())
        size[t] = p * (a.abs() + (p * a.abs()).sum())
        if dgates is not None and normalize:
            at = ids[t, there]
            w = p[at] / p[at].sum()
            g = dgates[t, there].double()
            dot, most = (w * g).sum(), (w * g.abs()).sum()
            for j, e in enumerate(at.tolist()):
                grad[t, e] += w[j] * (g[j] - dot)
                size[t, e] += w[j] * (g[j].abs() + most)
    return loss, grad, size


# ------------------------------------------------- activations in 8 bits

def kept(x):
    """(numbers (M, runs, 32) int8, bytes (M, runs)) of x, by Python's powers of
    two and numpy's rounding to even."""
    M, N = x.shape
    runs = -(-N // 32)
    y = np.zeros((M, runs * 32))
    y[:, :N] = x.double().numpy()
    y = y.reshape(M, runs, 32)
    numbers, byte = np.zeros((M, runs, 32), np.int8), np.zeros((M, runs), np.uint8)
    for m in range(M):
        for r in range(runs):
            v = y[m, r]
            if not np.all(np.isfinite(v)):
                byte[m, r] = 255
                continue
            top = np.abs(v).max()
            e = max(-126, math.frexp(top)[1] - 8) if top else -126
            while e < 121 and np.abs(np.rint(v * 2.0 ** -e)).max() > 127:
                e += 1
            numbers[m, r] = np.clip(np.rint(v * 2.0 ** -e), -127, 127)
            byte[m, r] = e + 127
    return numbers, byte


def fetched(numbers, byte, N):
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return torch.from_numpy((numbers * scale[:, :, None]).reshape(len(byte), -1)[:, :N])
