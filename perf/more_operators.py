"""More replica operators as cases that can be measured.

Three further parts of what a data-parallel replica computes between two
AllReduces: attention's relative position bias by buckets with its table's
gradient, the routing of tokens to experts with the experts' counts and the
balance loss with its gradient, and activation checkpoints in 8 bits with the
gated feed-forward block's backward pass from them.

A case is one pass.  ``prepare`` makes what a program holds before the call:
inputs, weights, what an earlier forward pass kept, and the vectors that
gradients and counts are written into (a replica's AllReduce buffers).
``run`` is the pass: with ``own`` through ``paper_2409_04202_amd.ops``,
without it in elementary torch operations in 32 bits (long sums and bucket
borders in 64), rounded once at the end.

Widths, lengths and numbers of experts are generic powers of two and odd
neighbours of them.
"""

import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
ESIZE = {"f32": 4, "bf16": 2}
COEFFICIENT = 0.01      # of the balance loss
BLOCK = 32              # elements that share a scale in a checkpoint


def _bias(name, way, dtype, B, H, Q, K, offset, causal, buckets=32, distance=128):
    c = {"op": "bias", "way": way, "dtype": dtype, "B": B, "H": H, "Q": Q, "K": K,
         "offset": offset, "causal": causal, "buckets": buckets, "distance": distance}
    return dict(c, name=name) if name else c


def _route(name, way, dtype, T, E, k, normalize, padded):
    c = {"op": "route", "way": way, "dtype": dtype, "T": T, "E": E, "k": k,
         "normalize": normalize, "padded": padded}
    return dict(c, name=name) if name else c


def _keep(name, dtype, M, N):
    c = {"op": "keep", "way": "keep", "dtype": dtype, "M": M, "N": N}
    return dict(c, name=name) if name else c


def _glu(name, way, dtype, M, D, F, act="silu"):
    c = {"op": "glu", "way": way, "dtype": dtype, "M": M, "D": D, "F": F, "act": act}
    return dict(c, name=name) if name else c


def listed():
    return [
        # Generation: the bias of one new query over the keys so far.
        _bias("bias_token_bf16", "bias", "bf16", 1, 32, 1, 4001, 4000, True),
        # An encoder's layer, made once a step for all sequences.
        _bias("bias_2k_bf16", "bias", "bf16", 1, 16, 2048, 2048, 0, False),
        # Its gradient from the scores' gradients of four sequences, 512 MiB.
        _bias("bias_grad_2k_bf16", "grad", "bf16", 4, 16, 2048, 2048, 0, False),
        # A decoder's second part of a sequence, odd sizes, in f32.
        _bias("bias_grad_odd_f32", "grad", "f32", 3, 5, 509, 1021, 512, True, 48, 300),
        # Generation, eight sequences a step: the router's latency.
        _route("route_8_bf16", "route", "bf16", 8, 64, 2, True, 0),
        # Training on a microbatch: routing, then loss and gradient.
        _route("route_step_16k_bf16", "step", "bf16", 16384, 128, 8, True, 1024),
        # A small replica with odd sizes in f32, a quarter padding.
        _route("route_step_odd_f32", "step", "f32", 5003, 61, 4, False, 1250),
        # Many tokens to many small experts.
        _route("route_step_64k_bf16", "step", "bf16", 65536, 512, 8, False, 0),
        # A small activation with odd sizes, kept and fetched again.
        _keep("keep_odd_f32", "f32", 1021, 1001),
        # A block's inner activation of a microbatch, kept and fetched again.
        _keep("keep_8k_bf16", "bf16", 8192, 16384),
        # A small replica's backward pass from 8 bits, no size a multiple of a tile.
        _glu("glu_back_odd_f32", "back", "f32", 777, 1003, 2731, "gelu"),
        # The largest: a training step of 8K tokens with everything kept in 8 bits.
        _glu("glu_step_8k_bf16", "step", "bf16", 8192, 4096, 16384),
    ]


_FLOPS = 2 * 10 ** 12       # a drawn matrix case at most (the largest listed one takes 6.6e12)
_BYTES = 6 * 10 ** 8        # a drawn memory case at most


def draw(rng):
    """One more case over the range of the listed ones: single rows to many,
    powers of two, multiples of eight and odd sizes, every way and type."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def size(lo, hi):
        v = log(lo, hi)
        kind = rng.choice(("round", "eight", "any"))
        if kind == "round":
            return 1 << max(0, int(round(math.log2(v))))
        return -(-v // 8) * 8 if kind == "eight" else v

    dtype = rng.choice(("f32", "bf16", "bf16"))
    op = rng.choice(("bias", "route", "keep", "glu"))
    if op == "bias":
        way = rng.choice(("bias", "grad", "grad"))
        causal = rng.random() < 0.5
        K = size(16, 8192)
        Q = rng.choice((1, K, size(1, 4096)))
        offset = max(0, K - Q) if causal else rng.choice((0, max(0, K - Q)))
        B, H = (1 if way == "bias" else rng.randint(1, 8)), rng.randint(1, 32)
        while B * H * Q * K * ESIZE[dtype] > _BYTES:
            B, H = (B + 1) // 2, H // 2 + 1 if B == 1 else H
            Q = Q // 2 + 1 if H <= 2 else Q
        return _bias("", way, dtype, B, H, Q, K, offset, causal, 4 * rng.randint(4, 32),
                     rng.choice((128, 256, log(100, 4000))))
    if op == "route":
        way = rng.choice(("route", "step", "step"))
        T, E = max(1, size(1, 65536)), max(4, size(4, 1024))
        while T * E * ESIZE[dtype] > _BYTES // 4:
            T = T // 2 + 1
        return _route("", way, dtype, T, E, rng.randint(1, min(E, 16)), rng.random() < 0.5,
                      rng.choice((0, 0, T // 8, T // 3)))
    if op == "keep":
        M, N = max(1, size(1, 16384)), max(1, size(16, 16384))
        while M * N * ESIZE[dtype] > _BYTES // 2:
            M = M // 2 + 1
        return _keep("", dtype, M, N)
    M, D, F = max(1, size(1, 8192)), size(64, 4096), size(128, 16384)
    while 12 * M * D * F > _FLOPS // (8 if dtype == "f32" else 1):
        M = M // 2 + 1
    way = "back" if dtype == "f32" else rng.choice(("back", "step"))
    return _glu("", way, dtype, M, D, F, rng.choice(("silu", "gelu")))


# ---------------------------------------------------------------- inputs

class State:
    pass


def _pitch(width):
    """Bytes of a checkpoint's row: codes in whole blocks, a scale a block, and
    room up to 16 bytes."""
    blocks = -(-width // BLOCK)
    return -(-blocks * (BLOCK + 1) // 16) * 16


def _block_scales(x):
    """x (M, N) in 32 bits as blocks (M, blocks, 32), zeros behind a row, and
    each block's exponent: the least for which no code leaves [-127, 127]."""
    M, N = x.shape
    blocks = -(-N // BLOCK)
    y = torch.zeros(M, blocks * BLOCK, dtype=torch.float32, device=x.device)
    y[:, :N] = x
    y = y.view(M, blocks, BLOCK)
    top = y.abs().amax(2)
    significand, exponent = torch.frexp(top)
    e = torch.where(significand * 128 < 127.5, exponent - 7, exponent - 6)
    e = torch.where(top == 0, torch.full_like(e, -126), e).clamp_(-126, 121)
    return y, e, torch.isfinite(top)


def _power(e):
    """2^e in 32 bits, exactly."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _codes(x):
    """(codes, exponents, whether a block is finite) of x (M, N)."""
    y, e, fine = _block_scales(x)
    codes = torch.round(y * _power(-e)[:, :, None]).clamp_(-127, 127)
    return torch.where(fine[:, :, None], codes, torch.zeros((), device=x.device)), e, fine


def _values(x):
    """What a checkpoint of x (M, N) stands for, in 32 bits."""
    codes, e, fine = _codes(x)
    v = codes * _power(e)[:, :, None]
    v = torch.where(fine[:, :, None], v, torch.full((), math.nan, device=x.device))
    return v.flatten(1)[:, :x.shape[1]]


def _rows_kept(x):
    """A checkpoint of x (M, N), as an earlier forward pass left it."""
    M, N = x.shape
    codes, e, fine = _codes(x)
    blocks = e.shape[1]
    kept = torch.zeros(M, _pitch(N), dtype=torch.uint8, device=x.device)
    kept[:, :blocks * BLOCK] = codes.flatten(1).to(torch.int8).view(torch.uint8)
    kept[:, blocks * BLOCK:blocks * (BLOCK + 1)] = torch.where(
        fine, e + 127, torch.full_like(e, 255)).to(torch.uint8)
    return kept


def _read_kept(kept, N):
    """The values that a checkpoint's rows stand for, in 32 bits."""
    blocks = -(-N // BLOCK)
    codes = kept[:, :blocks * BLOCK].view(torch.int8).float().view(-1, blocks, BLOCK)
    s = kept[:, blocks * BLOCK:blocks * (BLOCK + 1)].to(torch.int32)
    scale = torch.where(s == 255, torch.full((), math.nan, device=kept.device), _power(s - 127))
    return (codes * scale[:, :, None]).flatten(1)[:, :N]


def prepare(case, seed):
    s = State()
    s.case = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = TORCH[case["dtype"]]

    def normal(*shape, scale=1.0):
        out = torch.empty(shape, dtype=dt, device="cuda")
        step = max(1, (1 << 28) // max(1, out[0].numel()))
        for i in range(0, shape[0], step):      # no second copy of everything
            n = min(step, shape[0] - i)
            out[i:i + n] = torch.randn((n,) + shape[1:], generator=g, device="cuda") * scale
        return out

    if case["op"] == "bias":
        B, H, Q, K = case["B"], case["H"], case["Q"], case["K"]
        if case["way"] == "bias":
            s.table = normal(case["buckets"], H)
        else:
            s.dscores = normal(B, H, Q, K, scale=1e-2)
            if case["causal"]:      # softmax leaves no gradient at keys it does not see
                i = torch.arange(Q, device="cuda")[:, None] + case["offset"]
                s.dscores.mul_(torch.arange(K, device="cuda")[None, :] <= i)
            s.dtable = torch.empty(case["buckets"], H, dtype=dt, device="cuda")
    elif case["op"] == "route":
        T, E, k = case["T"], case["E"], case["k"]
        # some experts are liked more than others, which is what the loss is against
        s.logits = (torch.randn(T, E, generator=g, device="cuda") * 1.5
                    + torch.randn(E, generator=g, device="cuda")).to(dt)
        s.live = torch.ones(T, dtype=torch.bool, device="cuda")
        s.live[torch.randperm(T, generator=g, device="cuda")[:case["padded"]]] = False
        s.counts = torch.empty(E + 1, dtype=torch.int32, device="cuda")
        s.mass = torch.empty(E, device="cuda")
        if case["way"] == "step":
            s.dgates = torch.randn(T, k, generator=g, device="cuda") * (0.1 / T)
            s.grad = torch.empty(T, E, dtype=dt, device="cuda")
    elif case["op"] == "keep":
        s.x = normal(case["M"], case["N"])
        # activations have columns that are larger than the others
        s.x.mul_(torch.exp(torch.randn(case["N"], generator=g, device="cuda")).to(dt))
    else:
        M, D, F = case["M"], case["D"], case["F"]
        s.wg = normal(F, D, scale=1 / math.sqrt(D))
        s.wu = normal(F, D, scale=1 / math.sqrt(D))
        s.dh = normal(M, F, scale=1e-2)
        s.dwg, s.dwu = torch.empty(2 * F * D, dtype=dt, device="cuda").view(2, F, D).unbind(0)
        x = normal(M, D)
        if case["way"] == "step":
            s.x = x
        else:
            gate = torch.randn(M, F, generator=g, device="cuda")
            up = torch.randn(M, F, generator=g, device="cuda")
            a, da = _act(case["act"], gate)
            s.saved = torch.stack([_rows_kept(da * up), _rows_kept(a)])
            s.kept = _rows_kept(x.float())
    return s


# ------------------------------------------------------------------- run

def _buckets(c):
    """The bucket of each distance j - (offset + i), from -(Q - 1) - offset up,
    and whether a causal bias leaves it visible."""
    d = torch.arange(c["Q"] + c["K"] - 1, device="cuda") - (c["Q"] - 1) - c["offset"]
    a_side = c["buckets"] if c["causal"] else c["buckets"] // 2
    exact_ones = a_side // 2
    n = (-d).clamp(min=0) if c["causal"] else d.abs()
    # far ones in 64 bits; a distance on a border belongs to the bucket above it
    far = torch.floor(torch.log(n.clamp(min=1).double() / exact_ones) * (a_side - exact_ones)
                      / math.log(c["distance"] / exact_ones) + 1e-9).long() + exact_ones
    b = torch.where(n < exact_ones, n, far.clamp(max=a_side - 1))
    return (b, d <= 0) if c["causal"] else (b + a_side * (d > 0), d == d)


def _plain_bias(s):
    c = s.case
    Q, K, H = c["Q"], c["K"], c["H"]
    b, seen = _buckets(c)
    if c["way"] == "bias":
        row = torch.where(seen[:, None], s.table.float()[b],
                          torch.full((), -math.inf, device="cuda")).t()
        at = (torch.arange(K, device="cuda")[None, :] + (Q - 1)
              - torch.arange(Q, device="cuda")[:, None])
        return row[:, at].to(s.table.dtype)
    # rows from the last to the first, each one element wider than the one above, so that
    # a diagonal becomes a column
    x = torch.zeros(H, Q, K + Q, dtype=torch.float64, device="cuda")
    x[:, :, :K] = s.dscores.double().sum(0).flip(1)
    columns = x.flatten(1)[:, :Q * (K + Q - 1)].view(H, Q, K + Q - 1).sum(1)
    d = torch.zeros(c["buckets"], H, dtype=torch.float64, device="cuda")
    d.index_add_(0, b, (columns * seen).t().contiguous())
    return d.to(s.dscores.dtype)


def _plain_route(s):
    c = s.case
    T, E, k = c["T"], c["E"], c["k"]
    z = s.logits.float()
    live = s.live[:, None]
    e = torch.exp(z - z.max(1, keepdim=True).values)
    p = torch.where(live, e / e.sum(1, keepdim=True), torch.zeros((), device="cuda"))
    # a stable sort: of equal logits the lowest index
    ids = z.sort(dim=1, descending=True, stable=True).indices[:, :k]
    chosen = p.gather(1, ids)
    gates = chosen / chosen.sum(1, keepdim=True).clamp(min=1e-30) if c["normalize"] else chosen
    counts = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    counts.index_add_(0, ids.flatten(), live.expand(T, k).flatten().int())
    counts[E] = s.live.sum()
    mass = p.double().sum(0)
    ids = torch.where(live, ids, torch.full((), -1, device="cuda"))
    if c["way"] == "route":
        return ids, gates, counts, mass.float()
    rate = counts[:E].double() * (COEFFICIENT * E / k) / counts[E].double().square()
    loss = (rate * mass).sum().float()
    rate = rate.float()[None, :]
    grad = p * (rate - (p * rate).sum(1, keepdim=True))
    w = s.dgates * gates
    part = w - gates * w.sum(1, keepdim=True) if c["normalize"] else w
    grad.scatter_add_(1, ids.clamp(min=0), part)
    if not c["normalize"]:
        grad -= p * w.sum(1, keepdim=True)
    return ids, gates, counts, mass.float(), loss, grad.to(s.logits.dtype)


def _act(name, g):
    """The activation and its derivative."""
    if name == "silu":
        e = 1 / (1 + torch.exp(-g))
        return g * e, e * (1 + g * (1 - e))
    phi = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def _plain_glu(s):
    c, dt = s.case, s.wg.dtype
    wg, wu = s.wg.float(), s.wu.float()
    if c["way"] == "step":
        x = s.x.float()
        g, u = x @ wg.t(), x @ wu.t()
        a, da = _act(c["act"], g)
        h = (a * u).to(dt)
        to_gate, to_up, x = _values(da * u), _values(a), _values(x)
    else:
        h = None
        to_gate, to_up = _read_kept(s.saved[0], c["F"]), _read_kept(s.saved[1], c["F"])
        x = _read_kept(s.kept, c["D"])
    dh = s.dh.float()
    dg, du = dh * to_gate, dh * to_up
    dx = dg @ wg + du @ wu
    grads = dx.to(dt), (dg.t() @ x).to(dt), (du.t() @ x).to(dt)
    return grads if h is None else (h,) + grads


def run(s):
    c = s.case
    op, way = c["op"], c["way"]
    if not own:
        if op == "keep":
            return _values(s.x.float()).to(s.x.dtype)
        return {"bias": _plain_bias, "route": _plain_route, "glu": _plain_glu}[op](s)
    from paper_2409_04202_amd import ops
    if op == "bias":
        where = {"max_distance": c["distance"], "offset": c["offset"], "causal": c["causal"]}
        if way == "bias":
            return ops.position_bias(s.table, c["Q"], c["K"], **where)
        return ops.position_bias_grad(s.dscores, s.dtable, **where)
    if op == "route":
        out = ops.route(s.logits, c["k"], live=s.live, normalize=c["normalize"], counts=s.counts,
                        mass=s.mass)
        if way == "route":
            return out
        loss, grad = ops.balance(s.logits, out[0], s.counts, s.mass, coefficient=COEFFICIENT,
                                 normalize=c["normalize"], dgates=s.dgates, grad=s.grad)
        return out + (loss, grad)
    if op == "keep":
        return ops.checkpoint_load(ops.checkpoint_store(s.x), c["N"], s.x.dtype)
    if way == "back":
        x = ops.checkpoint_load(s.kept, c["D"], s.wg.dtype)
        return ops.glu_backward(s.dh, x, s.wg, s.wu, s.saved, dwg=s.dwg, dwu=s.dwu)
    kept = ops.checkpoint_store(s.x)
    h, saved = ops.glu_forward(s.x, s.wg, s.wu, act=c["act"], save=torch.uint8)
    x = ops.checkpoint_load(kept, c["D"], s.x.dtype)
    return (h,) + ops.glu_backward(s.dh, x, s.wg, s.wu, saved, dwg=s.dwg, dwu=s.dwu)


# ------------------------------------------------------------------ work

def work(case):
    """Inputs read once, outputs written once; the operations of the products
    (an element-wise operator: a few operations an element)."""
    c, e = case, ESIZE[case["dtype"]]
    if c["op"] == "bias":
        B, H, Q, K = c["B"], c["H"], c["Q"], c["K"]
        seen = Q * K
        if c["causal"] and c["way"] == "grad":
            seen = sum(min(K, max(0, c["offset"] + i + 1)) for i in range(Q))
        return {"bytes": (B * H * seen + c["buckets"] * H) * e, "flops": B * H * seen}
    if c["op"] == "route":
        T, E, k = c["T"], c["E"], c["k"]
        b = T * E * e + T + T * k * 12 + 8 * E + 4
        if c["way"] == "step":
            b += T * E * e + T * k * 4 + 4
        return {"bytes": b, "flops": (4 if c["way"] == "route" else 8) * T * E}
    if c["op"] == "keep":
        M, N = c["M"], c["N"]
        return {"bytes": 2 * M * N * e + 2 * M * -(-N // BLOCK) * (BLOCK + 1), "flops": 4 * M * N}
    M, D, F = c["M"], c["D"], c["F"]
    kept = M * (-(-D // BLOCK) + 2 * -(-F // BLOCK)) * (BLOCK + 1)
    if c["way"] == "back":
        return {"bytes": (M * D + M * F + 4 * F * D) * e + kept, "flops": 8 * M * D * F}
    return {"bytes": (2 * M * D + 2 * M * F + 4 * F * D) * e + 2 * kept, "flops": 12 * M * D * F}


# ----------------------------------------------------------------- exact

def _border(m, ones, a_side, distance):
    """The least distance of far bucket m, by whole numbers."""
    q = a_side - ones
    goal = ones ** (q - m) * distance ** m
    low, high = 0, distance
    while high - low > 1:
        mid = (low + high) // 2
        low, high = (low, mid) if mid ** q >= goal else (mid, high)
    return high


def _exact_bias(s):
    c, f64 = s.case, torch.float64
    Q, K, H = c["Q"], c["K"], c["H"]
    a_side = c["buckets"] if c["causal"] else c["buckets"] // 2
    ones = a_side // 2
    borders = list(range(1, ones + 1)) + [_border(m, ones, a_side, c["distance"])
                                          for m in range(1, a_side - ones)]
    borders = torch.tensor(borders, device="cuda")
    i = torch.arange(Q, device="cuda")[:, None] + c["offset"]
    j = torch.arange(K, device="cuda")[None, :]
    b = torch.bucketize((i - j).abs(), borders, right=True)
    if not c["causal"]:
        b = b + a_side * (j > i)
    hidden = (j > i) if c["causal"] else torch.zeros_like(b, dtype=torch.bool)
    if c["way"] == "bias":
        t = s.table.to(f64)
        return torch.stack([t[:, h][b].masked_fill(hidden, -math.inf) for h in range(H)])
    out = torch.zeros(c["buckets"], H, dtype=f64, device="cuda")
    flat = b.masked_fill(hidden, -1).flatten()
    for at in range(0, Q * K, 1 << 20):
        part = flat[at:at + (1 << 20)]
        which = (part[:, None] == torch.arange(c["buckets"], device="cuda")).to(f64)
        for n in range(c["B"]):
            d = s.dscores[n].reshape(H, Q * K)[:, at:at + (1 << 20)].to(f64)
            out += torch.mm(d, which).T
    return out


def _exact_route(s):
    c, f64 = s.case, torch.float64
    E, k = c["E"], c["k"]
    z = s.logits.to(f64)
    p = torch.softmax(z, 1) * s.live[:, None]
    # rank: how many logits are larger, or equal at a lower index
    ids = torch.argsort(-z, dim=1, stable=True)[:, :k]
    sel = p.gather(1, ids)
    total = sel.sum(1, keepdim=True)
    gates = sel / total.masked_fill(total == 0, 1) if c["normalize"] else sel
    kept = ids[s.live]
    counts = torch.cat([torch.bincount(kept.flatten(), minlength=E),
                        torch.tensor([kept.shape[0]], device="cuda")]).int()
    out = (ids.masked_fill(~s.live[:, None], -1), gates, counts, p.sum(0))
    if c["way"] == "route":
        return out
    N = kept.shape[0]
    slope = COEFFICIENT * E * counts[:E].to(f64) / (k * N * N)
    at_p = slope.expand_as(p).clone()
    G = s.dgates.to(f64)
    if c["normalize"]:
        # gate j = p_j / sum: its slope at the chosen probabilities
        inner = (G * gates).sum(1, keepdim=True)
        G = (G - inner) / total.masked_fill(total == 0, 1)
    at_p.scatter_add_(1, ids, G)
    grad = p * (at_p - (p * at_p).sum(1, keepdim=True))
    return out + ((slope * p.sum(0)).sum(), grad)


def _unit(e):
    """2^e in 64 bits, from Python's powers of two."""
    e = e.clamp(-1000, 1000).long()
    return torch.tensor([2.0 ** i for i in range(-1000, 1001)], dtype=torch.float64,
                        device=e.device)[e + 1000]


def _exact_values(x):
    """The same values as a checkpoint's, from 64 bits."""
    M, N = x.shape
    out = torch.empty_like(x)
    for at in range(0, N, BLOCK * 64):
        part = x[:, at:at + BLOCK * 64]
        w = part.shape[1]
        blocks = torch.nn.functional.pad(part, (0, -w % BLOCK)).view(M, -1, BLOCK)
        top = blocks.abs().amax(2, keepdim=True)
        e = torch.frexp(top).exponent - 7
        unit = _unit(e)
        e = torch.where(torch.round(top / unit) > 127, e + 1, e)
        e = e.masked_fill(top == 0, -126).clamp(-126, 121)
        unit = _unit(e)
        out[:, at:at + w] = (torch.round(blocks / unit).clamp(-127, 127) * unit).flatten(1)[:, :w]
    return out


def exact(case, seed):
    """The same outputs from the definitions, in 64 bits."""
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "bias":
        return _exact_bias(s)
    if case["op"] == "route":
        return _exact_route(s)
    if case["op"] == "keep":
        return _exact_values(s.x.to(f64))
    wg, wu, dh = s.wg.to(f64), s.wu.to(f64), s.dh.to(f64)
    h = ()
    if case["way"] == "step":
        x = s.x.to(f64)
        gate, up = torch.mm(x, wg.T.contiguous()), torch.mm(x, wu.T.contiguous())
        if case["act"] == "silu":
            sig = torch.sigmoid(gate)
            value, slope = gate * sig, sig + gate * sig * (1 - sig)
        else:
            cdf = torch.special.ndtr(gate)
            value = gate * cdf
            slope = cdf + gate * torch.exp(-gate.square() / 2) / math.sqrt(2 * math.pi)
        h = (value * up,)
        to_gate, to_up, x = _exact_values(slope * up), _exact_values(value), _exact_values(x)
    else:
        def values(kept, width):
            blocks = -(-width // BLOCK)
            unit = _unit(kept[:, BLOCK * blocks:(BLOCK + 1) * blocks].int() - 127)
            codes = kept[:, :BLOCK * blocks].contiguous().view(torch.int8).to(f64)
            return (codes * unit.repeat_interleave(BLOCK, 1))[:, :width]

        to_gate, to_up = values(s.saved[0], case["F"]), values(s.saved[1], case["F"])
        x = values(s.kept, case["D"])
    dgate, dup = dh * to_gate, dh * to_up
    return h + (torch.mm(dgate, wg) + torch.mm(dup, wu), torch.mm(dgate.T.contiguous(), x),
                torch.mm(dup.T.contiguous(), x))
