"""The replica operators as cases that can be measured.

Between two AllReduces a data-parallel replica turns tokens into gradients.
Three operators of that step are measured here: the embedding lookup and its
gradient, the gated feed-forward block with its backward pass, and the
distillation loss from a teacher's top logits with its gradient.

A case is one pass through one operator.  ``prepare`` makes what a program
holds before the call: inputs, weights and, where a pass leaves weight
gradients, the vector they are written into (a replica's AllReduce buffer).
``run`` is the pass: with ``own`` through ``paper_2409_04202_amd.ops``,
without it in elementary torch operations in 32 bits, rounded once at the end.

Widths and vocabularies are generic powers of two and odd neighbours of them.
"""

import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
ESIZE = {"f32": 4, "bf16": 2}


def _embed(name, way, dtype, T, V, D):
    c = {"op": "embed", "way": way, "dtype": dtype, "T": T, "V": V, "D": D}
    return dict(c, name=name) if name else c


def _glu(name, way, dtype, M, D, F, act="silu"):
    c = {"op": "glu", "way": way, "dtype": dtype, "M": M, "D": D, "F": F, "act": act}
    return dict(c, name=name) if name else c


def _distill(name, way, dtype, T, V, K, tau, masked):
    c = {"op": "distill", "way": way, "dtype": dtype, "T": T, "V": V, "K": K, "tau": tau,
         "masked": masked}
    return dict(c, name=name) if name else c


def listed():
    return [
        # Generation, eight sequences a step: latency of a small lookup.
        _embed("lookup_8_f32", "lookup", "f32", 8, 32768, 1024),
        # A replica's microbatch of 16K tokens from a large vocabulary.
        _embed("lookup_16k_bf16", "lookup", "bf16", 16384, 131072, 4096),
        # Its dense gradient, the part of the AllReduce vector that the table
        # takes; token frequencies fall as 1/rank, so a few rows get very many.
        _embed("embed_grad_16k_bf16", "grad", "bf16", 16384, 131072, 4096),
        # A small replica with odd sizes in f32.
        _embed("embed_grad_odd_f32", "grad", "f32", 5003, 32003, 1001),
        # Evaluation of a few positions against the teacher: few long rows.
        _distill("distill_loss_8_bf16", "loss", "bf16", 8, 131072, 32, 1.0, 0),
        # Evaluation over a validation batch, odd vocabulary, f32.
        _distill("distill_loss_odd_f32", "loss", "f32", 1021, 32003, 10, 1.0, 0),
        # Training on one sequence in f32, the prompt's positions masked.
        _distill("distill_step_odd_f32", "step", "f32", 509, 50021, 20, 2.0, 128),
        # Training on a microbatch: 1 GiB of logits and as much gradient.
        _distill("distill_step_4k_bf16", "step", "bf16", 4096, 131072, 64, 2.0, 512),
        # Generation with one sequence: one row against both weights.
        _glu("glu_infer_1_bf16", "infer", "bf16", 1, 4096, 16384),
        # A prompt, or evaluation of a batch: forward only.
        _glu("glu_infer_2k_bf16", "infer", "bf16", 2048, 4096, 16384),
        # A small replica's training step in f32, no size a multiple of a tile.
        _glu("glu_train_odd_f32", "train", "f32", 777, 1003, 2731, "gelu"),
        # The largest: a microbatch of 8K tokens, forward and backward.
        _glu("glu_train_8k_bf16", "train", "bf16", 8192, 4096, 16384),
    ]


_FLOPS = 2 * 10 ** 12       # a drawn matrix case at most (the largest listed one takes 6.6e12)
_BYTES = 2 * 10 ** 9        # a drawn memory case at most


def draw(rng):
    """One more case over the range of the listed ones: one row to many, powers
    of two, multiples of eight and odd sizes, every way and type."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def size(lo, hi):
        v = log(lo, hi)
        kind = rng.choice(("round", "eight", "any"))
        if kind == "round":
            return 1 << max(0, int(round(math.log2(v))))
        return -(-v // 8) * 8 if kind == "eight" else v

    dtype = rng.choice(("f32", "bf16", "bf16"))
    op = rng.choice(("embed", "glu", "distill"))
    if op == "embed":
        way = rng.choice(("lookup", "grad"))
        V, D = size(1000, 131072), size(64, 4096)
        while V * D * ESIZE[dtype] > _BYTES // 2:
            V = V // 2 + 1
        return _embed("", way, dtype, max(1, size(1, 16384)), V, D)
    if op == "glu":
        way = rng.choice(("infer", "train", "train"))
        M, D, F = max(1, size(1, 8192)), size(64, 4096), size(128, 16384)
        while 12 * M * D * F > _FLOPS // (8 if dtype == "f32" else 1):
            M = M // 2 + 1
        return _glu("", way, dtype, M, D, F, rng.choice(("silu", "gelu")))
    way = rng.choice(("loss", "step", "step"))
    T, V = size(1, 4096), size(1000, 131072)
    while T * V * ESIZE[dtype] > _BYTES // 2:
        T = T // 2 + 1
    return _distill("", way, dtype, T, V, size(1, 128), rng.choice((1.0, 2.0, 4.0)),
                    rng.choice((0, T // 8, T // 3)))


# ---------------------------------------------------------------- inputs

class State:
    pass


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _tokens(g, T, V):
    """Token ids with frequencies that fall as 1/rank; one position in 32 is
    padding (-1), except in very short lists."""
    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(V)).long() - 1).clamp_(0, V - 1)
    ids = (rank * 7919) % V     # ranks spread over the table
    if T >= 32:
        ids[torch.rand(T, generator=g, device="cuda") < 1 / 32] = -1
    return ids


def prepare(case, seed):
    s = State()
    s.case = case
    g = _generator(seed)
    dt = TORCH[case["dtype"]]

    def normal(*shape, scale=1.0):
        out = torch.empty(shape, dtype=dt, device="cuda")
        step = max(1, (1 << 28) // max(1, out[0].numel()))
        for i in range(0, shape[0], step):      # no second copy of everything
            n = min(step, shape[0] - i)
            out[i:i + n] = torch.randn((n,) + shape[1:], generator=g, device="cuda") * scale
        return out

    if case["op"] == "embed":
        T, V, D = case["T"], case["V"], case["D"]
        s.ids = _tokens(g, T, V)
        s.scale = float(torch.tensor(math.sqrt(D), dtype=torch.float32))
        if case["way"] == "lookup":
            s.table = normal(V, D, scale=1 / math.sqrt(D))
        else:
            s.dout = normal(T, D, scale=1e-3)
            s.dtable = torch.empty(V, D, dtype=dt, device="cuda")
    elif case["op"] == "glu":
        M, D, F = case["M"], case["D"], case["F"]
        s.x = normal(M, D)
        s.wg = normal(F, D, scale=1 / math.sqrt(D))
        s.wu = normal(F, D, scale=1 / math.sqrt(D))
        if case["way"] == "train":
            s.dh = normal(M, F, scale=1e-2)
            vector = torch.empty(2 * F * D, dtype=dt, device="cuda")
            s.dwg, s.dwu = vector.view(2, F, D).unbind(0)
    else:
        T, V, K = case["T"], case["V"], case["K"]
        s.tau = case["tau"]
        # K distinct ids a row, in the order of the teacher's logits; up to
        # half of a row's entries are absent
        gaps = torch.randint(1, max(2, V // K + 1), (T, K), generator=g, device="cuda")
        ids = gaps.cumsum(1) - 1
        order = torch.rand(T, K, generator=g, device="cuda").argsort(1)
        s.ids = ids.gather(1, order)
        s.teacher = (torch.randn(T, K, generator=g, device="cuda") * 2 + 8).sort(
            1, descending=True).values.to(dt)
        present = torch.randint((K + 1) // 2, K + 1, (T, 1), generator=g, device="cuda")
        s.ids[torch.arange(K, device="cuda")[None, :] >= present] = -1
        s.logits = normal(T, V, scale=2.0)
        # the student has learnt something: its logits rise where the teacher's are high
        row, k = torch.nonzero(s.ids >= 0, as_tuple=True)
        s.logits[row, s.ids[row, k]] = (s.teacher[row, k].float() * 0.75).to(dt)
        s.weights = torch.full((T,), 1.0 / max(1, T - case["masked"]), device="cuda")
        s.weights[torch.randperm(T, generator=g, device="cuda")[:case["masked"]]] = 0
        if case["way"] == "step":
            s.grad = torch.empty(T, V, dtype=dt, device="cuda")
    return s


# ------------------------------------------------------------------- run

def _plain_embed(s):
    c = s.case
    here = (s.ids >= 0) & (s.ids < c["V"])
    if c["way"] == "lookup":
        rows = s.table[s.ids.clamp(0, c["V"] - 1)].float() * s.scale
        return (rows * here[:, None]).to(s.table.dtype)
    d = torch.zeros(c["V"], c["D"], dtype=torch.float32, device="cuda")
    d.index_add_(0, s.ids[here], s.dout[here].float() * s.scale)
    return d.to(s.dout.dtype)


def _act(name, g):
    """The activation and its derivative."""
    if name == "silu":
        e = 1 / (1 + torch.exp(-g))
        return g * e, e * (1 + g * (1 - e))
    phi = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def _plain_glu(s):
    c, dt = s.case, s.x.dtype
    x, wg, wu = s.x.float(), s.wg.float(), s.wu.float()
    g, u = x @ wg.t(), x @ wu.t()
    a, da = _act(c["act"], g)
    h = (a * u).to(dt)
    if c["way"] == "infer":
        return h
    dh = s.dh.float()
    dg, du = dh * u * da, dh * a
    dx = dg @ wg + du @ wu
    return h, dx.to(dt), (dg.t() @ x).to(dt), (du.t() @ x).to(dt)


def _plain_distill(s):
    c = s.case
    tau, w = s.tau, s.weights[:, None]
    here = s.ids >= 0
    at = s.ids.clamp(min=0)
    none = torch.full((), -math.inf, device="cuda")
    t = torch.where(here, s.teacher.float() / tau, none)
    t = t - t.max(1, keepdim=True).values
    e = torch.exp(t)
    total = e.sum(1, keepdim=True)
    p = e / total
    logp = t - torch.log(total)
    z = s.logits.float() / tau
    z = z - z.max(1, keepdim=True).values
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    logq = z.gather(1, at) - torch.log(total)
    terms = torch.where(here, p * (logp - logq), torch.zeros((), device="cuda"))
    loss = w[:, 0] * tau * tau * terms.sum(1)
    if c["way"] == "loss":
        return loss
    q = e / total
    q.scatter_add_(1, at, -p)
    return loss, (q * (w * tau)).to(s.logits.dtype)


def run(s):
    op, way = s.case["op"], s.case["way"]
    if not own:
        return {"embed": _plain_embed, "glu": _plain_glu, "distill": _plain_distill}[op](s)
    from paper_2409_04202_amd import ops
    if op == "embed":
        if way == "lookup":
            return ops.embed_lookup(s.table, s.ids, scale=s.scale)
        return ops.embed_grad(s.dout, s.ids, s.dtable, scale=s.scale)
    if op == "glu":
        if way == "infer":
            return ops.glu_forward(s.x, s.wg, s.wu, act=s.case["act"])
        h, saved = ops.glu_forward(s.x, s.wg, s.wu, act=s.case["act"], save=True)
        dx, dwg, dwu = ops.glu_backward(s.dh, s.x, s.wg, s.wu, saved, dwg=s.dwg, dwu=s.dwu)
        return h, dx, dwg, dwu
    if way == "loss":
        return ops.distill(s.logits, s.teacher, s.ids, temperature=s.tau, weights=s.weights)
    return ops.distill(s.logits, s.teacher, s.ids, temperature=s.tau, weights=s.weights,
                       grad=s.grad)


# ------------------------------------------------------------------ work

def work(case):
    """Inputs read once, outputs written once; the operations of the products
    (an element-wise operator: a few operations an element)."""
    e = ESIZE[case["dtype"]]
    if case["op"] == "embed":
        T, V, D = case["T"], case["V"], case["D"]
        if case["way"] == "lookup":
            distinct = min(T, V)
            return {"bytes": 8 * T + (distinct + T) * D * e, "flops": T * D}
        return {"bytes": 8 * T + (T + V) * D * e, "flops": 2 * T * D}
    if case["op"] == "glu":
        M, D, F = case["M"], case["D"], case["F"]
        if case["way"] == "infer":
            return {"bytes": (M * D + 2 * F * D + M * F) * e, "flops": 4 * M * D * F}
        return {"bytes": (2 * M * D + 4 * F * D + 2 * M * F) * e, "flops": 12 * M * D * F}
    T, V, K = case["T"], case["V"], case["K"]
    live = T - case["masked"]
    b = live * V * e + live * K * (8 + e) + 8 * T
    if case["way"] == "step":
        b += T * V * e
    return {"bytes": b, "flops": (3 if case["way"] == "loss" else 6) * live * V}


# ----------------------------------------------------------------- exact

def _rows(n, width):
    """Row ranges of about 2^28 elements."""
    step = max(1, (1 << 28) // max(1, width))
    return [(i, min(n, i + step)) for i in range(0, n, step)]


def exact(case, seed):
    """The same outputs from the definitions, in 64 bits."""
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "embed":
        V, D = case["V"], case["D"]
        valid = torch.nonzero((s.ids >= 0) & (s.ids < V)).flatten()
        if case["way"] == "lookup":
            out = torch.zeros(case["T"], D, dtype=f64, device="cuda")
            out[valid] = s.table.index_select(0, s.ids[valid]).to(f64) * s.scale
            return out
        out = torch.zeros(V, D, dtype=f64, device="cuda")
        for i, j in _rows(valid.numel(), D):
            t = valid[i:j]
            out.index_put_((s.ids[t],), s.dout[t].to(f64), accumulate=True)
        return out.mul_(s.scale)
    if case["op"] == "glu":
        x, wg, wu = s.x.to(f64), s.wg.to(f64), s.wu.to(f64)
        gate, up = torch.mm(x, wg.T.contiguous()), torch.mm(x, wu.T.contiguous())
        if case["act"] == "silu":
            sig = torch.sigmoid(gate)
            value, slope = gate * sig, sig + gate * sig * (1 - sig)
        else:
            cdf = torch.special.ndtr(gate)
            value = gate * cdf
            slope = cdf + gate * torch.exp(-gate.square() / 2) / math.sqrt(2 * math.pi)
        h = value * up
        if case["way"] == "infer":
            return h
        dh = s.dh.to(f64)
        dgate, dup = dh * up * slope, dh * value
        dx = torch.mm(dgate, wg) + torch.mm(dup, wu)
        return (h, dx, torch.mm(dgate.T.contiguous(), x), torch.mm(dup.T.contiguous(), x))
    T, K = case["T"], case["K"]
    step = case["way"] == "step"
    loss = torch.zeros(T, dtype=f64, device="cuda")
    grad = torch.zeros(T, case["V"], dtype=f64, device="cuda") if step else None
    for i, j in _rows(T, case["V"]):
        z = s.logits[i:j].to(f64) / case["tau"]
        lse = torch.logsumexp(z, 1, keepdim=True)
        there = s.ids[i:j] >= 0
        t = (s.teacher[i:j].to(f64) / case["tau"]).masked_fill(~there, -math.inf)
        logp = t - torch.logsumexp(t, 1, keepdim=True)
        weight = s.weights[i:j].to(f64)
        rows, cols = torch.nonzero(there, as_tuple=True)
        lp, ids = logp[rows, cols], s.ids[i:j][rows, cols]
        terms = torch.exp(lp) * (lp - (z[rows, ids] - lse[rows, 0]))
        part = torch.zeros(j - i, dtype=f64, device="cuda").index_add_(0, rows, terms)
        loss[i:j] = part * weight * case["tau"] ** 2
        if step:
            q = torch.exp(z - lse)
            q.index_put_((rows, ids), -torch.exp(lp), accumulate=True)
            grad[i:j] = q * (weight * case["tau"])[:, None]
    return (loss, grad) if step else loss
