"""Position bias, routing with its balance loss and activations in 8 bits on the
GPU, against plain definitions in 64 bits."""

import math

import numpy as np
import pytest
import torch

import more_ops_reference as ref

arplan = pytest.importorskip(
    "paper_2409_04202_amd.arplan",
    reason="HIP library not built (run python -m paper_2409_04202_amd.build)")
from paper_2409_04202_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu
DTYPES = ("f32", "bf16")
U, UB = ref.U, ref.UB


def rnd(seed, *shape, dtype="f32", scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(ref.TORCH[dtype])


def wide(x, value=float("nan")):
    """x on the GPU inside a tensor with wider rows of other values, at an odd element."""
    m = torch.full(x.shape[:-1] + (x.shape[-1] + 5,), value, dtype=x.dtype, device="cuda")
    at = m[..., 3:3 + x.shape[-1]]
    at.copy_(x)
    return at


def stored(x, dtype):
    return x.abs() * (UB if dtype == "bf16" else U) + 1e-38


def near(got, want, bound):
    off = (got.double().cpu() - want).abs()
    assert bool((off <= bound).all()), (float(off.max()), float((off / bound).max()))


# --------------------------------------------------------- position bias

BIAS = [    # H, Q, K, offset, buckets, max_distance, causal
    (1, 1, 1, 0, 32, 128, False), (3, 1, 700, 699, 32, 128, True), (2, 5, 3, 0, 4, 3, False),
    (2, 130, 70, 0, 32, 128, False), (1, 65, 1030, 965, 48, 300, True), (5, 64, 64, 0, 2, 2, True),
    (2, 3, 600, 10 ** 12, 32, 128, False), (2, 67, 9, -20, 32, 128, False),
    (1, 4, 20, -30, 16, 100, True), (1, 300, 40, 0, 256, 129, True), (3, 129, 515, 2, 256, 5000, False),
    (2, 40, 90, 50, 7, 31, True), (1, 17, 2050, 2033, 32, 128, True)]


@pytest.mark.parametrize("layout", ("rows", "wide", "heads within"))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,Q,K,offset,buckets,most,causal", BIAS)
def test_position_bias(H, Q, K, offset, buckets, most, causal, dtype, layout):
    table = rnd(1, buckets, H, dtype=dtype)
    want = ref.position_bias(table, Q, K, offset, most, causal)
    given = table.cuda() if layout == "rows" else wide(table)
    out, around = None, None
    if layout == "wide":
        around = torch.full((H, Q + 1, K + 5), 7.0, dtype=table.dtype, device="cuda")
        out = around[:, :Q, 3:3 + K]
    elif layout == "heads within":
        around = torch.full((Q, H + 1, K), 7.0, dtype=table.dtype, device="cuda")
        out = around[:, :H].transpose(0, 1)
    got = ops.position_bias(given, Q, K, max_distance=most, offset=offset, causal=causal, out=out)
    assert torch.equal(got.cpu(), want)
    if around is not None:
        out.fill_(7.0)
        assert bool((around == 7.0).all()), "elements around the output were written"


@pytest.mark.parametrize("buckets,most,causal", [
    (32, 128, False), (32, 128, True), (64, 256, False), (20, 1000, True), (8, 3000, False),
    (48, 2187, True), (4, 4096, False), (256, 2048, False), (3, 100, True), (16, 2 ** 31 - 1, True)])
def test_position_buckets_at_their_borders(buckets, most, causal):
    """The bucket of every distance up to 3000, by whole numbers: the table holds its rows' numbers."""
    table = torch.arange(buckets, dtype=torch.float32)[:, None]
    got = ops.position_bias(table.cuda(), 1, 3001, max_distance=most, offset=3000, causal=causal)
    want = ref.buckets(1, 3001, 3000, buckets, most, causal)
    assert torch.equal(got.cpu()[0, 0].long(), want[0])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("K", (8, 13, 519))
def test_position_bias_copies_bits(K, dtype):
    """Every bit of the table's values, those of NaN among them, at whole vectors and parts."""
    bits = torch.int16 if dtype == "bf16" else torch.int32
    top = 1 << 15 if dtype == "bf16" else 1 << 31
    g = torch.Generator().manual_seed(9)
    table = torch.randint(-top, top, (32, 3), generator=g).to(bits)
    table[::2] = (table[::2] | (0x7F80 if dtype == "bf16" else 0x7F800000))     # NaN of all kinds
    want = ref.position_bias(table.view(ref.TORCH[dtype]), 21, K, 3, 128, False)
    got = ops.position_bias(table.view(ref.TORCH[dtype]).cuda(), 21, K, offset=3)
    assert torch.equal(got.cpu().view(bits), want.view(bits))


@pytest.mark.parametrize("accumulate", (False, True))
@pytest.mark.parametrize("layout", ("rows", "wide"))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B", (1, 5))
@pytest.mark.parametrize("H,Q,K,offset,buckets,most,causal", BIAS)
def test_position_bias_grad(H, Q, K, offset, buckets, most, causal, B, dtype, layout, accumulate):
    """Whole numbers, whose sums are exact in any order: bit for bit."""
    g = torch.Generator().manual_seed(2)
    d = torch.randint(-8, 9, (B, H, Q, K), generator=g).to(ref.TORCH[dtype])
    old = torch.randint(-8, 9, (buckets, H), generator=g).to(d.dtype)
    want, _ = ref.position_bias_grad(d, buckets, offset, most, causal)
    if causal:      # what lies at keys that are not seen has no effect
        d[..., ref.buckets(Q, K, offset, buckets, most, True) < 0] = math.nan
    given = d.cuda() if layout == "rows" else wide(d)
    out = old.cuda() if layout == "rows" else wide(old, 7.0)
    ops.position_bias_grad(given, out, max_distance=most, offset=offset, causal=causal,
                           accumulate=accumulate)
    want = want.float() + (old.float() if accumulate else 0)
    assert torch.equal(out.cpu(), want.to(d.dtype))
    if layout == "wide":
        around = out._base
        out.fill_(7.0)
        assert bool((around == 7.0).all()), "elements around the output were written"


@pytest.mark.parametrize("dtype", DTYPES)
def test_position_bias_grad_of_real_numbers(dtype):
    """An element passes through at most 8 batches of 32 rows in its lane, 3 additions
    over the wavefronts, 8 along the diagonals, 6 over the lanes, and so again where
    the slots (16 a lane at most here) are joined."""
    B, H, Q, K = 3, 2, 413, 601
    d = rnd(3, B, H, Q, K, dtype=dtype)
    want, size = ref.position_bias_grad(d, 32, 0, 128, False)
    out = torch.empty(32, H, dtype=d.dtype, device="cuda")
    ops.position_bias_grad(d.cuda(), out)
    near(out, want, size * (8 * 32 + 3 + 8 + 6 + 16 + 6) * U + stored(want, dtype))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,H,Q,K,offset,causal", [
    (70, 2, 1, 40, 39, True), (33, 1, 5, 1600, 0, False), (9, 3, 17, 30, 0, False),
    (2, 1, 1, 100003, 99000, False), (1, 2, 700, 1, 0, False), (1, 1, 300, 300, 1 << 62, True),
    (1, 1, 30, 300, -(1 << 62), True), (1, 1, 30, 300, -(1 << 62), False), (2, 40, 90, 2100, 0, False)])
def test_position_bias_grad_at_its_ends(B, H, Q, K, offset, causal, dtype):
    """Many sequences, single rows and columns, distances beyond 32 bits: whole numbers."""
    g = torch.Generator().manual_seed(10)
    d = torch.randint(-1, 2, (B, H, Q, K), generator=g).to(ref.TORCH[dtype])
    want, _ = ref.position_bias_grad(d, 32, offset, 128, causal)
    out = torch.empty(32, H, dtype=d.dtype, device="cuda")
    ops.position_bias_grad(d.cuda(), out, offset=offset, causal=causal)
    assert torch.equal(out.cpu(), want.float().to(d.dtype))
    table = rnd(11, 32, H, dtype=dtype)
    assert torch.equal(ops.position_bias(table.cuda(), Q, K, offset=offset, causal=causal).cpu(),
                       ref.position_bias(table, Q, K, offset, 128, causal))


def test_position_bias_grad_of_shared_heads_and_batches():
    """A gradient that is the same for several heads and sequences has strides of zero."""
    g = torch.Generator().manual_seed(4)
    d = torch.randint(-8, 9, (1, 1, 70, 90), generator=g).float()
    want, _ = ref.position_bias_grad(d.expand(3, 4, 70, 90), 32, 0, 128, False)
    out = torch.empty(32, 4, device="cuda")
    ops.position_bias_grad(d.cuda().expand(3, 4, 70, 90), out)
    assert torch.equal(out.cpu(), want.float())
    one = ops.position_bias_grad(d.cuda()[0], torch.empty(32, 1, device="cuda"))
    assert torch.equal(one.cpu() * 3, want[:, :1].float())


def test_position_bias_is_linear_in_its_table():
    """<bias(table), d> = <table, gradient(d)> for whole numbers, exactly."""
    g = torch.Generator().manual_seed(5)
    table = torch.randint(-8, 9, (32, 3), generator=g).float().cuda()
    d = torch.randint(-8, 9, (3, 80, 100), generator=g).float().cuda()
    left = (ops.position_bias(table, 80, 100, offset=20).double() * d.double()).sum()
    grad = ops.position_bias_grad(d, torch.empty_like(table), offset=20)
    assert float(left) == float((table.double() * grad.double()).sum())


def test_position_bias_far_offsets():
    """Rows and heads whose elements lie beyond 2^31 of the first."""
    step = (1 << 30) + 12345
    flat = torch.zeros(4 * step, dtype=torch.bfloat16, device="cuda")
    out = flat.as_strided((2, 2, 100), (2 * step, step, 1))
    table = rnd(6, 32, 2, dtype="bf16")
    ops.position_bias(table.cuda(), 2, 100, offset=98, out=out)
    assert torch.equal(out.cpu(), ref.position_bias(table, 2, 100, 98, 128, False))
    g = torch.Generator().manual_seed(7)
    d = torch.randint(-8, 9, (1, 2, 2, 100), generator=g).bfloat16()
    out.copy_(d[0])
    got = ops.position_bias_grad(out, torch.empty(32, 2, dtype=torch.bfloat16, device="cuda"),
                                 offset=98)
    want, _ = ref.position_bias_grad(d, 32, 98, 128, False)
    assert torch.equal(got.cpu(), want.bfloat16())


def test_position_bias_of_nothing():
    table = rnd(8, 32, 2).cuda()
    assert ops.position_bias(table, 0, 5).shape == (2, 0, 5)
    assert ops.position_bias(table, 5, 0).shape == (2, 5, 0)
    for shape in ((0, 2, 5, 5), (3, 2, 0, 5), (3, 2, 5, 0)):
        d = torch.empty(shape, device="cuda")
        out = table.clone()
        assert torch.equal(ops.position_bias_grad(d, out, accumulate=True), table)
        assert bool((ops.position_bias_grad(d, out) == 0).all())
    assert ops.position_bias_grad(torch.empty(3, 0, 5, 5, device="cuda"),
                                  torch.empty(32, 0, device="cuda")).shape == (32, 0)


# --------------------------------------------------------------- routing

def logits_of(seed, T, E, dtype, kind):
    z = rnd(seed, T, E, dtype=dtype, scale=2.0)
    g = torch.Generator().manual_seed(seed + 100)
    if kind == "ties":      # few values, zeros of both signs among them
        z = (torch.randint(-2, 3, (T, E), generator=g).float() * 0.5).to(z.dtype)
        z[torch.rand(T, E, generator=g) < 0.2] = -0.0
    if kind == "holes":     # absent experts, whole rows of them among the rows
        z[torch.rand(T, E, generator=g) < 0.6] = -math.inf
        z[::3] = -math.inf
        if T > 1:
            z[1] = torch.finfo(z.dtype).min
    return z


ROUTES = [  # T, E, k, kind
    (1, 4, 1, ""), (8, 64, 2, ""), (9, 1, 1, ""), (70, 8, 8, "ties"), (33, 9, 3, "holes"),
    (300, 16, 5, "ties"), (200, 31, 31, "holes"), (129, 61, 4, ""), (500, 64, 8, "ties"),
    (250, 100, 32, "holes"), (1500, 128, 8, ""), (100, 130, 6, "ties"), (60, 256, 8, "holes"),
    (70, 511, 7, ""), (40, 513, 9, "ties"), (30, 1024, 32, "holes"), (0, 8, 2, ""),
    (9000, 300, 3, "ties"), (4500, 600, 8, "")]     # (more rows than a launch's wavefronts)


@pytest.mark.parametrize("E,k", [(66, 8), (100, 3), (129, 8), (250, 1), (300, 5), (512, 8)])
def test_route_of_many_rows(E, k):
    """The form for many rows chooses as that for few does, ties and holes among them, bit for
    bit; its sums over rows are the few rows' sums up to the additions."""
    T, step = 70000, 5000
    z = torch.cat([logits_of(90 + i, T // 7, E, "bf16", ("", "ties", "holes")[i % 3]) for i in range(7)])
    z = z[:, torch.randperm(E, generator=torch.Generator().manual_seed(91))].cuda()
    live = (torch.rand(T, generator=torch.Generator().manual_seed(92)) < 0.8).cuda()
    ids, gates, counts, mass = ops.route(z, k, live=live, normalize=True)
    parts = [ops.route(z[i:i + step], k, live=live[i:i + step], normalize=True)
             for i in range(0, T, step)]
    assert torch.equal(ids, torch.cat([p[0] for p in parts]))
    assert torch.equal(counts, sum(p[2] for p in parts))
    few = torch.cat([p[1] for p in parts])
    near(gates, few.double().cpu(), few.double().cpu() * 2 * gate_bound(E, k) + 2e-36)
    want = sum(p[3].double() for p in parts).cpu()
    near(mass, want, want * 2 * (E + 16 + T / 512) * U + T * 1e-36)


def gate_bound(E, k):
    """exp to 4 units, the sum's E additions, its inverse and a product, twice where gates
    are normalized (by a sum of k); what underflows is below 1e-36."""
    return (2 * (E + 12) + k + 4) * U


@pytest.mark.parametrize("padded", (False, True))
@pytest.mark.parametrize("normalize", (False, True))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,E,k,kind", ROUTES)
def test_route(T, E, k, kind, dtype, normalize, padded):
    z = logits_of(11, T, E, dtype, kind)
    live = torch.rand(T, generator=torch.Generator().manual_seed(12)) < 0.7 if padded else None
    if padded:      # padding holds anything
        z[~live] = math.nan
    ids, gates, counts, mass = ref.route(z, k, live, normalize)
    got = ops.route(wide(z) if padded else z.cuda(), k, live=None if live is None else live.cuda(),
                    normalize=normalize)
    assert torch.equal(got[0].cpu(), ids)
    assert torch.equal(got[2].cpu().long(), counts)
    near(got[1], gates, gates * gate_bound(E, k) + 1e-36)
    near(got[3], mass, mass * (E + 16 + T) * U + T * 1e-36)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("value", (math.nan, -math.nan, math.inf))
def test_route_of_numbers_that_are_none(value, dtype):
    z = rnd(13, 20, 40, dtype=dtype)
    z[7, 30] = value
    ids, gates, counts, mass = ops.route(z.cuda(), 4)
    want, there, _, _ = ref.route(z[torch.arange(20) != 7], 4)
    rest = torch.arange(20) != 7
    assert torch.equal(ids.cpu()[rest], want)
    near(gates[rest.cuda()], there, there * gate_bound(40, 4))
    assert int(ids[7, 0]) == 30 and len(set(ids[7].tolist())) == 4
    assert bool(gates[7].isnan().all()) and bool(mass.isnan().all())
    assert int(counts[40]) == 20 and int(counts[:40].sum()) == 80


BALANCES = [c for c in ROUTES if c[0]]


@pytest.mark.parametrize("gates", ("none", "plain", "normalized"))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,E,k,kind", BALANCES)
def test_balance(T, E, k, kind, dtype, gates):
    z = logits_of(14, T, E, dtype, kind)
    z[z.float().abs() > 1e30] = -math.inf
    normalize = gates == "normalized"
    ids, _, counts, mass = ref.route(z, k, None, normalize)
    counts = counts * 3 + 1     # other replicas' among them
    dgates = None if gates == "none" else rnd(15, T, k)
    mass = mass.float()
    loss, grad, size = ref.balance(z, ids, counts, mass, 0.37, normalize, dgates)
    out = torch.full((T, E + 3), 7.0, dtype=z.dtype, device="cuda")
    args = (ids.cuda(), counts.int().cuda(), mass.cuda())
    got, _ = ops.balance(z.cuda(), *args, coefficient=0.37, normalize=normalize,
                         dgates=None if dgates is None else dgates.cuda(), grad=out[:, 1:1 + E])
    assert abs(float(got) - loss) <= 8 * U * abs(loss) + 1e-38
    # probabilities as gates' above; a_te of a few operations and k additions; a sum of E
    bound = size * (3 * (E + 16) + 2 * k + 16) * U + stored(grad, dtype) + 1e-36
    near(out[:, 1:1 + E], grad, bound)
    out[:, 1:1 + E] = 7.0
    assert bool((out == 7.0).all()), "elements around the output were written"
    alone = ops.balance(z.cuda(), *args, coefficient=0.37, normalize=normalize)
    assert float(alone) == float(got)
    place = z.cuda()
    ops.balance(place, *args, coefficient=0.37, normalize=normalize,
                dgates=None if dgates is None else dgates.cuda(), grad=place)
    assert torch.equal(place, ops.balance(z.cuda(), *args, coefficient=0.37, normalize=normalize,
                                          dgates=None if dgates is None else dgates.cuda(),
                                          grad=torch.empty_like(place))[1])


@pytest.mark.parametrize("normalize", (False, True))
def test_balance_against_differences(normalize):
    """The loss for fixed counts and the gates' part, in 64 bits, against the gradient."""
    T, E, k = 6, 10, 3
    z = rnd(16, T, E)
    ids, _, counts, _ = ref.route(z, k)
    G = rnd(17, T, k).double()

    def value(x):
        p = torch.softmax(x, 1)
        w = p.gather(1, ids)
        if normalize:
            w = w / w.sum(1, keepdim=True)
        return float((p.sum(0) * counts[:E].double()).sum() * 0.5 * E / (k * T * T) + (w * G).sum())
    mass = torch.softmax(z.double(), 1).sum(0).float()
    _, got = ops.balance(z.cuda(), ids.cuda(), counts.int().cuda(), mass.cuda(), coefficient=0.5,
                         normalize=normalize, dgates=G.float().cuda(),
                         grad=torch.empty(T, E, device="cuda"))
    for t in range(T):
        for e in range(E):
            step = torch.zeros(T, E).double()
            step[t, e] = 1e-4
            diff = (value(z.double() + step) - value(z.double() - step)) / 2e-4
            assert abs(diff - float(got[t, e])) < 1e-5


def test_balance_with_ids_that_are_none():
    """An id that is given twice counts twice, one outside the experts not at all."""
    z = rnd(18, 5, 12)
    ids = torch.tensor([[3, 3, 5], [-1, 2, 2], [0, 12, -7], [11, 2 ** 40, 11], [4, -1, -1]])
    counts, mass, G = torch.full((13,), 5, dtype=torch.int32), torch.ones(12), rnd(19, 5, 3)
    for normalize in (False, True):
        _, want, size = ref.balance(z, ids, counts, mass, 1.0, normalize, G)
        _, got = ops.balance(z.cuda(), ids.cuda(), counts.cuda(), mass.cuda(), 1.0, normalize,
                             G.cuda(), torch.empty(5, 12, device="cuda"))
        near(got, want, size * (3 * 28 + 6 + 16) * U + stored(want, "f32"))
    loss = ops.balance(z.cuda(), ids.cuda(), torch.zeros_like(counts).cuda(), mass.cuda())
    assert float(loss) == 0


def test_replicas_losses_add_up():
    """Counts summed by an int32 plan: the replicas' losses and gradients are the whole batch's."""
    n, T, E, k = 4, 96, 24, 3
    z = rnd(20, n * T, E).cuda()
    parts = [ops.route(z[i * T:(i + 1) * T], k) for i in range(n)]
    with arplan.Plan(n, E + 1, "i32", "ring") as p:
        p.execute([x[2] for x in parts], torch.cuda.current_stream())
    ids, _, counts, mass = ops.route(z, k)
    for x in parts:
        assert torch.equal(x[2], counts)
    whole, grad = ops.balance(z, ids, counts, mass, 0.1, grad=torch.empty_like(z))
    total = 0.0
    for i, x in enumerate(parts):
        loss, g = ops.balance(z[i * T:(i + 1) * T], x[0], x[2], x[3], 0.1,
                              grad=torch.empty(T, E, device="cuda"))
        total += float(loss)
        assert torch.equal(g, grad[i * T:(i + 1) * T])
    assert abs(total - float(whole)) <= (n * T + 40) * U * float(whole)


# ------------------------------------------------- activations in 8 bits

def activations(seed, M, N, dtype, kind):
    x = rnd(seed, M, N, dtype="f32")
    g = torch.Generator().manual_seed(seed + 1)
    if kind == "spread":    # every power of two, zeros, the smallest and the largest
        x = x * 2.0 ** torch.randint(-149, 128, (M, N), generator=g).float()
        x[torch.rand(M, N, generator=g) < 0.1] = 0
        x = x.clamp(-3.3e38, 3.3e38)
    if kind == "ties":      # whole numbers of halves of a unit, and the borders of a power
        x = torch.randint(-255, 256, (M, N), generator=g).float() * 0.5
        x[:, ::32] = torch.tensor([127.0, 127.25, 127.5, 127.75, 63.75, 63.5])[
            torch.randint(0, 6, (M, len(range(0, N, 32))), generator=g)]
    if kind == "nan":
        x[torch.rand(M, N, generator=g) < 0.01] = math.nan
        x[torch.rand(M, N, generator=g) < 0.01] = -math.inf
        x[-1, -1] = math.inf
    return x.to(ref.TORCH[dtype])


@pytest.mark.parametrize("layout", ("rows", "wide"))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ("", "spread", "ties", "nan"))
@pytest.mark.parametrize("M,N", [(1, 1), (3, 32), (2, 33), (5, 31), (7, 16), (4, 4096), (3, 4100),
                                 (2, 9000), (200, 40), (33, 1001)])
def test_checkpoint(M, N, kind, dtype, layout):
    x = activations(21, M, N, dtype, kind)
    numbers, byte = ref.kept(x)
    runs, row = byte.shape[1], arplan.ar_checkpoint_row(N)
    assert row % 16 == 0 and 33 * runs <= row < 33 * runs + 16
    around = torch.full((M + 1, row + 16), 99, dtype=torch.uint8, device="cuda")
    out = None if layout == "rows" else around[:M, :row]
    kept = ops.checkpoint_store(x.cuda() if layout == "rows" else wide(x), out=out)
    got = kept.cpu().numpy()
    assert np.array_equal(got[:, :32 * runs].view(np.int8).reshape(M, runs, 32), numbers)
    assert np.array_equal(got[:, 32 * runs:33 * runs], byte)
    want = ref.fetched(numbers, byte, N)
    for as_dtype in DTYPES:
        back = ops.checkpoint_load(kept, N, ref.TORCH[as_dtype])
        assert torch.equal(back.cpu().double().nan_to_num(7e300), want.nan_to_num(7e300))
    fine = (x.double().abs() < 3.3e38) & ~want.isnan()
    unit = torch.from_numpy(2.0 ** (byte.astype(np.float64) - 127)).repeat_interleave(32, 1)[:, :N]
    assert bool(((want - x.double()).abs() <= unit / 2)[fine & (want.abs() < 127 * 2.0 ** 121)].all())
    if layout == "wide":
        res = torch.full((M + 1, N + 5), 7.0, dtype=x.dtype, device="cuda")
        ops.checkpoint_load(kept, N, out=res[:M, 3:3 + N])
        assert torch.equal(res[:M, 3:3 + N], ops.checkpoint_load(kept, N, x.dtype)) or kind == "nan"
        res[:M, 3:3 + N] = 7.0
        assert bool((res == 7.0).all()), "elements around the output were written"
        around[:M, :33 * runs] = 99
        assert bool((around == 99).all()), "bytes behind the rows were written"


def test_checkpoint_of_the_largest_numbers():
    x = torch.tensor([[3.4028235e38, -3.4e38, 1.0] + [0.0] * 29, [2.0 ** 121 * 127] * 32])
    back = ops.checkpoint_load(ops.checkpoint_store(x.cuda()), 32, torch.float32).cpu()
    assert back[0, :3].tolist() == [127 * 2.0 ** 121, -127 * 2.0 ** 121, 0.0]
    assert torch.equal(back[1], x[1])


def test_checkpoint_of_nothing():
    for M, N in ((0, 40), (5, 0)):
        kept = ops.checkpoint_store(torch.empty(M, N, device="cuda"))
        assert ops.checkpoint_load(kept, N, torch.bfloat16).shape == (M, N)


def test_checkpoint_far_rows():
    """Rows beyond 2^32 bytes of the first, in x and in what is kept."""
    M, N = 3, 1000
    x = torch.zeros(M, 1 << 31, dtype=torch.bfloat16, device="cuda")[:, 7:7 + N]
    x.copy_(rnd(22, M, N, dtype="bf16"))
    room = torch.zeros(M, (1 << 32) + 4096, dtype=torch.uint8, device="cuda")
    kept = ops.checkpoint_store(x, out=room[:, 64:64 + arplan.ar_checkpoint_row(N)])
    want = ref.fetched(*ref.kept(x.cpu()), N)
    assert torch.equal(ops.checkpoint_load(kept, N, torch.float32).cpu().double(), want)


GLU = [(9, 64, 33), (16, 8, 1), (33, 129, 65), (65, 1000, 130), (130, 72, 300), (300, 512, 1000),
       (777, 200, 513), (40, 2048, 96)]


@pytest.mark.parametrize("act", ("silu", "gelu"))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,D,F", GLU)
def test_glu_saves_in_8_bits(M, D, F, dtype, act):
    """What the forward pass keeps is the fp32 factors as checkpoint_store keeps them, and the
    backward pass from it is that from its values in fp32: bit for bit."""
    x, wg, wu = (rnd(30 + i, *s, dtype=dtype).cuda() for i, s in enumerate(((M, D), (F, D), (F, D))))
    h, saved = ops.glu_forward(x, wg, wu, act=act, save=torch.uint8)
    want, factors = ops.glu_forward(x, wg, wu, act=act, save=True)
    assert torch.equal(h, want)
    n = 33 * (-(-F // 32))
    values = torch.empty_like(factors)
    for i in range(2):
        assert torch.equal(saved[i][:, :n], ops.checkpoint_store(factors[i])[:, :n])
        ops.checkpoint_load(saved[i], F, out=values[i])
    dh = rnd(33, M, F, dtype=dtype).cuda()
    for got, plain in zip(ops.glu_backward(dh, x, wg, wu, saved),
                          ops.glu_backward(dh, x, wg, wu, values)):
        assert torch.equal(got, plain)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,D,F", [(1, 64, 40), (2, 100, 37), (5, 72, 300), (8, 512, 1000), (3, 0, 50),
                                   (20, 0, 50)])
def test_glu_saves_few_rows_in_8_bits(M, D, F, dtype):
    """Against the definition in 64 bits: half a unit, and the sums' and the activation's error,
    D + 32 units of the magnitudes (a factor is at most 1.2 of those)."""
    x, wg, wu = (rnd(40 + i, *s, dtype=dtype) for i, s in enumerate(((M, D), (F, D), (F, D))))
    h, saved = ops.glu_forward(x.cuda(), wg.cuda(), wu.cuda(), save=torch.uint8)
    X, G, W = x.double(), wg.double(), wu.double()
    g, u = X @ G.T, X @ W.T
    mg, mu = X.abs() @ G.abs().T, X.abs() @ W.abs().T
    s = torch.sigmoid(g)
    slope = s * (1 + g * (1 - s))
    off = (D + 32) * U * 1.2
    if dtype == "bf16":     # the hardware's exponential: |g| more units
        off = off + g.abs() * U * 4 + 16 * U
    near(h, g * s * u, off * (mg * mu + mg + mu) * 2 + (g * s * u).abs() * (UB if dtype == "bf16" else U) + 1e-38)
    for i, (want, size) in enumerate(((slope * u, mu + mg * mu), (g * s, mg))):
        runs = -(-F // 32)
        byte = saved[i][:, 32 * runs:33 * runs].cpu().double()
        unit = (2.0 ** (byte - 127)).repeat_interleave(32, 1)[:, :F]
        near(ops.checkpoint_load(saved[i], F, torch.float32), want, unit / 2 + off * size * 2 + 1e-38)


@pytest.mark.parametrize("dtype", DTYPES)
def test_glu_backward_from_8_bits(dtype):
    """Gradients against the formula in 64 bits on the kept values."""
    M, D, F = 70, 90, 110
    x, wg, wu, dh = (rnd(50 + i, *s, dtype=dtype) for i, s in
                     enumerate(((M, D), (F, D), (F, D), (M, F))))
    factors = torch.stack([rnd(54, M, F), rnd(55, M, F)])
    saved = torch.stack([ops.checkpoint_store(factors[i].cuda()) for i in range(2)])
    a, b = (ref.fetched(*ref.kept(factors[i]), F) for i in range(2))
    kept = ops.checkpoint_store(x.cuda())
    X = ref.fetched(*ref.kept(x), D)
    got = ops.glu_backward(dh.cuda(), ops.checkpoint_load(kept, D, x.dtype), wg.cuda(), wu.cuda(), saved)
    dg, du = dh.double() * a, dh.double() * b
    rounding = UB if dtype == "bf16" else U      # of dg and du
    for out, want, size, n in (
            (got[0], dg @ wg.double() + du @ wu.double(),
             dg.abs() @ wg.double().abs() + du.abs() @ wu.double().abs(), 2 * F),
            (got[1], dg.T @ X, dg.T.abs() @ X.abs(), M), (got[2], du.T @ X, du.T.abs() @ X.abs(), M)):
        near(out, want, size * (rounding + (n + 2) * U) + stored(want, dtype))


def test_glu_runs_of_nan():
    """A factor that is no number reads as NaN with its run, and with nothing else."""
    M, D, F = 20, 24, 100
    x, wg, wu, dh = (rnd(60 + i, *s).cuda() for i, s in enumerate(((M, D), (F, D), (F, D), (M, F))))
    x[3] = math.nan
    h, saved = ops.glu_forward(x, wg, wu, save=torch.uint8)
    dx, _, _ = ops.glu_backward(dh, x, wg, wu, saved)
    assert bool(dx[3].isnan().all()) and bool(dx[torch.arange(M) != 3].isfinite().all())


# --------------------------------------------------------- a step of them

def step(s):
    """A replica's step around one gated block: bias, routing, block, and back."""
    bias = ops.position_bias(s["table"], 48, 64, offset=16, causal=True, out=s["bias"])
    ids, gates, counts, mass = ops.route(s["logits"], 2, normalize=True, counts=s["counts"])
    kept = ops.checkpoint_store(s["x"])
    h, saved = ops.glu_forward(s["x"], s["wg"], s["wu"], save=torch.uint8)
    loss, dlogits = ops.balance(s["logits"], ids, counts, mass, normalize=True, dgates=gates,
                                grad=s["dlogits"])
    x = ops.checkpoint_load(kept, s["x"].shape[1], s["x"].dtype)
    dx, dwg, dwu = ops.glu_backward(h, x, s["wg"], s["wu"], saved, dwg=s["dwg"], dwu=s["dwu"])
    dtable = ops.position_bias_grad(s["dbias"], s["dtable"], offset=16, causal=True)
    return [t.clone() for t in (bias, ids, gates, counts, mass, loss, dlogits, h, dx, dwg, dwu, dtable)]


def state(dtype="bf16"):
    n = lambda i, *shape: rnd(70 + i, *shape, dtype=dtype).cuda()   # noqa: E731
    e = lambda *shape: torch.empty(*shape, dtype=ref.TORCH[dtype], device="cuda")   # noqa: E731
    return {"table": n(0, 32, 3), "bias": e(3, 48, 64), "logits": n(1, 200, 40),
            "counts": torch.empty(41, dtype=torch.int32, device="cuda"), "x": n(2, 200, 72),
            "wg": n(3, 100, 72), "wu": n(4, 100, 72), "dlogits": e(200, 40), "dwg": e(100, 72),
            "dwu": e(100, 72), "dbias": n(5, 2, 3, 48, 64), "dtable": e(32, 3)}


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_step_captured_and_replayed(dtype):
    s = state(dtype)
    want = step(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(s)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(s)
    fresh = state(dtype)
    for i in range(4):
        for k, v in fresh.items():
            if k in ("x", "logits", "dbias", "table"):
                s[k].copy_(v * (1.0 if i % 2 else 0.5))
        eager = step(s)
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, eager):
            assert torch.equal(a, b)
        if i % 2:
            for a, b in zip(got, want):
                assert torch.equal(a, b)


def test_calls_on_another_stream():
    s = state()
    want = step(s)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    bias = ops.position_bias(s["table"], 48, 64, offset=16, causal=True, stream=other)
    ids, gates, counts, mass = ops.route(s["logits"], 2, normalize=True, stream=other)
    _, dlogits = ops.balance(s["logits"], ids, counts, mass, normalize=True, dgates=gates,
                             grad=s["dlogits"], stream=other)
    kept = ops.checkpoint_store(s["x"], stream=other)
    x = ops.checkpoint_load(kept, 72, torch.bfloat16, stream=other)
    dtable = ops.position_bias_grad(s["dbias"], s["dtable"], offset=16, causal=True, stream=other)
    other.synchronize()
    for a, b in zip((bias, ids, gates, counts, mass, dlogits, dtable), want[:5] + [want[6], want[11]]):
        assert torch.equal(a, b)
    assert torch.equal(x, ops.checkpoint_load(ops.checkpoint_store(s["x"]), 72, torch.bfloat16))


def test_two_streams_at_once():
    """Calls that overlap, each with what it allocates itself."""
    a, b = state("bf16"), state("f32")
    want = [[t.clone() for t in step(s)] for s in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(5):
        for i, s in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i] = step(s)
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        for p, q in zip(x, y):
            assert torch.equal(p, q)


def test_counts_in_a_slice_of_a_vector():
    """Counts and mass at any element of a vector that a plan sums, and nothing beside them."""
    z = rnd(81, 3000, 61, dtype="bf16").cuda()
    ids, _, counts, mass = ops.route(z, 3)
    loss, grad = ops.balance(z, ids, counts, mass, grad=torch.empty_like(z))
    whole, sums = torch.full((100,), -5, dtype=torch.int32, device="cuda"), torch.full((99,), 7.0, device="cuda")
    ops.route(z, 3, counts=whole[7:69], mass=sums[5:66])
    assert torch.equal(whole[7:69], counts) and torch.equal(sums[5:66], mass)
    assert bool((whole[:7] == -5).all()) and bool((whole[69:] == -5).all())
    assert bool((sums[:5] == 7).all()) and bool((sums[66:] == 7).all())
    again, other = ops.balance(z, ids, whole[7:69], sums[5:66], grad=torch.empty_like(z))
    assert torch.equal(again, loss) and torch.equal(other, grad)


def test_given_workspaces_and_what_counts_as_changed():
    s = state("f32")
    need = arplan.ar_position_bias_grad_workspace("f32", 32, 2, 3, 48, 64)
    space = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    before = s["dtable"]._version
    a = ops.position_bias_grad(s["dbias"], s["dtable"], workspace=space[:need]).clone()
    assert s["dtable"]._version > before
    assert torch.equal(a, ops.position_bias_grad(s["dbias"], torch.empty_like(a)))
    z = rnd(80, 3000, 24).cuda()
    need = arplan.ar_route_workspace(3000, 24, 2)
    assert need > 0
    room = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    for got, want in zip(ops.route(z, 2, workspace=room[:need]), ops.route(z, 2)):
        assert torch.equal(got, want)
    assert bool((room[need:] == 255).all()) and bool((space[-64:] == 255).all())
    with pytest.raises(ValueError):
        ops.position_bias_grad(s["dbias"].requires_grad_(), s["dtable"])
