"""Position bias, routing with its balance loss and activations in 8 bits at the ends of
what they accept, on the GPU, against plain definitions in 64 bits."""

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
LARGEST = float(np.finfo(np.float32).max)


def rnd(seed, *shape, dtype="f32", scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(ref.TORCH[dtype])


def near(got, want, bound):
    off = (got.double().cpu() - want).abs()
    assert bool((off <= bound).all()), (float(off.max()), float((off / bound).max()))


# --------------------------------------------------------- position bias

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,H,Q,K", [(4, 3, 32, 32), (5, 3, 32, 32), (8, 3, 32, 32), (1, 3, 250, 250),
                                     (1, 3, 256, 256), (32, 3, 8, 8), (8, 3, 32, 256), (3, 3, 64, 1000)])
def test_position_bias_grad_on_both_sides_of_the_join(B, H, Q, K, dtype):
    """A head in one block or in several: whole numbers, bit for bit."""
    g = torch.Generator().manual_seed(5)
    d = torch.randint(-4, 5, (B, H, Q, K), generator=g).to(ref.TORCH[dtype])
    for causal in (False, True):
        want, _ = ref.position_bias_grad(d, 32, 0, 128, causal)
        got = ops.position_bias_grad(d.cuda(), torch.empty(32, H, dtype=d.dtype, device="cuda"),
                                     causal=causal)
        assert torch.equal(got.cpu(), want.float().to(d.dtype))


# --------------------------------------------------------------- routing

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("E", (2, 8, 60, 128, 512, 1000))
def test_mass_of_far_experts(E, dtype):
    """Each probability of one row whose logits go down to 85 below the largest, which is 0, so
    that no difference is rounded: an exponential to 4 units, one in the sum, whose 16 + 6
    additions (of a lane's and over the lanes) and inverse follow, and the product."""
    g = torch.Generator().manual_seed(2)
    z = (torch.rand(1, E, generator=g) * -85).to(ref.TORCH[dtype])
    z[0, E // 2], z[0, 0] = 0, -84
    p = torch.softmax(z.double(), 1)[0]
    ids, gates, counts, mass = ops.route(z.cuda(), min(E, 32))
    near(mass, p, p * (4 + 4 + 22 + 2) * U)
    near(gates[0], p[ids[0].cpu()], p[ids[0].cpu()] * (4 + 4 + 22 + 2) * U)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,E,k", [
    (1024, 8, 8), (1025, 8, 8), (2048, 8, 8), (2049, 8, 8), (1536, 16, 7), (1537, 16, 7), (128, 61, 9),
    (129, 61, 32), (257, 61, 9), (64, 128, 32), (65, 128, 32), (129, 128, 32), (128, 128, 8), (129, 128, 8),
    (192, 128, 8), (193, 128, 8), (49, 512, 8), (33, 512, 9), (8, 1024, 32), (9, 1024, 32), (17, 1024, 32),
    (25, 1024, 8)])
def test_route_on_both_sides_of_the_join(T, E, k, dtype):
    """The largest calls of one block and the smallest of several, with ties among the logits."""
    g = torch.Generator().manual_seed(3)
    z = (torch.randint(-6, 7, (T, E), generator=g).float() * 0.5).to(ref.TORCH[dtype])
    ids, gates, counts, mass = ref.route(z, k, None, True)
    got = ops.route(z.cuda(), k, normalize=True)
    assert torch.equal(got[0].cpu(), ids) and torch.equal(got[2].cpu().long(), counts)
    # exponentials, sums over experts and rows, inverses and products, twice where normalized
    near(got[1], gates, gates * (2 * (E + 12) + k + 4) * U)
    near(got[3], mass, mass * (E + 16 + T) * U)


@pytest.mark.parametrize("E,k,T,step", [
    (66, 8, 16385, 8192), (100, 3, 17000, 8500), (128, 8, 30001, 15001), (129, 8, 33000, 16500),
    (256, 1, 32769, 16385), (300, 5, 16385, 8193), (512, 8, 20011, 10006)])
def test_route_of_many_rows_and_of_their_halves(E, k, T, step):
    """bf16 rows past the limits of 16 logits a lane, with ties, absent experts and padding: what
    is chosen is bit for bit what the halves of the rows choose, with 8."""
    g = torch.Generator().manual_seed(4)
    z = torch.randint(-9, 10, (T, E), generator=g).float() * 0.5 + torch.randn(1, E, generator=g).bfloat16()
    z[torch.rand(T, E, generator=g) < 0.05] = -math.inf
    z = z.bfloat16().cuda()
    live = (torch.rand(T, generator=g) < 0.8).cuda()
    ids, gates, counts, mass = ops.route(z, k, live=live, normalize=True)
    parts = [ops.route(z[i:i + step], k, live=live[i:i + step], normalize=True)
             for i in range(0, T, step)]
    assert torch.equal(ids, torch.cat([p[0] for p in parts]))
    assert torch.equal(counts, sum(p[2] for p in parts))
    few = torch.cat([p[1] for p in parts]).double().cpu()
    near(gates, few, few * 2 * (2 * (E + 12) + k + 4) * U + 2e-36)
    want = sum(p[3].double() for p in parts).cpu()
    near(mass, want, want * 2 * (E + 16 + T / 512) * U + T * 1e-36)


def test_route_refuses_a_number_of_choices():
    z = rnd(7, 4, 8).cuda()
    for k in (2.0, None, -1, (1 << 64) + 2, torch.tensor(2.0)):
        with pytest.raises(ValueError):
            ops.route(z, k)
    for k in (0, 9):
        with pytest.raises(arplan.ArError):
            ops.route(z, k)


def test_whole_numbers_of_other_types():
    """numpy's and torch's whole numbers are whole numbers."""
    z, table = rnd(7, 4, 8).cuda(), rnd(8, 32, 2).cuda()
    for k in (np.int64(2), np.int32(2), torch.tensor(2)):
        for a, b in zip(ops.route(z, k), ops.route(z, 2)):
            assert torch.equal(a, b)
        got = ops.position_bias(table, k, np.int64(5), max_distance=np.int64(100), offset=k)
        assert torch.equal(got, ops.position_bias(table, 2, 5, max_distance=100, offset=2))
        kept = ops.checkpoint_store(z)
        assert torch.equal(ops.checkpoint_load(kept, np.int64(8), torch.float32),
                           ops.checkpoint_load(kept, 8, torch.float32))


# --------------------------------------------------------------- balance

@pytest.mark.parametrize("normalize", (False, True))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,E,k,coefficient,many", [
    (600, 1024, 2, 1e36, 0), (600, 1024, 2, -LARGEST, 0), (300, 512, 8, LARGEST, 0),
    (40, 4, 1, 1e-24, 1 << 31), (40, 16, 2, 1e-22, 1 << 30)])
def test_balance_of_extreme_coefficients(T, E, k, coefficient, many, dtype, normalize):
    """Coefficients whose product with E leaves fp32, and counts of so many replicas that
    E / N^2 does; an expert without choices among them.  The slopes are rounded once, the
    gradient as in any other call."""
    z = rnd(1, T, E, dtype=dtype)
    ids, _, counts, mass = ref.route(z, k, None, normalize)
    counts[3] = 0
    if many:
        counts[:3], counts[E] = many - 1 - torch.arange(3) * 1000003, many - 1
    mass = mass.float()
    loss, grad, size = ref.balance(z, ids, counts, mass, float(np.float32(coefficient)), normalize)
    got, out = ops.balance(z.cuda(), ids.cuda(), counts.int().cuda(), mass.cuda(), coefficient,
                           normalize, grad=torch.empty(T, E, dtype=z.dtype, device="cuda"))
    # (a loss of 3.485e38 lies beyond the largest fp32 number, 3.403e38, by more than half of
    # that one's last place, 2^103: rounded, it is infinite)
    if abs(loss) >= LARGEST + 2.0 ** 103:
        assert float(got) == math.copysign(math.inf, loss)
    else:
        assert abs(float(got) - loss) <= 8 * U * abs(loss)
    # a slope of one rounding, probabilities of E + 16, a sum of E and three operations; half
    # of the least bf16 number, and a few of fp32's
    near(out, grad, size * (3 * (E + 16) + 16) * U
         + (grad.abs() * UB + 2.0 ** -134 if dtype == "bf16" else grad.abs() * U) + 1e-44)


# ------------------------------------------------- calls, streams, graphs

def test_calls_through_torchs_public_stream_functions(monkeypatch):
    """What the functions fall back to where torch has no others: the same stream."""
    monkeypatch.setattr(ops, "_current_device", torch.cuda.current_device)
    monkeypatch.setattr(ops, "_current_stream", lambda d: torch.cuda.current_stream(d).cuda_stream)
    x = rnd(6, 40, 100).cuda()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        kept = ops.checkpoint_store(x)
    other.synchronize()
    monkeypatch.undo()
    assert torch.equal(kept[:, :33 * 4], ops.checkpoint_store(x)[:, :33 * 4])


def state(dtype):
    """A replica's tensors of sizes whose routing and whose bias gradient leave parts in a
    workspace, which another launch joins."""
    n = lambda i, *shape: rnd(10 + i, *shape, dtype=dtype).cuda()   # noqa: E731
    e = lambda *shape: torch.empty(*shape, dtype=ref.TORCH[dtype], device="cuda")   # noqa: E731
    s = {"table": n(0, 32, 3), "bias": e(3, 130, 1100), "logits": n(1, 600, 40),
         "counts": torch.empty(41, dtype=torch.int32, device="cuda"), "x": n(2, 600, 72),
         "dlogits": e(600, 40), "dbias": n(3, 2, 3, 130, 1100), "dtable": e(32, 3)}
    s["needs"] = (arplan.ar_route_workspace(600, 40, 2),
                  arplan.ar_position_bias_grad_workspace(dtype, 32, 2, 3, 130, 1100))
    assert min(s["needs"]) > 0
    s["spaces"] = (None, None)
    return s


def step(s, stream=None):
    on = {"stream": stream}
    bias = ops.position_bias(s["table"], 130, 1100, offset=970, causal=True, out=s["bias"], **on)
    ids, gates, counts, mass = ops.route(s["logits"], 2, normalize=True, counts=s["counts"],
                                         workspace=s["spaces"][0], **on)
    loss, dlogits = ops.balance(s["logits"], ids, counts, mass, normalize=True, dgates=gates,
                                grad=s["dlogits"], **on)
    x = ops.checkpoint_load(ops.checkpoint_store(s["x"], **on), 72, s["x"].dtype, **on)
    dtable = ops.position_bias_grad(s["dbias"], s["dtable"], offset=970, causal=True,
                                    workspace=s["spaces"][1], **on)
    return bias, ids, gates, counts, mass, loss, dlogits, x, dtable


def copies(got):
    return [t.clone() for t in got]


def checked(got, want):
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a, b), i


def test_a_step_of_several_blocks_against_definitions():
    """The step that the tests below repeat, against 64 bits."""
    s = state("f32")
    bias, ids, gates, counts, mass, loss, dlogits, x, dtable = step(s)
    assert torch.equal(bias.cpu(), ref.position_bias(s["table"].cpu(), 130, 1100, 970, 128, True))
    want = ref.route(s["logits"].cpu(), 2, None, True)
    assert torch.equal(ids.cpu(), want[0]) and torch.equal(counts.cpu().long(), want[2])
    near(gates, want[1], want[1] * (2 * (40 + 12) + 6) * U)
    near(mass, want[3], want[3] * (40 + 16 + 600) * U)
    total, grad, size = ref.balance(s["logits"].cpu(), want[0], want[2], mass.cpu(), 0.01, True, gates.cpu())
    assert abs(float(loss) - total) <= 8 * U * total
    near(dlogits, grad, size * (3 * (40 + 16) + 4 + 16) * U + grad.abs() * U + 1e-36)
    want, size = ref.position_bias_grad(s["dbias"].cpu(), 32, 970, 128, True)
    # a lane's additions: rows of both batches; those over the wavefronts, the diagonals, the lanes
    # and the slots' join, at most 64 of each
    near(dtable, want, size * (2 * 64 + 4 * 64) * U + want.abs() * U)
    values = ref.fetched(*ref.kept(s["x"].cpu()), 72)
    assert torch.equal(x.cpu().double(), values)


@pytest.mark.parametrize("given", (False, True))
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_step_of_several_blocks_captured_and_replayed(dtype, given):
    """Two graphs of it, with workspaces of their own or sharing given ones, replayed in turn with
    the program's own work between the replays; inputs change."""
    s = state(dtype)
    if given:
        s["spaces"] = tuple(torch.full((n + 64,), 255, dtype=torch.uint8, device="cuda") for n in s["needs"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(s)
    torch.cuda.current_stream().wait_stream(side)
    graphs, got = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            got.append(step(s))
    fresh = state(dtype)
    for i in range(5):
        for k in ("x", "logits", "dbias", "table"):
            s[k].copy_(fresh[k] * (1.0 if i % 2 else 0.5))
        eager = copies(step(s))
        for g, out in zip(graphs, got):
            for t in out:
                t.zero_()
            if given:
                for w in s["spaces"]:
                    w.fill_(255)
            g.replay()
            torch.cuda.synchronize()
            checked(out, eager)
            for w, n in zip(s["spaces"], s["needs"]) if given else ():
                assert bool((w[n:] == 255).all()) and not bool((w[:n] == 255).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_step_of_several_blocks_on_another_stream(dtype):
    s = state(dtype)
    want = copies(step(s))
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for t in want:
        t.record_stream(other)
    got = step(s, other)
    other.synchronize()
    checked(got, want)


def test_steps_of_several_blocks_on_two_streams_at_once():
    a, b = state("bf16"), state("f32")
    want = [copies(step(s)) for s in (a, b)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(5):
        for i, s in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i] = copies(step(s))
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        checked(x, y)


@pytest.mark.parametrize("dtype", DTYPES)
def test_given_workspaces_of_several_blocks(dtype):
    """The bytes that were asked for and no others are written, and what they held has no effect;
    one byte less is refused."""
    s = state(dtype)
    want = copies(step(s))
    rooms = [torch.full((n + 64,), 255, dtype=torch.uint8, device="cuda") for n in s["needs"]]
    s["spaces"] = tuple(r[:n] for r, n in zip(rooms, s["needs"]))
    checked(step(s), want)
    for r, n in zip(rooms, s["needs"]):
        assert bool((r[n:] == 255).all()) and not bool((r[:n] == 255).all())
    with pytest.raises(arplan.ArError):
        ops.route(s["logits"], 2, workspace=rooms[0][:s["needs"][0] - 1])
    with pytest.raises(arplan.ArError):
        ops.position_bias_grad(s["dbias"], s["dtable"], workspace=rooms[1][:s["needs"][1] - 1])


# ------------------------------------------------- activations in 8 bits

@pytest.mark.parametrize("as_dtype", DTYPES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N", [(1, 1), (2, 33), (5, 31), (3, 4100), (200, 40), (33, 1001)])
def test_runs_of_nan_into_strided_rows(M, N, dtype, as_dtype):
    """Runs with NaN and infinities, loaded to an odd element of wider rows, and nothing beside
    them."""
    x = rnd(8, M, N)
    g = torch.Generator().manual_seed(9)
    x[torch.rand(M, N, generator=g) < 0.02] = math.nan
    x[torch.rand(M, N, generator=g) < 0.02] = -math.inf
    x[-1, -1] = math.inf
    x = x.to(ref.TORCH[dtype])
    want = ref.fetched(*ref.kept(x), N)
    assert bool(want.isnan().any())
    around = torch.full((M + 1, N + 5), 7.0, dtype=ref.TORCH[as_dtype], device="cuda")
    ops.checkpoint_load(ops.checkpoint_store(x.cuda()), N, out=around[:M, 3:3 + N])
    got = around[:M, 3:3 + N].cpu().double()
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))
    around[:M, 3:3 + N] = 7.0
    assert bool((around == 7.0).all()), "elements around the output were written"


@pytest.mark.parametrize("M,D,F", [(70, 90, 110), (300, 200, 515), (1, 64, 40), (777, 130, 64)])
def test_glu_gradients_from_8_bits_lose_the_rounding_of_dg_and_du_alone(M, D, F):
    """bf16: 64-bit products of dg and du, each rounded to bf16 once as the matrices are (before
    that they are exact: 8 bits times 7), up to fp32 sums and the result's own rounding."""
    x, wg, wu, dh = (rnd(20 + i, *s, dtype="bf16") for i, s in
                     enumerate(((M, D), (F, D), (F, D), (M, F))))
    factors = [rnd(24 + i, M, F) for i in range(2)]
    saved = torch.stack([ops.checkpoint_store(f.cuda()) for f in factors])
    dg, du = ((dh.double() * ref.fetched(*ref.kept(f), F)).float().bfloat16().double() for f in factors)
    X, G, W = x.double(), wg.double(), wu.double()
    got = ops.glu_backward(dh.cuda(), x.cuda(), wg.cuda(), wu.cuda(), saved)
    for out, want, size, n in ((got[0], dg @ G + du @ W, dg.abs() @ G.abs() + du.abs() @ W.abs(), 2 * F),
                               (got[1], dg.T @ X, dg.T.abs() @ X.abs(), M),
                               (got[2], du.T @ X, du.T.abs() @ X.abs(), M)):
        near(out, want, size * (n + 2) * U + want.abs() * UB + 1e-38)
