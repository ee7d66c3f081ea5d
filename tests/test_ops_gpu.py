"""The replica operators on the GPU against plain definitions in 64 bits."""

import math

import pytest
import torch

import ops_reference as ref
from gpu_helpers import say

arplan = pytest.importorskip(
    "paper_2409_04202_amd.arplan",
    reason="HIP library not built (run python -m paper_2409_04202_amd.build)")
from paper_2409_04202_amd import ops  # noqa: E402

pytestmark = pytest.mark.gpu
DTYPES = ("f32", "bf16")


def rnd(seed, *shape, dtype="f32", scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(ref.TORCH[dtype])


def laid(x, layout):
    """x on the GPU: its rows adjacent ("rows"), or inside a wider matrix of
    other values, at an odd element ("wide")."""
    if layout == "rows" or x.numel() == 0:
        return x.cuda()
    r, c = x.shape
    m = torch.full((r, c + 5), float("nan"), dtype=x.dtype, device="cuda")
    m[:, 3:3 + c] = x.cuda()
    return m[:, 3:3 + c]


def room(rows, cols, dtype, layout):
    """An output like that, and a check that nothing around it was written."""
    if layout == "rows":
        return torch.full((rows, cols), 7.0, dtype=ref.TORCH[dtype], device="cuda"), lambda: None
    m = torch.full((rows + 1, cols + 5), 7.0, dtype=ref.TORCH[dtype], device="cuda")

    def check():
        m[:rows, 3:3 + cols] = 7.0
        assert bool((m == 7.0).all()), "elements around the output were written"
    return m[:rows, 3:3 + cols], check


def ids_of(seed, T, V, kind):
    g = torch.Generator().manual_seed(seed)
    if kind == "one":
        return torch.full((T,), V // 2, dtype=torch.int64)
    if kind == "none":
        return torch.randint(0, 2, (T,), generator=g) * (V + 5) - 3
    u = torch.rand(T, generator=g).double()
    ids = (torch.exp(u * math.log(V)).long() - 1).clamp(0, V - 1)
    if kind == "edges":
        far = torch.tensor([-1, V, -2 ** 63, 2 ** 63 - 1, 2 ** 32, V - 1, 0, 2 ** 32 + 1])
        pick = torch.randint(0, 16, (T,), generator=g)
        ids = torch.where(pick < 8, far[pick.clamp(max=7)], ids)
    return ids


# ------------------------------------------------------------- embedding

@pytest.mark.parametrize("layout", ("rows", "wide"))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,V,D,kind", [
    (1, 7, 64, "zipf"), (5, 1, 1, "edges"), (300, 130, 513, "edges"), (64, 1000, 8, "none"),
    (33, 257, 2051, "zipf")])
def test_embed_lookup(T, V, D, kind, dtype, layout):
    table, ids = rnd(1, V, D, dtype=dtype), ids_of(2, T, V, kind)
    out, check = room(T, D, dtype, layout)
    ops.embed_lookup(laid(table, layout), ids.cuda(), scale=1.7, out=out)
    assert torch.equal(out.cpu(), ref.embed_lookup(table, ids, 1.7))
    check()


@pytest.mark.parametrize("accumulate", (False, True))
@pytest.mark.parametrize("layout", ("rows", "wide"))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,V,D,kind", [
    (1, 7, 64, "zipf"), (0, 5, 9, "zipf"), (31, 1, 3, "one"), (32, 3, 16, "one"),
    (33, 3, 16, "one"), (700, 300, 257, "edges"), (1000, 9, 40, "zipf"), (64, 1000, 8, "none"),
    (4097, 70001, 24, "zipf"), (9000, 2, 12, "zipf"), (16384, 300000, 4, "zipf"),
    (16385, 511, 9, "zipf"), (20011, 400, 16, "zipf"), (16383, 512, 5, "one"),
    (40000, 100000, 8, "edges")])
def test_embed_grad(T, V, D, kind, dtype, layout, accumulate):
    dout, ids = rnd(3, T, D, dtype=dtype), ids_of(4, T, V, kind)
    out, check = room(V, D, dtype, layout)
    old = out.cpu() if accumulate else None
    ops.embed_grad(laid(dout, layout), ids.cuda(), out, scale=0.37, accumulate=accumulate)
    got = out.cpu()
    assert torch.equal(got, ref.embed_grad(dout, ids, V, 0.37, arplan.AR_EMBED_RUN, old))
    if not accumulate:
        want, e = ref.embed_grad64(dout, ids, V, 0.37)
        ref.compare("gradient", got, want, e + ref.stored(want, dtype))
    check()


def test_embed_far_rows():
    """Offsets beyond 32 bits, in elements and in bytes."""
    V, D = 1100000, 4096
    table = torch.empty(V, D, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([0, V - 1, 600000, V - 2, V - 1])
    for i in set(ids.tolist()):
        table[i] = rnd(i, 1, D, dtype="bf16")[0].cuda()
    out = ops.embed_lookup(table, ids.cuda(), scale=2.0)
    for t, i in enumerate(ids.tolist()):
        assert torch.equal(out[t].cpu(), (rnd(i, 1, D, dtype="bf16")[0].float() * 2).bfloat16())
    dout = rnd(9, 5, D, dtype="bf16")
    ops.embed_grad(dout.cuda(), ids.cuda(), table, scale=1.0, accumulate=True)
    want = (dout[1].float() + dout[4].float()) + rnd(V - 1, 1, D, dtype="bf16")[0].float()
    assert torch.equal(table[V - 1].cpu(), want.bfloat16())
    want = dout[2].float() + rnd(600000, 1, D, dtype="bf16")[0].float()
    assert torch.equal(table[600000].cpu(), want.bfloat16())


def test_embed_grad_is_the_lookups_derivative():
    """Against central differences of <lookup, dout> in the table."""
    T, V, D = 19, 6, 5
    table, dout, ids = rnd(1, V, D).double(), rnd(2, T, D), ids_of(3, T, V, "edges")
    out = torch.empty(V, D, device="cuda")
    got = ops.embed_grad(dout.cuda(), ids.cuda(), out, scale=1.5).cpu().double()
    ok = (ids >= 0) & (ids < V)

    def value(tab):
        return float((1.5 * tab[ids[ok]] * dout[ok].double()).sum())
    for v in range(V):
        for d in range(D):
            e = torch.zeros(V, D).double()
            e[v, d] = 1e-3
            diff = (value(table + e) - value(table - e)) / 2e-3
            assert abs(diff - float(got[v, d])) < 1e-5


# ------------------------------------------------------ gated feed-forward

GLU_SIZES = [
    (1, 64, 128), (1, 1, 1), (2, 8, 16), (3, 100, 37), (16, 256, 512), (17, 264, 200),
    (33, 129, 65), (64, 64, 64), (65, 1000, 130), (130, 72, 300), (256, 512, 256),
    (300, 333, 515), (257, 520, 776)]


@pytest.mark.parametrize("layout", ("rows", "wide"))
@pytest.mark.parametrize("act", ("silu", "gelu"))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,D,F", GLU_SIZES)
def test_glu(M, D, F, dtype, act, layout):
    x, wg = rnd(1, M, D, dtype=dtype), rnd(2, F, D, dtype=dtype, scale=D ** -0.5)
    wu, dh = rnd(3, F, D, dtype=dtype, scale=D ** -0.5), rnd(4, M, F, dtype=dtype)
    h, dx, dwg, dwu = ref.glu(x, wg, wu, act, dh, dtype)
    gx, gg, gu, gd = (laid(t, layout) for t in (x, wg, wu, dh))
    out, check = room(M, F, dtype, layout)
    ops.glu_forward(gx, gg, gu, act=act, out=out)
    ref.compare("h", out, *h)
    alone = out.clone()
    check()
    got, saved = ops.glu_forward(gx, gg, gu, act=act, save=True)
    ref.compare("h", got, *h)
    if M > 16:
        assert torch.equal(alone, got)
    (ox, c0), (og, c1), (ou, c2) = (room(r, D, dtype, layout) for r in (M, F, F))
    ops.glu_backward(gd, gx, gg, gu, saved, dx=ox, dwg=og, dwu=ou)
    for name, o, w in (("dx", ox, dx), ("dwg", og, dwg), ("dwu", ou, dwu)):
        ref.compare(name, o, *w)
    first = [t.clone() for t in (ox, og, ou)]
    # once more, adding: the sum's own rounding on top
    ops.glu_backward(gd, gx, gg, gu, saved, dx=ox, dwg=og, dwu=ou, accumulate=True)
    assert torch.equal(ox, first[0])
    for name, o, w, f in (("dwg", og, dwg, first[1]), ("dwu", ou, dwu, first[2])):
        v = w[0] + f.double().cpu()
        ref.compare(name + " added", o, v, w[1] + ref.stored(v, dtype))
    for c in (c0, c1, c2):
        c()


@pytest.mark.parametrize("layout", ("rows", "wide"))
@pytest.mark.parametrize("act", ("silu", "gelu"))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,F", [(1, 5), (7, 33), (513, 100), (2500, 67), (4104, 130)])
@pytest.mark.parametrize("M", (2, 3, 4, 5, 6, 7, 8, 9))
def test_glu_few_rows(M, D, F, dtype, act, layout):
    """Every number of rows that takes the weights in whole rows, and one more:
    lanes with nothing, one vector and several, an odd last feature."""
    test_glu(M, D, F, dtype, act, layout)


GLU_EXACT = [
    (1, 1, 1), (8, 2051, 37), (9, 72, 64), (20, 3000, 70), (70, 130, 2500), (1500, 65, 130),
    (130, 2, 67), (5000, 65, 9), (2309, 5800, 40), (50, 3849, 3081), (203, 133, 301),
    (645, 1319, 2731), (777, 1003, 2731), (1290, 1500, 5380), (1531, 264, 520), (2050, 504, 520),
    (600, 1003, 1000)]


def whole(seed, *shape, far=2):
    """Whole numbers up to ``far`` in magnitude."""
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-far, far + 1, shape, generator=g).double()


@pytest.mark.parametrize("layout", ("rows", "wide"))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,D,F", GLU_EXACT)
def test_glu_products_are_exact(M, D, F, dtype, layout):
    """On small whole numbers every product and sum is exact in fp32 (the largest
    sum, of 2 F terms up to 8, stays below 2^24), the factors in bf16 too: each
    result is the exact one rounded once, and a term lost, or added twice, at
    any place of a sum shows."""
    dt = ref.TORCH[dtype]
    x, wg, wu, dh = whole(1, M, D), whole(2, F, D), whole(3, F, D), whole(4, M, F)
    sg, su = whole(5, M, F), whole(6, M, F)
    dg, du = dh * sg, dh * su
    gpu = lambda t: laid(t.to(dt), layout)  # noqa: E731
    gx, gg, gu, gd = (gpu(t) for t in (x, wg, wu, dh))
    for kind in {torch.float32, dt}:
        saved = torch.stack((sg, su)).to(kind).cuda()
        (ox, c0), (og, c1), (ou, c2) = (room(r, D, dtype, layout) for r in (M, F, F))
        og.copy_(whole(7, F, D))
        ou.copy_(whole(8, F, D))
        for add in (True, False):   # (first onto whole numbers)
            ops.glu_backward(gd, gx, gg, gu, saved, dx=ox, dwg=og, dwu=ou, accumulate=add)
            assert torch.equal(ox.cpu(), (dg @ wg + du @ wu).to(dt))
            for i, (o, d) in enumerate(((og, dg), (ou, du))):
                want = d.t() @ x + (whole(7 + i, F, D) if add else 0)
                assert torch.equal(o.cpu(), want.to(dt)), (i, add)
        for c in (c0, c1, c2):
            c()
    # the forward: a(g) is g for gates this large, and the other projection 1
    x[:, 0] = 1
    far, one = wg.clone(), torch.zeros(F, D).double()
    far[:, 0], one[:, 0] = 4096, 1
    x[:, 1:] = x[:, 1:].clamp(-1, 1)
    out, check = room(M, F, dtype, layout)
    ops.glu_forward(gpu(x), gpu(far), gpu(one), out=out)
    g = x @ far.t()
    assert bool((g > 64).all())
    assert torch.equal(out.cpu(), g.to(dt))
    gate = one * 64
    out.fill_(7.0)
    ops.glu_forward(gpu(x), gpu(gate), gpu(wu), out=out)
    assert torch.equal(out.cpu(), (64 * (x @ wu.t())).to(dt))
    check()


@pytest.mark.parametrize("layout", ("rows", "wide"))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,D,F", [(20, 3000, 70), (70, 130, 2500), (1500, 65, 130), (130, 2, 67),
                                   (5000, 65, 9), (3, 2049, 4097)])
def test_glu_long_sums(M, D, F, dtype, layout):
    """Products of few tiles and long sums, which are split, and of a few
    columns beyond a tile."""
    test_glu(M, D, F, dtype, "gelu", layout)


@pytest.mark.parametrize("dtype", DTYPES)
def test_glu_rows_within_a_matrix(dtype):
    """Row strides at 16 bytes with widths that are not: the last chunk of a
    row is incomplete, and what follows it in memory is NaN."""
    M, D, F = 203, 133, 301
    x, wg = rnd(1, M, D, dtype=dtype), rnd(2, F, D, dtype=dtype, scale=D ** -0.5)
    wu, dh = rnd(3, F, D, dtype=dtype, scale=D ** -0.5), rnd(4, M, F, dtype=dtype)
    want = ref.glu(x, wg, wu, "silu", dh, dtype)

    def inside(t):
        m = torch.full((t.shape[0], -(-t.shape[1] // 16) * 16 + 16), float("nan"), dtype=t.dtype,
                       device="cuda")
        m[:, :t.shape[1]] = t.cuda()
        return m[:, :t.shape[1]]
    x, wg, wu, dh = (inside(t) for t in (x, wg, wu, dh))
    h, saved = ops.glu_forward(x, wg, wu, save=True)
    got = (h,) + ops.glu_backward(dh, x, wg, wu, saved)
    for name, g, w in zip(("h", "dx", "dwg", "dwu"), got, want):
        ref.compare(name, g, *w)
    more = ops.glu_backward(dh, x, wg, wu, saved, dwg=got[2], dwu=got[3], accumulate=True)
    for name, g, w in zip(("dwg", "dwu"), more[1:], want[2:]):
        ref.compare(name, g, 2 * w[0], 2 * w[1] + ref.stored(2 * w[0], dtype))


@pytest.mark.parametrize("layout", ("rows", "wide"))
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,D,F", [(2050, 72, 3000), (2309, 5800, 40), (50, 3849, 3081)])
def test_glu_many_tiles(M, D, F, dtype, layout):
    """Products of so many tiles that the largest ones are taken: h's, dx's and
    the weight gradients', in turn."""
    test_glu(M, D, F, dtype, "silu", layout)


@pytest.mark.parametrize("layout", ("rows", "wide"))
@pytest.mark.parametrize("dtype,M,D,F", [
    ("f32", 777, 1003, 2731), ("f32", 700, 520, 1000), ("f32", 785, 1299, 323),
    ("bf16", 645, 1319, 2731), ("bf16", 1273, 1177, 1621), ("bf16", 1290, 1500, 5380)])
def test_glu_uneven_tiles(dtype, M, D, F, layout):
    """Some tiles more than whole rounds of the card: whole ones first, and the
    others split."""
    test_glu(M, D, F, dtype, "silu", layout)


@pytest.mark.parametrize("which", ("x", "weights", "both"))
@pytest.mark.parametrize("M,D,F", [(800, 1024, 776), (2050, 520, 776)])
def test_glu_views_of_a_flat_vector(M, D, F, which):
    """Whole vectors wide, but at an odd place of a flat vector: the same bits as
    at 16 bytes, and the definition's values."""
    x, wg = rnd(1, M, D, dtype="bf16"), rnd(2, F, D, dtype="bf16", scale=D ** -0.5)
    wu, dh = rnd(3, F, D, dtype="bf16", scale=D ** -0.5), rnd(4, M, F, dtype="bf16")
    want = ref.glu(x, wg, wu, "silu", dh, "bf16")

    def odd(t):
        v = torch.full((t.numel() + 6,), float("nan"), dtype=t.dtype, device="cuda")
        v[3:3 + t.numel()] = t.flatten().cuda()
        return v[3:3 + t.numel()].view(t.shape)
    gx, gg, gu, gd = (t.cuda() for t in (x, wg, wu, dh))
    ox = gx if which == "weights" else odd(x)
    og, ou = (gg, gu) if which == "x" else (odd(wg), odd(wu))
    h, saved = ops.glu_forward(gx, gg, gu, save=True)
    even = (h, saved) + ops.glu_backward(gd, gx, gg, gu, saved)
    h, saved = ops.glu_forward(ox, og, ou, save=True)
    got = (h, saved) + ops.glu_backward(gd, ox, og, ou, saved)
    for a, b in zip(got, even):
        assert torch.equal(a, b)
    for name, g, w in zip(("h", "dx", "dwg", "dwu"), (got[0],) + got[2:], want):
        ref.compare(name, g, *w)


@pytest.mark.parametrize("M,D,F", [(65, 130, 129), (200, 4000, 70)])
def test_glu_compact_factors(M, D, F):
    """Factors saved in bf16, half of the memory: within the bound, which
    allows them a rounding, and the same where nothing is rounded by it."""
    x, wg = rnd(1, M, D, dtype="bf16"), rnd(2, F, D, dtype="bf16", scale=D ** -0.5)
    wu, dh = rnd(3, F, D, dtype="bf16", scale=D ** -0.5), rnd(4, M, F, dtype="bf16")
    want = ref.glu(x, wg, wu, "silu", dh, "bf16")
    x, wg, wu, dh = (t.cuda() for t in (x, wg, wu, dh))
    h, saved = ops.glu_forward(x, wg, wu, save=torch.bfloat16)
    _, full = ops.glu_forward(x, wg, wu, save=True)
    assert saved.dtype == torch.bfloat16 and full.dtype == torch.float32
    assert torch.equal(saved, full.bfloat16())
    got = (h,) + ops.glu_backward(dh, x, wg, wu, saved)
    for name, g, w in zip(("h", "dx", "dwg", "dwu"), got, want):
        ref.compare(name, g, *w)
    for a, b in zip(ops.glu_backward(dh, x, wg, wu, saved.float()), got[1:]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES)
def test_glu_empty(dtype):
    dt = ref.TORCH[dtype]
    e = lambda *s: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    assert ops.glu_forward(e(0, 8), e(4, 8), e(4, 8)).shape == (0, 4)
    # an empty sum: g = u = 0
    h, saved = ops.glu_forward(e(3, 0), e(4, 0), e(4, 0), save=True)
    assert bool((h == 0).all())
    dwg, dwu = e(4, 8) + 5, e(4, 8) + 5
    ops.glu_backward(e(0, 4), e(0, 8), e(4, 8), e(4, 8), e(2, 0, 4), dwg=dwg, dwu=dwu,
                     accumulate=True)
    assert bool((dwg == 5).all()) and bool((dwu == 5).all())
    ops.glu_backward(e(0, 4), e(0, 8), e(4, 8), e(4, 8), e(2, 0, 4), dwg=dwg, dwu=dwu)
    assert bool((dwg == 0).all()) and bool((dwu == 0).all())
    dx, _, _ = ops.glu_backward(e(3, 0), e(3, 8), e(0, 8), e(0, 8), e(2, 3, 0))
    assert bool((dx == 0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ("silu", "gelu"))
@pytest.mark.parametrize("M", (1, 40))
def test_glu_extremes(M, act, dtype):
    """Gates at the ends of the range: the activation's limits, no NaN; and a
    NaN or an infinity stays in its own row."""
    D, F = 8, 48
    x = torch.zeros(M, D)
    x[:, 0] = 1
    wg, wu = torch.zeros(F, D), torch.zeros(F, D)
    wg[:, 0] = torch.tensor([0.0, 1e30, -1e30, 200.0, -200.0, 50.0, -50.0, -88.0] * 6)
    wu[:, 0] = 1
    x, wg, wu = (t.to(ref.TORCH[dtype]) for t in (x, wg, wu))
    h, saved = ops.glu_forward(x.cuda(), wg.cuda(), wu.cuda(), act=act, save=True)
    g = wg[:, 0].double()
    a, da = ref.activate(act, g)
    a, da = torch.where(a.isnan(), 0.0, a), torch.where(da.isnan(), (g > 0).double(), da)
    for name, got, want in (("h", h, a), ("a", saved[1], a), ("a'", saved[0], da)):
        want = want[None, :].expand(M, F)
        ref.compare(name, got, want, want.abs() * 2.0 ** -8 + 1e-30)
    if M > 1:
        y = x.clone()
        y[3, 5], y[7, 2] = float("nan"), float("inf")
        h2 = ops.glu_forward(y.cuda(), wg.cuda(), wu.cuda(), act=act)
        keep = [r for r in range(M) if r not in (3, 7)]
        assert torch.equal(h2[keep], h[keep]) and bool(h2[3].isnan().all())


@pytest.mark.parametrize("M", (5, 40))
@pytest.mark.parametrize("act", ("silu", "gelu"))
def test_glu_activations_in_their_tails(M, act):
    """fp32, gates from -12 to 12 that are exact, against 64 bits and relative to
    the value: an argument off by a unit moves the tail of the normal
    distribution by g^2 units, and the functions are off by some tens of units of
    their own.  The slope, which has a zero, relative to its two terms."""
    F = 4801
    g = torch.linspace(-12, 12, F).double().float()
    x, wg, wu = torch.zeros(M, 3), torch.zeros(F, 3), torch.zeros(F, 3)
    x[:, 1], wg[:, 1], wu[:, 1] = 1, g, 1
    h, saved = ops.glu_forward(x.cuda(), wg.cuda(), wu.cuda(), act=act, save=True)
    g = g.double()
    value, slope = ref.activate(act, g)
    if act == "silu":
        s = torch.sigmoid(g)
        terms = s * (1 + (g * torch.sigmoid(-g)).abs())
        slope = s * (1 + g * torch.sigmoid(-g))
    else:
        pdf = torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        terms = 0.5 * torch.special.erfc(-g / math.sqrt(2.0)) + g.abs() * pdf
    rel = (64 + 4 * g * g) * ref.U
    for name, got, want, size in (("h", h, value, value.abs()), ("a", saved[1], value, value.abs()),
                                  ("a'", saved[0], slope, terms)):
        ref.compare(name, got, want[None, :].expand(M, F), (rel * size)[None, :].expand(M, F))


def test_glu_gradients_are_derivatives():
    """Against central differences of <h, dh> in 64 bits."""
    M, D, F = 5, 4, 3
    for act in ("silu", "gelu"):
        args = [rnd(i, *s) for i, s in enumerate(((M, D), (F, D), (F, D)))]
        dh = rnd(9, M, F)
        _, saved = ops.glu_forward(*(a.cuda() for a in args), act=act, save=True)
        got = ops.glu_backward(dh.cuda(), *(a.cuda() for a in args), saved)

        def value(x, wg, wu):
            return float((ref.activate(act, x @ wg.t())[0] * (x @ wu.t()) * dh.double()).sum())
        for i, a in enumerate(args):
            for j in range(a.numel()):
                e = torch.zeros(a.numel()).double()
                e[j] = 1e-4
                lo, hi = [b.double() for b in args], [b.double() for b in args]
                lo[i], hi[i] = lo[i] - e.view(a.shape), hi[i] + e.view(a.shape)
                diff = (value(*hi) - value(*lo)) / 2e-4
                assert abs(diff - float(got[i].flatten()[j])) < 2e-5


def test_glu_side_by_side():
    """Both weight gradients as columns of one wider matrix."""
    M, D, F = 40, 24, 56
    x, wg, wu, dh = (rnd(i, *s).cuda() for i, s in enumerate(((M, D), (F, D), (F, D), (M, F))))
    _, saved = ops.glu_forward(x, wg, wu, save=True)
    _, a, b = ops.glu_backward(dh, x, wg, wu, saved)
    both = torch.empty(F, 2 * D, device="cuda")
    ops.glu_backward(dh, x, wg, wu, saved, dwg=both[:, :D], dwu=both[:, D:])
    assert torch.equal(both, torch.cat((a, b), 1))


# ----------------------------------------------------------- distillation

def teacher_of(seed, T, V, K, repeat=False):
    g = torch.Generator().manual_seed(seed)
    if repeat:
        ids = torch.randint(0, max(1, V // 2), (T, K), generator=g)
    else:
        ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)]) if T else \
            torch.zeros(0, K, dtype=torch.int64)
    return ids, torch.randn(T, K, generator=g) * 3


@pytest.mark.parametrize("layout", ("rows", "wide"))
@pytest.mark.parametrize("dtype,tdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"),
                                          ("f32", "bf16")])
@pytest.mark.parametrize("T,V,K,tau", [
    (1, 1, 1, 1.0), (3, 7, 7, 2.0), (5, 1000, 20, 1.0), (4, 4099, 64, 4.0), (2, 65536, 10, 0.5),
    (9, 33001, 1, 1.0), (3, 140001, 33, 2.0), (300, 513, 8, 1.0)])
def test_distill(T, V, K, tau, dtype, tdtype, layout):
    z = rnd(1, T, V, dtype=dtype, scale=4.0)
    ids, tea = teacher_of(2, T, V, K)
    tea = tea.to(ref.TORCH[tdtype])
    wt = torch.rand(T, generator=torch.Generator().manual_seed(3))
    (loss, el), (grad, eg) = ref.distill(z, tea, ids, tau, wt, dtype)
    gz, gt, gi, gw = laid(z, layout), laid(tea, layout), ids.cuda(), wt.cuda()
    ref.compare("loss", ops.distill(gz, gt, gi, temperature=tau, weights=gw), loss, el)
    out, check = room(T, V, dtype, layout)
    got, g = ops.distill(gz, gt, gi, temperature=tau, weights=gw, grad=out)
    ref.compare("loss", got, loss, el)
    ref.compare("gradient", g, grad, eg)
    there = g.clone()
    check()
    # in place
    ops.distill(gz, gt, gi, temperature=tau, weights=gw, grad=gz)
    assert torch.equal(gz, there)


@pytest.mark.parametrize("V,copies", [(2051, 1), (2051, 13), (20011, 1), (20011, 13), (70001, 13)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_distill_masks(dtype, V, copies):
    """Every kind of mask, in few rows and in many."""
    inf, nan, low = float("inf"), float("nan"), torch.finfo(ref.TORCH[dtype]).min
    T, K = 16, 6
    z = rnd(1, T, V, dtype=dtype, scale=3.0)
    ids, tea = teacher_of(2, T, V, K)
    w = torch.ones(T)
    w[0] = 0
    z[0], tea[0, 1] = nan, nan                      # weight 0: whatever it holds
    ids[1] = torch.tensor([-1, V, 2 ** 40, -2 ** 63, V + 1, -7])   # no entry
    z[1, 5] = nan
    tea[2] = -inf                                   # no entry either
    z[3] = -inf                                     # no logit
    z[4] = low                                      # the mask's value throughout: uniform
    z[5], z[5, :3] = low, z[6, :3]                  # three logits left
    ids[5] = torch.tensor([0, 1, 2, -1, -1, -1])
    z[6, ids[6, 0]] = -inf                          # the student excludes an entry
    z[7, ids[7, 0]], tea[7, 0] = -inf, -inf         # that the teacher excludes too
    tea[8] = low                                    # entries at the lowest value: uniform
    tea[9, 1:] = low
    z[10, 7] = nan
    z[11, 7] = inf
    tea[12, 2] = nan
    ids[13, 1:] = ids[13, 0]                        # one id in every entry
    ids[14, 3] = ids[14, 1]
    z[15, 1000:] = -inf
    ids[15] = torch.tensor([5, 2, 999, -1, 0, 1])
    (loss, el), (grad, eg) = ref.distill(z, tea.to(ref.TORCH[dtype]), ids, 1.3, w, dtype)
    assert bool(loss[6] == inf) and bool(grad[6].isfinite().all())
    assert bool(loss[10].isnan()) and bool(loss[11].isnan()) and bool(loss[12].isnan())
    args = [x.cuda().repeat(copies, 1) for x in (z, tea.to(ref.TORCH[dtype]), ids)]
    weights = w.cuda().repeat(copies)
    got, g = ops.distill(*args, temperature=1.3, weights=weights,
                         grad=torch.empty(copies * T, V, dtype=z.dtype, device="cuda"))
    only = ops.distill(*args, temperature=1.3, weights=weights)
    assert torch.equal(only.nan_to_num(nan=-5.0), got.nan_to_num(nan=-5.0))
    bits = g.view(torch.int32 if dtype == "f32" else torch.int16).view(copies, T, V)
    assert bool((bits == bits[:1]).all())
    ops.distill(*args, temperature=1.3, weights=weights, grad=args[0])
    assert torch.equal(args[0].view(bits.dtype).view(bits.shape), bits)
    got, g = got[-T:], g[-T:]
    ref.compare("loss", got, loss, el)
    for t in range(T):
        if t != 12:     # (a NaN in the teacher: below)
            ref.compare("gradient of row %d" % t, g[t], grad[t], eg[t])
    at = ids[12][(ids[12] >= 0) & (ids[12] < V)]
    assert bool(g[12, at.cuda()].isnan().all())
    rest = torch.ones(V, dtype=torch.bool)
    rest[at] = False
    ref.compare("gradient beside a NaN entry", g[12].cpu()[rest], grad[12][rest],
                ref.stored(grad[12][rest], dtype) + 1e-5 * grad[12][rest])


@pytest.mark.parametrize("V,copies", [(2051, 1), (2051, 13), (20011, 1), (20011, 13), (70001, 13)])
@pytest.mark.parametrize("tau", (0.5, 1.0, 2.0))
@pytest.mark.parametrize("dtype", DTYPES)
def test_distill_entries_at_the_masks_value(V, copies, tau, dtype):
    """The student's logit at entries of the teacher is the type's lowest value:
    the loss is that far off, and finite in fp32."""
    T, K = 16, 6
    low = torch.finfo(ref.TORCH[dtype]).min
    z = rnd(1, T, V, dtype=dtype, scale=3.0)
    ids, tea = teacher_of(2, T, V, K)
    for t in range(T):
        z[t, ids[t, :1 + t % (K - 1)]] = low        # one to all but one
    w = torch.full((T,), 0.25)
    (loss, el), (grad, eg) = ref.distill(z, tea, ids, tau, w, dtype)
    assert bool((loss > 1e28).all()) and bool((loss < 3.4e38).all())
    # (the reference's bound leaves numbers of this size out: K terms, each off
    # by its probability's error, 6 units a unit of its logarithm, that is above
    # -45, and some roundings)
    el = loss * (K + 64 + 6 * 45) * ref.U
    args = [x.cuda().repeat(copies, 1) for x in (z, tea, ids)]
    got, g = ops.distill(*args, temperature=tau, weights=w.cuda().repeat(copies),
                         grad=torch.empty(copies * T, V, dtype=z.dtype, device="cuda"))
    ref.compare("loss", got, loss.repeat(copies), el.repeat(copies))
    for i in (0, copies - 1):
        ref.compare("gradient", g[i * T:(i + 1) * T], grad, eg)


@pytest.mark.parametrize("K", (6, 64, 65, 1500, 4096))
@pytest.mark.parametrize("dtype,V,T", [
    ("bf16", 2051, 9001), ("f32", 2051, 9001), ("bf16", 12001, 5000), ("f32", 6001, 5000),
    ("bf16", 20011, 2600), ("f32", 10007, 2600), ("bf16", 50021, 1300), ("f32", 20011, 1300),
    ("bf16", 100003, 650), ("f32", 50021, 650), ("bf16", 131072, 300), ("f32", 65536, 300)])
def test_distill_rows_in_turn(dtype, V, T, K):
    """More rows than blocks, so that each takes several in turn, at every size of
    a block: eleven rows of every kind over and over, whose successor within a
    block is another kind.  Every copy of a row has its bits."""
    inf, nan, low = float("inf"), float("nan"), torch.finfo(ref.TORCH[dtype]).min
    P = 11
    z = rnd(1, P, V, dtype=dtype, scale=3.0)
    ids, tea = teacher_of(2, P, V, K, repeat=K > V // 2)
    w = torch.rand(P, generator=torch.Generator().manual_seed(3)) + 0.1
    w[1], z[1] = 0, nan                             # weight 0, whatever it holds
    ids[2], z[2, 3] = -1, nan                       # no entry
    z[3] = -inf                                     # no logit
    z[4] = low                                      # the mask's value throughout
    z[6, V // 2] = inf
    z[7, 10:] = -inf                                # few logits left
    z[8, :V // 2] = -300                            # the maximum far from the first vectors
    z[9, :V // 2] = -30
    ids[10, K // 2:] = ids[10, 0]                   # one id many times
    tea = tea.to(ref.TORCH[dtype])
    (loss, el), (grad, eg) = ref.distill(z, tea, ids, 1.5, w, dtype)
    # a base that lies 30 below the maximum: differences of 30 log2(e) / 1.5 and
    # as large a logarithm of the sum, each off by a few units, against the 64
    # that the bound has for a row
    el[9], eg[9] = 4 * el[9], 4 * eg[9]
    n = -(-T // P)
    args = [x.cuda().repeat(n, 1)[:T].contiguous() for x in (z, tea, ids)]
    weights = w.cuda().repeat(n)[:T].contiguous()
    kind = torch.int32 if dtype == "f32" else torch.int16

    def copies_agree(loss, g):
        b = g.view(kind)
        for i in range(P, T, P):
            m = min(P, T - i)
            assert torch.equal(b[i:i + m], b[:m])
            assert torch.equal(loss[i:i + m].view(torch.int32), loss[:m].view(torch.int32))
    got, g = ops.distill(*args, temperature=1.5, weights=weights,
                         grad=torch.full((T, V), 7.0, dtype=z.dtype, device="cuda"))
    copies_agree(got, g)
    ref.compare("loss", got[:P], loss, el)
    for t in range(P):
        ref.compare("gradient of row %d" % t, g[t], grad[t], eg[t])
    only = ops.distill(*args, temperature=1.5, weights=weights)
    assert torch.equal(only.view(torch.int32), got.view(torch.int32))
    again, _ = ops.distill(*args, temperature=1.5, weights=weights, grad=args[0])
    assert torch.equal(args[0].view(kind), g.view(kind))
    assert torch.equal(again.view(torch.int32), got.view(torch.int32))


@pytest.mark.parametrize("tau", (arplan.AR_DISTILL_MIN_TEMPERATURE, 1e-20, 1e-3, 1e6,
                                 arplan.AR_DISTILL_MAX_TEMPERATURE))
@pytest.mark.parametrize("V,copies", [(2051, 1), (20011, 1), (20011, 64)])
def test_distill_temperatures(V, copies, tau):
    """The ends of the range: one logit takes all, and all the same."""
    T, K = 3, 6
    z, w = rnd(1, T, V, scale=3.0), torch.full((T,), 1e-2)
    ids, tea = teacher_of(2, T, V, K)
    (loss, el), (grad, eg) = ref.distill(z, tea, ids, tau, w, "f32")
    got, g = ops.distill(*(x.cuda().repeat(copies, 1) for x in (z, tea, ids)), temperature=tau,
                         weights=w.cuda().repeat(copies),
                         grad=torch.empty(copies * T, V, device="cuda"))
    ref.compare("loss", got, loss.repeat(copies), el.repeat(copies))
    ref.compare("gradient", g[-T:], grad, eg)


@pytest.mark.parametrize("K", (0, 1000, 4096))
def test_distill_numbers_of_entries(K):
    T, V = 3, 5003
    z = rnd(1, T, V)
    ids, tea = teacher_of(2, T, V, K, repeat=True)
    (loss, el), (grad, eg) = ref.distill(z, tea, ids, 1.0, None, "f32")
    got, g = ops.distill(z.cuda(), tea.cuda(), ids.cuda(), grad=torch.empty(T, V, device="cuda"))
    ref.compare("loss", got, loss, el)
    ref.compare("gradient", g, grad, eg)


def test_distill_gradient_is_the_losses_derivative():
    T, V, K = 3, 6, 4
    z, (ids, tea) = rnd(1, T, V), teacher_of(2, T, V, K, repeat=True)
    w = torch.tensor([1.0, 0.25, 2.0])
    _, g = ops.distill(z.cuda(), tea.cuda(), ids.cuda(), temperature=1.7, weights=w.cuda(),
                       grad=torch.empty(T, V, device="cuda"))
    for t in range(T):
        for j in range(V):
            e = torch.zeros(T, V).double()
            e[t, j] = 1e-4
            up = ref.distill(z.double() + e, tea, ids, 1.7, w, "f32")[0][0]
            down = ref.distill(z.double() - e, tea, ids, 1.7, w, "f32")[0][0]
            assert abs(float((up - down).sum()) / 2e-4 - float(g[t, j])) < 1e-5


def test_distill_far_rows():
    """Row offsets beyond 32 bits."""
    T, V, stride = 3, 1003, (1 << 31) + 11
    m = torch.empty(2 * stride + V, dtype=torch.bfloat16, device="cuda")
    far = m.as_strided((T, V), (stride, 1))
    z = rnd(1, T, V, dtype="bf16")
    far.copy_(z.cuda())
    ids, tea = teacher_of(2, T, V, 5)
    (loss, el), (grad, eg) = ref.distill(z, tea, ids, 1.0, None, "bf16")
    got, g = ops.distill(far, tea.cuda(), ids.cuda(), grad=far)
    ref.compare("loss", got, loss, el)
    ref.compare("gradient", g, grad, eg)


def test_distill_more_rows_than_a_pair_of_launches():
    """Long rows, over 4 GiB of them: every copy of a row has its bits."""
    T, V, K, copies = 5, (1 << 20) + 3, 7, 206
    z = rnd(1, T, V, scale=3.0)
    ids, tea = teacher_of(2, T, V, K)
    (loss, el), (grad, eg) = ref.distill(z, tea, ids, 2.0, None, "f32")
    big = z.cuda().repeat(copies, 1)
    got, g = ops.distill(big, tea.cuda().repeat(copies, 1), ids.cuda().repeat(copies, 1),
                         temperature=2.0, grad=big)
    ref.compare("loss", got[-T:], loss, el)
    ref.compare("gradient", g[-T:], grad, eg)
    assert torch.equal(got.view(copies, T), got[:T].expand(copies, T))
    assert all(torch.equal(g[i:i + T], g[:T]) for i in range(0, copies * T, T))


# ------------------------------------------------------ streams and graphs

def _pass(dtype="bf16"):
    """One pass through every operator on fixed buffers, as a function."""
    dt = ref.TORCH[dtype]
    T, V, D, F, K = 300, 1000, 128, 192, 8
    table, ids = rnd(1, V, D, dtype=dtype).cuda(), ids_of(2, T, V, "edges").cuda()
    wg, wu = (rnd(i, F, D, dtype=dtype, scale=D ** -0.5).cuda() for i in (3, 4))
    dh = rnd(5, T, F, dtype=dtype).cuda()
    tid, tea = teacher_of(6, T, F, K)
    tid, tea = tid.cuda(), tea.cuda()
    dtable = torch.empty(V, D, dtype=dt, device="cuda")

    def go(stream=None):
        x = ops.embed_lookup(table, ids, scale=3.0, stream=stream)
        h, saved = ops.glu_forward(x, wg, wu, save=True, stream=stream)
        loss, g = ops.distill(h, tea, tid, temperature=2.0, grad=torch.empty_like(h), stream=stream)
        dx, dwg, dwu = ops.glu_backward(dh, x, wg, wu, saved, stream=stream)
        ops.embed_grad(dx, ids, dtable, scale=3.0, stream=stream)
        return x, h, loss, g, dx, dwg, dwu, dtable
    return go, table


def test_ops_repeat_bit_for_bit_and_on_another_stream():
    go, _ = _pass()
    first = [t.clone() for t in go()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        out = go(side)
        side.synchronize()
        for a, b in zip(first, out):
            assert torch.equal(a, b)


def _tensors():
    """(function, arguments, the names of what it writes) of every operator."""
    M, D, F, V, K = 4, 8, 16, 32, 3
    e = lambda *s: rnd(1, *s).cuda()  # noqa: E731
    ids = torch.zeros(M, dtype=torch.int64, device="cuda")
    return [
        (ops.embed_lookup, dict(table=e(V, D), ids=ids, out=e(M, D)), ("out",)),
        (ops.embed_grad, dict(dout=e(M, D), ids=ids, dtable=e(V, D)), ("dtable",)),
        (ops.glu_forward, dict(x=e(M, D), wg=e(F, D), wu=e(F, D), out=e(M, F)), ("out",)),
        (ops.glu_backward, dict(dh=e(M, F), x=e(M, D), wg=e(F, D), wu=e(F, D), saved=e(2, M, F),
                                dx=e(M, D), dwg=e(F, D), dwu=e(F, D)), ("dx", "dwg", "dwu")),
        (ops.distill, dict(logits=e(M, V), teacher=e(M, K), ids=ids[:, None].repeat(1, K),
                           weights=e(M, 1)[:, 0].contiguous(), grad=e(M, V)), ("grad",))]


def test_tensors_that_require_a_gradient_are_refused():
    for f, args, _ in _tensors():
        for name, t in args.items():
            if not t.is_floating_point():
                continue
            t.requires_grad_()
            with pytest.raises(ValueError, match="gradient"):
                f(**args)
            with torch.no_grad():
                f(**args)
            t.requires_grad_(False)


def test_a_stream_of_another_device_is_refused():
    class Other:
        device, cuda_stream = torch.device("cuda", torch.cuda.device_count()), 0
    for f, args, _ in _tensors():
        with pytest.raises(ValueError, match="stream"):
            f(stream=Other(), **args)


def test_written_tensors_count_as_changed():
    for f, args, written in _tensors():
        before = {name: t._version for name, t in args.items()}
        f(**args)
        for name, t in args.items():
            assert (t._version > before[name]) == (name in written), (f.__name__, name)
    # an in-place gradient over logits that autograd has saved
    w = torch.ones(4, 32, device="cuda", requires_grad=True)
    logits = rnd(1, 4, 32).cuda()
    y = (w * logits).sum()
    ops.distill(logits, rnd(2, 4, 3).cuda(), torch.zeros(4, 3, dtype=torch.int64, device="cuda"),
                grad=logits)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_ops_in_a_graph():
    go, table = _pass()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        go()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = go()
    for i in range(3):
        table.copy_(rnd(20 + i, *table.shape, dtype="bf16"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = go()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        say("replay", i)
