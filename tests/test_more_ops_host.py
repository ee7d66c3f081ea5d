"""What position bias, routing, balance loss and activations in 8 bits refuse, and the
workspaces they ask for (no GPU call is made: every check comes before the first launch)."""

import ctypes
import os
import shutil
import subprocess

import pytest

arplan = pytest.importorskip(
    "paper_2409_04202_amd.arplan",
    reason="HIP library not built (run python -m paper_2409_04202_amd.build)")

P = 1 << 40     # an address that is never used
BIG = 1 << 30   # apart from the next
INVALID, UNSUPPORTED = arplan.AR_ERR_INVALID_ARG, arplan.AR_ERR_UNSUPPORTED


def at(i, off=0):
    return P + i * BIG + off


def refuses(f, args, status, **change):
    args = dict(args, **change)
    with pytest.raises(arplan.ArError) as e:
        f(**args)
    assert e.value.status == status and str(e.value)


BIAS = dict(dtype="bf16", buckets=32, max_distance=128, causal=0, H=4, Q=8, K=16, offset=0,
            table=at(0), table_stride=4, out=at(1), head_stride=128, row_stride=16)
BIAS_GRAD = dict(dtype="bf16", buckets=32, max_distance=128, causal=0, B=2, H=4, Q=8, K=16, offset=0,
                 dbias=at(0), batch_stride=512, head_stride=128, row_stride=16, accumulate=0,
                 dtable=at(1), table_stride=4, workspace=at(2), workspace_bytes=BIG)
ROUTE = dict(dtype="bf16", T=4, E=16, k=2, logits=at(0), logits_stride=16, live=at(1), normalize=1,
             ids=at(2), gates=at(3), counts=at(4), mass=at(5), workspace=at(6), workspace_bytes=BIG)
BALANCE = dict(dtype="bf16", T=4, E=16, k=2, logits=at(0), logits_stride=16, ids=at(1), counts=at(2),
               mass=at(3), coefficient=0.01, normalize=1, dgates=at(4), loss=at(5), grad=at(6),
               grad_stride=16)
STORE = dict(dtype="bf16", M=4, N=40, x=at(0), x_stride=40, kept=at(1), kept_stride=80)
FORWARD = dict(dtype="bf16", act="silu", M=4, D=8, F=16, x=at(0), x_stride=8, wg=at(1), wu=at(2),
               w_stride=8, h=at(3), h_stride=16, saved_gate=at(4), saved_up=at(5), saved_stride=48,
               saved_dtype=arplan.AR_BLOCK8, workspace=at(6), workspace_bytes=BIG)
BACKWARD = dict(dtype="bf16", M=4, D=8, F=16, dh=at(0), dh_stride=16, x=at(1), x_stride=8, wg=at(2),
                wu=at(3), w_stride=8, saved_gate=at(4), saved_up=at(5), saved_stride=48,
                saved_dtype=arplan.AR_BLOCK8, accumulate=0, dx=at(6), dx_stride=8, dwg=at(7),
                dwu=at(8), dw_stride=8, workspace=at(9), workspace_bytes=BIG)
CALLS = [(arplan.ar_position_bias, BIAS, ("out",)),
         (arplan.ar_position_bias_grad, BIAS_GRAD, ("dtable",)),
         (arplan.ar_route, ROUTE, ("ids", "gates", "counts", "mass")),
         (arplan.ar_balance, BALANCE, ("loss", "grad")),
         (arplan.ar_checkpoint_store, STORE, ("kept",)),
         (arplan.ar_checkpoint_load, STORE, ("x",))]
NAMES = lambda v: getattr(v, "__name__", "")    # noqa: E731


@pytest.mark.parametrize("f,args,outs", CALLS, ids=NAMES)
def test_common_refusals(f, args, outs):
    refuses(f, args, UNSUPPORTED, dtype="i32")
    refuses(f, args, INVALID, dtype=9)
    for k in ("B", "H", "Q", "K", "T", "E", "k", "M", "N"):
        if k in args:
            refuses(f, args, INVALID, **{k: -1})
            refuses(f, args, UNSUPPORTED, **{k: 1 << 31})
    for k in args:
        if isinstance(args[k], int) and args[k] >= P and k != "workspace":
            if k not in ("live", "grad", "dgates"):     # may be absent
                refuses(f, args, INVALID, **{k: None})
            if k != "live":
                refuses(f, args, INVALID, **{k: args[k] + 1})   # below the element's alignment
        if k.endswith("_stride"):
            refuses(f, args, INVALID, **{k: 1 << 62})
            refuses(f, args, INVALID, **{k: -1})
            if not (f is arplan.ar_position_bias_grad and k != "table_stride"):
                refuses(f, args, INVALID, **{k: args[k] - 1})


@pytest.mark.parametrize("f,args,outs", CALLS, ids=NAMES)
def test_overlaps_are_refused(f, args, outs):
    pointers = [k for k in args if isinstance(args[k], int) and args[k] >= P]
    for o in outs:
        for k in pointers:
            if k == o or k == "workspace":
                continue
            refuses(f, args, INVALID, **{o: args[k]} if (o, k) != ("grad", "logits")
                    else {o: args[k] + 4})
    # in place, but not with another stride
    refuses(arplan.ar_balance, BALANCE, INVALID, grad=BALANCE["logits"], grad_stride=17)


def test_workspaces():
    need = arplan.ar_position_bias_grad_workspace("bf16", 32, 2, 4, 8, 16)
    if need:
        refuses(arplan.ar_position_bias_grad, BIAS_GRAD, INVALID, workspace_bytes=need - 1)
    long = dict(BIAS_GRAD, Q=3000, K=5000, head_stride=3000 * 5000, row_stride=5000,
                batch_stride=4 * 3000 * 5000, dtable=at(200), workspace=at(300))
    need = arplan.ar_position_bias_grad_workspace("bf16", 32, 2, 4, 3000, 5000)
    assert need > 0
    for change in (dict(workspace_bytes=need - 1), dict(workspace=None), dict(workspace=at(300) + 8),
                   dict(workspace=long["dbias"]), dict(workspace=long["dtable"])):
        refuses(arplan.ar_position_bias_grad, long, INVALID, **change)
    need = arplan.ar_route_workspace(5000, 16, 2)
    assert need > 0
    for change in (dict(workspace_bytes=need - 1), dict(workspace=None), dict(workspace=at(6) + 8),
                   dict(workspace=ROUTE["logits"]), dict(workspace=ROUTE["ids"])):
        refuses(arplan.ar_route, dict(ROUTE, T=5000), INVALID, **change)
    assert arplan.ar_route_workspace(1, 16, 2) == 0
    assert arplan.ar_position_bias_grad_workspace("f32", 32, 0, 4, 8, 16) == 0
    for f, a in ((arplan._lib.ar_position_bias_grad_workspace, (0, 32, 1, 1, 1, 1)),
                 (arplan._lib.ar_route_workspace, (1, 1, 1)), (arplan._lib.ar_checkpoint_row, (1,))):
        assert f(*a, None) == INVALID
        b = ctypes.c_int64(-7)
        assert f(*(-1 for _ in a), ctypes.byref(b)) == INVALID
        assert b.value == -7        # written on success only


def test_refusals_of_the_position_bias():
    for f, args in ((arplan.ar_position_bias, BIAS), (arplan.ar_position_bias_grad, BIAS_GRAD)):
        refuses(f, args, UNSUPPORTED, buckets=arplan.AR_POSITION_MAX_BUCKETS + 2)
        for n in (-4, 0, 2, 31):
            refuses(f, args, INVALID, buckets=n)
        refuses(f, dict(args, causal=1), INVALID, buckets=1)
        for most in (-1, 0, 8):
            refuses(f, args, INVALID, max_distance=most)
        refuses(f, dict(args, causal=1), INVALID, max_distance=16)
        for offset in ((1 << 62) + 1, -(1 << 62) - 1):
            refuses(f, args, INVALID, offset=offset)
        refuses(f, args, UNSUPPORTED, H=1 << 21, Q=1 << 21, K=1 << 21, table_stride=1 << 21)
    # rows in heads or heads in rows, and no other order
    refuses(arplan.ar_position_bias, BIAS, INVALID, head_stride=127)
    refuses(arplan.ar_position_bias, BIAS, INVALID, head_stride=16, row_stride=63)
    refuses(arplan.ar_position_bias, BIAS, INVALID, head_stride=16, row_stride=16)


def test_refusals_of_the_routing():
    for f, args in ((arplan.ar_route, ROUTE), (arplan.ar_balance, BALANCE)):
        refuses(f, args, UNSUPPORTED, E=arplan.AR_ROUTE_MAX_EXPERTS + 1)
        refuses(f, args, UNSUPPORTED, k=arplan.AR_ROUTE_MAX_K + 1)
        refuses(f, args, INVALID, k=0)
        refuses(f, args, INVALID, k=17)
        refuses(f, args, INVALID, E=0)
    for c in (float("inf"), float("-inf"), float("nan")):
        refuses(arplan.ar_balance, BALANCE, INVALID, coefficient=c)


def test_refusals_of_rows_in_8_bits():
    for f in (arplan.ar_checkpoint_store, arplan.ar_checkpoint_load):
        refuses(f, STORE, INVALID, kept=STORE["kept"] + 8)
        refuses(f, STORE, INVALID, kept_stride=88)      # no multiple of 16
        refuses(f, STORE, INVALID, kept_stride=64)      # below a row's 80 bytes
    for f, args in ((arplan.ar_glu_forward, FORWARD), (arplan.ar_glu_backward, BACKWARD)):
        for k in ("saved_gate", "saved_up"):
            refuses(f, args, INVALID, **{k: args[k] + 8})
            refuses(f, args, INVALID, **{k: None})
        for stride in (16, 32, 40, 47, 56):
            refuses(f, args, INVALID, saved_stride=stride)
        refuses(f, args, INVALID, saved_dtype=7)
    for k in ("saved_gate", "saved_up"):
        refuses(arplan.ar_glu_forward, FORWARD, INVALID, **{k: FORWARD["h"]})
        refuses(arplan.ar_glu_backward, BACKWARD, INVALID, **{k: BACKWARD["dx"]})


def test_rows():
    for N, row in ((0, 0), (1, 48), (32, 48), (33, 80), (512, 528), (513, 576), (16384, 16896)):
        assert arplan.ar_checkpoint_row(N) == row
    ops = pytest.importorskip("paper_2409_04202_amd.ops")
    for N in list(range(600)) + [10 ** 6 + 7, (1 << 31) - 1]:
        assert ops._row(N) == arplan.ar_checkpoint_row(N)


def test_empty_calls_need_no_pointers():
    arplan.ar_position_bias("f32", 32, 128, 0, 4, 0, 5, 0, at(0), 4, None, 0, 5)
    arplan.ar_position_bias("f32", 32, 128, 0, 0, 5, 5, 0, None, 1, None, 25, 5)
    arplan.ar_position_bias_grad("f32", 32, 128, 0, 3, 0, 5, 5, 0, None, 0, 25, 5, 0, None, 1, None, 0)
    arplan.ar_checkpoint_store("f32", 0, 8, None, 8, None, 48)
    arplan.ar_checkpoint_load("bf16", 5, 0, None, 48, None, 1)


def test_tensors_are_checked():
    torch = pytest.importorskip("torch")
    from paper_2409_04202_amd import ops
    x = torch.zeros(4, 8)
    i = torch.zeros(4, 2, dtype=torch.int64)
    for call in (lambda: ops.position_bias(x, 4, 4), lambda: ops.position_bias_grad(x, x),
                 lambda: ops.position_bias_grad(torch.zeros(1, 8, 4, 4), x), lambda: ops.route(x, 2),
                 lambda: ops.balance(x, i, torch.zeros(9, dtype=torch.int32), torch.zeros(8)),
                 lambda: ops.checkpoint_store(x), lambda: ops.checkpoint_load(x, 8, torch.float32),
                 lambda: ops.glu_forward(x, x, x, save=torch.uint8)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.skipif(not shutil.which("g++"), reason="no C++ compiler")
def test_no_exception_leaves_an_entry(tmp_path):
    here = os.path.dirname(os.path.abspath(__file__))
    exe = str(tmp_path / "more_ops_no_memory")
    lib = os.path.dirname(arplan._lib._name)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror",
                    "-I", os.path.join(os.path.dirname(here), "include"),
                    os.path.join(here, "c_abi", "more_ops_no_memory.cpp"), "-o", exe,
                    "-L", lib, "-larplan", "-Wl,-rpath," + lib], check=True)
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.count(": %d\n" % arplan.AR_ERR_OOM) == 9, r.stdout
