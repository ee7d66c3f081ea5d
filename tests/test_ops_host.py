"""What the replica operators refuse, and the workspaces they ask for (no GPU
call is made: every check comes before the first launch)."""

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


def at(i, off=0):
    return P + i * BIG + off


def refuses(f, args, status, **change):
    args = dict(args, **change)
    with pytest.raises(arplan.ArError) as e:
        f(**args)
    assert e.value.status == status and str(e.value)


INVALID, UNSUPPORTED = arplan.AR_ERR_INVALID_ARG, arplan.AR_ERR_UNSUPPORTED

LOOKUP = dict(dtype="f32", V=10, D=8, T=4, table=at(0), table_stride=8, ids=at(1), scale=1.0,
              out=at(2), out_stride=8)
GRAD = dict(dtype="bf16", V=10, D=8, T=4, dout=at(0), dout_stride=8, ids=at(1), scale=1.0,
            accumulate=0, dtable=at(2), dtable_stride=8, workspace=at(3), workspace_bytes=BIG)
FORWARD = dict(dtype="bf16", act="silu", M=4, D=8, F=16, x=at(0), x_stride=8, wg=at(1), wu=at(2),
               w_stride=8, h=at(3), h_stride=16, saved_gate=at(4), saved_up=at(5), saved_stride=16,
               workspace=at(6), workspace_bytes=BIG)
BACKWARD = dict(dtype="bf16", M=4, D=8, F=16, dh=at(0), dh_stride=16, x=at(1), x_stride=8, wg=at(2),
                wu=at(3), w_stride=8, saved_gate=at(4), saved_up=at(5), saved_stride=16,
                accumulate=0, dx=at(6), dx_stride=8, dwg=at(7), dwu=at(8), dw_stride=8,
                workspace=at(9), workspace_bytes=BIG)
DISTILL = dict(dtype="bf16", T=4, V=100, K=5, logits=at(0), logits_stride=100, teacher_dtype="f32",
               teacher=at(1), teacher_stride=5, ids=at(2), ids_stride=5, temperature=1.0,
               weights=at(3), loss=at(4), grad=at(5), grad_stride=100, workspace=at(6),
               workspace_bytes=BIG)
CALLS = [(arplan.ar_embed_lookup, LOOKUP), (arplan.ar_embed_grad, GRAD),
         (arplan.ar_glu_forward, FORWARD), (arplan.ar_glu_backward, BACKWARD),
         (arplan.ar_distill, DISTILL)]


@pytest.mark.parametrize("f,args", CALLS, ids=lambda v: getattr(v, "__name__", ""))
def test_common_refusals(f, args):
    refuses(f, args, UNSUPPORTED, dtype="i32")
    refuses(f, args, INVALID, dtype=9)
    sizes = [k for k in ("V", "D", "T", "M", "F", "K") if k in args]
    for k in sizes:
        refuses(f, args, INVALID, **{k: -1})
        refuses(f, args, UNSUPPORTED, **{k: 1 << 31})
    esize = 4 if args["dtype"] == "f32" else 2
    for k in args:
        if not (isinstance(args[k], int) and args[k] >= P):
            continue
        if k not in ("workspace", "weights", "grad", "dx", "saved_gate", "dwg"):  # may be absent
            refuses(f, args, INVALID, **{k: None})
        if k == "workspace":
            continue
        refuses(f, args, INVALID, **{k: args[k] + 1})       # below the element's alignment
    for k in args:
        if k.endswith("_stride"):
            refuses(f, args, INVALID, **{k: args[k] - 1})
            refuses(f, args, INVALID, **{k: 1 << 62})
    assert esize in (2, 4)


@pytest.mark.parametrize("f,args,outs", [
    (arplan.ar_embed_lookup, LOOKUP, ("out",)), (arplan.ar_embed_grad, GRAD, ("dtable",)),
    (arplan.ar_glu_forward, FORWARD, ("h", "saved_gate", "saved_up")),
    (arplan.ar_glu_backward, BACKWARD, ("dx", "dwg", "dwu")),
    (arplan.ar_distill, DISTILL, ("loss", "grad"))], ids=lambda v: getattr(v, "__name__", ""))
def test_overlaps_are_refused(f, args, outs):
    pointers = [k for k in args if isinstance(args[k], int) and args[k] >= P and k != "workspace"]
    for o in outs:
        for k in pointers:
            if k != o:
                refuses(f, args, INVALID, **{o: args[k] + 4})


def test_one_row_beside_the_columns_of_a_matrix():
    """A table of one row within the output's rows, in columns that the output
    leaves out, is no overlap: the call is refused for its size, which is checked
    after that."""
    T, D = (1 << 31) - 1, 1024
    args = dict(LOOKUP, V=1, T=T, D=D, table=at(0, 4 * (5 * 4096 + D)), table_stride=D,
                ids=at(1 << 20), out=at(0), out_stride=4096)
    refuses(arplan.ar_embed_lookup, args, UNSUPPORTED)
    refuses(arplan.ar_embed_lookup, args, UNSUPPORTED, table=at(0, 4 * (5 * 4096 + 3 * D)))
    refuses(arplan.ar_embed_lookup, args, INVALID, table=at(0, 4 * (5 * 4096 + D - 1)))
    refuses(arplan.ar_embed_lookup, args, INVALID, table=at(0, 4 * (5 * 4096 + 3 * D + 1)))


def test_workspaces():
    need = arplan.ar_embed_grad_workspace(10, 8, 4)
    assert need > 0
    refuses(arplan.ar_embed_grad, GRAD, INVALID, workspace_bytes=need - 1)
    refuses(arplan.ar_embed_grad, GRAD, INVALID, workspace=None)
    refuses(arplan.ar_embed_grad, GRAD, INVALID, workspace=at(3) + 8)
    refuses(arplan.ar_embed_grad, GRAD, INVALID, workspace=GRAD["dout"])
    need = arplan.ar_glu_workspace("bf16", 4, 8, 16, True)
    assert need >= 2 * 4 * 16 * 2
    refuses(arplan.ar_glu_backward, BACKWARD, INVALID, workspace_bytes=need - 1)
    refuses(arplan.ar_glu_backward, BACKWARD, INVALID, workspace=None)
    assert arplan.ar_embed_grad_workspace(10, 8, 0) == 0
    for f, a in ((arplan._lib.ar_embed_grad_workspace, (1, 1, 1)),
                 (arplan._lib.ar_glu_workspace, (0, 1, 1, 1, 1)),
                 (arplan._lib.ar_distill_workspace, (1, 1, 1))):
        assert f(*a, None) == INVALID
        b = ctypes.c_int64(-7)
        assert f(*[x if i else (9 if len(a) == 5 else -1) for i, x in enumerate(a)],
                 ctypes.byref(b)) == INVALID
        assert b.value == -7        # written on success only


@pytest.mark.parametrize("M,D,F", [(2048, 1024, 2048), (4000, 2051, 5465)])
def test_workspace_for_rows_laid_out_anew(M, D, F):
    """Whether rows lie at 16 bytes is known by their addresses and strides, not by
    their width: a long bf16 product's workspace has room for x and the weights."""
    rows = (M + 2 * F) * (-(-D // 8) * 8) * 2
    assert arplan.ar_glu_workspace("bf16", M, D, F, False) >= rows
    assert arplan.ar_glu_workspace("bf16", M, D, F, True) >= rows + 2 * M * F * 2


def test_refusals_of_one_call():
    refuses(arplan.ar_glu_forward, FORWARD, INVALID, act=2)
    refuses(arplan.ar_glu_forward, FORWARD, INVALID, saved_up=None)
    refuses(arplan.ar_glu_forward, FORWARD, UNSUPPORTED, M=arplan.AR_GLU_MAX_EXTENT + 1)
    refuses(arplan.ar_glu_backward, BACKWARD, INVALID, dwu=None)
    for f, args in ((arplan.ar_glu_forward, FORWARD), (arplan.ar_glu_backward, BACKWARD)):
        refuses(f, args, UNSUPPORTED, saved_dtype="i32")
        refuses(f, args, INVALID, saved_dtype=7)
        refuses(f, dict(args, dtype="f32"), UNSUPPORTED, saved_dtype="bf16")
    refuses(arplan.ar_distill, DISTILL, UNSUPPORTED, K=arplan.AR_DISTILL_MAX_K + 1)
    for t in (0.0, -1.0, float("inf"), float("nan")):
        refuses(arplan.ar_distill, DISTILL, INVALID, temperature=t)
    refuses(arplan.ar_distill, DISTILL, UNSUPPORTED, teacher_dtype="i32")
    # in place, but not with another stride
    refuses(arplan.ar_distill, DISTILL, INVALID, grad=DISTILL["logits"], grad_stride=101)


def test_temperatures_beyond_the_range_are_refused():
    for t in (1e-45, 4e-39, 0.9 * arplan.AR_DISTILL_MIN_TEMPERATURE,
              1.1 * arplan.AR_DISTILL_MAX_TEMPERATURE, 2e19, 3e38):
        refuses(arplan.ar_distill, DISTILL, UNSUPPORTED, temperature=t)


def test_empty_calls_need_no_pointers():
    arplan.ar_embed_lookup("f32", 0, 8, 0, None, 8, None, 1.0, None, 8)
    arplan.ar_embed_grad("f32", 0, 8, 5, at(0), 8, at(1), 1.0, 0, None, 8, None, 0)
    arplan.ar_glu_forward("f32", "silu", 0, 8, 4, None, 8, at(1), at(2), 8, None, 4, None, None, 0,
                          None, 0)
    arplan.ar_distill("f32", 0, 8, 4, None, 8, "f32", None, 4, None, 4, 1.0, None, None, None, 0,
                      None, 0)


def test_tensors_are_checked():
    torch = pytest.importorskip("torch")
    from paper_2409_04202_amd import ops
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        ops.embed_lookup(x, torch.zeros(4, dtype=torch.int64))      # not on a GPU
    with pytest.raises(ValueError):
        ops.embed_lookup(torch.zeros(4), torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError):
        ops.glu_forward(x, x, x)
    with pytest.raises(ValueError):
        ops.distill(x, x, torch.zeros(4, 8, dtype=torch.int64))


@pytest.mark.skipif(not shutil.which("g++"), reason="no C++ compiler")
def test_no_exception_leaves_an_entry(tmp_path):
    here = os.path.dirname(os.path.abspath(__file__))
    exe = str(tmp_path / "ops_no_memory")
    lib = os.path.dirname(arplan._lib._name)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror",
                    "-I", os.path.join(os.path.dirname(here), "include"),
                    os.path.join(here, "c_abi", "ops_no_memory.cpp"), "-o", exe,
                    "-L", lib, "-larplan", "-Wl,-rpath," + lib], check=True)
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.count(": %d\n" % arplan.AR_ERR_OOM) == 8, r.stdout
