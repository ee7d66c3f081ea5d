"""The replica operators on torch tensors.

What a data-parallel replica computes between two AllReduces: an embedding
lookup and its gradient, attention's relative position bias and its gradient,
the first half of a gated feed-forward block (both projections, the activation
and the product) and its gradients, activations kept in 8 bits, the routing of
tokens to experts with a balance loss and its gradient, a distillation loss
and its gradient.  The functions here check their tensors,
allocate what the caller did not give and call the C functions of the same
names in ``paper_2409_04202_amd.arplan``, whose header says what each
computes.  There is no fallback: all work is the library's kernels.

Tensors are float32 or bfloat16 matrices on one GPU whose rows may have any
stride (adjacent elements within a row), so gradients can be written straight
into a slice of the vector that an AllReduce plan sums.  A call runs on
``stream`` (a ``torch.cuda.Stream``), by default the device's current stream,
and returns without waiting.  With another stream than the current one the
caller orders it after the work that made the inputs, as for any torch call;
what the call itself allocates belongs to the stream it runs on.  A
``workspace`` (a uint8 tensor of at least the bytes the ``*_workspace``
function of ``arplan`` names) is allocated where it is not given.

Wrong shapes, types or devices raise ValueError; what the library refuses
raises ``arplan.ArError``.

Autograd does not see these calls: the gradients are calls of their own.  With
gradients enabled a tensor that requires one raises ValueError (call under
``torch.no_grad()``, or with detached tensors), and what a call writes into a
given tensor counts as a change of it, as of any torch call in place.
"""

from operator import index

import torch
from torch.autograd.graph import increment_version

from . import arplan

_DT = {torch.float32: arplan.AR_F32, torch.bfloat16: arplan.AR_BF16}
_MOST = (1 << 31) - 1
_SAVED = {**_DT, torch.uint8: arplan.AR_BLOCK8}


def _matrix(name, x, shape=None, like=None):
    """The tensor's row stride, after checking that it is a matrix the library
    takes: of ``like``'s type and device, of ``shape`` where that is given."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError("%s: a two-dimensional tensor expected" % name)
    if not x.is_cuda:
        raise ValueError("%s: a GPU tensor expected" % name)
    if like is None:
        if x.dtype not in _DT:
            raise ValueError("%s: float32 or bfloat16 expected, got %s" % (name, x.dtype))
    elif x.dtype != like.dtype or x.get_device() != like.get_device():
        raise ValueError("%s: type and device differ from the first operand's" % name)
    if shape is not None and x.shape != shape:
        raise ValueError("%s: shape %s expected, got %s" % (name, tuple(shape), tuple(x.shape)))
    rows, cols = x.shape
    if cols > 1 and x.stride(1) != 1:
        raise ValueError("%s: the elements of a row have to be adjacent" % name)
    return x.stride(0) if rows > 1 else max(cols, 1)


def _strides(name, x, shape, like):
    """The strides of all but the last dimension, after the checks."""
    if not isinstance(x, torch.Tensor) or x.shape != shape:
        raise ValueError("%s: shape %s expected" % (name, tuple(shape)))
    if x.dtype != like.dtype or x.get_device() != like.get_device():
        raise ValueError("%s: type and device differ from the first operand's" % name)
    if x.shape[-1] > 1 and x.stride(-1) != 1:
        raise ValueError("%s: the elements of a row have to be adjacent" % name)
    return x.stride()[:-1]


def _whole(name, v, low, high):
    """The whole number, of any type that is one."""
    try:
        n = index(v)
    except TypeError:
        n = low - 1
    if not low <= n <= high:
        raise ValueError("%s: a whole number from %d to %d expected" % (name, low, high))
    return n


def _ids(name, ids, like):
    if not isinstance(ids, torch.Tensor) or ids.dtype != torch.int64 or ids.device != like.device:
        raise ValueError("%s: an int64 tensor on the operands' device expected" % name)


# The current device and its current stream as numbers, without the objects around them,
# whose making takes longer than a short call's launch (4 us of 13); with them where torch
# has no such functions, as one without GPU support has not.
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_current_stream = (getattr(torch._C, "_cuda_getCurrentRawStream", None)
                   or (lambda device: torch.cuda.current_stream(device).cuda_stream))


class _on:
    """The stream a call runs on, as a handle: its allocations are made there,
    and the tensors it is given are marked as used there, those in ``written`` as
    changed."""

    __slots__ = ("like", "stream", "tensors", "written", "entered")

    def __init__(self, like, stream, tensors, written=()):
        if torch.is_grad_enabled():
            for t in tensors:
                if t is not None and t.requires_grad:
                    raise ValueError("a tensor requires a gradient, and none is recorded here: "
                                     "call under torch.no_grad() or with detached tensors")
        self.like, self.stream, self.tensors, self.entered = like, stream, tensors, ()
        self.written = written

    def __enter__(self):
        if self.stream is None:
            device = self.like.get_device()
            if device != _current_device():
                self.entered = (torch.cuda.device(device),)
                self.entered[0].__enter__()
            return _current_stream(device)
        if self.stream.device != self.like.device:
            raise ValueError("stream: one of the operands' device expected")
        self.entered = (torch.cuda.device(self.like.device), torch.cuda.stream(self.stream))
        for e in self.entered:
            e.__enter__()
        return self.stream.cuda_stream

    def __exit__(self, *exc):
        if self.entered:
            for e in reversed(self.entered):
                e.__exit__(*exc)
        for t in self.written:
            if t is not None:
                increment_version(t)
        if self.stream is not None:
            for t in self.tensors:
                if t is not None:
                    t.record_stream(self.stream)


def _space(workspace, need, like):
    """(pointer, bytes) of the workspace, and what keeps it alive."""
    if workspace is None:
        if need == 0:
            return None, 0, None
        workspace = torch.empty(need, dtype=torch.uint8, device=like.device)
    elif (workspace.dtype != torch.uint8 or workspace.device != like.device
          or not workspace.is_contiguous()):
        raise ValueError("workspace: a contiguous uint8 tensor on the operands' device expected")
    return workspace.data_ptr(), workspace.numel(), workspace


# ------------------------------------------------------------- embedding

def embed_lookup(table, ids, scale=1.0, out=None, stream=None):
    """``scale * table[ids]``, a row of zeros where an id is outside the table:
    (..., D) for ids of shape (...), or ``out`` (T, D)."""
    st = _matrix("table", table)
    _ids("ids", ids, table)
    V, D = table.shape
    T = ids.numel()
    with _on(table, stream, (table, ids, out), (out,)) as s:
        flat = ids if ids.is_contiguous() else ids.contiguous()
        if out is None:
            res = torch.empty(ids.shape + (D,), dtype=table.dtype, device=table.device)
            so = max(D, 1)
        else:
            res, so = out, _matrix("out", out, (T, D), table)
        arplan.ar_embed_lookup(_DT[table.dtype], V, D, T, table, st, flat, scale, res, so, s)
    return res


def embed_grad(dout, ids, dtable, scale=1.0, accumulate=False, workspace=None, stream=None):
    """The gradient of ``embed_lookup``'s table for ``dout`` (T, D), stored
    into ``dtable`` (V, D), all of it, or added to it; returns ``dtable``."""
    sd = _matrix("dout", dout)
    st = _matrix("dtable", dtable, None, dout)
    _ids("ids", ids, dout)
    T, D = dout.shape
    V = dtable.shape[0]
    if dtable.shape[1] != D or ids.numel() != T:
        raise ValueError("dtable has to be as wide as dout, and ids one a row of dout")
    with _on(dout, stream, (dout, ids, dtable, workspace), (dtable,)) as s:
        flat = ids if ids.is_contiguous() else ids.contiguous()
        w, n, keep = _space(workspace, arplan.ar_embed_grad_workspace(V, D, T), dout)
        arplan.ar_embed_grad(_DT[dout.dtype], V, D, T, dout, sd, flat, scale, accumulate, dtable,
                             st, w, n, s)
    return dtable


# --------------------------------------------------------- position bias

def position_bias(table, queries, keys, max_distance=128, offset=0, causal=False, out=None,
                  stream=None):
    """Attention's relative position bias (H, queries, keys) from ``table``
    (buckets, H), for queries at positions ``offset`` on and keys at 0 on; with
    ``causal`` all buckets are the past's and later keys have -inf.  ``out``
    may have any strides of heads and rows, a slice of a wider tensor's among
    them."""
    st = _matrix("table", table)
    buckets, H = table.shape
    queries, keys = _whole("queries", queries, 0, _MOST), _whole("keys", keys, 0, _MOST)
    max_distance = _whole("max_distance", max_distance, 1, _MOST)
    offset = _whole("offset", offset, -1 << 62, 1 << 62)
    with _on(table, stream, (table, out), (out,)) as s:
        if out is None:
            res = torch.empty(H, queries, keys, dtype=table.dtype, device=table.device)
            sh, sr = queries * keys, keys
        else:
            res = out
            sh, sr = _strides("out", out, (H, queries, keys), table)
        arplan.ar_position_bias(_DT[table.dtype], buckets, max_distance, causal, H, queries, keys,
                                offset, table, st, res, sh, sr, s)
    return res


def position_bias_grad(dbias, dtable, max_distance=128, offset=0, causal=False, accumulate=False,
                       workspace=None, stream=None):
    """The gradient of ``position_bias``'s table for ``dbias`` (B, H, queries,
    keys) or (H, queries, keys), summed over the batch and stored into
    ``dtable`` (buckets, H), all of it, or added to it; returns ``dtable``."""
    st = _matrix("dtable", dtable)
    if isinstance(dbias, torch.Tensor) and dbias.dim() == 3:
        dbias = dbias[None]
    if not isinstance(dbias, torch.Tensor) or dbias.dim() != 4:
        raise ValueError("dbias: a (batch, heads, queries, keys) tensor expected")
    max_distance = _whole("max_distance", max_distance, 1, _MOST)
    offset = _whole("offset", offset, -1 << 62, 1 << 62)
    B, H, Q, K = dbias.shape
    buckets = dtable.shape[0]
    if dtable.shape[1] != H:
        raise ValueError("dtable: a column for each of dbias's heads expected")
    sb, sh, sr = _strides("dbias", dbias, (B, H, Q, K), dtable)
    with _on(dbias, stream, (dbias, dtable, workspace), (dtable,)) as s:
        need = arplan.ar_position_bias_grad_workspace(_DT[dbias.dtype], buckets, B, H, Q, K)
        w, n, keep = _space(workspace, need, dbias)
        arplan.ar_position_bias_grad(_DT[dbias.dtype], buckets, max_distance, causal, B, H, Q, K,
                                     offset, dbias, sb, sh, sr, accumulate, dtable, st, w, n, s)
    return dtable


# ---------------------------------------------------- gated feed-forward

def glu_forward(x, wg, wu, act="silu", save=False, out=None, workspace=None, stream=None):
    """``act(x wg^T) * (x wu^T)`` for x (M, D) and wg, wu (F, D): (M, F).  With
    ``save`` returns it and what ``glu_backward`` needs, a (2, M, F) tensor:
    ``True`` in float32, a dtype (float32 or x's) in that; ``torch.uint8`` in 8
    bits, a (2, M, row) tensor of rows as ``checkpoint_store`` makes them."""
    sx = _matrix("x", x)
    M, D = x.shape
    sw = _matrix("wg", wg, None, x)
    F = wg.shape[0]
    su = _matrix("wu", wu, (F, D), x)
    if wg.shape[1] != D:
        raise ValueError("wg: as wide as x expected")
    if su != sw:
        raise ValueError("wg and wu: one row stride expected")
    if act not in arplan.ACTS:
        raise ValueError("act: one of %s expected" % ", ".join(sorted(arplan.ACTS)))
    with _on(x, stream, (x, wg, wu, out, workspace), (out,)) as s:
        h = torch.empty(M, F, dtype=x.dtype, device=x.device) if out is None else out
        sh = _matrix("out", h, (M, F), x)
        kind = torch.float32 if save in (True, False, None) else save
        if kind not in (torch.float32, x.dtype, torch.uint8):
            raise ValueError("save: True, float32, x's type or uint8 expected")
        width = arplan.ar_checkpoint_row(F) if kind == torch.uint8 else F
        saved = torch.empty(2, M, width, dtype=kind, device=x.device) if save else None
        a, b = (saved[0], saved[1]) if save else (None, None)
        w, n, keep = _space(workspace, arplan.ar_glu_workspace(_DT[x.dtype], M, D, F, False), x)
        arplan.ar_glu_forward(_DT[x.dtype], act, M, D, F, x, sx, wg, wu, sw, h, sh, a, b,
                              max(width, 1), w, n, s, saved_dtype=_SAVED[kind])
    return (h, saved) if save else h


def glu_backward(dh, x, wg, wu, saved, dx=None, dwg=None, dwu=None, accumulate=False,
                 workspace=None, stream=None):
    """(dx, dwg, dwu) for ``dh`` (M, F), the gradient at ``glu_forward``'s
    result, and what that saved.  With bfloat16 the gradients at the two
    projections are rounded to it before the products, and the results again.
    Outputs that are given are written in place; with ``accumulate`` dwg and dwu
    are added to (and have to be given)."""
    sh = _matrix("dh", dh)
    M, F = dh.shape
    sx = _matrix("x", x, None, dh)
    D = x.shape[1]
    if x.shape[0] != M:
        raise ValueError("x: a row for each of dh's expected")
    sw = _matrix("wg", wg, (F, D), dh)
    if _matrix("wu", wu, (F, D), dh) != sw:
        raise ValueError("wg and wu: one row stride expected")
    if (not isinstance(saved, torch.Tensor) or saved.dim() != 3 or saved.shape[0] != 2):
        raise ValueError("saved: what glu_forward saved expected")
    sg, su = saved[0], saved[1]
    if saved.dtype not in (torch.float32, dh.dtype, torch.uint8) or saved.device != dh.device:
        raise ValueError("saved: float32, dh's type or uint8 on dh's device expected")
    if saved.dtype == torch.uint8:
        ss = _kept("saved", sg, M, F)
        _kept("saved", su, M, F)
    else:
        ss = _matrix("saved", sg, (M, F))
        if _matrix("saved", su, (M, F)) != ss:
            raise ValueError("saved: one row stride expected")
    if (dwg is None) != (dwu is None):
        raise ValueError("dwg and dwu are given together")
    if accumulate and dwg is None:
        raise ValueError("accumulate: dwg and dwu have to be given")
    with _on(dh, stream, (dh, x, wg, wu, saved, dx, dwg, dwu, workspace), (dx, dwg, dwu)) as s:
        if dx is None:
            dx = torch.empty(M, D, dtype=dh.dtype, device=dh.device)
        if dwg is None:
            dwg, dwu = torch.empty(2, F, D, dtype=dh.dtype, device=dh.device).unbind(0)
        sdx = _matrix("dx", dx, (M, D), dh)
        sdw = _matrix("dwg", dwg, (F, D), dh)
        if _matrix("dwu", dwu, (F, D), dh) != sdw:
            raise ValueError("dwg and dwu: one row stride expected")
        w, n, keep = _space(workspace, arplan.ar_glu_workspace(_DT[dh.dtype], M, D, F, True), dh)
        arplan.ar_glu_backward(_DT[dh.dtype], M, D, F, dh, sh, x, sx, wg, wu, sw, sg, su, ss,
                               accumulate, dx, sdx, dwg, dwu, sdw, w, n, s,
                               saved_dtype=_SAVED[saved.dtype])
    return dx, dwg, dwu


# ------------------------------------------------- activations in 8 bits

def _row(width):
    """A row's bytes, as ``arplan.ar_checkpoint_row`` has them."""
    return ((width + 31) // 32 * 33 + 15) & -16


def _kept(name, x, rows, width):
    """The row stride of rows in 8 bits."""
    if (not isinstance(x, torch.Tensor) or x.dim() != 2 or x.dtype != torch.uint8 or not x.is_cuda):
        raise ValueError("%s: a two-dimensional uint8 tensor on a GPU expected" % name)
    if rows is not None and x.shape[0] != rows:
        raise ValueError("%s: %d rows expected, got %d" % (name, rows, x.shape[0]))
    need = _row(width)
    if x.shape[1] < need or (need > 1 and x.stride(1) != 1):
        raise ValueError("%s: rows of %d adjacent bytes expected" % (name, need))
    return x.stride(0) if x.shape[0] > 1 else need


def checkpoint_store(x, out=None, stream=None):
    """``x`` (M, N) in 8 bits for a later pass: a uint8 (M, row) tensor, ``row``
    being ``arplan.ar_checkpoint_row(N)``, or ``out``, which may be wider.  32
    elements of a row share a power of two; each is off by half a unit of that at
    most, 2^-7 of the largest of the 32."""
    sx = _matrix("x", x)
    M, N = x.shape
    with _on(x, stream, (x, out), (out,)) as s:
        res = out
        if out is None:
            sk = _row(N)
            res = torch.empty(M, sk, dtype=torch.uint8, device=x.device)
        else:
            sk = _kept("out", out, M, N)
            if out.device != x.device:
                raise ValueError("out: on x's device expected")
        arplan.ar_checkpoint_store(_DT[x.dtype], M, N, x, sx, res, sk, s)
    return res


def checkpoint_load(kept, width, dtype=None, out=None, stream=None):
    """The (M, ``width``) values that ``kept`` holds, exactly, as ``dtype``
    (float32 or bfloat16) or into ``out``."""
    width = _whole("width", width, 0, _MOST)
    sk = _kept("kept", kept, None, width)
    M = kept.shape[0]
    if out is None and dtype not in _DT:
        raise ValueError("dtype: float32 or bfloat16 expected")
    with _on(kept, stream, (kept, out), (out,)) as s:
        if out is None:
            res, sx = torch.empty(M, width, dtype=dtype, device=kept.device), max(width, 1)
        else:
            res, sx = out, _matrix("out", out, (M, width))
            if out.device != kept.device or (dtype is not None and out.dtype != dtype):
                raise ValueError("out: of dtype and on kept's device expected")
        arplan.ar_checkpoint_load(_DT[res.dtype], M, width, kept, sk, res, sx, s)
    return res


# --------------------------------------------------------------- routing

def _whole_rows(name, x, shape, dtype, like):
    if (not isinstance(x, torch.Tensor) or x.shape != shape or x.dtype != dtype
            or x.get_device() != like.get_device() or not x.is_contiguous()):
        raise ValueError("%s: a contiguous %s tensor of shape %s on the operands' device expected"
                         % (name, str(dtype)[6:], tuple(shape)))


def route(logits, k, live=None, normalize=False, counts=None, mass=None, workspace=None,
          stream=None):
    """The ``k`` experts of each row of ``logits`` (T, E): (ids, gates, counts,
    mass) with int64 ids (T, k), -1 where there is none, float32 gates (T, k) (the
    softmax there; with ``normalize`` over their sum), int32 counts (E + 1,) (how
    often each expert was chosen, and how many rows were routed) and float32 mass
    (E,) (the probabilities' sums).  Rows whose ``live`` (bool (T,)) is false are
    padding.  ``counts`` and ``mass`` may be given, such as a slice of the vector
    that an int32 plan sums."""
    k = _whole("k", k, 0, _MOST)
    sl = _matrix("logits", logits)
    T, E = logits.shape
    if live is not None:
        _whole_rows("live", live, (T,), torch.bool, logits)
    with _on(logits, stream, (logits, live, counts, mass, workspace), (counts, mass)) as s:
        dev = logits.device
        w, n, keep = _space(workspace, arplan.ar_route_workspace(T, E, k), logits)
        if counts is None:
            counts = torch.empty(E + 1, dtype=torch.int32, device=dev)
        else:
            _whole_rows("counts", counts, (E + 1,), torch.int32, logits)
        if mass is None:
            mass = torch.empty(E, dtype=torch.float32, device=dev)
        else:
            _whole_rows("mass", mass, (E,), torch.float32, logits)
        ids = torch.empty(T, k, dtype=torch.int64, device=dev)
        gates = torch.empty(T, k, dtype=torch.float32, device=dev)
        arplan.ar_route(_DT[logits.dtype], T, E, k, logits, sl, live, normalize, ids, gates, counts,
                        mass, w, n, s)
    return ids, gates, counts, mass


def balance(logits, ids, counts, mass, coefficient=0.01, normalize=False, dgates=None, grad=None,
            stream=None):
    """The balance loss of a routing, a float32 scalar: ``coefficient`` times E
    times the sum over experts of the share of choices times the mean probability.
    With ``grad`` (T, E; ``logits`` itself for a gradient in place) returns the loss
    and ``grad``, holding its gradient and that of the gates for ``dgates`` (float32
    (T, k)).  ``counts`` may be all replicas' (summed by a plan): the replicas'
    losses and gradients then add up to the whole batch's."""
    sl = _matrix("logits", logits)
    T, E = logits.shape
    if not isinstance(ids, torch.Tensor) or ids.dim() != 2:
        raise ValueError("ids: a row for each of logits' expected")
    k = ids.shape[1]
    _whole_rows("ids", ids, (T, k), torch.int64, logits)
    _whole_rows("counts", counts, (E + 1,), torch.int32, logits)
    _whole_rows("mass", mass, (E,), torch.float32, logits)
    if dgates is not None:
        _whole_rows("dgates", dgates, (T, k), torch.float32, logits)
        if grad is None:
            raise ValueError("dgates: grad has to be given")
    sg = _matrix("grad", grad, (T, E), logits) if grad is not None else 0
    with _on(logits, stream, (logits, ids, counts, mass, dgates, grad), (grad,)) as s:
        loss = torch.empty((), dtype=torch.float32, device=logits.device)
        arplan.ar_balance(_DT[logits.dtype], T, E, k, logits, sl, ids, counts, mass, coefficient,
                          normalize, dgates, loss, grad, sg, s)
    return (loss, grad) if grad is not None else loss


# ----------------------------------------------------------- distillation

def distill(logits, teacher, ids, temperature=1.0, weights=None, grad=None, workspace=None,
            stream=None):
    """The distillation loss of each row of ``logits`` (T, V) from the
    teacher's top logits ``teacher`` (T, K) at ``ids`` (T, K), times
    ``weights`` (T,): a float32 (T,) tensor.  With ``grad`` (T, V; ``logits``
    itself for a gradient in place) returns the losses and ``grad``, holding
    the gradient of their sum."""
    sl = _matrix("logits", logits)
    T, V = logits.shape
    st = _matrix("teacher", teacher)
    K = teacher.shape[1]
    _ids("ids", ids, logits)
    if teacher.device != logits.device or teacher.shape[0] != T or ids.shape != teacher.shape:
        raise ValueError("teacher and ids: a (rows of logits, K) tensor each expected")
    if K > 1 and ids.stride(1) != 1:
        raise ValueError("ids: the elements of a row have to be adjacent")
    si = ids.stride(0) if T > 1 else max(K, 1)
    if weights is not None and (weights.shape != (T,) or weights.dtype != torch.float32
                                or weights.device != logits.device or not weights.is_contiguous()):
        raise ValueError("weights: a contiguous float32 vector, one a row, expected")
    sg = _matrix("grad", grad, (T, V), logits) if grad is not None else 0
    with _on(logits, stream, (logits, teacher, ids, weights, grad, workspace), (grad,)) as s:
        loss = torch.empty(T, dtype=torch.float32, device=logits.device)
        w, n, keep = _space(workspace, arplan.ar_distill_workspace(T, V, K), logits)
        arplan.ar_distill(_DT[logits.dtype], T, V, K, logits, sl, _DT[teacher.dtype], teacher, st,
                          ids, si, temperature, weights, loss, grad, sg, w, n, s)
    return (loss, grad) if grad is not None else loss
