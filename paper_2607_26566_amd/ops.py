"""Block operators (``include/t2i_ops.h``): 8-bit linear layer, gated
feed-forward, query / key norm with rotation, the residual's addition with an RMS norm, a
linear layer with a low-rank adapter per row, and their gradients.

Argument marshalling only, as in the package's other calls.  Tensors are device
tensors of one device whose last dimension is contiguous (rows may be strided);
results are new tensors of that device.  The work runs on ``stream``, by default
the device's current stream, and results and workspaces are allocated for that
stream: a caller that uses another stream on either side orders the two itself and
keeps the operands until the work is done.  Nothing here is recorded for automatic
differentiation: the ``_backward`` calls are the gradients, and an operand that requires a
gradient while gradients are recorded (outside ``torch.no_grad()`` and the passes of a
``torch.autograd.Function``), or that carries a tangent, is refused, as the result would
lose it.  Wrong arguments raise :class:`T2IError` before anything is launched.
"""
from __future__ import annotations

import contextlib
from typing import Optional, Tuple

import torch
from torch.autograd import forward_ad

from . import _lib
from ._lib import T2I_BF16, T2I_F32, T2IError, load

EPILOGUES = {"store": _lib.T2I_EPI_STORE, "gelu": _lib.T2I_EPI_GELU, "silu": _lib.T2I_EPI_SILU,
             "resid": _lib.T2I_EPI_RESID, "resid_gated": _lib.T2I_EPI_RESID_GATED}
ACTS = {"gelu": _lib.T2I_EPI_GELU, "silu": _lib.T2I_EPI_SILU}
PAIRINGS = {"pairs": _lib.T2I_ROPE_PAIRS, "halves": _lib.T2I_ROPE_HALVES}
_DTYPES = {torch.bfloat16: T2I_BF16, torch.float32: T2I_F32}
_INT = 2 ** 31   # the library's sizes are 32-bit integers, and ctypes drops what lies above


def _check(status: int):
    if status != 0:
        raise T2IError(status, load().t2i_ops_last_error().decode())


def _need(ok: bool, what: str, status: int = 2):
    if not ok:
        raise T2IError(status, what)


def _of(table: dict, key, what: str):
    v = table.get(key)
    if v is None:
        raise T2IError(1, f"{what} must be one of {', '.join(map(str, table))}")
    return v


def _device(first: torch.Tensor, *others) -> int:
    """Index of the one device of all given tensors (None entries left out), none of
    which automatic differentiation follows."""
    dev = first.get_device()
    if dev < 0:
        raise T2IError(1, "operands must be device tensors")
    followed = torch.is_grad_enabled()
    for t in (first, *others):
        if t is not None:
            if t.get_device() != dev:
                raise T2IError(1, "operands must be device tensors of one device")
            if followed and t.requires_grad:
                raise T2IError(1, "an operand requires a gradient, which this call does not record: "
                                  "detach it or call under torch.no_grad()")
    if getattr(forward_ad, "_current_level", 0) >= 0:   # (within a dual level)
        for t in (first, *others):
            if t is not None and forward_ad.unpack_dual(t).tangent is not None:
                raise T2IError(1, "an operand carries a tangent, which this call does not pass on")
    return dev


# A call's own work is a few microseconds, so the common case -- contiguous operands on
# the current device, no stream given -- goes without strides, stream objects and
# contexts.

def _rows(t: torch.Tensor, rows: int, cols: int, dtype, what: str) -> int:
    """Row stride of a matrix of this shape and type (its columns contiguous)."""
    if t.dtype is not dtype or t.shape != (rows, cols):
        raise T2IError(2, f"{what}: expected ({rows}, {cols}) {dtype}, got {tuple(t.shape)} {t.dtype}")
    if rows >= _INT or cols >= _INT:
        raise T2IError(2, f"{what}: 2^31 rows or columns, or more")
    if t.is_contiguous():
        return cols
    ld, step = t.stride()
    if cols != 1 and step != 1:
        raise T2IError(2, f"{what}: columns must be contiguous")
    if rows == 1:       # a single row may come with any stride
        ld = cols
    if not cols <= ld < _INT:
        raise T2IError(2, f"{what}: rows must not overlap")
    return ld


def _vec(t: Optional[torch.Tensor], n: int, dtype, what: str):
    if t is not None and (t.dtype is not dtype or t.shape != (n,) or not t.is_contiguous()):
        raise T2IError(2, f"{what}: expected ({n},) {dtype}, contiguous")


def _p(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _written(*tensors):
    """Operands that were written to: differentiation that has saved one of them finds out
    (as with torch's own operations in place) instead of using the new values."""
    for t in tensors:
        if t is not None:
            torch.autograd.graph.increment_version(t)


def _elsewhere(dev: int, stream) -> bool:
    return stream is not None or dev != torch._C._cuda_getDevice()


@contextlib.contextmanager
def _switch(dev: int, stream):
    """The operands' device and the stream asked for (or that device's own) made current."""
    if stream is None:
        stream = torch.cuda.current_stream(dev)
    elif stream.device.index != dev:
        raise T2IError(1, "stream belongs to another device than the operands")
    with torch.cuda.device(dev), torch.cuda.stream(stream):
        yield


def _stream(dev: int) -> int:
    # (looked up here, not at import: a torch without a GPU back end has no such name)
    return torch._C._cuda_getCurrentRawStream(dev)


def quant_rows(x: torch.Tensor, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Rows of ``x [rows, K]`` (bf16 or fp32) in 8 bits with a scale each
    (``t2i_op_quant_rows``): ``(q int8 [rows, K rounded up to 128], scale fp32
    [rows])``, zeros behind column K."""
    dev = _device(x)
    if _elsewhere(dev, stream):
        with _switch(dev, stream):
            return quant_rows(x)
    dt = _of(_DTYPES, x.dtype, "dtype")
    _need(x.dim() == 2, "x must be [rows, K]")
    rows, K = x.shape
    ld = _rows(x, rows, K, x.dtype, "x")
    ldq = (K + 127) // 128 * 128
    q = x.new_empty((rows, ldq), dtype=torch.int8)
    scale = x.new_empty(rows, dtype=torch.float32)
    _check(load().t2i_op_quant_rows(dt, rows, K, x.data_ptr(), ld, q.data_ptr(), ldq, scale.data_ptr(),
                                    _stream(dev)))
    return q, scale


def linear_i8(a: torch.Tensor, a_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor,
              bias: Optional[torch.Tensor] = None, *, K: int, epilogue: str = "store",
              dtype: torch.dtype = torch.bfloat16, resid: Optional[torch.Tensor] = None,
              resid_copy: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
              stream=None) -> torch.Tensor:
    """8-bit linear layer (``t2i_op_linear_i8``) of ``a [M, >= K]`` and ``w [N, >= K]``
    as :func:`quant_rows` makes them, with the epilogues of the bf16 layer:
    ``store``, ``gelu``, ``silu`` return ``[M, N]`` of ``dtype``; ``resid`` and
    ``resid_gated`` add to the fp32 ``resid [M, N]`` in place (and write the bf16
    ``resid_copy``, if given) and return it."""
    dev = _device(a, a_scale, w, w_scale, bias, resid, resid_copy, gate)
    if _elsewhere(dev, stream):
        with _switch(dev, stream):
            return linear_i8(a, a_scale, w, w_scale, bias, K=K, epilogue=epilogue, dtype=dtype, resid=resid,
                             resid_copy=resid_copy, gate=gate)
    dt, epi = _of(_DTYPES, dtype, "dtype"), _of(EPILOGUES, epilogue, "epilogue")
    _need(a.dim() == 2 and w.dim() == 2, "a and w must be matrices")
    (M, ka), (N, kw) = a.shape, w.shape
    need = (K + 127) // 128 * 128
    _need(K >= 1 and ka >= need and kw >= need, "a and w must reach K rounded up to 128")
    lda, ldw = _rows(a, M, ka, torch.int8, "a"), _rows(w, N, kw, torch.int8, "w")
    lda, ldw = (need if M == 1 else lda), (need if N == 1 else ldw)
    _vec(a_scale, M, torch.float32, "a_scale")
    _vec(w_scale, N, torch.float32, "w_scale")
    _vec(bias, N, dtype, "bias")
    _vec(gate, N, torch.float32, "gate")
    ldr = N
    if epi >= _lib.T2I_EPI_RESID:
        _need(resid is not None, "the resid epilogues need resid", 1)
        ldr = _rows(resid, M, N, torch.float32, "resid")
        if resid_copy is not None:
            ldc = _rows(resid_copy, M, N, torch.bfloat16, "resid_copy")
            _need(M == 1 or ldc == ldr, "resid_copy must have resid's row stride")
    else:
        _need(resid is None and resid_copy is None, "resid goes with the resid epilogues", 1)
    _need((gate is not None) == (epilogue == "resid_gated"), "gate goes with resid_gated", 1)
    out = None
    if epi < _lib.T2I_EPI_RESID:
        out = a.new_empty((M, N), dtype=dtype)
    _check(load().t2i_op_linear_i8(dt, epi, M, N, K, a.data_ptr(), lda, a_scale.data_ptr(), w.data_ptr(),
                                   ldw, w_scale.data_ptr(), _p(bias), _p(out), N, _p(resid), ldr,
                                   _p(resid_copy), _p(gate), _stream(dev)))
    if out is not None:
        return out
    _written(resid, resid_copy)
    return resid


def _gated_args(x, wg, wu):
    dt = _of(_DTYPES, x.dtype, "dtype")
    _need(x.dim() == 2 and wg.dim() == 2, "x and the weights must be matrices")
    (M, K), F = x.shape, wg.shape[0]
    lda = _rows(x, M, K, x.dtype, "x")
    ldw = _rows(wg, F, K, x.dtype, "wg")
    _need(_rows(wu, F, K, x.dtype, "wu") == ldw, "wg and wu must have one row stride")
    return dt, M, F, K, lda, ldw


def gated_linear(x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor,
                 bg: Optional[torch.Tensor] = None, bu: Optional[torch.Tensor] = None, *,
                 act: str = "silu", save_pre: bool = False, stream=None):
    """``act(x wg^T + bg) * (x wu^T + bu)`` (``t2i_op_gated_linear``): ``x [M, K]``,
    ``wg``, ``wu`` ``[F, K]``, one dtype (bf16 or fp32); ``[M, F]``.  With ``save_pre``
    also the fp32 pre-activations ``[M, 2F]`` that :func:`gated_linear_backward` takes."""
    dev = _device(x, wg, wu, bg, bu)
    if _elsewhere(dev, stream):
        with _switch(dev, stream):
            return gated_linear(x, wg, wu, bg, bu, act=act, save_pre=save_pre)
    dt, M, F, K, lda, ldw = _gated_args(x, wg, wu)
    a = _of(ACTS, act, "act")
    _vec(bg, F, x.dtype, "bg")
    _vec(bu, F, x.dtype, "bu")
    out = x.new_empty((M, F))
    pre = x.new_empty((M, 2 * F), dtype=torch.float32) if save_pre else None
    _check(load().t2i_op_gated_linear(dt, a, M, F, K, x.data_ptr(), lda, wg.data_ptr(), wu.data_ptr(), ldw,
                                      _p(bg), _p(bu), out.data_ptr(), F, _p(pre), 2 * F, _stream(dev)))
    return (out, pre) if save_pre else out


def gated_linear_backward(dout: torch.Tensor, x: torch.Tensor, wg: torch.Tensor, wu: torch.Tensor,
                          pre: torch.Tensor, *, act: str = "silu", bias: bool = False,
                          need_dx: bool = True, need_dw: bool = True, stream=None):
    """Gradients of :func:`gated_linear` (``t2i_op_gated_linear_backward``):
    ``(dx, dwg, dwu, dbg, dbu)``, None for those not asked for."""
    dev = _device(dout, x, wg, wu, pre)
    if _elsewhere(dev, stream):
        with _switch(dev, stream):
            return gated_linear_backward(dout, x, wg, wu, pre, act=act, bias=bias, need_dx=need_dx,
                                         need_dw=need_dw)
    dt, M, F, K, lda, ldw = _gated_args(x, wg, wu)
    a = _of(ACTS, act, "act")
    ldd = _rows(dout, M, F, x.dtype, "dout")
    ldp = _rows(pre, M, 2 * F, torch.float32, "pre")
    lib = load()
    dx = x.new_empty((M, K)) if need_dx else None
    dwg, dwu = (x.new_empty((F, K)), x.new_empty((F, K))) if need_dw else (None, None)
    dbg, dbu = (x.new_empty(F), x.new_empty(F)) if bias else (None, None)
    n = lib.t2i_op_gated_linear_backward_ws_bytes(dt, M, F, K)
    ws = x.new_empty(n, dtype=torch.uint8)
    _check(lib.t2i_op_gated_linear_backward(
        dt, a, M, F, K, x.data_ptr(), lda, wg.data_ptr(), wu.data_ptr(), ldw, pre.data_ptr(), ldp,
        dout.data_ptr(), ldd, _p(dx), K, _p(dwg), _p(dwu), K, _p(dbg), _p(dbu), ws.data_ptr(), n,
        _stream(dev)))
    return dx, dwg, dwu, dbg, dbu


def _heads(t: torch.Tensor, rows: int, d: int, dtype, what: str):
    """(heads, row stride) of a [rows, heads, d] tensor whose heads lie side by side."""
    shape = t.shape
    if t.dtype is not dtype or len(shape) != 3 or shape[0] != rows or shape[2] != d:
        raise T2IError(2, f"{what}: expected ({rows}, heads, {d}) {dtype}, got {tuple(shape)} {t.dtype}")
    h = shape[1]
    if t.is_contiguous():
        ld = h * d
    else:
        ld, head, step = t.stride()
        if step != 1 or (h > 1 and head != d):
            raise T2IError(2, f"{what}: heads must be side by side")
        if rows == 1:
            ld = h * d
    if rows >= _INT:
        raise T2IError(2, f"{what}: 2^31 rows or more")
    if not h * d <= ld < _INT:
        raise T2IError(2, f"{what}: rows must not overlap")
    return h, ld


def _qk_args(q, k, wq, wk, table, pos, pairing):
    dt = _of(_DTYPES, q.dtype, "dtype")
    pr = _of(PAIRINGS, pairing, "pairing")
    _need(q.dim() == 3, "q must be [rows, heads, head_dim]")
    rows, _, d = q.shape
    hq, ldq = _heads(q, rows, d, q.dtype, "q")
    hk, ldk = _heads(k, rows, d, q.dtype, "k")
    _vec(wq, d, q.dtype, "wq")
    _vec(wk, d, q.dtype, "wk")
    n_pos = 0
    if table is not None:
        n_pos = table.shape[0] if table.dim() == 3 else -1
        if table.dtype != torch.float32 or table.shape != (n_pos, d // 2, 2) or not table.is_contiguous():
            raise T2IError(2, f"table must be fp32 [n_pos, {d // 2}, 2], contiguous")
        _need(n_pos < _INT, "table: 2^31 positions or more")
    _need(pos is None or table is not None, "pos goes with a table", 1)
    _vec(pos, rows, torch.int32, "pos")
    return dt, pr, rows, hq, hk, d, ldq, ldk, n_pos


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, wq: Optional[torch.Tensor] = None,
                 wk: Optional[torch.Tensor] = None, *, table: Optional[torch.Tensor] = None,
                 pos: Optional[torch.Tensor] = None, eps: float = 1e-6, pairing: str = "pairs",
                 inplace: bool = False, stream=None):
    """RMS norm of every head of ``q [rows, heads_q, d]`` and ``k [rows, heads_k, d]``
    with weights ``wq``, ``wk`` ``[d]`` (or None), then the rotation by
    ``table[pos[row]]`` (``t2i_op_qk_norm_rope``): ``table`` fp32 ``[n_pos, d/2, 2]`` of
    (cos, sin) or None, ``pos`` int32 ``[rows]`` (negative: not turned) or None (row r
    at position r).  Returns new ``(q, k)``, or with ``inplace`` the given ones."""
    dev = _device(q, k, wq, wk, table, pos)
    if _elsewhere(dev, stream):
        with _switch(dev, stream):
            return qk_norm_rope(q, k, wq, wk, table=table, pos=pos, eps=eps, pairing=pairing, inplace=inplace)
    dt, pr, rows, hq, hk, d, ldq, ldk, n_pos = _qk_args(q, k, wq, wk, table, pos, pairing)
    if inplace:
        oq, ok, ldoq, ldok = q, k, ldq, ldk
    else:
        oq, ok, ldoq, ldok = q.new_empty((rows, hq, d)), q.new_empty((rows, hk, d)), hq * d, hk * d
    _check(load().t2i_op_qk_norm_rope(
        dt, rows, hq, hk, d, q.data_ptr(), ldq, k.data_ptr(), ldk, _p(wq), _p(wk), eps, pr, _p(table), n_pos,
        _p(pos), oq.data_ptr(), ldoq, ok.data_ptr(), ldok, _stream(dev)))
    if inplace:
        _written(q, k)
    return oq, ok


def qk_norm_rope_backward(dq: torch.Tensor, dk: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                          wq: Optional[torch.Tensor] = None, wk: Optional[torch.Tensor] = None, *,
                          table: Optional[torch.Tensor] = None, pos: Optional[torch.Tensor] = None,
                          eps: float = 1e-6, pairing: str = "pairs", stream=None):
    """Gradients of :func:`qk_norm_rope` (``t2i_op_qk_norm_rope_backward``) from those of
    its outputs and its inputs: ``(dq, dk, dwq, dwk)``, None for a weight that is None."""
    dev = _device(q, k, wq, wk, table, pos, dq, dk)
    if _elsewhere(dev, stream):
        with _switch(dev, stream):
            return qk_norm_rope_backward(dq, dk, q, k, wq, wk, table=table, pos=pos, eps=eps, pairing=pairing)
    dt, pr, rows, hq, hk, d, ldq, ldk, n_pos = _qk_args(q, k, wq, wk, table, pos, pairing)
    h1, lddq = _heads(dq, rows, d, q.dtype, "dq")
    h2, lddk = _heads(dk, rows, d, q.dtype, "dk")
    _need(h1 == hq and h2 == hk, "gradients must have the heads of q and k")
    lib = load()
    oq, ok = q.new_empty((rows, hq, d)), q.new_empty((rows, hk, d))
    dwq = q.new_empty(d) if wq is not None else None
    dwk = q.new_empty(d) if wk is not None else None
    n, ws = 0, None
    if wq is not None or wk is not None:
        n = lib.t2i_op_qk_norm_rope_backward_ws_bytes(rows, hq, hk, d)
        ws = q.new_empty(n, dtype=torch.uint8)
    _check(lib.t2i_op_qk_norm_rope_backward(
        dt, rows, hq, hk, d, dq.data_ptr(), lddq, dk.data_ptr(), lddk, q.data_ptr(), ldq, k.data_ptr(), ldk,
        _p(wq), _p(wk), eps, pr, _p(table), n_pos, _p(pos), oq.data_ptr(), hq * d, ok.data_ptr(), hk * d,
        _p(dwq), _p(dwk), _p(ws), n, _stream(dev)))
    return oq, ok, dwq, dwk


def _norm_args(x, w, resid, what="x"):
    dt = _of(_DTYPES, x.dtype, "dtype")
    _need(x.dim() == 2, f"{what} must be [rows, K]")
    rows, K = x.shape
    ldx = _rows(x, rows, K, x.dtype, what)
    _vec(w, K, x.dtype, "w")
    if resid is None:
        return dt, dt, rows, K, ldx, K
    rt = _of(_DTYPES, resid.dtype, "the residual's dtype")
    _need(rt in (dt, T2I_F32), "the residual must have the operands' dtype or be fp32", 1)
    return dt, rt, rows, K, ldx, _rows(resid, rows, K, resid.dtype, "the residual")


def _norm_sum(resid, rows, K, ldr, inplace):
    """(tensor, pointer, stride) of the sum"""
    if resid is None:
        _need(not inplace, "inplace goes with a residual", 1)
        return None, None, K
    if inplace:
        return resid, resid.data_ptr(), ldr
    h = resid.new_empty((rows, K))
    return h, h.data_ptr(), K


def add_rms_norm(x: torch.Tensor, w: Optional[torch.Tensor] = None, resid: Optional[torch.Tensor] = None, *,
                 eps: float = 1e-6, inplace: bool = False, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The residual's addition and an RMS norm (``t2i_op_add_rms_norm``): ``h = resid + x``,
    ``y = h / sqrt(mean(h^2) + eps) * w`` for ``x [rows, K]``, ``w [K]`` (or None: ones) of
    bf16 or fp32 and ``resid [rows, K]`` of that type or fp32.  Returns ``(y, h)``; with
    ``inplace`` h is written over ``resid``; without a residual h is ``x``."""
    dev = _device(x, w, resid)
    if _elsewhere(dev, stream):
        with _switch(dev, stream):
            return add_rms_norm(x, w, resid, eps=eps, inplace=inplace)
    dt, rt, rows, K, ldx, ldr = _norm_args(x, w, resid)
    h, hp, ldh = _norm_sum(resid, rows, K, ldr, inplace)
    y = x.new_empty((rows, K))
    _check(load().t2i_op_add_rms_norm(dt, rt, rows, K, x.data_ptr(), ldx, _p(resid), ldr, _p(w), eps, hp, ldh,
                                      y.data_ptr(), K, _stream(dev)))
    if inplace:
        _written(resid)
    return y, (x if h is None else h)


def add_rms_norm_i8(x: torch.Tensor, w: Optional[torch.Tensor] = None, resid: Optional[torch.Tensor] = None, *,
                    eps: float = 1e-6, inplace: bool = False,
                    stream=None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """:func:`add_rms_norm` with y in 8 bits (``t2i_op_add_rms_norm_i8``): ``(q int8 [rows, K
    rounded up to 128], scale fp32 [rows], h)``, what :func:`linear_i8` takes."""
    dev = _device(x, w, resid)
    if _elsewhere(dev, stream):
        with _switch(dev, stream):
            return add_rms_norm_i8(x, w, resid, eps=eps, inplace=inplace)
    dt, rt, rows, K, ldx, ldr = _norm_args(x, w, resid)
    h, hp, ldh = _norm_sum(resid, rows, K, ldr, inplace)
    ldq = (K + 127) // 128 * 128
    q = x.new_empty((rows, ldq), dtype=torch.int8)
    scale = x.new_empty(rows, dtype=torch.float32)
    _check(load().t2i_op_add_rms_norm_i8(dt, rt, rows, K, x.data_ptr(), ldx, _p(resid), ldr, _p(w), eps, hp, ldh,
                                         q.data_ptr(), ldq, scale.data_ptr(), _stream(dev)))
    if inplace:
        _written(resid)
    return q, scale, (x if h is None else h)


def add_rms_norm_backward(dy: torch.Tensor, h: torch.Tensor, w: Optional[torch.Tensor] = None,
                          dh: Optional[torch.Tensor] = None, *, eps: float = 1e-6,
                          stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor]]:
    """Gradients of :func:`add_rms_norm` (``t2i_op_add_rms_norm_backward``) from y's, ``dy``,
    the sum ``h`` that it returned and the gradient ``dh`` that reaches the sum from elsewhere
    (or None): ``(dx, dresid, dw)``.  dx, of dy's type, is the gradient of x and of the
    residual alike; where the residual is fp32 beside bf16 operands it comes in both types,
    else dresid is None.  dw is None without a weight."""
    dev = _device(dy, h, w, dh)
    if _elsewhere(dev, stream):
        with _switch(dev, stream):
            return add_rms_norm_backward(dy, h, w, dh, eps=eps)
    dt, rt, rows, K, lddy, ldh = _norm_args(dy, w, h, "dy")
    lddh = K if dh is None else _rows(dh, rows, K, h.dtype, "dh")
    lib = load()
    dx = dy.new_empty((rows, K))
    dresid = h.new_empty((rows, K)) if rt != dt else None
    dw, n, ws = None, 0, None
    if w is not None:
        dw = w.new_empty(K)
        n = lib.t2i_op_add_rms_norm_backward_ws_bytes(rows, K)
        ws = dy.new_empty(n, dtype=torch.uint8) if n else None
    _check(lib.t2i_op_add_rms_norm_backward(dt, rt, rows, K, dy.data_ptr(), lddy, h.data_ptr(), ldh, _p(w), eps,
                                            _p(dh), lddh, dx.data_ptr(), K, _p(dresid), K, _p(dw), _p(ws), n,
                                            _stream(dev)))
    return dx, dresid, dw


def _adapter_args(x, w, a, b, index, scale):
    dt = _of(_DTYPES, x.dtype, "dtype")
    _need(x.dim() == 2 and w.dim() == 2 and a.dim() == 3, "x and w must be matrices, a [n, rank, K]")
    (M, K), N, (n, r, _) = x.shape, w.shape[0], a.shape
    ldx, ldw = _rows(x, M, K, x.dtype, "x"), _rows(w, N, K, x.dtype, "w")
    for t, shape, what in ((a, (n, r, K), "a"), (b, (n, N, r), "b")):
        if t.dtype is not x.dtype or t.shape != shape or not t.is_contiguous():
            raise T2IError(2, f"{what}: expected {shape} {x.dtype}, contiguous")
    _need(n < _INT and r < _INT, "2^31 adapters or ranks, or more")
    _vec(index, M, torch.int32, "index")
    _vec(scale, n, torch.float32, "scale")
    return dt, M, N, K, n, r, ldx, ldw


def adapter_linear(x: torch.Tensor, w: torch.Tensor, a: torch.Tensor, b: torch.Tensor,
                   bias: Optional[torch.Tensor] = None, *, index: Optional[torch.Tensor] = None,
                   scale: Optional[torch.Tensor] = None, epilogue: str = "store",
                   resid: Optional[torch.Tensor] = None, resid_copy: Optional[torch.Tensor] = None,
                   gate: Optional[torch.Tensor] = None, save_t: bool = False, stream=None):
    """A linear layer shared by rows with low-rank adapters of their own
    (``t2i_op_adapter_linear``): ``y = x w^T + bias + s_i (x a_i^T) b_i^T`` with ``i =
    index[row]`` (int32 ``[M]``; outside ``0 .. n-1``: no adapter; None: adapter 0 for all) for
    ``x [M, K]``, ``w [N, K]``, ``a [n, rank, K]``, ``b [n, N, rank]`` of one dtype (bf16 or
    fp32) and ``scale`` fp32 ``[n]`` (None: ones), with the epilogues of :func:`linear_i8`.
    With ``save_t`` also ``t = s_i x a_i^T`` (fp32 ``[M, rank rounded up to 32]``) that
    :func:`adapter_linear_backward` takes."""
    dev = _device(x, w, a, b, bias, index, scale, resid, resid_copy, gate)
    if _elsewhere(dev, stream):
        with _switch(dev, stream):
            return adapter_linear(x, w, a, b, bias, index=index, scale=scale, epilogue=epilogue, resid=resid,
                                  resid_copy=resid_copy, gate=gate, save_t=save_t)
    dt, M, N, K, n, r, ldx, ldw = _adapter_args(x, w, a, b, index, scale)
    epi = _of(EPILOGUES, epilogue, "epilogue")
    _vec(bias, N, x.dtype, "bias")
    _vec(gate, N, torch.float32, "gate")
    ldr, out = N, None
    if epi >= _lib.T2I_EPI_RESID:
        _need(resid is not None, "the resid epilogues need resid", 1)
        ldr = _rows(resid, M, N, torch.float32, "resid")
        if resid_copy is not None:
            ldc = _rows(resid_copy, M, N, torch.bfloat16, "resid_copy")
            _need(M == 1 or ldc == ldr, "resid_copy must have resid's row stride")
    else:
        _need(resid is None and resid_copy is None, "resid goes with the resid epilogues", 1)
        out = x.new_empty((M, N))
    _need((gate is not None) == (epilogue == "resid_gated"), "gate goes with resid_gated", 1)
    ldt = (r + 31) // 32 * 32
    t = x.new_empty((M, ldt), dtype=torch.float32)
    _check(load().t2i_op_adapter_linear(dt, epi, M, N, K, x.data_ptr(), ldx, w.data_ptr(), ldw, _p(bias), n, r,
                                        a.data_ptr(), b.data_ptr(), _p(scale), _p(index), t.data_ptr(), ldt, _p(out),
                                        N, _p(resid), ldr, _p(resid_copy), _p(gate), _stream(dev)))
    if out is None:
        _written(resid, resid_copy)
        out = resid
    return (out, t) if save_t else out


def adapter_linear_backward(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor, a: torch.Tensor, b: torch.Tensor,
                            t: torch.Tensor, *, index: Optional[torch.Tensor] = None,
                            scale: Optional[torch.Tensor] = None, need_dx: bool = True, need_dab: bool = True,
                            stream=None):
    """Gradients of :func:`adapter_linear` (epilogue ``store``) for adapters trained beside a
    frozen layer (``t2i_op_adapter_linear_backward``): ``(dx, da, db)`` from y's gradient ``dy
    [M, N]``, the forward pass's operands and its ``t``; None for those not asked for."""
    dev = _device(dy, x, w, a, b, t, index, scale)
    if _elsewhere(dev, stream):
        with _switch(dev, stream):
            return adapter_linear_backward(dy, x, w, a, b, t, index=index, scale=scale, need_dx=need_dx,
                                           need_dab=need_dab)
    dt, M, N, K, n, r, ldx, ldw = _adapter_args(x, w, a, b, index, scale)
    lddy = _rows(dy, M, N, x.dtype, "dy")
    ldt = _rows(t, M, (r + 31) // 32 * 32, torch.float32, "t")
    lib = load()
    dx = x.new_empty((M, K)) if need_dx else None
    da, db = (a.new_empty(a.shape), b.new_empty(b.shape)) if need_dab else (None, None)
    nb = lib.t2i_op_adapter_linear_backward_ws_bytes(dt, M, N, K, n, r)
    ws = x.new_empty(nb, dtype=torch.uint8)
    _check(lib.t2i_op_adapter_linear_backward(
        dt, M, N, K, dy.data_ptr(), lddy, x.data_ptr(), ldx, w.data_ptr(), ldw, n, r, a.data_ptr(), b.data_ptr(),
        _p(scale), _p(index), t.data_ptr(), ldt, _p(dx), K, _p(da), _p(db), ws.data_ptr(), nb, _stream(dev)))
    return dx, da, db
