"""The block operators on the host: the oracle's formulas against differences,
and every refusal of the entry points (nothing here reaches a GPU: each call
fails its argument checks)."""
import ctypes as C
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2607_26566_amd as t2i
from paper_2607_26566_amd import _lib
from conftest import ROOT
from oracle import blocks

F32, BF16 = _lib.T2I_F32, _lib.T2I_BF16
INVALID, SHAPE, WORKSPACE = 1, 2, 4
P = 1 << 20   # an aligned address that no call here reads


def rng(seed):
    return np.random.default_rng(seed)


# ------------------------------------------------------------------ oracle

@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_gated_gradients_against_differences(act):
    r = rng(1)
    M, F, K = 3, 4, 5
    p = dict(x=r.normal(size=(M, K)), wg=r.normal(size=(F, K)), wu=r.normal(size=(F, K)),
             bg=r.normal(size=F), bu=r.normal(size=F))
    dout = r.normal(size=(M, F))
    loss = lambda q: (blocks.gated(act, *blocks.gated_pre(**q)) * dout).sum()  # noqa: E731
    g, u = blocks.gated_pre(**p)
    got = blocks.gated_grads(act, dout, p["x"], p["wg"], p["wu"], g, u)
    for name in p:
        num = np.zeros_like(p[name])
        for i in np.ndindex(*p[name].shape):
            hi, lo = ({**p, name: p[name].copy()} for _ in range(2))
            hi[name][i] += 1e-6
            lo[name][i] -= 1e-6
            num[i] = (loss(hi) - loss(lo)) / 2e-6
        # central differences: h^2 f''' / 6 + 2^-53 |f| / h, both below 1e-8 here
        assert np.allclose(got["d" + name], num, rtol=1e-6, atol=1e-7), name


@pytest.mark.parametrize("pairing", ["pairs", "halves"])
def test_qk_gradients_against_differences(pairing):
    r = rng(2)
    rows, H, d, eps = 3, 2, 16, 1e-5
    x, w, dy = r.normal(size=(rows, H, d)), r.normal(size=d), r.normal(size=(rows, H, d))
    ang = r.uniform(-3, 3, size=(4, d // 2))
    rot = dict(table=np.stack([np.cos(ang), np.sin(ang)], -1), pos=np.array([2, -1, 0]), pairing=pairing)
    loss = lambda a, b: (blocks.qk_norm_rope(a, b, eps, **rot) * dy).sum()  # noqa: E731
    dx, dw = blocks.qk_norm_rope_grads(dy, x, w, eps, **rot)
    for v, got, f in ((x, dx, lambda t: loss(t, w)), (w, dw, lambda t: loss(x, t))):
        num = np.zeros_like(v)
        for i in np.ndindex(*v.shape):
            hi, lo = v.copy(), v.copy()
            hi[i] += 1e-6
            lo[i] -= 1e-6
            num[i] = (f(hi) - f(lo)) / 2e-6
        assert np.allclose(got, num, rtol=1e-6, atol=1e-7)


def test_rotation_by_complex_numbers():
    r = rng(3)
    x, ang = r.normal(size=(5, 3, 8)), r.uniform(-9, 9, size=(5, 4))
    t = np.stack([np.cos(ang), np.sin(ang)], -1)
    z = np.exp(1j * ang)[:, None]
    pairs = blocks.rotate(x, t, np.arange(5), "pairs")
    halves = blocks.rotate(x, t, np.arange(5), "halves")
    assert np.allclose(pairs[..., 0::2] + 1j * pairs[..., 1::2], (x[..., 0::2] + 1j * x[..., 1::2]) * z)
    assert np.allclose(halves[..., :4] + 1j * halves[..., 4:], (x[..., :4] + 1j * x[..., 4:]) * z)
    assert np.allclose(blocks.rotate(pairs, t, np.arange(5), "pairs", inverse=True), x)


def test_quantising_by_whole_number_arithmetic():
    """Against fractions: every q is the nearest, and even where two are equally near."""
    from fractions import Fraction
    x = np.array([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -126.5, 126.5], [3.0, 1.0, -2.0, 0.1, 0, 0, 0, 1e-30]])
    q, s = blocks.quant_rows(x)
    assert s[0] == 1 and list(q[0]) == [127, 0, 2, 2, 0, -2, -126, 126]
    for row, qs, sc in zip(x, q, s):
        for v, n in zip(row, qs):
            f = Fraction(float(v)) / Fraction(float(sc))
            assert abs(f - int(n)) < Fraction(1, 2) or (abs(f - int(n)) == Fraction(1, 2) and n % 2 == 0)
    q, s = blocks.quant_rows(np.array([[0.0, 0.0], [np.nan, 1.0], [np.inf, 1.0]]))
    assert s[0] == np.float32(2.0 ** -126) and np.isnan(s[1:]).all() and not q.any()


# ------------------------------------------------------------------ refusals of the C entry points

def call(name, spec, **change):
    """Status of the call with the spec's arguments, some changed."""
    args = dict(spec)
    assert set(change) <= set(args), change
    args.update(change)
    return getattr(t2i.load(), name)(*args.values())


def check_refusals(name, spec, cases):
    for change, status in cases:
        assert call(name, spec, **change) == status, (name, change)
        assert t2i.load().t2i_ops_last_error(), (name, change)


QUANT = dict(dtype=BF16, rows=3, K=130, x=P, ldx=130, q=P, ldq=256, scale=P, stream=None)


def test_quant_rows_refuses():
    check_refusals("t2i_op_quant_rows", QUANT, [
        (dict(dtype=2), INVALID), (dict(rows=0), SHAPE), (dict(rows=-1), SHAPE), (dict(K=0), SHAPE),
        (dict(x=None), INVALID), (dict(q=None), INVALID), (dict(scale=None), INVALID),
        (dict(ldx=129), SHAPE), (dict(ldq=240), SHAPE), (dict(ldq=264), SHAPE),
        (dict(x=P + 1), INVALID), (dict(dtype=F32, x=P + 2), INVALID), (dict(q=P + 8), INVALID),
        (dict(scale=P + 2), INVALID)])


I8 = dict(dtype=BF16, epilogue=0, M=3, N=5, K=130, A=P, lda=256, a_scale=P, W=P, ldw=256, w_scale=P,
          bias=None, out=P, ldo=5, resid=None, ldr=5, resid_copy=None, gate=None, stream=None)


def test_linear_i8_refuses():
    res = dict(epilogue=_lib.T2I_EPI_RESID, out=None, resid=P)
    gated = dict(res, epilogue=_lib.T2I_EPI_RESID_GATED, gate=P)
    check_refusals("t2i_op_linear_i8", I8, [
        (dict(dtype=3), INVALID), (dict(epilogue=5), INVALID), (dict(epilogue=-1), INVALID),
        (dict(M=0), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(K=131072), SHAPE),
        (dict(M=2 ** 30, N=2 ** 30), SHAPE), (dict(A=None), INVALID), (dict(W=None), INVALID),
        (dict(a_scale=None), INVALID), (dict(w_scale=None), INVALID), (dict(out=None), INVALID),
        (dict(lda=240), SHAPE), (dict(lda=264), SHAPE), (dict(ldw=130), SHAPE), (dict(lda=2 ** 24), SHAPE),
        (dict(ldw=2 ** 24), SHAPE), (dict(ldo=4), INVALID),
        (dict(A=P + 8), INVALID), (dict(W=P + 1), INVALID), (dict(a_scale=P + 1), INVALID),
        (dict(w_scale=P + 2), INVALID), (dict(bias=P + 1), INVALID), (dict(out=P + 1), INVALID),
        (dict(res, resid=None), INVALID), (dict(res, ldr=4), INVALID), (dict(res, resid=P + 2), INVALID),
        (dict(res, resid_copy=P + 1), INVALID), (dict(gated, gate=None), INVALID),
        (dict(gated, gate=P + 2), INVALID)])


GATED = dict(dtype=BF16, act=_lib.T2I_EPI_SILU, M=3, F=8, K=16, A=P, lda=16, Wg=P, Wu=P, ldw=16, bg=None,
             bu=None, out=P, ldo=8, pre=None, ldp=16, stream=None)


def test_gated_linear_refuses():
    check_refusals("t2i_op_gated_linear", GATED, [
        (dict(dtype=2), INVALID), (dict(act=0), INVALID), (dict(act=3), INVALID), (dict(M=0), SHAPE),
        (dict(F=0), SHAPE), (dict(K=0), SHAPE), (dict(F=2 ** 29), SHAPE), (dict(A=None), INVALID),
        (dict(Wg=None), INVALID), (dict(Wu=None), INVALID), (dict(out=None), INVALID),
        (dict(bg=P), INVALID), (dict(bu=P), INVALID), (dict(lda=8), SHAPE), (dict(ldw=8), SHAPE),
        (dict(ldo=0), SHAPE), (dict(pre=P, ldp=8), SHAPE), (dict(F=12, ldo=16), SHAPE),
        (dict(K=12), SHAPE), (dict(lda=20), SHAPE), (dict(ldw=20), SHAPE), (dict(ldo=12), SHAPE),
        (dict(lda=2 ** 23), SHAPE), (dict(ldw=2 ** 23), SHAPE),
        (dict(pre=P, ldp=18), SHAPE), (dict(A=P + 8), INVALID), (dict(Wg=P + 8), INVALID),
        (dict(Wu=P + 8), INVALID), (dict(out=P + 8), INVALID), (dict(pre=P + 8), INVALID),
        (dict(bg=P + 8, bu=P), INVALID), (dict(dtype=F32, A=P + 2), INVALID)])


GBWD = dict(dtype=BF16, act=_lib.T2I_EPI_SILU, M=3, F=8, K=16, A=P, lda=16, Wg=P, Wu=P, ldw=16, pre=P,
            ldp=16, dout=P, ldd=8, dA=P, ldda=16, dWg=P, dWu=P, lddw=16, dbg=P, dbu=P, ws=P,
            ws_bytes=1 << 20, stream=None)


def test_gated_linear_backward_refuses():
    need = t2i.load().t2i_op_gated_linear_backward_ws_bytes(BF16, 3, 8, 16)
    assert 0 < need <= 1 << 20
    check_refusals("t2i_op_gated_linear_backward", GBWD, [
        (dict(dtype=2), INVALID), (dict(act=4), INVALID), (dict(M=0), SHAPE), (dict(F=0), SHAPE),
        (dict(K=0), SHAPE), (dict(A=None), INVALID), (dict(Wg=None), INVALID), (dict(Wu=None), INVALID),
        (dict(pre=None), INVALID), (dict(dout=None), INVALID), (dict(ws=None), INVALID),
        (dict(dbg=None), INVALID), (dict(dbu=None), INVALID),
        (dict(dA=None, dWg=None, dWu=None, dbg=None, dbu=None), INVALID),
        (dict(lda=8), SHAPE), (dict(ldw=8), SHAPE), (dict(ldp=8), SHAPE), (dict(ldd=0), SHAPE),
        (dict(ldda=8), SHAPE), (dict(lddw=8), SHAPE), (dict(K=12), SHAPE), (dict(F=4), SHAPE),
        (dict(ldda=20), SHAPE), (dict(lddw=20), SHAPE), (dict(ldd=12), SHAPE), (dict(ldp=18), SHAPE), (dict(lda=2 ** 23), SHAPE),
        (dict(ldw=2 ** 23), SHAPE), (dict(dA=P + 8), INVALID),
        (dict(dWg=P + 8), INVALID), (dict(dWu=P + 8), INVALID), (dict(dbg=P + 8), INVALID),
        (dict(ws=P + 128), INVALID), (dict(ws_bytes=need - 1), WORKSPACE)])
    ws = t2i.load().t2i_op_gated_linear_backward_ws_bytes
    assert ws(2, 3, 8, 8) == 0 and ws(BF16, 0, 8, 8) == 0 and ws(BF16, 3, 0, 8) == 0 and ws(F32, 3, 8, 0) == 0


QK = dict(dtype=BF16, rows=3, heads_q=2, heads_k=1, head_dim=16, q=P, ldq=32, k=P, ldk=16, wq=None, wk=None,
          eps=1e-6, pairing=0, table=P, n_pos=3, pos=None, q_out=P, ldqo=32, k_out=P, ldko=16, stream=None)
QK_BAD = [
    (dict(dtype=2), INVALID), (dict(pairing=2), INVALID), (dict(rows=0), SHAPE),
    (dict(heads_q=0, heads_k=0), SHAPE), (dict(heads_q=-1), SHAPE), (dict(head_dim=12), SHAPE),
    (dict(head_dim=264, ldq=528, ldk=264), SHAPE), (dict(head_dim=8, pairing=1), SHAPE),
    (dict(rows=2 ** 30, pos=P), SHAPE), (dict(q=None), INVALID), (dict(k=None), INVALID),
    (dict(ldq=24), SHAPE), (dict(ldk=8), SHAPE), (dict(ldq=36), SHAPE), (dict(q=P + 8), INVALID),
    (dict(k=P + 8), INVALID), (dict(wq=P + 8), INVALID), (dict(wk=P + 2), INVALID),
    (dict(table=P + 8), INVALID), (dict(pos=P + 2), INVALID), (dict(eps=-1e-6), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(n_pos=2), SHAPE),
    (dict(n_pos=0, pos=P), SHAPE)]


def test_qk_norm_rope_refuses():
    check_refusals("t2i_op_qk_norm_rope", QK, QK_BAD + [
        (dict(q_out=None), INVALID), (dict(k_out=None), INVALID), (dict(ldqo=24), SHAPE),
        (dict(ldko=20), SHAPE), (dict(q_out=P + 8), INVALID), (dict(k_out=P + 8), INVALID)])


QKB = dict(dtype=BF16, rows=3, heads_q=2, heads_k=1, head_dim=16, dq=P, lddq=32, dk=P, lddk=16, q=P, ldq=32,
           k=P, ldk=16, wq=None, wk=None, eps=1e-6, pairing=0, table=P, n_pos=3, pos=None, dq_in=P,
           lddqi=32, dk_in=P, lddki=16, dwq=P, dwk=P, ws=P, ws_bytes=1 << 20, stream=None)


def test_qk_norm_rope_backward_refuses():
    need = t2i.load().t2i_op_qk_norm_rope_backward_ws_bytes(3, 2, 1, 16)
    assert 0 < need <= 1 << 20
    check_refusals("t2i_op_qk_norm_rope_backward", QKB, QK_BAD + [
        (dict(dq=None), INVALID), (dict(dk=None), INVALID), (dict(lddq=24), SHAPE), (dict(lddk=20), SHAPE),
        (dict(dq=P + 8), INVALID), (dict(dk=P + 8), INVALID), (dict(dq_in=None), INVALID),
        (dict(lddki=8), SHAPE), (dict(dwq=P + 1), INVALID), (dict(ws=P + 64), INVALID),
        (dict(ws=None), WORKSPACE), (dict(ws_bytes=need - 1), WORKSPACE)])
    ws = t2i.load().t2i_op_qk_norm_rope_backward_ws_bytes
    assert ws(0, 1, 1, 16) == 0 and ws(3, 0, 0, 16) == 0 and ws(3, 1, 1, 12) == 0 and ws(3, 1, 1, 264) == 0


def test_launches_of_too_many_threads_are_refused():
    """A launch holds fewer than 2^32 threads: sizes past that are refused here, not
    by the launch (for the gradients: before the first of their kernels)."""
    need = t2i.load().t2i_op_gated_linear_backward_ws_bytes
    check_refusals("t2i_op_quant_rows", QUANT, [
        (dict(rows=2 ** 26 - 4), SHAPE), (dict(rows=2 ** 24 - 4, K=2056, ldx=2056, ldq=2176), SHAPE)])
    check_refusals("t2i_op_linear_i8", I8, [
        (dict(M=2 ** 29, N=1), SHAPE), (dict(M=2 ** 18, N=2 ** 17, ldo=2 ** 17), SHAPE)])
    check_refusals("t2i_op_gated_linear", GATED, [
        (dict(M=2 ** 29, F=8, ldo=8, ldp=16), SHAPE), (dict(M=2 ** 18, F=2 ** 16, ldo=2 ** 16, ldp=2 ** 17), SHAPE)])
    big = dict(M=2 ** 21, F=2 ** 13, ldp=2 ** 14, ldd=2 ** 13)
    check_refusals("t2i_op_gated_linear_backward", GBWD, [(big, SHAPE)])
    assert need(BF16, big["M"], big["F"], 16) == 0 and need(BF16, big["M"] // 2, big["F"], 16) > 0
    wide = dict(rows=2 ** 26, heads_q=1, heads_k=0, head_dim=256, ldq=256, ldqo=256, pos=P)
    check_refusals("t2i_op_qk_norm_rope", QK, [(wide, SHAPE)])


# ------------------------------------------------------------------ refusals of the Python calls

def test_python_calls_refuse_host_tensors():
    x, w = torch.zeros(4, 128), torch.zeros(8, 128)
    q = torch.zeros(4, 128, dtype=torch.int8)
    h = torch.zeros(4, 2, 64)
    for f in (lambda: t2i.quant_rows(x), lambda: t2i.linear_i8(q, x[:, 0], q, x[:, 0], K=128),
              lambda: t2i.gated_linear(x, w, w), lambda: t2i.gated_linear_backward(x, x, w, w, x),
              lambda: t2i.qk_norm_rope(h, h), lambda: t2i.qk_norm_rope_backward(h, h, h, h)):
        with pytest.raises(t2i.T2IError) as e:
            f()
        assert e.value.status == INVALID


def test_the_package_imports_with_a_torch_that_has_no_gpu():
    """Such a torch lacks the names behind the current device and stream; the calls still
    refuse host tensors."""
    code = """
import torch
for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
import paper_2607_26566_amd as t2i
x = torch.zeros(4, 128)
try:
    t2i.quant_rows(x)
except t2i.T2IError as e:
    assert e.status == 1
else:
    raise SystemExit("not refused")
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_python_calls_refuse_sizes_past_32_bits(monkeypatch):
    """2^32 + 8 of anything would reach the library as 8."""
    from paper_2607_26566_amd import ops
    monkeypatch.setattr(ops, "_device", lambda *a: 0)
    monkeypatch.setattr(ops, "_elsewhere", lambda *a: False)
    monkeypatch.setattr(ops, "_stream", lambda dev: 0)
    big = 2 ** 32 + 8

    def of(*shape, dtype=torch.bfloat16):   # (no memory behind it)
        return torch.empty(shape, dtype=dtype, device="meta")
    x, w, h = of(big, 8), of(8, 8), of(big, 1, 8)
    q8, s8 = of(big, 128, dtype=torch.int8), of(big, dtype=torch.float32)
    w8, ws = of(8, 128, dtype=torch.int8), of(8, dtype=torch.float32)
    pre, few, table = of(big, 16, dtype=torch.float32), of(8, 1, 8), of(big, 4, 2, dtype=torch.float32)
    for f in (lambda: t2i.quant_rows(x), lambda: t2i.quant_rows(of(1, big)),
              lambda: t2i.linear_i8(q8, s8, w8, ws, K=8), lambda: t2i.linear_i8(w8, ws, q8, s8, K=8),
              lambda: t2i.linear_i8(of(8, 2 ** 32 + 128, dtype=torch.int8), ws, w8, ws, K=8),
              lambda: t2i.gated_linear(x, w, w), lambda: t2i.gated_linear(w, x, x),
              lambda: t2i.gated_linear_backward(x, x, w, w, pre), lambda: t2i.qk_norm_rope(h, h),
              lambda: t2i.qk_norm_rope(few, few, table=table), lambda: t2i.qk_norm_rope_backward(h, h, h, h)):
        with pytest.raises(t2i.T2IError, match=r"2\^31") as e:
            f()
        assert e.value.status == SHAPE


class OnDevice(torch.Tensor):
    """A host tensor that says it lies on device 0."""

    def get_device(self):
        return 0


def block_calls(mk):
    """(call, its floating operands) of every Python call, on operands that mk makes."""
    x, wg, wu, b, dout, pre, g = mk(4, 64), mk(8, 64), mk(8, 64), mk(8), mk(4, 8), mk(4, 16), mk(8)
    q8, w8 = torch.zeros(4, 128, dtype=torch.int8).as_subclass(OnDevice), torch.zeros(8, 128, dtype=torch.int8)
    w8, sa, sw, r, c = w8.as_subclass(OnDevice), mk(4), mk(8), mk(4, 8), mk(4, 8)
    q, k, dq, dk, nq, nk, t = mk(4, 2, 16), mk(4, 1, 16), mk(4, 2, 16), mk(4, 1, 16), mk(16), mk(16), mk(4, 8, 2)
    return [
        (lambda x: t2i.quant_rows(x), [x]),
        (lambda sa, sw, b, r, c, g: t2i.linear_i8(q8, sa, w8, sw, b, K=64, epilogue="resid_gated", resid=r,
                                                  resid_copy=c, gate=g), [sa, sw, b, r, c, g]),
        (lambda x, wg, wu, b, c: t2i.gated_linear(x, wg, wu, b, c), [x, wg, wu, b, g]),
        (lambda *a: t2i.gated_linear_backward(*a), [dout, x, wg, wu, pre]),
        (lambda q, k, nq, nk, t: t2i.qk_norm_rope(q, k, nq, nk, table=t), [q, k, nq, nk, t]),
        (lambda dq, dk, q, k, nq, nk, t: t2i.qk_norm_rope_backward(dq, dk, q, k, nq, nk, table=t),
         [dq, dk, q, k, nq, nk, t])]


def test_python_calls_refuse_what_differentiation_follows(monkeypatch):
    from torch.autograd import forward_ad
    from paper_2607_26566_amd import ops

    class Through(Exception):
        pass

    def through(*a):
        raise Through
    monkeypatch.setattr(ops, "_elsewhere", through)   # what follows the checks of the operands
    for call, operands in block_calls(lambda *s: torch.ones(s).as_subclass(OnDevice)):
        with pytest.raises(Through):
            call(*operands)
        for i, t in enumerate(operands):
            leaf = t.clone().requires_grad_()
            for v in (leaf, leaf * 1):
                args = [*operands[:i], v, *operands[i + 1:]]
                with pytest.raises(t2i.T2IError, match="requires a gradient") as e:
                    call(*args)
                assert e.value.status == INVALID
                with torch.no_grad(), pytest.raises(Through):
                    call(*args)
                with pytest.raises(Through):
                    call(*(a.detach() for a in args))
            with forward_ad.dual_level():
                dual = forward_ad.make_dual(t, torch.ones_like(t))
                with pytest.raises(t2i.T2IError, match="tangent"):
                    call(*operands[:i], dual, *operands[i + 1:])
                with pytest.raises(Through):
                    call(*operands)


def test_operands_written_in_place_are_marked(monkeypatch):
    """Differentiation that saved them has to find out that their values are gone."""
    from paper_2607_26566_amd import ops

    class Done:   # (a library whose calls succeed)
        t2i_op_linear_i8 = t2i_op_qk_norm_rope = staticmethod(lambda *a: 0)
    monkeypatch.setattr(ops, "load", Done)
    monkeypatch.setattr(ops, "_elsewhere", lambda *a: False)
    monkeypatch.setattr(ops, "_stream", lambda dev: 0)

    def mk(*s, dtype=torch.float32):
        return torch.ones(s, dtype=dtype).as_subclass(OnDevice)
    weight = torch.ones(4, 16, requires_grad=True)
    q8, s8 = mk(4, 128, dtype=torch.int8), mk(4)

    def spoiled(t, call):
        """Whether the gradient of weight * t fails once the call has written t."""
        y = (weight * t.as_subclass(torch.Tensor).reshape(4, 16)).sum()
        call()
        try:
            y.backward()
        except RuntimeError as e:
            assert "inplace" in str(e)
            return True
        return False
    q, k, r, c = mk(4, 1, 16), mk(4, 1, 16), mk(4, 4), mk(4, 4, dtype=torch.bfloat16)
    for t in (q, k):
        assert spoiled(t, lambda: t2i.qk_norm_rope(q, k, inplace=True))
        assert not spoiled(t, lambda: t2i.qk_norm_rope(q, k))
    before = r._version, c._version
    t2i.linear_i8(q8, s8, q8, s8, K=128, epilogue="resid", resid=r, resid_copy=c)
    assert (r._version, c._version) == (before[0] + 1, before[1] + 1)
    with torch.inference_mode():
        q, k = mk(4, 1, 16), mk(4, 1, 16)
        t2i.qk_norm_rope(q, k, inplace=True)


def launched_threads(op, dtype, M, F, K):
    """Threads of the launch that a product takes (op as in t2i_test_block_tile)."""
    v = [C.c_int() for _ in range(4)]
    assert t2i.load().t2i_test_block_tile(op, int(dtype == BF16), M, F, K, *map(C.byref, v))
    bm, bn, _, slices = (x.value for x in v)
    rows, cols = {0: (M, F), 1: (M, 2 * F), 2: (M, K), 3: (F, K)}[op]
    tiles = -(-rows // bm) * -(-cols // bn) * (2 if op == 3 else 1)
    waves = {(256, 256): 8, (128, 128): 8, (64, 128): 8, (32, 128): 4, (64, 64): 4, (32, 64): 4, (16, 32): 1}
    return tiles * waves[bm, bn] * 64 * slices


@pytest.mark.parametrize("op,dtype", [(0, BF16), (1, BF16), (1, F32), (2, BF16), (2, F32), (3, BF16), (3, F32)])
def test_no_allowed_product_launches_too_many_threads(op, dtype):
    """Sizes just inside the limit of 2^23 pieces of 64 x 64 outputs, of every form."""
    r, most = rng(5 + op), 2 ** 23 - 1
    cases = 0
    for i in range(4000):
        short = int(2 ** r.uniform(0, 20)) if i % 4 else int(r.integers(1, 65))
        long = most // -(-short // 64) * 64 - int(r.integers(0, 200))
        deep = int(2 ** r.uniform(0, 14))
        rows, cols = (long, short) if r.random() < 0.5 else (short, long)
        if op == 0:
            sizes = rows, cols, deep
        elif op == 1:
            sizes = rows, max(1, cols // 2), deep
        elif op == 2:
            sizes = rows, deep, cols
        else:
            sizes = deep, max(1, rows // 2), cols
        M, F, K = sizes
        # (an operand's rows lie less than 8 MiB apart)
        if F > 2 ** 28 or op > 1 and F >= 2 ** 20 or op and K * (2 if dtype == BF16 else 4) >= 2 ** 23:
            continue
        cases += 1
        assert launched_threads(op, dtype, M, F, K) < 2 ** 32, sizes
    assert cases > 500
