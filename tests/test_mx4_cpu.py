"""Refusals of the microscaled 4-bit operators, the norms around a block and the
gated activation, without a GPU, and the references that the GPU tests use."""
import ctypes as C
import math

import pytest
import torch

import paper_2605_28803_amd as oq
from paper_2605_28803_amd import _lib
from tests import mx4_ref as R

OK, NULL, SHAPE, ALIGN, ARG = 0, -1, -2, -3, -7
P16, P4, P2, P1 = (C.c_void_p(0x10000 + x) for x in (0, 4, 2, 1))  # never dereferenced on error paths


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def test_step_bytes(lib):
    for K, want in ((1, 16), (32, 16), (512, 16), (513, 32), (544, 32), (2048, 64), (65536, 2048)):
        assert lib.oq_mx4_step_bytes(K) == oq.mx4_step_bytes(K) == want
    assert lib.oq_mx4_step_bytes(0) == 0


def _quantize(lib, X=P16, M=4, K=64, ldx=64, dtype=0, had=1, q=P16, s=P16):
    return lib.oq_mx4_quantize(X, M, K, ldx, dtype, had, q, s, None)


CODES = [(dict(M=-1), SHAPE), (dict(K=0), SHAPE), (dict(K=48), SHAPE), (dict(K=65568, ldx=65568), SHAPE), (dict(ldx=56), SHAPE),
         (dict(ldx=68), ALIGN), (dict(dtype=5), ARG), (dict(X=None), NULL), (dict(q=None), NULL), (dict(s=None), NULL),
         (dict(X=P4), ALIGN), (dict(q=P4), ALIGN), (dict(s=P4), ALIGN), (dict(M=0, X=None, q=None, s=None), OK)]


@pytest.mark.parametrize("change,status", CODES + [
    (dict(dtype=2), ARG), (dict(had=0), ARG), (dict(had=16), ARG), (dict(had=256, K=256, ldx=256), ARG), (dict(had=128), SHAPE),
    (dict(had=64, K=96, ldx=96), SHAPE)])
def test_quantize_refusals(lib, change, status):
    assert _quantize(lib, **change) == status


@pytest.mark.parametrize("change,status", CODES)
def test_dequantize_refusals(lib, change, status):
    a = dict(dict(X=P16, M=4, K=64, ldx=64, dtype=0, q=P16, s=P16), **change)
    assert lib.oq_mx4_dequantize(a["q"], a["s"], a["M"], a["K"], a["X"], a["ldx"], a["dtype"], None) == status


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), SHAPE), (dict(N=0), SHAPE), (dict(K=16), SHAPE), (dict(K=80), SHAPE), (dict(K=65568), SHAPE), (dict(ldy=8), SHAPE),
    (dict(ldy=20), ALIGN), (dict(out=3), ARG), (dict(out=-1), ARG), (dict(x=None), NULL), (dict(xs=None), NULL), (dict(w=None), NULL),
    (dict(ws=None), NULL), (dict(Y=None), NULL), (dict(x=P4), ALIGN), (dict(xs=P4), ALIGN), (dict(w=P4), ALIGN), (dict(ws=P4), ALIGN),
    (dict(Y=P4), ALIGN), (dict(b=P1), ALIGN), (dict(M=0, x=None, xs=None, w=None, ws=None, Y=None), OK)])
def test_linear_refusals(lib, change, status):
    a = dict(dict(x=P16, xs=P16, M=4, w=P16, ws=P16, b=None, N=16, K=64, Y=P16, ldy=16, out=0), **change)
    assert lib.oq_mx4_linear(a["x"], a["xs"], a["M"], a["w"], a["ws"], a["b"], a["N"], a["K"], a["Y"], a["ldy"], a["out"],
                             None) == status


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), SHAPE), (dict(F=4), SHAPE), (dict(F=12, ld=24), SHAPE), (dict(F=65544, ld=131088), SHAPE), (dict(ld=120), SHAPE),
    (dict(ld=132), ALIGN), (dict(ldh=56), SHAPE), (dict(ldh=68), ALIGN), (dict(dtype=2), ARG), (dict(act=2), ARG), (dict(act=-1), ARG),
    (dict(q=P16, s=P16), ARG), (dict(H=None), NULL), (dict(GU=None), NULL), (dict(GU=P4), ALIGN), (dict(H=P4), ALIGN),
    (dict(H=None, q=P16), NULL), (dict(H=None, s=P16), NULL), (dict(H=None, q=P4, s=P16), ALIGN),
    (dict(H=None, q=P16, s=P16, F=40, ld=80), SHAPE), (dict(M=0, GU=None, H=None), OK)])
def test_activation_refusals(lib, change, status):
    a = dict(dict(GU=P16, M=4, F=64, ld=128, dtype=0, act=0, H=P16, ldh=64, q=None, s=None), **change)
    assert lib.oq_gated_activation(a["GU"], a["M"], a["F"], a["ld"], a["dtype"], a["act"], a["H"], a["ldh"], a["q"], a["s"],
                                   None) == status


def _norm(kind=1, eps=1e-6, offset=0.0, gain=0x10000, bias=None):
    return _lib.oq_norm(kind, eps, offset, gain, bias)


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), SHAPE), (dict(D=0), SHAPE), (dict(D=12), SHAPE), (dict(D=16392, ld=16392), SHAPE), (dict(ldr=56), SHAPE), (dict(ldy=56), SHAPE),
    (dict(ldro=56), SHAPE), (dict(ldh=56), SHAPE), (dict(ldr=68), ALIGN), (dict(ldy=68), ALIGN), (dict(ldro=68), ALIGN), (dict(ldh=68), ALIGN),
    (dict(dtype=2), ARG), (dict(dtype=1), ARG), (dict(rd=3), ARG), (dict(alpha=math.inf), ARG), (dict(alpha=math.nan), ARG),
    (dict(pre=_norm(kind=3)), ARG), (dict(pre=_norm(eps=0.0)), ARG), (dict(post=_norm(eps=2.0)), ARG), (dict(post=_norm(eps=math.nan)), ARG),
    (dict(post=_norm(offset=math.inf)), ARG), (dict(pre=_norm(gain=0x10004)), ALIGN), (dict(post=_norm(bias=0x10002)), ALIGN),
    (dict(q=P16, s=P16), ARG), (dict(H=None, q=P16), NULL), (dict(H=None, s=P16), NULL), (dict(H=None), NULL),
    (dict(pre=None), ARG), (dict(pre=None, H=None, scale=P16), ARG), (dict(pre=None, H=None, Ro=None), NULL), (dict(pre=_norm(kind=0)), ARG),
    (dict(R=None, Y=None), NULL), (dict(gate=P16, n_mod=0), SHAPE), (dict(shift=P16, ldm=56), SHAPE), (dict(scale=P16, ldm=68), ALIGN),
    (dict(gate=P4), ALIGN), (dict(R=P4), ALIGN), (dict(Y=P2), ALIGN), (dict(Ro=P4), ALIGN), (dict(H=P4), ALIGN), (dict(rows=P2, gate=P16), ALIGN),
    (dict(H=None, q=P16, s=P16, D=40), SHAPE), (dict(M=0, R=None, Y=None, Ro=None, H=None), OK)])
def test_residual_norm_refusals(lib, change, status):
    a = dict(R=P16, ldr=64, rd=0, Y=P16, ldy=64, dtype=0, M=4, D=64, post=None, pre=_norm(), alpha=1.0, gate=None, scale=None, shift=None,
             ldm=64, n_mod=1, rows=None, Ro=P16, ldro=64, H=P16, ldh=64, q=None, s=None)
    if "ld" in change:
        a.update(ldr=change["ld"], ldy=change["ld"], ldro=change["ld"], ldh=change["ld"])
    a.update({k: v for k, v in change.items() if k != "ld"})
    ref = lambda n: None if n is None else C.byref(n)  # noqa: E731
    assert lib.oq_residual_norm(a["R"], a["ldr"], a["rd"], a["Y"], a["ldy"], a["dtype"], a["M"], a["D"], ref(a["post"]), ref(a["pre"]),
                                a["alpha"], a["gate"], a["scale"], a["shift"], a["ldm"], a["n_mod"], a["rows"], a["Ro"], a["ldro"],
                                a["H"], a["ldh"], a["q"], a["s"], None) == status


def _z(*shape, dt=torch.float16):
    return torch.zeros(shape, dtype=dt)


@pytest.mark.parametrize("call", [
    lambda: oq.mx4_quantize(_z(4, 64)),                                        # not on a GPU
    lambda: oq.mx4_quantize(_z(4, 64, dt=torch.float32)),
    lambda: oq.mx4_quantize(_z(4, 40)),
    lambda: oq.mx4_quantize(_z(64)),
    lambda: oq.mx4_quantize(_z(64, 64).T[:, ::2]),
    lambda: oq.mx4_quantize(_z(4, 64), Xq=_z(4, 31, dt=torch.uint8)),
    lambda: oq.mx4_dequantize(_z(4, 32, dt=torch.uint8), _z(4, 2, dt=torch.uint8)),
    lambda: oq.mx4_dequantize(_z(4, 32, dt=torch.uint8), _z(4, 16, dt=torch.uint8), out_dtype=7),
    lambda: oq.mx4_linear(_z(4, 32, dt=torch.uint8), _z(4, 16, dt=torch.uint8), _z(8, 16, dt=torch.uint8), _z(8, 16, dt=torch.uint8)),
    lambda: oq.mx4_linear(_z(4, 32, dt=torch.uint8), _z(4, 16, dt=torch.uint8), _z(8, 32, dt=torch.uint8), _z(8, 16, dt=torch.uint8),
                          bias=_z(9)),
    lambda: oq.mx4_linear(_z(4, 32, dt=torch.uint8), _z(4, 16, dt=torch.uint8), _z(8, 32, dt=torch.uint8), _z(8, 16, dt=torch.uint8),
                          Y=_z(4, 8, dt=torch.bfloat16)),
    lambda: oq.gated_activation(_z(4, 65)),
    lambda: oq.gated_activation(_z(4, 80), mx4=True),
    lambda: oq.gated_activation(_z(4, 64), H=_z(4, 64)),
    lambda: oq.Norm("batch"),
    lambda: oq.Norm("rms", _z(4, 4)),
    lambda: oq.residual_norm(None),
    lambda: oq.residual_norm(_z(4, 64, dt=torch.float32)),                     # what type is h?
    lambda: oq.residual_norm(_z(4, 64), _z(4, 64, dt=torch.bfloat16)),
    lambda: oq.residual_norm(_z(4, 64), _z(5, 64)),
    lambda: oq.residual_norm(_z(4, 64), _z(4, 64), pre=oq.Norm("rms", _z(32))),
    lambda: oq.residual_norm(_z(4, 64), _z(4, 64), pre=oq.Norm("rms", _z(64, dt=torch.bfloat16))),
    lambda: oq.residual_norm(_z(4, 64), _z(4, 64), gate=_z(2, 64), scale=_z(3, 64), pre=oq.Norm("rms")),
    lambda: oq.residual_norm(_z(4, 64), _z(4, 64), gate=_z(2, 64), mod_row=_z(4, dt=torch.int64)),
    lambda: oq.residual_norm(_z(4, 64), _z(4, 64), mx4=True),
    lambda: oq.residual_norm(_z(4, 40), _z(4, 40), pre=oq.Norm("rms"), mx4=True),
    lambda: oq.residual_norm(_z(4, 64), _z(4, 64), pre=oq.Norm("rms"), H=_z(4, 32)),
])
def test_binding_refusals(call):
    with pytest.raises(ValueError):
        call()


def test_reference_codes_by_hand():
    x = torch.zeros((4, 32), dtype=torch.float64)
    # A block of max 6 has step 1: every border, and a value beside it.
    x[0, :16] = torch.tensor([6, -6, 0.25, 0.26, 0.75, 0.74, 1.25, 1.26, 1.75, 1.74, 2.5, 2.51, 3.5, 3.49, 5, -5.01])
    x[1, 0], x[1, 1] = 7.99, 7.0          # saturates
    x[2, 3] = math.inf
    index, byte = R.quantize(x)
    assert index[0, :16].tolist() == [7, 15, 0, 1, 2, 1, 2, 3, 4, 3, 4, 5, 6, 5, 6, 15]
    assert index[1, :2].tolist() == [7, 7] and byte.flatten().tolist() == [127, 127, 255, 0]
    assert R.values(index, byte)[0, 1] == -6 and torch.isnan(R.values(index, byte)[2]).all()
    q, s = R.pack(index, byte, "cpu")
    i2, b2 = R.unpack(q, s)
    assert torch.equal(i2, index) and torch.equal(b2, byte)
    tiny = torch.full((1, 32), 2.0 ** -127, dtype=torch.float64)
    assert R.quantize(tiny)[1].item() == 0 and (R.quantize(tiny)[0] == 2).all()
