"""Linears in microscaled 4-bit floating point and the operators between them
(binding of oq_mx4_*, oq_gated_activation and oq_residual_norm in include/oq.h).

Marshalling only.  Shapes, types and devices are checked here, because the C
entry points see pointers alone.  MX4 codes travel as the pair (codes uint8
[M, K / 2], steps uint8 [M, mx4_step_bytes(K)]).
"""
from __future__ import annotations

import ctypes as C

import torch

from . import OUT_BF16, OUT_F16, _check, _empty, _lib, _on, _one_gpu, _ptr  # (the package has these before it imports this module)

ACT_GELU_TANH, ACT_SILU = 0, 1

_DTYPE = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
_TORCH = {0: torch.float16, 1: torch.bfloat16, 2: torch.float32}


def _want(ok, what):
    if not ok:
        raise ValueError(what)


def mx4_step_bytes(K: int) -> int:
    """Bytes from one row's steps to the next."""
    return 16 * ((K + 511) // 512)


def _rows(t, name, ok_types=(torch.float16, torch.bfloat16)):
    """Leading dimension of a 2-D tensor of rows."""
    if t.dim() != 2 or t.dtype not in ok_types or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name}: rows [n, channels] of {' or '.join(str(x) for x in ok_types)} expected")
    return t.stride(0) if t.shape[0] > 1 else (t.shape[1] + 7) // 8 * 8


def _codes(q, steps, name):
    """(rows, K) of a pair of codes and steps."""
    if q.dim() == 2 and q.dtype is torch.uint8 and steps.dtype is torch.uint8 and q.is_contiguous() and steps.is_contiguous():
        n, K = q.shape[0], 2 * q.shape[1]
        if steps.shape == (n, mx4_step_bytes(K)):
            return n, K
    raise ValueError(f"{name}: contiguous uint8 codes [n, K / 2] and steps [n, mx4_step_bytes(K)] expected")


def _new_codes(like, M, K, Xq, steps, stream):
    if Xq is None:
        Xq = _empty(like, (M, K // 2), torch.uint8, stream)
    if steps is None:
        steps = _empty(like, (M, mx4_step_bytes(K)), torch.uint8, stream)
    _want(_codes(Xq, steps, "Xq, steps") == (M, K), f"Xq, steps: codes of {M} rows of {K} channels expected")
    return Xq, steps


def mx4_quantize(X, had_block=1, Xq=None, steps=None, stream=None):
    """Codes and steps of X (fp16 or bf16 [M, K], activations or a weight),
    rotated in Hadamard blocks of had_block (1: none, 32, 64, 128) channels."""
    ldx = _rows(X, "X")
    M, K = X.shape
    _want(K % 32 == 0, "X: a multiple of 32 channels expected")
    Xq, steps = _new_codes(X, M, K, Xq, steps, stream)
    dev = _one_gpu(X, Xq, steps)
    _check(_lib.load().oq_mx4_quantize(_ptr(X), M, K, ldx, _DTYPE[X.dtype], had_block, _ptr(Xq), _ptr(steps),
                                       _on(stream, dev)), "oq_mx4_quantize")
    return Xq, steps


def mx4_dequantize(Xq, steps, out_dtype=OUT_BF16, X=None, stream=None):
    """The values [M, K] of codes, in fp16, bf16 or fp32 by out_dtype (OUT_F16,
    OUT_BF16, OUT_F32)."""
    M, K = _codes(Xq, steps, "Xq, steps")
    dt = _TORCH.get(out_dtype)
    _want(dt is not None, "out_dtype: OUT_F16, OUT_BF16 or OUT_F32 expected")
    if X is None:
        X = _empty(Xq, (M, K), dt, stream)
    _want(X.shape == (M, K), f"X: [{M}, {K}] expected")
    ldx = _rows(X, "X", (dt,))
    dev = _one_gpu(Xq, steps, X)
    _check(_lib.load().oq_mx4_dequantize(_ptr(Xq), _ptr(steps), M, K, _ptr(X), ldx, out_dtype, _on(stream, dev)),
           "oq_mx4_dequantize")
    return X


def mx4_linear(Xq, x_steps, Wq, w_steps, bias=None, out_dtype=OUT_F16, Y=None, stream=None):
    """Y [M, N] = x . w^T + bias (fp16 [N]) of the values of both operands' codes, in
    fp16, bf16 or fp32 by out_dtype.  (Made here, Y has rows of a multiple of 8
    elements: for another N it is a view of its first N columns.)"""
    M, K = _codes(Xq, x_steps, "Xq, x_steps")
    N, Kw = _codes(Wq, w_steps, "Wq, w_steps")
    _want(Kw == K, "the operands need equal K")
    dt = _TORCH.get(out_dtype)
    _want(dt is not None, "out_dtype: OUT_F16, OUT_BF16 or OUT_F32 expected")
    if bias is not None:
        _want(bias.shape == (N,) and bias.dtype is torch.float16 and bias.is_contiguous(), "bias: contiguous float16 [N] expected")
    if Y is None:
        ldy = (N + 7) // 8 * 8
        Y = _empty(Xq, (M, ldy), dt, stream)
        Y = Y if ldy == N else Y[:, :N]
    else:
        _want(Y.shape == (M, N), f"Y: [{M}, {N}] expected")
        ldy = _rows(Y, "Y", (dt,))
    dev = _one_gpu(Xq, x_steps, Wq, w_steps, Y) if bias is None else _one_gpu(Xq, x_steps, Wq, w_steps, Y, bias)
    _check(_lib.load().oq_mx4_linear(_ptr(Xq), _ptr(x_steps), M, _ptr(Wq), _ptr(w_steps), _ptr(bias), N, K, _ptr(Y), ldy,
                                     out_dtype, _on(stream, dev)), "oq_mx4_linear")
    return Y


def gated_activation(GU, act=ACT_GELU_TANH, mx4=False, H=None, stream=None):
    """act(g) u of rows GU [M, 2 F] = [g | u] (fp16 or bf16): H [M, F] of GU's
    type, or with mx4 the pair (codes, steps) of the next linear (H: such a pair)."""
    ld = _rows(GU, "GU")
    M, F = GU.shape[0], GU.shape[1] // 2
    _want(GU.shape[1] == 2 * F, "GU: an even number of columns expected")
    ldh, q, steps = 0, None, None
    if mx4:
        _want(F % 32 == 0, "GU: 2 F columns, F a multiple of 32, expected")
        q, steps = H = _new_codes(GU, M, F, *(H or (None, None)), stream)
        dev = _one_gpu(GU, q, steps)
    else:
        H = _empty(GU, (M, F), GU.dtype, stream) if H is None else H
        _want(H.shape == (M, F), f"H: [{M}, {F}] expected")
        ldh = _rows(H, "H", (GU.dtype,))
        dev = _one_gpu(GU, H)
    _check(_lib.load().oq_gated_activation(_ptr(GU), M, F, ld, _DTYPE[GU.dtype], act, None if mx4 else _ptr(H), ldh, _ptr(q),
                                           _ptr(steps), _on(stream, dev)), "oq_gated_activation")
    return H


class Norm:
    """A norm's parameters (oq_norm): kind "rms" or "layer", gain and bias [D]
    (fp16 or bf16) or None; the gain used is gain_offset + gain."""

    KINDS = {"rms": 1, "layer": 2}

    def __init__(self, kind, gain=None, bias=None, eps=1e-6, gain_offset=0.0):
        _want(kind in self.KINDS, "kind: 'rms' or 'layer' expected")
        for t, name in ((gain, "gain"), (bias, "bias")):
            _want(t is None or (t.dim() == 1 and t.is_contiguous() and t.dtype in (torch.float16, torch.bfloat16)),
                  f"{name}: contiguous float16 or bfloat16 [D] expected")
        self.kind, self.gain, self.bias = kind, gain, bias
        self._c = _lib.oq_norm(self.KINDS[kind], eps, gain_offset, _ptr(gain), _ptr(bias))
        self.ref = C.byref(self._c)


def residual_norm(R, Y=None, pre=None, post=None, alpha=1.0, gate=None, scale=None, shift=None, mod_row=None, mx4=False,
                  R_out=None, H=None, dtype=None, stream=None):
    """(r', h): r' = alpha R + gate post(Y), h = pre(r') (1 + scale) + shift.

    Y [M, D] fp16 or bf16 (or None: 0); R [M, D] of Y's type or fp32 (or None: 0,
    r' of Y's type unless R_out says otherwise); post, pre: Norm or None (pre
    None: h is None); gate, scale, shift: [n, D] of Y's type with one row stride,
    or [D], or None; mod_row int32 [M]: their row for each token (None: row 0;
    out of range: the token is skipped).  h is in Y's type (`dtype` where there is
    no Y), or with mx4 the pair (codes, steps) of the next linear.  R_out may be R,
    H may be Y."""
    first = Y if Y is not None else R
    _want(first is not None, "R or Y expected")
    M, D = first.shape
    dt = Y.dtype if Y is not None else dtype if dtype is not None else R.dtype
    _want(dt in (torch.float16, torch.bfloat16), "Y: fp16 or bf16 expected (dtype where there is no Y)")
    half = (dt,)
    tensors = [first]
    ldy = ldr = ldh = ldm = n_mod = 0
    if Y is not None:
        ldy = _rows(Y, "Y", half)
    rt = R.dtype if R is not None else R_out.dtype if R_out is not None else dt
    _want(rt == dt or rt is torch.float32, "R: Y's type or float32 expected")
    if R is not None:
        _want(R.shape == (M, D), f"R: [{M}, {D}] expected")
        ldr = _rows(R, "R", (rt,))
        tensors.append(R)
    for n, name in ((post, "post"), (pre, "pre")):
        if n is not None:
            for t in (n.gain, n.bias):
                if t is not None:
                    _want(t.shape[0] == D and t.dtype == dt, f"{name}: gain and bias [{D}] of {dt} expected")
                    tensors.append(t)
    for t, name in ((gate, "gate"), (scale, "scale"), (shift, "shift")):
        if t is None:
            continue
        t2 = t if t.dim() == 2 else t[None]
        ld = _rows(t2, name, half)
        _want(t2.shape[1] == D and t2.shape[0] >= 1 and (n_mod == 0 or (t2.shape[0] == n_mod and ld == ldm)),
              f"{name}: [n, {D}] rows like the others' expected")
        n_mod, ldm = t2.shape[0], ld
        tensors.append(t)
    if mod_row is not None:
        _want(mod_row.dtype is torch.int32 and mod_row.shape == (M,) and mod_row.is_contiguous(),
              f"mod_row: contiguous int32 [{M}] expected")
        tensors.append(mod_row)
    if R_out is None:
        R_out = _empty(first, (M, D), rt, stream)
    _want(R_out.shape == (M, D), f"R_out: [{M}, {D}] expected")
    ldro = _rows(R_out, "R_out", (rt,))
    tensors.append(R_out)
    q = steps = None
    if pre is None:
        _want(H is None and not mx4, "without pre there is no h")
    elif mx4:
        _want(D % 32 == 0, "codes need a multiple of 32 channels")
        q, steps = H = _new_codes(first, M, D, *(H or (None, None)), stream)
        tensors += H
    else:
        H = _empty(first, (M, D), dt, stream) if H is None else H
        _want(H.shape == (M, D), f"H: [{M}, {D}] expected")
        ldh = _rows(H, "H", half)
        tensors.append(H)
    dev = _one_gpu(*tensors)
    _check(_lib.load().oq_residual_norm(
        _ptr(R), ldr, _DTYPE[rt], _ptr(Y), ldy, _DTYPE[dt], M, D, post and post.ref, pre and pre.ref, alpha, _ptr(gate),
        _ptr(scale), _ptr(shift), ldm, n_mod, _ptr(mod_row), _ptr(R_out), ldro, None if mx4 else _ptr(H), ldh, _ptr(q),
        _ptr(steps), _on(stream, dev)), "oq_residual_norm")
    return R_out, H
