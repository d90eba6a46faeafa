"""Linears in microscaled 4-bit floating point and the operators between them
(binding of oq_mx4_*, oq_gated_activation and oq_residual_norm in include/oq.h).

Marshalling only.  Shapes, types and devices are checked here, because the C
entry points see pointers alone.  MX4 codes travel as the pair (codes uint8
[M, K / 2], steps uint8 [M, mx4_step_bytes(K)]).
"""
from __future__ import annotations

import ctypes as C

import torch

from . import OUT_BF16, OUT_F16, _check, _current_device, _empty, _lib, _on, _ptr  # (the package has these before it imports this module)

ACT_GELU_TANH, ACT_SILU = 0, 1

_DTYPE = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
_HALF = {torch.float16: 0, torch.bfloat16: 1}
_TORCH = {0: torch.float16, 1: torch.bfloat16, 2: torch.float32}
_U8 = torch.uint8

# The host's time bounds the smallest calls, so the checks below ask a tensor as little as they can.


def _want(ok, what):
    if not ok:
        raise ValueError(what)


def _dev(t):
    """Index of t's device, which has to be the current one (the library launches there)."""
    dev = t.get_device()
    if dev < 0:
        raise ValueError("the tensors must be on one GPU")
    if dev != _current_device():
        raise ValueError(f"cuda:{dev} is not the current device")
    return dev


def mx4_step_bytes(K: int) -> int:
    """Bytes from one row's steps to the next."""
    return 16 * ((K + 511) // 512)


def _ld(t, name, M, N, dtype, dev):
    """Leading dimension of rows t [M, N] of dtype on device dev."""
    if t.dtype is dtype and t.get_device() == dev and t.shape == (M, N):
        ld, one = t.stride()
        if one == 1 or N == 1:
            return ld if M > 1 else (N + 7) // 8 * 8
    raise ValueError(f"{name}: rows [{M}, {N}] of {dtype} on cuda:{dev} expected")


def _codes(q, steps, name, dev):
    """(rows, K) of a pair of codes and steps."""
    if (q.dtype is _U8 and steps.dtype is _U8 and q.get_device() == dev and steps.get_device() == dev and q.dim() == 2
            and q.is_contiguous() and steps.is_contiguous()):
        n, half = q.shape
        if steps.shape == (n, 16 * ((half + 255) // 256)):
            return n, 2 * half
    raise ValueError(f"{name}: contiguous uint8 codes [n, K / 2] and steps [n, mx4_step_bytes(K)] on one GPU expected")


def _out_codes(like, M, K, Xq, steps, dev, stream):
    _want(K % 32 == 0, "codes need a multiple of 32 channels")
    made = Xq is None and steps is None
    if Xq is None:
        Xq = _empty(like, (M, K // 2), _U8, stream)
    if steps is None:
        steps = _empty(like, (M, mx4_step_bytes(K)), _U8, stream)
    _want(made or _codes(Xq, steps, "Xq, steps", dev) == (M, K), f"Xq, steps: codes of {M} rows of {K} channels expected")
    return Xq, steps


def mx4_quantize(X, had_block=1, Xq=None, steps=None, stream=None):
    """Codes and steps of X (fp16 or bf16 [M, K], activations or a weight),
    rotated in Hadamard blocks of had_block (1: none, 32, 64, 128) channels."""
    dt = _HALF.get(X.dtype)
    _want(dt is not None and X.dim() == 2, "X: fp16 or bf16 [M, K] expected")
    M, K = X.shape
    dev = _dev(X)
    ldx = _ld(X, "X", M, K, X.dtype, dev)
    Xq, steps = _out_codes(X, M, K, Xq, steps, dev, stream)
    _check(_lib.load().oq_mx4_quantize(X.data_ptr(), M, K, ldx, dt, had_block, Xq.data_ptr(), steps.data_ptr(), _on(stream, dev)),
           "oq_mx4_quantize")
    return Xq, steps


def mx4_dequantize(Xq, steps, out_dtype=OUT_BF16, X=None, stream=None):
    """The values [M, K] of codes, in fp16, bf16 or fp32 by out_dtype (OUT_F16,
    OUT_BF16, OUT_F32)."""
    dev = _dev(Xq)
    M, K = _codes(Xq, steps, "Xq, steps", dev)
    dt = _TORCH.get(out_dtype)
    _want(dt is not None, "out_dtype: OUT_F16, OUT_BF16 or OUT_F32 expected")
    if X is None:
        X, ldx = _empty(Xq, (M, K), dt, stream), K
    else:
        ldx = _ld(X, "X", M, K, dt, dev)
    _check(_lib.load().oq_mx4_dequantize(Xq.data_ptr(), steps.data_ptr(), M, K, X.data_ptr(), ldx, out_dtype, _on(stream, dev)),
           "oq_mx4_dequantize")
    return X


def mx4_linear(Xq, x_steps, Wq, w_steps, bias=None, out_dtype=OUT_F16, Y=None, stream=None):
    """Y [M, N] = x . w^T + bias (fp16 [N]) of the values of both operands' codes, in
    fp16, bf16 or fp32 by out_dtype.  (Made here, Y has rows of a multiple of 8
    elements: for another N it is a view of its first N columns.)"""
    dev = _dev(Xq)
    M, K = _codes(Xq, x_steps, "Xq, x_steps", dev)
    N, Kw = _codes(Wq, w_steps, "Wq, w_steps", dev)
    _want(Kw == K, "the operands need equal K")
    dt = _TORCH.get(out_dtype)
    _want(dt is not None, "out_dtype: OUT_F16, OUT_BF16 or OUT_F32 expected")
    if bias is not None:
        _want(bias.dtype is torch.float16 and bias.shape == (N,) and bias.is_contiguous() and bias.get_device() == dev,
              f"bias: contiguous float16 [{N}] on cuda:{dev} expected")
    if Y is None:
        ldy = (N + 7) // 8 * 8
        Y = _empty(Xq, (M, ldy), dt, stream)
        Y = Y if ldy == N else Y[:, :N]
    else:
        ldy = _ld(Y, "Y", M, N, dt, dev)
    _check(_lib.load().oq_mx4_linear(Xq.data_ptr(), x_steps.data_ptr(), M, Wq.data_ptr(), w_steps.data_ptr(), _ptr(bias), N, K,
                                     Y.data_ptr(), ldy, out_dtype, _on(stream, dev)), "oq_mx4_linear")
    return Y


def gated_activation(GU, act=ACT_GELU_TANH, mx4=False, H=None, stream=None):
    """act(g) u of rows GU [M, 2 F] = [g | u] (fp16 or bf16): H [M, F] of GU's
    type, or with mx4 the pair (codes, steps) of the next linear (H: such a pair)."""
    dt = _HALF.get(GU.dtype)
    _want(dt is not None and GU.dim() == 2 and GU.shape[1] % 2 == 0, "GU: fp16 or bf16 [M, 2 F] expected")
    M, F = GU.shape
    dev = _dev(GU)
    ld = _ld(GU, "GU", M, F, GU.dtype, dev)
    F //= 2
    ldh, h, q, steps = 0, None, None, None
    if mx4:
        H = _out_codes(GU, M, F, *(H or (None, None)), dev, stream)
        q, steps = H[0].data_ptr(), H[1].data_ptr()
    else:
        if H is None:
            H, ldh = _empty(GU, (M, F), GU.dtype, stream), F
        else:
            ldh = _ld(H, "H", M, F, GU.dtype, dev)
        h = H.data_ptr()
    _check(_lib.load().oq_gated_activation(GU.data_ptr(), M, F, ld, dt, act, h, ldh, q, steps, _on(stream, dev)),
           "oq_gated_activation")
    return H


class Norm:
    """A norm's parameters (oq_norm): kind "rms" or "layer", gain and bias [D]
    (fp16 or bf16) or None; the gain used is gain_offset + gain.  It holds the
    memory that the tensors have now: values written in place are seen, another
    storage given to them later (module.to(), .data =) needs another Norm."""

    KINDS = {"rms": 1, "layer": 2}

    def __init__(self, kind, gain=None, bias=None, eps=1e-6, gain_offset=0.0):
        _want(kind in self.KINDS, "kind: 'rms' or 'layer' expected")
        there = [t for t in (gain, bias) if t is not None]
        for t in there:
            _want(t.dim() == 1 and t.is_contiguous() and t.dtype in _HALF, "gain, bias: contiguous float16 or bfloat16 [D] expected")
        _want(len({(t.dtype, t.shape, t.device) for t in there}) < 2, "gain and bias need one type, length and device")
        self.kind = kind
        # (Aliases, so that the memory stays whatever becomes of the tensors.)
        self._gain, self._bias = (None if t is None else t.detach() for t in (gain, bias))
        # What a call checks: (type, channels, device), or None without parameters.
        self.of = (there[0].dtype, there[0].shape[0], there[0].get_device()) if there else None
        self._c = _lib.oq_norm(self.KINDS[kind], eps, gain_offset, _ptr(gain), _ptr(bias))
        self.ref = C.byref(self._c)

    gain = property(lambda self: self._gain)
    bias = property(lambda self: self._bias)


def residual_norm(R, Y=None, pre=None, post=None, alpha=1.0, gate=None, scale=None, shift=None, mod_row=None, mx4=False,
                  R_out=None, H=None, dtype=None, stream=None):
    """(r', h): r' = alpha R + gate post(Y), h = pre(r') (1 + scale) + shift.

    Y [M, D] fp16 or bf16 (or None: 0); R [M, D] of Y's type or fp32 (or None: 0,
    r' of Y's type unless R_out says otherwise); post, pre: Norm or None (pre
    None: h is None); gate, scale, shift: [n, D] of Y's type with one row stride,
    or [D], or None; mod_row int32 [M]: their row for each token (None: row 0;
    out of range: the token is skipped).  h is in Y's type (`dtype` where there is
    no Y), or with mx4 the pair (codes, steps) of the next linear.  R_out may be R,
    H may be Y.  R_out False: r' is not written (None), as for a first norm whose
    residual is R itself."""
    first = R if Y is None else Y
    _want(first is not None and first.dim() == 2, "R or Y [M, D] expected")
    M, D = first.shape
    half = Y.dtype if Y is not None else dtype or R.dtype
    dt = _HALF.get(half)
    _want(dt is not None, "Y: fp16 or bf16 expected (dtype where there is no Y)")
    dev = _dev(first)
    ldy = ldr = ldh = ldm = n_mod = 0
    y = r = row = h = q = steps = pg = ps = pt = None
    if Y is not None:
        ldy, y = _ld(Y, "Y", M, D, half, dev), Y.data_ptr()
    if R is not None:
        rt = R.dtype
        _want(rt is half or rt is torch.float32, "R: Y's type or float32 expected")
        ldr, r = _ld(R, "R", M, D, rt, dev), R.data_ptr()
    else:
        rt = half if R_out is None or R_out is False else R_out.dtype
        _want(rt is half or rt is torch.float32, "R_out: Y's type or float32 expected")
    of = (half, D, dev)
    _want((pre is None or pre.of in (None, of)) and (post is None or post.of in (None, of)),
          f"pre, post: gain and bias [{D}] of {half} on cuda:{dev} expected")
    if gate is not None or scale is not None or shift is not None:
        ptrs = []
        for t in (gate, scale, shift):
            if t is None:
                ptrs.append(None)
                continue
            n = t.shape[0] if t.dim() == 2 else 1
            ld = _ld(t if t.dim() == 2 else t[None], "gate, scale, shift", n, D, half, dev)
            _want(n >= 1 and (n_mod == 0 or (n == n_mod and ld == ldm)), "gate, scale, shift: as many rows of one stride expected")
            n_mod, ldm = n, ld
            ptrs.append(t.data_ptr())
        pg, ps, pt = ptrs
    if mod_row is not None:
        _want(mod_row.dtype is torch.int32 and mod_row.shape == (M,) and mod_row.is_contiguous() and mod_row.get_device() == dev,
              f"mod_row: contiguous int32 [{M}] on cuda:{dev} expected")
        row = mod_row.data_ptr()
    ldro, ro = D, None
    if R_out is False:
        _want(pre is not None, "without pre and R_out there is no output")
        R_out = None
    else:
        if R_out is None:
            R_out = _empty(first, (M, D), rt, stream)
        else:
            ldro = _ld(R_out, "R_out", M, D, rt, dev)
        ro = R_out.data_ptr()
    if pre is None:
        _want(H is None and not mx4, "without pre there is no h")
    elif mx4:
        H = _out_codes(first, M, D, *(H or (None, None)), dev, stream)
        q, steps = H[0].data_ptr(), H[1].data_ptr()
    else:
        if H is None:
            H, ldh = _empty(first, (M, D), half, stream), D
        else:
            ldh = _ld(H, "H", M, D, half, dev)
        h = H.data_ptr()
    _check(_lib.load().oq_residual_norm(r, ldr, _DTYPE[rt], y, ldy, dt, M, D, None if post is None else post.ref,
                                        None if pre is None else pre.ref, alpha, pg, ps, pt, ldm, n_mod, row, ro, ldro,
                                        h, ldh, q, steps, _on(stream, dev)), "oq_residual_norm")
    return R_out, H
