"""Plain 64-bit references of the microscaled 4-bit operators on the CPU, and
the error bounds that the GPU tests hold their results to."""
import math

import torch

from tests.serving_ref import hadamard

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # half a step, relative
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}  # half the smallest number
F = 2.0 ** -24
GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
MIDDLES = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)


def rotate(x, b):
    return x if b == 1 else ((x.reshape(-1, b) @ hadamard(b)) / math.sqrt(b)).reshape(x.shape)


def quantize(x):
    """(index with sign int64 [M, K], bytes int64 [M, K / 32]) of x float64 [M, K]."""
    b = x.reshape(x.shape[0], -1, 32)
    top = b.abs().amax(-1)
    bad = ~torch.isfinite(b).all(-1)
    _, e = torch.frexp(torch.where(bad | (top == 0), torch.ones_like(top), top))
    s = torch.where(top == 0, torch.full_like(e, -127), e.to(torch.int32) - 3).clamp(-127, 127).to(torch.int64)
    a = torch.where(bad[..., None], torch.zeros_like(b), b.abs()) * 2.0 ** -s[..., None].double()
    low = torch.searchsorted(MIDDLES, a, right=False)   # borders below a
    up = torch.searchsorted(MIDDLES, a, right=True)     # and those equal to it
    index = torch.where(low % 2 == 0, low, up)          # at a border: the even neighbour
    index = index + 8 * (torch.signbit(b) & (index >= 0)).to(torch.int64)
    index[bad] = 0
    return index.reshape(x.shape), torch.where(bad, torch.full_like(s, 255), s + 127)


def values(index, byte):
    v = torch.where(index % 16 >= 8, -1.0, 1.0).double() * GRID[index % 8]
    step = torch.where(byte == 255, torch.full(byte.shape, math.nan, dtype=torch.float64), 2.0 ** (byte.double() - 127))
    return (v.reshape(v.shape[0], -1, 32) * step[..., None]).reshape(v.shape)


def unpack(q, steps):
    """(index, bytes) of the library's codes and steps."""
    q, K = q.cpu().to(torch.int64), 2 * q.shape[1]
    return torch.stack((q & 15, q >> 4), -1).reshape(q.shape[0], K), steps.cpu()[:, : K // 32].to(torch.int64)


def pack(index, byte, device, fill=255):
    """Codes and steps as the library takes them (unused bytes of a row: `fill`)."""
    q = (index[:, 0::2] | index[:, 1::2] << 4).to(torch.uint8)
    steps = torch.full((byte.shape[0], 16 * -(-index.shape[1] // 512)), fill, dtype=torch.uint8)
    steps[:, : byte.shape[1]] = byte.to(torch.uint8)
    return q.to(device), steps.to(device)


def check_codes(got, want64):
    """Codes and steps that the library wrote against those of float64 values."""
    index, byte = unpack(*got)
    wi, wb = quantize(want64)
    assert torch.equal(byte, wb)
    ok = (index == wi) | ((index % 8 == 0) & (wi % 8 == 0))  # (a zero's sign is free)
    assert bool(ok.all()), f"{int((~ok).sum())} of {ok.numel()} codes differ"


def linear(xi, xb, wi, wb, bias=None):
    """(Y, bound) in float64.  The matrix instruction's sum of 64 or 128 exact
    products and its accumulator is taken to be within 2^-23 of the sum of their
    magnitudes (a 32-bit result, truncated), one instruction behind the other, and
    the partial sums of up to 16 waves add as many roundings."""
    x, w = values(xi, xb), values(wi, wb)
    y, mag = x @ w.T, x.abs() @ w.abs().T
    if bias is not None:
        y, mag = y + bias.double(), mag + bias.double().abs()
    return y, (x.shape[1] / 64 + 17) * 2 * F * mag


def norm(x, kind, gain, bias, offset, eps):
    """float64 (normed rows, normed rows before gain and bias, 1 / deviation, mean)."""
    mean = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + eps)
    n = (x - mean) * rstd
    g = torch.ones_like(x[0]) if gain is None else gain.double() + offset
    return n * g + (0 if bias is None else bias.double()), n, rstd, mean, g


def residual_norm(R, Y, pre, post, alpha, gate, scale, shift):
    """pre, post: None or (kind, gain, bias, offset, eps); gate, scale, shift: rows
    for each token, or None.  Returns float64 (r', bound of r' in float arithmetic, h,
    bound of h), the bounds without the outputs' own rounding.

    Float arithmetic rounds each operation by F, relative.  A norm's result has at
    most six of them and its 1 / deviation: sums of squares of at most 32 values a
    thread (16 F for half of it: the root halves), the value's own rounding.  x - mean adds
    F (|x| + |mean|), and the mean is off by 16 F mean|x|.  An error d of r' (at most D in a
    row) moves h by |g| rstd (d + 2 D) + |n g| rstd D."""
    M, D = (Y if Y is not None else R).shape
    y = torch.zeros((M, D), dtype=torch.float64) if Y is None else Y.double()
    err = torch.zeros_like(y)
    if post is not None:
        x = y
        y, n, rstd, mean, g = norm(x, *post)
        far = F * (x.abs() + mean.abs() + 16 * x.abs().mean(-1, keepdim=True)) if post[0] == "layer" else 0 * x
        worst = far.amax(-1, keepdim=True)
        err = (g.abs() * rstd * far + (n * g).abs() * (24 * F + rstd * worst) + 2 * F * y.abs())
    if gate is not None:
        y, err = y * gate.double(), err * gate.double().abs() + F * (y * gate.double()).abs()
    old = torch.zeros_like(y) if R is None else alpha * R.double()
    r = old + y
    err = err + F * (r.abs() + y.abs() + old.abs())
    if pre is None:
        return r, err, None, None
    h, n, rstd, mean, g = norm(r, *pre)
    worst = err.amax(-1, keepdim=True)
    far = F * (r.abs() + mean.abs() + 16 * r.abs().mean(-1, keepdim=True)) + worst if pre[0] == "layer" else 0 * r
    e = g.abs() * rstd * (err + far + worst) + (n * g).abs() * (24 * F + rstd * (worst + far.amax(-1, keepdim=True))) + 2 * F * h.abs()
    e = e + 2 * F * (0 if pre[2] is None else pre[2].double().abs())
    s = 1.0 if scale is None else 1 + scale.double()
    t = 0.0 if shift is None else shift.double()
    out = h * s + t
    return r, err, out, e * (s.abs() if scale is not None else 1) + 3 * F * (h * s).abs() + F * out.abs()


def activation(GU, act):
    """(h, bound of h in float arithmetic) in float64: t has four roundings and its
    product with log2 e one, all relative to it, then at most 8 more units.  The
    reciprocal of 1 + e^-t is 0 where it is below the smallest normal float, 2^-126:
    an error of at most 2^-126 |g u|, which bf16 can hold."""
    g, u = GU.double().chunk(2, dim=1)
    t = g if act == 1 else 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
    h = g / (1 + torch.exp(-t)) * u
    return h, h.abs() * (6 * F * t.abs().clamp(max=200) + 10 * F) + 2.0 ** -126 * (g * u).abs()


def check(got, want, bound, dtype):
    got = got.cpu().double()
    tol = bound + (U[dtype] * (want.abs() + bound) + TINY[dtype])
    bad = (got - want).abs() > tol
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, at worst {((got - want).abs() / tol).max():.3g} of the bound"
