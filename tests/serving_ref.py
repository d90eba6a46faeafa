"""Plain 64-bit references of the serving operators (8-bit product, prompt
attention, 4-bit key/value cache) on the CPU, and the error bounds that the
GPU tests hold their results to."""
import math

import numpy as np
import torch

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # half a step, relative


def hadamard(d):
    i = np.arange(d)
    bits = i[:, None] & i[None, :]
    odd = np.zeros_like(bits)
    while bits.any():
        odd ^= bits & 1
        bits >>= 1
    return torch.from_numpy(1.0 - 2.0 * odd)


def codes(x, rotate):
    """(codes, steps) of rows x [..., d] float64; the quotient is formed from the
    unnormalized rotation, where inputs and sums are exact."""
    d = x.shape[-1]
    u = x @ hadamard(d) if rotate else x
    top = u.abs().amax(-1, keepdim=True)
    q = torch.round(7 * u / torch.where(top > 0, top, torch.ones_like(top)))
    return q, top[..., 0] / (7 * (math.sqrt(d) if rotate else 1.0))


def pack(q):
    n = q.to(torch.int64) & 15
    return (n[..., 0::2] | n[..., 1::2] << 4).to(torch.uint8)


def unpack(p):
    n = torch.stack((p & 15, p >> 4), -1).flatten(-2).to(torch.int64)
    return torch.where(n >= 8, n - 16, n).double()


def put(bufs, slots, k, v, rotate):
    """Write tokens into CPU copies of a cache's buffers (k_codes, v_codes, k_scale, v_scale)."""
    kc, vc, ks, vs = bufs
    page = kc.shape[2]
    for i, s in enumerate(slots.tolist()):
        if not 0 <= s < kc.shape[0] * page:
            continue
        p, t = divmod(s, page)
        for x, rot, c, sc in ((k[i], rotate, kc, ks), (v[i], False, vc, vs)):
            q, step = codes(x.double(), rot)
            sc[p, :, t] = step.float()
            if c is kc:
                kc[p, :, t] = pack(q)
            else:
                vc[p, :, t // 16, :, t % 16] = pack(q)


def take(bufs, slots, d, rotate):
    """(K, V) float64 values of slots, keys in the cache's own (rotated) basis."""
    kc, vc, ks, vs = bufs
    page = kc.shape[2]
    p, t = slots // page, slots % page
    k = unpack(kc[p, :, t]) * ks[p, :, t].double()[..., None]
    v = unpack(vc[p, :, t // 16, :, t % 16]) * vs[p, :, t].double()[..., None]
    return k, v


def attend(q, k, v, scale, visible):
    """One head in float64: rows q [n, d], k, v [L, d], row i sees the keys where
    visible[i].  Returns o, sum p |v|, and p."""
    if k.shape[0] == 0:
        return torch.zeros_like(q), torch.zeros_like(q), torch.zeros((q.shape[0], 1), dtype=q.dtype)
    s = scale * (q @ k.T)
    s = s.masked_fill(~visible, -math.inf)
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    p = e / torch.where(total > 0, total, torch.ones_like(total))
    return p @ v, p @ v.abs(), p


def check(got, ref, spread, extra, dtype, p_round):
    """|got - ref| <= u |ref| (the output's rounding) + spread (2 p_round + extra)
    + the type's smallest step: every probability is off by at most p_round (its
    rounding) in the product and in the sum, and by `extra` (twice the largest
    error of a score, and fp32 exponentials)."""
    u = U[dtype]
    tiny = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -130
    err = (got.double() - ref).abs()
    bound = u * ref.abs() + spread * (2 * p_round + extra) + tiny
    assert torch.isfinite(got.double()).all()
    worst = (err / bound).max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"error {worst:.2f} of the bound"
    norm = ref.norm().item()
    if norm > 0:
        rel = err.norm().item() / norm
        # Rounding errors are independent over outputs and keys: their root mean
        # square is below u (output) plus 2 p_round spread.
        lim = 2 * (u + 2 * p_round * spread.norm().item() / norm)
        assert rel <= lim, f"relative error {rel:.2e} over {lim:.2e}"


def score_error(q, k, scale):
    """Largest error of a score that fp32 sums of d products make, and of its exponential's argument."""
    d = q.shape[-1]
    top = (scale * (q.abs() @ k.abs().T)).max().item() if k.numel() and q.numel() else 0.0
    return 2 * (d + 8) * 2.0 ** -24 * top + 2.0 ** -20 * (1 + top / 8)
