"""Attention over the 4-bit cache where its numbers are extreme: rows of zero
values under strongly negative scores, values near the smallest normal numbers,
scores far past 2^24.
All expected values are float64's."""
import pytest
import torch

import paper_2605_28803_amd as oq
from tests import serving_ref as R

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def _call(q, k, v, scale, rotate=False, page=64, causal=True):
    """q [nq, hq, d] over one sequence k, v [L, hk, d]: (output, the cache's keys and values as float64)."""
    L, hk, d = k.shape
    pages = -(-L // page)
    bufs = [torch.zeros((pages, hk, page, d // 2), dtype=torch.uint8),
            torch.zeros((pages, hk, page // 16, d // 2, 16), dtype=torch.uint8),
            torch.full((pages, hk, page), float("nan")), torch.full((pages, hk, page), float("nan"))]
    order = torch.arange(L)
    R.put(bufs, order, k, v, rotate)
    cache = oq.KV4Cache(*(b.to(DEV) for b in bufs), rotate_k=rotate)
    cu = None if q.shape[0] == 1 else torch.tensor([0, q.shape[0]], dtype=torch.int32, device=DEV)
    o = oq.attention_kv4(q.to(DEV), cache, torch.arange(pages, dtype=torch.int32, device=DEV)[None],
                         torch.tensor([L], dtype=torch.int32, device=DEV), cu, max_q=q.shape[0], max_len=L, causal=causal,
                         scale=scale)
    torch.cuda.synchronize()
    return o.cpu(), *R.take(bufs, order, d, rotate)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d,rotate", [(64, False), (128, True), (256, False)])
@pytest.mark.parametrize("below", [90.0, 100.0, 150.0, 1000.0])
@pytest.mark.parametrize("L", [1, 64, 700, 6000])
def test_zero_values_under_low_scores(L, below, d, rotate, dtype):
    """Every score is -below and every value 0: the output is 0, exactly."""
    q, k = torch.zeros((1, 4, d), dtype=dtype), torch.zeros((L, 2, d), dtype=dtype)
    q[:, :, 0], k[:, :, 0] = 1.0, -1.0
    o, _, _ = _call(q, k, torch.zeros_like(k), below, rotate)
    assert (o == 0).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("nq", [1, 3, 10])
@pytest.mark.parametrize("L,start,stop", [(128, 0, 64), (700, 64, 600), (6000, 0, 2500), (6000, 2000, 5990)])
def test_zero_values_beside_others(L, start, stop, nq, dtype):
    """A run of tokens with zero values and scores of -below, between tokens of
    score 0: it weighs nothing, in whatever wave or split it lies."""
    d = 128
    g = torch.Generator().manual_seed(L + nq)
    for below in (95.0, 110.0, 400.0):
        q, k = torch.zeros((nq, 4, d), dtype=dtype), torch.zeros((L, 2, d), dtype=dtype)
        v = torch.randn((L, 2, d), generator=g).to(dtype)
        q[:, :, 0] = 1.0
        k[start:stop, :, 0], v[start:stop] = -1.0, 0.0
        o, kk, vv = _call(q, k, v, below)
        see = torch.arange(L)[None, :] <= (L - nq + torch.arange(nq))[:, None]
        for h in range(4):
            ref, spread, _ = R.attend(q[:, h].double(), kk[:, h // 2], vv[:, h // 2], below, see)
            # (The other tokens' keys have step 0: their scores are 0 exactly.)
            R.check(o[:, h], ref, spread, 2.0 ** -18, dtype, 2.0 ** -11)


@pytest.mark.parametrize("e", [100, 104, 106, 110, 116, 122])
@pytest.mark.parametrize("L,nq,hq,d", [(1, 1, 2, 64), (64, 3, 4, 128), (700, 1, 8, 128), (6000, 2, 2, 256), (900, 12, 4, 64)])
def test_small_steps(L, nq, hq, d, e):
    """Steps of 2^-e, alone and among steps of up to 2^20 times as much.  2^126 of the
    largest contribution is above 2^3, so that a contribution has fp16's 11 bits down to 2^-17 of it."""
    g = torch.Generator().manual_seed(L + e)
    for spread in (0, 20):
        q, k = torch.randn((nq, hq, d), generator=g).bfloat16(), torch.randn((L, 2, d), generator=g).bfloat16()
        v = torch.randint(-7, 8, (L, 2, d), generator=g).double()
        v[:, :, 1] = 7.0
        v = (v * 2.0 ** (torch.randint(0, spread + 1, (L, 1, 1), generator=g) - e)).bfloat16()
        o, kk, vv = _call(q, k, v, 0.125)
        see = torch.arange(L)[None, :] <= (L - nq + torch.arange(nq))[:, None]
        for h in range(hq):
            qq, one = q[:, h].double(), kk[:, h // (hq // 2)]
            ref, size, p = R.attend(qq, one, vv[:, h // (hq // 2)], 0.125, see)
            # The accumulator starts at 72 sum(q) in units of the step (max / 7).
            extra = 2 * R.score_error(qq, one, 0.125)
            extra += 2 * 0.125 * qq.abs().sum(-1).max().item() * one.abs().max().item() / 7 * 80 * (d + 8) * 2.0 ** -24
            # ... and below that a contribution is off by half of fp16's smallest step, 2^-25, over 2^126, times 7
            # (size is taken times 2^-10).
            size = size + 7 * see.sum(-1, keepdim=True) * 2.0 ** -141
            R.check(o[:, h], ref, size, extra, torch.bfloat16, 2.0 ** -11)


@pytest.mark.parametrize("dtype,q0,step,high,low", [
    (torch.float16, 700.0, 97.0, 1000.0, 500.0),
    (torch.float16, -20000.0, 1024.0, 29000.0, 30000.0),
    (torch.bfloat16, 700.0, 97.0, 1000.0, 500.0),
    (torch.bfloat16, 2.0 ** 30, 2.0 ** 27, 2.0 ** 30, 2.0 ** 29),
    (torch.bfloat16, -2.0 ** 30, -2.0 ** 27, 2.0 ** 29, 2.0 ** 30),
])
@pytest.mark.parametrize("L,nq,hq,d,rotate", [(1, 1, 2, 64, False), (300, 3, 4, 128, False), (300, 20, 2, 64, True), (700, 5, 8, 256, False),
                                              (6000, 1, 4, 128, True), (6000, 9, 2, 64, False), (3000, 20, 4, 128, False)])
def test_equal_large_scores(L, nq, hq, d, rotate, dtype, q0, step, high, low):
    """Keys that share the largest score share the weight, however large it is."""
    q = (q0 + step * torch.arange(nq * hq).view(nq, hq, 1)).expand(nq, hq, d).to(dtype).contiguous()
    k = torch.full((L, 2, d), low, dtype=dtype)
    k[::2] = high
    v = torch.randn((L, 2, d), generator=torch.Generator().manual_seed(L)).to(dtype)
    o, kk, vv = _call(q, k, v, d ** -0.5, rotate)
    see = torch.arange(L)[None, :] <= (L - nq + torch.arange(nq))[:, None]
    for h in range(hq):
        qq = q[:, h].double()
        ref, spread, _ = R.attend(qq @ R.hadamard(d) / d ** 0.5 if rotate else qq, kk[:, h // (hq // 2)], vv[:, h // (hq // 2)],
                                  d ** -0.5, see)
        # (Equal keys have equal scores, whatever they were rounded to; the others are too far below to count.)
        R.check(o[:, h], ref, spread, 2.0 ** -15, dtype, 2.0 ** -11)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("L", [300, 6000])
def test_maxima_that_grow(L, dtype):
    """Scores that double along the sequence, from 2^-3 to 2^29 and from -2^29 up."""
    d = 64
    v = torch.randn((L, 1, d), generator=torch.Generator().manual_seed(3)).to(dtype)
    for down in (False, True):
        q, k = torch.zeros((1, 3, d), dtype=dtype), torch.zeros((L, 1, d), dtype=dtype)
        q[:, :, 0] = 2.0 ** 15
        k[:, 0, 0] = 2.0 ** (torch.arange(L) * (33.0 / L) - 18).floor()
        if down:
            k = -k.flip(0)
        o, kk, vv = _call(q, k, v, 1.0)
        ref, spread, _ = R.attend(q[:, 0].double(), kk[:, 0], vv[:, 0], 1.0, torch.ones((1, L), dtype=torch.bool))
        # (Where several scores count they are below 2^6; the product, the step's and the factor's roundings and the
        # exponent's are four of 2^-24 of 2^6.5, which counts twice.)
        for h in range(3):
            R.check(o[:, h], ref, spread, 2.0 ** -14, dtype, 2.0 ** -11)


@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("e", [120, 126, 130, 133])
def test_small_queries_and_large_keys(e, rotate):
    """Queries down to bf16's smallest number against keys of up to 2^126: the
    row's factor is below fp32's normal numbers, the scores are not."""
    d, L = 64, 100
    q, k = torch.zeros((2, 2, d), dtype=torch.bfloat16), torch.zeros((L, 1, d), dtype=torch.bfloat16)
    q[:, 0, 3], q[:, 1, 5] = 2.0 ** -e, -(2.0 ** -e)
    k[:, 0, 3], k[:, 0, 5] = 2.0 ** (e - 8), 2.0 ** (e - 9)
    k[::3] = -k[::3]
    v = torch.randn((L, 1, d), generator=torch.Generator().manual_seed(e)).bfloat16()
    o, kk, vv = _call(q, k, v, 32.0, rotate, causal=False)
    o2, _, _ = _call(q, k, v, 0.25, rotate, causal=False)
    for scale, got in ((32.0, o), (0.25, o2)):
        for h in range(2):
            qq = q[:, h].double()
            qq = qq @ R.hadamard(d) / d ** 0.5 if rotate else qq
            ref, spread, _ = R.attend(qq, kk[:, 0], vv[:, 0], scale, torch.ones((2, L), dtype=torch.bool))
            # (2^-10: the factor has 11 bits at least.  The start of 72 sum(q) and 22 bits of a rotated query are below it.)
            extra = 2 * R.score_error(qq, kk[:, 0], scale) + 2.0 ** -9 * scale * (qq.abs() @ kk[:, 0].abs().T).max().item()
            R.check(got[:, h], ref, spread, extra, torch.bfloat16, 2.0 ** -11)
