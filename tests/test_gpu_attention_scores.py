"""Prompt attention under scores far past 2^24, where neighbouring fp32 numbers are
more than 1 apart: keys that share the largest score share the weight."""
import pytest
import torch

import paper_2605_28803_amd as oq
from tests import serving_ref as R

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def _check(q, k, v, causal, scale=None):
    n, hq, d = q.shape
    cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    got = oq.attention_prompt(q.to(DEV), k.to(DEV), v.to(DEV), cu, causal=causal, scale=scale).cpu()
    see = torch.ones((n, n), dtype=torch.bool)
    see = see.tril() if causal else see
    for h in range(hq):
        kv = h // (hq // k.shape[1])
        ref, spread, _ = R.attend(q[:, h].double(), k[:, kv].double(), v[:, kv].double(), d ** -0.5 if scale is None else scale, see)
        # (Equal keys have equal scores, whatever they were rounded to, and where others count the scores are
        # powers of two below 2^6: c's rounding and the exponent's, twice 2^-24 of 2^6.5 each, are below 2^-16 together.)
        R.check(got[:, h], ref, spread, 2.0 ** -15, q.dtype, R.U[q.dtype])


def _keys(n, hk, d, high, low, dtype):
    """high and low keys in turn, all channels alike."""
    k = torch.full((n, hk, d), float(low), dtype=dtype)
    k[::2] = high
    return k


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype,q0,step,high,low", [
    (torch.float16, 700.0, 4.0, 1000.0, 500.0),         # about 2^23 to 2^25 in units of log2
    (torch.float16, 20000.0, 32.0, 30000.0, 29000.0),   # 2^33 and more
    (torch.float16, -20000.0, 32.0, 29000.0, 30000.0),
    (torch.bfloat16, 700.0, 4.0, 1000.0, 500.0),
    (torch.bfloat16, 2.0 ** 40, 2.0 ** 34, 2.0 ** 40, 2.0 ** 39),
    (torch.bfloat16, -2.0 ** 40, -2.0 ** 34, 2.0 ** 39, 2.0 ** 40),
])
def test_equal_large_scores(dtype, q0, step, high, low, d, causal):
    g = torch.Generator().manual_seed(d)
    for n, hq, hk in ((300, 2, 1), (700, 44, 2) if d == 128 else (130, 4, 4)):
        q = (q0 + step * torch.arange(n)[:, None, None]).expand(n, hq, d).to(dtype)
        v = torch.randn((n, hk, d), generator=g).to(dtype)
        _check(q.contiguous(), _keys(n, hk, d, high, low, dtype), v, causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_maxima_that_grow(dtype, causal):
    """Scores that double about every 9 keys, from 2^-3 to 2^29 and from -2^29 up."""
    n, d = 300, 64
    v = torch.randn((n, 1, d), generator=torch.Generator().manual_seed(3)).to(dtype)
    for down in (False, True):
        q, k = torch.zeros((n, 2, d), dtype=dtype), torch.zeros((n, 1, d), dtype=dtype)
        q[:, :, 0] = 2.0 ** 15
        k[:, 0, 0] = 2.0 ** ((torch.arange(n) // 8).float() * 0.875 - 18).floor()
        if down:
            k = -k.flip(0)
        _check(q, k, v, causal, scale=1.0)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_rows_beside_a_growing_maximum(dtype, d):
    """Rows of equal scores up to 2^19 weigh their keys alike, though another
    row of the same wave meets a new maximum in every step."""
    n = 1500
    q, k = torch.zeros((n, 1, d), dtype=dtype), torch.zeros((n, 1, d), dtype=dtype)
    v = torch.randn((n, 1, d), generator=torch.Generator().manual_seed(d)).to(dtype)
    q[:, 0, 0] = (0.5 + torch.arange(n) % 29) * 16
    k[:, 0, 0] = 1023.0
    q[::16] = 0
    q[::16, 0, 1] = 1.0
    k[:, 0, 1] = torch.arange(n).to(dtype) / 64
    _check(q, k, v, False, scale=1.0)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,at", [(torch.float16, 25000.0), (torch.bfloat16, -2.0 ** 40)])
@pytest.mark.parametrize("n,hq,hk,d", [(100, 3, 1, 64), (100, 3, 1, 128), (100, 3, 1, 256), (700, 52, 4, 128)])
def test_equal_large_scores_without_key_groups(n, hq, hk, d, dtype, at, causal):
    # (at most 2 at: 50000 is finite in fp16)
    q = (at * (1 + torch.arange(n)[:, None, None] / n)).expand(n, hq, d).to(dtype).contiguous()
    assert torch.isfinite(q).all()
    v = torch.randn((n, hk, d), generator=torch.Generator().manual_seed(n + d)).to(dtype)
    _check(q, _keys(n, hk, d, at, at / 2, dtype), v, causal)
